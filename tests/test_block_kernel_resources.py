"""What the compiler made of the block operators' kernels, from the metadata of the library that was built here: kernels whose loops hold their
sums, fragments or pieces in registers keep them there."""
import pytest

from test_kernel_resources import kernels  # noqa: F401


@pytest.mark.parametrize("name", ["linear_gemm_kernel", "linear_direct_kernel", "linear_row_kernel", "linear_stream_kernel", "linear_join_kernel", "act_bwd_kernel",
                                  "norm_sums_kernel", "norm_apply_kernel", "norm_grad_sums_kernel", "norm_grad_apply_kernel", "norm_held_kernel",
                                  "norm_grad_held_kernel", "adamw_kernel"])
def test_no_register_goes_to_memory(kernels, name):  # noqa: F811
    mine = {n: k for n, k in kernels.items() if name in n}
    assert mine
    bad = {n: (k[".vgpr_spill_count"], k[".private_segment_fixed_size"]) for n, k in mine.items()
           if k[".vgpr_spill_count"] or k[".private_segment_fixed_size"]}
    assert not bad, bad
