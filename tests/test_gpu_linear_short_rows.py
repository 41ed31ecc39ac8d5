"""Few rows by many short rows of w, in every form that the choice between them may take, against 64 bits.

Bound (eps = 2^-24): C + 2 eps of the terms' magnitudes, and a bf16 rounding, 2^-8."""
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [4, 8, 16, 64, 72, 260])
@pytest.mark.parametrize("N,K", [(1, 4096), (2, 65537), (4, 65536), (1, 300007), (3, 300000), (4, 1 << 20), (16, 100000)])
def test_short_rows(N, C, K, dtype):
    import paper_1412_6249_amd as pa
    td, code = (torch.bfloat16, pa.PURINE_BF16) if dtype == "bf16" else (torch.float32, pa.PURINE_F32)
    g = torch.Generator(device=DEV).manual_seed(C)
    x, w, b = (torch.randn(s, generator=g, device=DEV, dtype=td) for s in ((N, C), (K, C), (K,)))
    y = torch.full((N, K), float("nan"), dtype=td, device=DEV)
    ws = torch.full((max(256, pa.purine_linear_workspace_bytes(pa.PURINE_CONV_FWD, N, C, K, code)),), 255, dtype=torch.uint8, device=DEV)
    pa.purine_linear_fwd(x, w, b, None, y, ws=ws)
    wt = w.double().t().contiguous()
    want = x.double() @ wt + b.double()
    tol = (C + 2) * EPS * (x.double().abs() @ wt.abs() + b.double().abs()) + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0.0)
    assert bool(torch.isfinite(y).all()) and bool(((y.double() - want).abs() <= tol).all())
