"""Few rows by a matrix of 2^31 bytes and more, past the 32-bit offsets of the one-launch forms, against 64 bits.

Bounds (eps = 2^-24): C + 2 eps of the terms' magnitudes, and a bf16 rounding, 2^-8. The activation's slope is 1.1 at most, and it has four
roundings of its own."""
import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
DEV = "cuda:0"


# rows, columns of x, rows of w, its columns in memory
@pytest.mark.parametrize("dtype,N,C,K,ld", [("bf16", 1, 8192, 140008, 8192), ("bf16", 4, 4096, 264000, 4096), ("f32", 2, 4096, 136000, 4096), ("bf16", 7, 8190, 132000, 8200),
                                            ("f32", 11, 1000, 40000, 16000)])
def test_far_matrix(dtype, N, C, K, ld):
    import paper_1412_6249_amd as pa
    td, code = (torch.bfloat16, pa.PURINE_BF16) if dtype == "bf16" else (torch.float32, pa.PURINE_F32)
    g = torch.Generator(device=DEV).manual_seed(N)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV, dtype=td)  # noqa: E731
    x, w, b, r = rnd(N, C), rnd(K, ld)[:, :C], rnd(K), rnd(N, K)
    assert ((K - 1) * ld + C) * x.element_size() >= 1 << 31
    y, pre = (torch.full((N, K), float("nan"), dtype=td, device=DEV) for _ in range(2))
    pa.purine_linear_fwd(x, w, b, r, y, pre, pa.PURINE_ACT_SILU, ws=torch.empty(max(256, pa.purine_linear_workspace_bytes(0, N, C, K, code)), dtype=torch.uint8, device=DEV))
    for k in range(0, K, 4096):
        n = min(4096, K - k)
        wk, bk = w[k:k + n].double().t().contiguous(), b[k:k + n].double()
        want = x.double() @ wk + bk
        tol = (C + 2) * EPS * (x.double().abs() @ wk.abs() + bk.abs()) + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0.0)
        assert bool(((pre[:, k:k + n].double() - want).abs() <= tol).all()), k
        z = ref.act(want, "silu") + r[:, k:k + n].double()
        tol = 1.1 * tol + 4 * EPS * want.abs() + (2.0 ** -8 * z.abs() if dtype == "bf16" else EPS * z.abs())
        assert bool(((y[:, k:k + n].double() - z).abs() <= tol).all()), k
