"""Products whose rows have 2^24 elements and more, past the offsets of the kernels on the matrix cores, against 64 bits.

Bound (eps = 2^-24): partial sums of K / splits terms one after the other; of terms with random signs their roundings add up as squares, and 2^-12 of the
terms' 2-norm times the square root of two is far above that; a bf16 result is rounded once, 2^-8."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ws(pa, which, N, C, K, code):
    return torch.full((max(256, pa.purine_linear_workspace_bytes(which, N, C, K, code)),), 255, dtype=torch.uint8, device=DEV)


def _dot(a, b):
    """Product of [n, K] and [m, K] in 64 bits, and the terms' 2-norms, by parts; few results pair by pair (the library takes a second for 2^25 terms of one)."""
    total = norm = 0.0
    for k in range(0, a.shape[1], 1 << 25):
        x, y = a[:, k:k + (1 << 25)].double(), b[:, k:k + (1 << 25)].double()
        if len(a) * len(b) > 100:
            total, norm = total + x @ y.t().contiguous(), norm + x.square() @ y.square().t().contiguous()
            continue
        terms = [[p * q for q in y] for p in x]
        total = total + torch.stack([torch.stack([t.sum() for t in row]) for row in terms])
        norm = norm + torch.stack([torch.stack([t.square().sum() for t in row]) for row in terms])
    return total, norm.sqrt()


def _check(got, want, norm, dtype):
    tol = 2.0 ** -11.5 * norm + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0.0)
    assert bool(torch.isfinite(got).all()) and bool(((got.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype,N,C,K", [("bf16", 2, (1 << 29) + 5, 3), ("f32", 1, (1 << 29) + 8, 2), ("bf16", 1, (1 << 31) - 1, 1), ("bf16", 70, (1 << 24) + 16, 100), ("f32", 3, (1 << 24) + 3, 5)])
def test_forward(dtype, N, C, K):
    import paper_1412_6249_amd as pa
    td, code = (torch.bfloat16, pa.PURINE_BF16) if dtype == "bf16" else (torch.float32, pa.PURINE_F32)
    g = torch.Generator(device=DEV).manual_seed(N)
    x, w, b = (torch.empty(s, dtype=td, device=DEV).normal_(generator=g) for s in ((N, C), (K, C), (K,)))
    y = torch.full((N, K), float("nan"), dtype=td, device=DEV)
    pa.purine_linear_fwd(x, w, b, None, y, ws=_ws(pa, pa.PURINE_CONV_FWD, N, C, K, code))
    want, norm = _dot(x, w)
    _check(y, want + b.double(), norm, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradients(dtype):
    """The data gradient whose reduction is the long side, and the weight gradient whose results it is."""
    import paper_1412_6249_amd as pa
    td, code = (torch.bfloat16, pa.PURINE_BF16) if dtype == "bf16" else (torch.float32, pa.PURINE_F32)
    N, C, K = 3, 5, (1 << 27) + 9
    g = torch.Generator(device=DEV).manual_seed(N)
    dy, w, x = (torch.empty(s, dtype=td, device=DEV).normal_(generator=g) for s in ((N, K), (K, C), (N, C)))
    dx, dw = torch.full((N, C), float("nan"), dtype=td, device=DEV), torch.full((K, C), float("nan"), dtype=td, device=DEV)
    pa.purine_linear_bwd_data(dy, w, None, dx, ws=_ws(pa, pa.PURINE_CONV_BWD_DATA, N, C, K, code))
    want, norm = _dot(dy, w.t())
    _check(dx, want, norm, dtype)
    pa.purine_linear_bwd_weight(x, dy, dw, None, ws=_ws(pa, pa.PURINE_CONV_BWD_WEIGHT, N, C, K, code))
    for k in range(0, K, 1 << 24):
        part = slice(k, min(K, k + (1 << 24)))
        d = dy[:, part].double().t().contiguous()
        _check(dw[part], d @ x.double(), (d.square() @ x.double().square()).sqrt(), dtype)
