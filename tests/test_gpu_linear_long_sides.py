"""Matrix products of more columns or rows than one launch has threads for (2^32), against 64 bits.

Bounds (eps = 2^-24): a result is a sum of K fp32 terms, K + 2 eps of the terms' magnitudes; bf16 results and gradients are rounded once more, 2^-8."""
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
DEV = "cuda:0"


def _ws(pa, which, N, C, K, code):
    return torch.full((max(256, pa.purine_linear_workspace_bytes(which, N, C, K, code)),), 255, dtype=torch.uint8, device=DEV)


def _check(got, want, mag, terms, dtype, what):
    tol = (terms + 2) * EPS * mag + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0.0)
    assert bool(torch.isfinite(got).all()), what
    assert bool(((got.double() - want).abs() <= tol).all()), what


@pytest.mark.parametrize("dtype,N,C", [("bf16", 1, 8), ("f32", 3, 4), ("bf16", 9, 12)])
def test_columns(dtype, N, C):
    """K = 2^27 + 40 rows of w: 2^32 threads at 64 or 32 a column and more."""
    import paper_1412_6249_amd as pa
    K, td, code = (1 << 27) + 40, *((torch.bfloat16, pa.PURINE_BF16) if dtype == "bf16" else (torch.float32, pa.PURINE_F32))
    g = torch.Generator(device=DEV).manual_seed(N)
    x = torch.randn(N, C, generator=g, device=DEV).to(td)
    w = torch.randn(K, C, generator=g, device=DEV, dtype=td)
    b = torch.randn(K, generator=g, device=DEV, dtype=td)
    y = torch.full((N, K), float("nan"), dtype=td, device=DEV)
    pa.purine_linear_fwd(x, w, b, None, y, ws=_ws(pa, pa.PURINE_CONV_FWD, N, C, K, code))
    for k in range(0, K, 1 << 23):
        wk, bk = w[k:k + (1 << 23)].double(), b[k:k + (1 << 23)].double()
        _check(y[:, k:k + (1 << 23)], x.double() @ wk.t().contiguous() + bk, x.double().abs() @ wk.abs().t().contiguous() + bk.abs(), C + 1, dtype, k)


def test_rows():
    """Weight and data gradients whose results have 2^26 + 24 rows."""
    import paper_1412_6249_amd as pa
    K, C, N = (1 << 26) + 24, 8, 5
    g = torch.Generator(device=DEV).manual_seed(1)
    x = torch.randn(N, C, generator=g, device=DEV).bfloat16()
    dy = torch.randn(N, K, generator=g, device=DEV, dtype=torch.bfloat16)
    dw, db = (torch.full(s, float("nan"), dtype=torch.bfloat16, device=DEV) for s in ((K, C), (K,)))
    pa.purine_linear_bwd_weight(x, dy, dw, db, ws=_ws(pa, pa.PURINE_CONV_BWD_WEIGHT, N, C, K, pa.PURINE_BF16))
    t = torch.full((K, N), float("nan"), dtype=torch.bfloat16, device=DEV)
    w = torch.randn(C, N, generator=g, device=DEV).bfloat16()
    pa.purine_linear_bwd_data(dw, w, None, t, ws=_ws(pa, pa.PURINE_CONV_BWD_DATA, K, N, C, pa.PURINE_BF16))
    for k in range(0, K, 1 << 23):
        part = slice(k, k + (1 << 23))
        d, xd = dy[:, part].double().t().contiguous(), x.double()
        _check(dw[part], d @ xd, d.abs() @ xd.abs(), N, "bf16", ("dw", k))
        _check(db[part], d.sum(1), d.abs().sum(1), N, "bf16", ("db", k))
        a = dw[part].double()
        _check(t[part], a @ w.double(), a.abs() @ w.double().abs(), C, "bf16", ("dx", k))


def test_column_sums():
    """K = 2^29 + 64 columns."""
    import paper_1412_6249_amd as pa
    N, K = 2, (1 << 29) + 64
    dy = torch.arange(K, device=DEV, dtype=torch.int32).remainder_(251).to(torch.bfloat16).expand(N, K).contiguous()
    g, db = torch.empty_like(dy), torch.full((K,), float("nan"), device=DEV)
    ws = torch.empty(pa.purine_act_bwd_workspace_bytes(N, K), dtype=torch.uint8, device=DEV)
    pa.purine_act_bwd(dy, dy, g, db, pa.PURINE_ACT_RELU, ws=ws)
    assert torch.equal(g, dy)
    for k in range(0, K, 1 << 25):
        part = slice(k, k + (1 << 25))
        assert torch.equal(db[part], 2 * dy[0, part].float())
