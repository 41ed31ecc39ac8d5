"""Streams of rows whose bytes lie past 31 bits, up to the limit of a tensor's elements: dense ones of many rows, and rows far apart. Bounds as in test_gpu_linear_stream."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV, BF16 = "cuda:0", torch.bfloat16


def _near(got, want, products, what):
    err, tol = float((got.double() - want).norm()), (2e-8 * products ** 0.5 + 1e-6 + 2 ** -8.5) * float(want.norm())
    assert err <= tol, (what, err, tol)


def test_many_rows():
    import paper_1412_6249_amd as pa
    N, C, K = 19000003, 112, 96                 # 4.3 GB of x, 3.6 GB of y
    g = torch.Generator(device=DEV).manual_seed(1)
    part = torch.randn(1000003, C, generator=g, device=DEV).to(BF16)
    x = part.repeat(19, 1)[:N]
    x[-5000:] = torch.randn(5000, C, generator=g, device=DEV).to(BF16)
    assert x.is_contiguous() and x.shape[0] == N
    w = (torch.randn(K, C, generator=g, device=DEV) * C ** -0.5).to(BF16)
    y = torch.full((N, K), float("nan"), dtype=BF16, device=DEV)
    ws = torch.empty(max(256, *(pa.purine_linear_workspace_bytes(p, N, C, K, pa.PURINE_BF16) for p in (0, 1))), dtype=torch.uint8, device=DEV)
    pa.purine_linear_fwd(x, w, None, None, y, ws=ws)
    for rows in (slice(0, 5000), slice(9600000, 9605000), slice(N - 5000, N)):
        _near(y[rows], x[rows].double() @ w.double().t(), C, "y")
    assert torch.equal(y[:1000003], y[1000003:2000006])
    dy, tail = y, x[-5000:].clone()
    pa.purine_linear_bwd_data(dy, w, None, x, beta=1.0, ws=ws)
    want = tail.double() + dy[-5000:].double() @ w.double()
    _near(x[-5000:], want, K, "dx")


def test_rows_far_apart():
    import paper_1412_6249_amd as pa
    N, C, K, ld = 4097, 64, 48, 524048
    g = torch.Generator(device=DEV).manual_seed(2)
    base = torch.zeros(N * ld, dtype=BF16, device=DEV)      # 4.3 GB; rows a megabyte apart
    x = base.as_strided((N, C), (ld, 1))
    r = base.as_strided((N, K), (ld, 1), C)
    y = base.as_strided((N, K), (ld, 1), C + 256)
    x.copy_(torch.randn(N, C, generator=g, device=DEV))
    r.copy_(torch.randn(N, K, generator=g, device=DEV))
    w = (torch.randn(K, C, generator=g, device=DEV) * C ** -0.5).to(BF16)
    ws = torch.empty(max(256, pa.purine_linear_workspace_bytes(0, N, C, K, pa.PURINE_BF16)), dtype=torch.uint8, device=DEV)
    pa.purine_linear_fwd(x, w, None, r, y, ws=ws)
    torch.cuda.synchronize()
    _near(y, x.double() @ w.double().t() + r.double(), C, "y")
    assert float(base.as_strided((N, 256 - K), (ld, 1), C + K).abs().max()) == 0.0
