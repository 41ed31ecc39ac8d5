"""The block operators at the limit of 2^31 elements, where sums of positions come near 2^31, against 64 bits.

Bounds (eps = 2^-24): a mean and a sum of squares are nested sums of a few to some thousand terms, 64 eps; a bf16 result is rounded once, 2^-8.5 in the
2-norm."""
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
DEV = "cuda:0"


def _noise(n, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.empty(n, dtype=torch.bfloat16, device=DEV).normal_(generator=g)


def _parts(n, step=1 << 27):
    return [slice(k, min(n, k + step)) for k in range(0, n, step)]


@pytest.mark.parametrize("n", [(1 << 31) - 1, (1 << 31) - 1000])
def test_group_norm(n):
    """One channel of n positions."""
    import paper_1412_6249_amd as pa
    shape = (1, n, 1)
    x = _noise(n, 1).view(shape)
    y = torch.full_like(x, float("nan"))
    mean, rstd = (torch.empty(1, 1, device=DEV) for _ in range(2))
    ws = torch.empty(max(pa.purine_group_norm_workspace_bytes(b, shape, 1, pa.PURINE_BF16) for b in (0, 1)), dtype=torch.uint8, device=DEV)
    pa.purine_group_norm_fwd(x, None, None, y, mean, rstd, 1, 1e-5, pa.PURINE_ACT_NONE, ws=ws)
    flat = x.view(-1)
    mu = sum(float(flat[p].double().sum()) for p in _parts(n)) / n
    var = sum(float((flat[p].double() - mu).square().sum()) for p in _parts(n)) / n
    want = (var + 1e-5) ** -0.5
    assert abs(float(mean) - mu) <= 64 * EPS and abs(float(rstd) / want - 1) <= 64 * EPS
    for p in _parts(n):
        z = (flat[p].double() - mu) * want
        assert float((y.view(-1)[p].double() - z).norm()) <= 2 ** -8.5 * float(z.norm())
    dy = _noise(n, 2).view(shape)
    dx = y.fill_(float("nan"))
    pa.purine_group_norm_bwd(x, None, None, mean, rstd, dy, dx, None, None, 1, pa.PURINE_ACT_NONE, ws=ws)
    xhat = lambda p: (flat[p].double() - mu) * want  # noqa: E731
    a = sum(float(dy.view(-1)[p].double().sum()) for p in _parts(n)) / n
    b = sum(float((dy.view(-1)[p].double() * xhat(p)).sum()) for p in _parts(n)) / n
    for p in _parts(n):
        g = want * (dy.view(-1)[p].double() - a - xhat(p) * b)
        assert float((dx.view(-1)[p].double() - g).norm()) <= 2 ** -8.5 * float(g.norm())


@pytest.mark.parametrize("N,K", [((1 << 31) - 1, 1), ((1 << 31) - 1000, 1), (1, (1 << 31) - 1)])
def test_activation_gradient(N, K):
    import paper_1412_6249_amd as pa
    pre = _noise(N * K, 3).view(N, K)
    g = torch.full_like(pre, float("nan"))
    db = torch.full((K,), float("nan"), device=DEV)
    ws = torch.empty(pa.purine_act_bwd_workspace_bytes(N, K), dtype=torch.uint8, device=DEV)
    pa.purine_act_bwd(pre, pre, g, db, pa.PURINE_ACT_RELU, ws=ws)
    total = size = 0.0
    for p in _parts(N * K):
        want = pre.view(-1)[p].clamp(min=0)
        assert torch.equal(g.view(-1)[p], want)
        if K == 1:
            total, size = total + float(want.double().sum()), size + float(want.double().abs().sum())
        else:
            assert torch.equal(db[p], want.float())
    if K == 1:
        assert abs(float(db) - total) <= 64 * EPS * size
