"""Mean and rstd of group normalization where a channel's first positions are unlike the others (padding, masks), in the held and in the sliced
form, against 64 bits.

Bounds (eps = 2^-24). A thread's squares are taken about a value within its few values' own range and joined as squares about joined means, so that
nothing cancels: a few roundings each of a dozen nested sums of a few terms to some hundred, 64 eps of rstd with room. A mean is a nested sum of
values up to the largest: 8 eps of that."""
import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
DEV = "cuda:0"

# images, positions, channels, groups: held, held by fp32 only, sliced; threads with a few positions and with more than a hundred
CASES = [(2, 784, 192, 32), (2, 784, 24, 4), (1, 12544, 64, 8), (1, 262144, 16, 4), (2, 65536, 1024, 4), (3, 1000, 7, 1), (64, 12544, 64, 32)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("where", ["first", "two", "half", "last", "none"])
@pytest.mark.parametrize("case", CASES, ids=["x".join(map(str, c)) for c in CASES])
def test_unlike_positions(case, where, dtype):
    import paper_1412_6249_amd as pa
    N, S, C, G = case
    code, td, spread = (pa.PURINE_F32, torch.float32, 1.0) if dtype == "f32" else (pa.PURINE_BF16, torch.bfloat16, 30.0)
    g = torch.Generator(device=DEV).manual_seed(S + C)
    x = torch.randn(N, S, C, generator=g, device=DEV).mul_(spread).add_(1000.0)
    if where != "none":
        x[:, {"first": slice(0, 1), "two": slice(0, 2), "half": slice(0, S // 2), "last": slice(S - 1, S)}[where]] = 0.0
    x = x.to(td)
    ws = torch.full((max(256, pa.purine_group_norm_workspace_bytes(0, (N, S, C), G, code)),), 255, dtype=torch.uint8, device=DEV)
    y = torch.empty_like(x)
    mean, rstd = (torch.full((N, G), float("nan"), device=DEV) for _ in range(2))
    pa.purine_group_norm_fwd(x, None, None, y, mean, rstd, G, 1e-5, pa.PURINE_ACT_NONE, ws=ws)
    for n in range(N):
        xg = x[n].double().reshape(S, G, C // G)
        mu = xg.mean((0, 2))
        want = ((xg - mu[:, None]).pow(2).mean((0, 2)) + 1e-5).rsqrt()
        most = float(xg.abs().max())
        assert float((mean[n].double() - mu).abs().max()) <= 8 * EPS * most, (n, float((mean[n].double() - mu).abs().max()) / most / EPS)
        off = float((rstd[n].double() / want - 1).abs().max())
        assert off <= 64 * EPS, (n, off / EPS)
        z = ((xg - mu[:, None]) * want[:, None]).reshape(S, C)
        off = float((y[n].double() - z).norm() / z.norm())
        assert off <= (64 * EPS + 8 * EPS * most * float(want.max()) if dtype == "f32" else 2 ** -8.5), (n, off)
