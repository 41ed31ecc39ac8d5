"""Group normalization whose groups have many channels, slices or both, so that a kernel of its own joins their sums, against 64 bits.

Bounds (eps = 2^-24) as in test_gpu_group_norm.py: statistics 32 eps of the largest magnitude, a bf16 result one rounding, 2^-8.5 in the 2-norm, an fp32 one
32 eps (1 + |mean| / std / 8), its gradient four times that."""
import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
DEV = "cuda:0"


# images, positions, channels, groups: slices, channels, many of both (several workgroups a group), channels of one position
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", [(1, 12544, 512, 32), (3, 4096, 320, 32), (2, 5000, 6144, 1), (1, 70000, 1030, 2), (5, 1, 50000, 1), (2, 3, 40000, 2), (1, 20001, 33, 3)],
                         ids=lambda c: "x".join(map(str, c)) if isinstance(c, tuple) else c)
def test_both_directions(case, dtype):
    import paper_1412_6249_amd as pa
    N, S, C, G = case
    td, code = (torch.float32, pa.PURINE_F32) if dtype == "f32" else (torch.bfloat16, pa.PURINE_BF16)
    g = torch.Generator(device=DEV).manual_seed(S + C)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    x, dy = (rnd(N, S, C) + rnd(C)).to(td), rnd(N, S, C).to(td)
    scale, shift = 1 + 0.3 * rnd(C), 0.3 * rnd(C)
    ws = torch.full((max(pa.purine_group_norm_workspace_bytes(b, case[:3], G, code) for b in (0, 1)),), 255, dtype=torch.uint8, device=DEV)
    nan = lambda *s, dt=torch.float32: torch.full(s, float("nan"), dtype=dt, device=DEV)  # noqa: E731
    y, dx, mean, rstd, ds, db = nan(N, S, C, dt=td), nan(N, S, C, dt=td), nan(N, G), nan(N, G), nan(C), nan(C)
    pa.purine_group_norm_fwd(x, scale, shift, y, mean, rstd, G, 1e-5, pa.PURINE_ACT_SILU, ws=ws)
    d = [t.double() for t in (x, scale, shift, dy)]
    wy, wm, wr, _, _ = ref.group_norm(*d[:3], G, 1e-5, "silu")
    tol = 32 * EPS * (1 + float(wm.abs().max() * wr.max()) / 8)
    assert float((mean.double() - wm).abs().max()) <= 32 * EPS * float(d[0].abs().max()) and float((rstd.double() / wr - 1).abs().max()) <= tol
    assert float((y.double() - wy).norm()) <= (tol if dtype == "f32" else 2 ** -8.5) * float(wy.norm())
    z = x.clone()
    ws.fill_(255)
    pa.purine_group_norm_fwd(z, scale, shift, z, None, None, G, 1e-5, pa.PURINE_ACT_SILU, ws=ws)
    assert torch.equal(z, y)
    ws.fill_(255)
    pa.purine_group_norm_bwd(x, scale, shift, mean, rstd, dy, dx, ds, db, G, pa.PURINE_ACT_SILU, ws=ws)
    wdx, wds, wdb, mags, magb, hnorm = ref.group_norm_grad(*d[:3], G, 1e-5, "silu", d[3])
    assert bool(((ds.double() - wds).abs() <= tol * mags).all()) and bool(((db.double() - wdb).abs() <= tol * magb).all())
    assert float((dx.double() - wdx).norm()) <= (4 * tol if dtype == "f32" else 2 ** -8.5) * float(hnorm)


def test_not_a_number_stays_in_its_group():
    import paper_1412_6249_amd as pa
    N, S, C, G = 2, 5000, 512, 2
    x = torch.randn(N, S, C, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    ws = torch.full((pa.purine_group_norm_workspace_bytes(0, (N, S, C), G),), 255, dtype=torch.uint8, device=DEV)
    clean, y = torch.empty_like(x), torch.empty_like(x)
    pa.purine_group_norm_fwd(x, None, None, clean, None, None, G, 1e-5, pa.PURINE_ACT_NONE, ws=ws)
    for bad in (float("nan"), float("inf"), float("-inf")):
        for pos in (0, 1, 4999):
            z = x.clone()
            z[1, pos, 300] = bad
            pa.purine_group_norm_fwd(z, None, None, y, None, None, G, 1e-5, pa.PURINE_ACT_NONE, ws=ws)
            assert torch.equal(y[0], clean[0]) and torch.equal(y[1, :, :256], clean[1, :, :256]) and bool(torch.isnan(y[1, :, 256:]).all())


@pytest.mark.parametrize("C", [(1 << 31) - 1, (1 << 31) - 1000])
def test_one_group_of_all(C):
    """One position: a group of 2^31 - 1 channels."""
    import paper_1412_6249_amd as pa
    x = torch.empty(1, C, dtype=torch.bfloat16, device=DEV).normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    y = torch.full_like(x, float("nan"))
    mean, rstd = (torch.empty(1, 1, device=DEV) for _ in range(2))
    ws = torch.empty(pa.purine_group_norm_workspace_bytes(0, (1, C), 1, pa.PURINE_BF16), dtype=torch.uint8, device=DEV)
    pa.purine_group_norm_fwd(x, None, None, y, mean, rstd, 1, 1e-5, pa.PURINE_ACT_NONE, ws=ws)
    parts = [slice(k, min(C, k + (1 << 27))) for k in range(0, C, 1 << 27)]
    mu = sum(float(x[0, p].double().sum()) for p in parts) / C
    want = (sum(float((x[0, p].double() - mu).square().sum()) for p in parts) / C + 1e-5) ** -0.5
    assert abs(float(mean) - mu) <= 64 * EPS and abs(float(rstd) / want - 1) <= 64 * EPS
    for p in parts:
        z = (x[0, p].double() - mu) * want
        assert float((y[0, p].double() - z).norm()) <= 2 ** -8.5 * float(z.norm())
    # y is xhat within its rounding: what its own gradient leaves is that
    pa.purine_group_norm_bwd(x, None, None, mean, rstd, y, y, None, None, 1, pa.PURINE_ACT_NONE, ws=ws)
    assert float(y[0, -1000:].float().abs().max()) < 0.05
