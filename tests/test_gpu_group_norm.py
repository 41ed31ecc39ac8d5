"""Group normalization with an activation, channels last, forward and backward, against its definition in 64 bits: one position, one
channel per group, one group, odd planes and channels, rows of 2, 4, 8 and 16 bytes, images apart in memory, large means, infinities and NaNs.

Bounds (eps = 2^-24, the rounding of an fp32 result). xhat carries the rounding of the mean, |mean| / std of them, and about ten operations of its own; the
activations' exponentials add a few: 32 eps (1 + |mean| / std / 8). A bf16 result is rounded once more, 2^-9 at most and 2^-8.5
with room in the 2-norm. Sums of gradients are off by at most a few eps of the sum
of what their terms' roundings are proportional to (block_ref.group_norm_grad): 32 eps."""
import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
DEV = "cuda:0"

# images, positions, channels, groups
CASES = [(2, 1, 64, 1), (1, 1, 4096, 2), (3, 5, 8, 8), (2, 784, 192, 32), (1, 3136, 64, 32), (5, 899, 150, 15), (4, 49, 21, 7), (2, 100, 34, 17),
         (7, 16, 36, 9), (1, 12544, 32, 1), (2, 33, 2056, 8), (70, 9, 24, 3), (1, 20000, 5, 1), (300, 1, 48, 4), (2, 2500, 320, 32), (3, 130, 1030, 5), (4, 1, 8, 8)]
IDS = ["x".join(map(str, c)) for c in CASES]


def _inputs(case, dtype, seed=0, mean=1.0):
    N, S, C, G = case
    g = torch.Generator().manual_seed(seed + N + 7 * S + 31 * C + G)
    rnd = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    t = {"x": (rnd(N, S, C) + mean * rnd(C)).to(td), "scale": 1 + 0.3 * rnd(C), "shift": 0.3 * rnd(C), "dy": rnd(N, S, C).to(td)}
    return {k: v.to(DEV) for k, v in t.items()}, td


def _ws(pa, backward, case, dtype):
    N, S, C, G = case
    n = pa.purine_group_norm_workspace_bytes(backward, (N, S, C), G, pa.PURINE_F32 if dtype == "f32" else pa.PURINE_BF16)
    return torch.full((max(256, n),), 255, dtype=torch.uint8, device=DEV)


def _near(got, want, tol, what):
    got, want = got.double(), want.double()
    assert bool(torch.isfinite(got).all()), what
    assert float((got - want).norm()) <= tol * float(want.norm()) + 1e-30, (what, float((got - want).norm() / want.norm()), tol)


def _forward(pa, t, td, case, dtype, act, eps=1e-5, stats=True):
    N, S, C, G = case
    nan = lambda *s, dt=td: torch.full(s, float("nan"), dtype=dt, device=DEV)  # noqa: E731
    y = nan(N, S, C)
    mean, rstd = (nan(N, G, dt=torch.float32), nan(N, G, dt=torch.float32)) if stats else (None, None)
    pa.purine_group_norm_fwd(t["x"], t["scale"], t["shift"], y, mean, rstd, G, eps, pa.ACTIVATIONS[act], ws=_ws(pa, 0, case, dtype))
    return y, mean, rstd


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_both_directions(case, dtype):
    import paper_1412_6249_amd as pa
    N, S, C, G = case
    act = ["none", "silu", "gelu", "gelu_tanh", "relu"][(N + S + C) % 5]
    t, td = _inputs(case, dtype)
    few = S * C // G == 1                       # (one value per group: xhat is 0, and the gradient of x)
    d = {k: v.double() for k, v in t.items()}
    y, mean, rstd = _forward(pa, t, td, case, dtype, act)
    wy, wm, wr, _, z = ref.group_norm(d["x"], d["scale"], d["shift"], G, 1e-5, act)
    spread = 1 / float(wr.min()) if not few else 1.0
    tol = 32 * EPS * (1 + float(wm.abs().max()) / max(spread, 1e-3) / 8)
    _near(mean, wm, tol, "mean")
    if not few:
        _near(rstd, wr, tol, "rstd")
    _near(y, wy, tol if dtype == "f32" else 2 ** -8.5, "y")
    y2, _, _ = _forward(pa, t, td, case, dtype, act, stats=False)
    assert torch.equal(y, y2)

    if act == "relu":                           # at z = 0 within rounding the slope may be either value: no gradient comes in there
        t["dy"][z.abs() < 1e-4] = 0
        d["dy"] = t["dy"].double()
    dx = torch.full_like(t["x"], float("nan"))
    ds, db = (torch.full((C,), float("nan"), device=DEV) for _ in range(2))
    pa.purine_group_norm_bwd(t["x"], t["scale"], t["shift"], mean, rstd, t["dy"], dx, ds, db, G, pa.ACTIVATIONS[act], ws=_ws(pa, 1, case, dtype))
    wdx, wds, wdb, mags, magb, hnorm = ref.group_norm_grad(d["x"], d["scale"], d["shift"], G, 1e-5, act, d["dy"])
    assert bool(((ds.double() - wds).abs() <= tol * mags + 1e-30).all()) and bool(((db.double() - wdb).abs() <= tol * magb + 1e-30).all())
    assert float((dx.double() - wdx).norm()) <= (4 * tol if dtype == "f32" else 2 ** -8.5) * float(hnorm) + 1e-30
    # accumulation into what dx holds, in place over dy, no parameters' gradients; the same bits every time
    dx2, dx3 = t["dy"].clone(), t["dy"].clone()
    pa.purine_group_norm_bwd(t["x"], t["scale"], t["shift"], mean, rstd, dx2, dx2, None, None, G, pa.ACTIVATIONS[act], ws=_ws(pa, 1, case, dtype))
    assert torch.equal(dx2, dx)
    pa.purine_group_norm_bwd(t["x"], t["scale"], t["shift"], mean, rstd, t["dy"], dx3, None, None, G, pa.ACTIVATIONS[act], beta=1.0, ws=_ws(pa, 1, case, dtype))
    want = wdx + d["dy"]
    assert float((dx3.double() - want).norm()) <= (4 * tol if dtype == "f32" else 2 ** -8.5) * float(hnorm + d["dy"].norm())


@pytest.mark.parametrize("act", ["none", "relu", "silu", "gelu", "gelu_tanh"])
def test_activations_at_their_ends(act):
    """scale and shift put z at any place: z = shift where scale is 0."""
    import paper_1412_6249_amd as pa
    shift = torch.tensor([0.0, -0.0, 1e-30, -1e-30, 1.0, -1.0, 9.0, -9.0, 30.0, -30.0, 1e4, -1e4, 3e38, -3e38, float("inf"), float("-inf")], device=DEV)
    C = shift.numel()
    x, dy = torch.randn(1, 6, C, device=DEV), torch.ones(1, 6, C, device=DEV)
    t = {"x": x, "scale": torch.zeros(C, device=DEV), "shift": shift}
    y, mean, rstd = _forward(pa, t, torch.float32, (1, 6, C, 1), "f32", act)
    z = shift.double().cpu()
    want = ref.act(z, act)
    ends = {"none": [float("inf"), float("-inf")]}.get(act, [float("inf"), 0.0])
    want[-2:] = torch.tensor(ends).double()
    want = torch.where(torch.isnan(want), torch.where(z > 0, z, torch.zeros_like(z)), want)
    got = y[0].double().cpu()
    fin = torch.isfinite(want)
    assert bool((got[:, ~fin] == want[~fin]).all())
    assert bool(((got[:, fin] - want[fin]).abs() <= 64 * EPS * want[fin].abs() + 1e-11).all())
    ds, db = torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    pa.purine_group_norm_bwd(x, t["scale"], shift, mean, rstd, dy, torch.empty_like(x), ds, db, 1, pa.ACTIVATIONS[act], ws=_ws(pa, 1, (1, 6, C, 1), "f32"))
    s = ref.slope(z.clamp(-1e4, 1e4), act)
    assert bool(((db.double().cpu() / 6 - s).abs() <= 128 * EPS).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_views_without_parameters_on_a_stream(dtype):
    import paper_1412_6249_amd as pa
    N, H, W, C, G = 3, 5, 7, 24, 4
    t, td = _inputs((N, 2 * H * W, C, G), dtype)
    big = t["x"].reshape(N, 2 * H, W, C)
    x = big[:, H:]                                         # images 2 H W C elements apart
    out = torch.full_like(big, 7.0)
    y = out[:, :H]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    pa.purine_group_norm_fwd(x, None, None, y, None, None, G, 1e-5, pa.PURINE_ACT_SILU, ws=_ws(pa, 0, (N, H * W, C, G), dtype), stream=side)
    side.synchronize()
    one = torch.ones(C, device=DEV).double()
    want, *_ = ref.group_norm(x.double().reshape(N, H * W, C), one, 0 * one, G, 1e-5, "silu")
    _near(y.reshape(N, H * W, C), want, 64 * EPS if dtype == "f32" else 2 ** -8.5, "y")
    assert bool((out[:, H:] == 7.0).all())
    with torch.cuda.stream(side):                          # the current stream, in place
        pa.purine_group_norm_fwd(x, None, None, x, None, None, G, 1e-5, pa.PURINE_ACT_SILU, ws=_ws(pa, 0, (N, H * W, C, G), dtype))
    side.synchronize()
    assert torch.equal(x, y)


def test_large_means_and_small_spreads():
    import paper_1412_6249_amd as pa
    case = (2, 600, 24, 4)
    g = torch.Generator().manual_seed(3)
    x = (1000.0 + torch.randn(2, 600, 24, generator=g)).to(DEV)
    t = {"x": x, "scale": torch.ones(24, device=DEV), "shift": torch.zeros(24, device=DEV)}
    y, mean, rstd = _forward(pa, t, torch.float32, case, "f32", "none")
    wy, wm, wr, *_ = ref.group_norm(x.double(), t["scale"].double(), t["shift"].double(), 4, 1e-5, "none")
    _near(mean, wm, 4 * EPS, "mean")
    _near(rstd, wr, 64 * EPS, "rstd")                      # (about the mean's own value: its size does not come in)
    _near(y, wy, 1001 * 2 * EPS, "y")
    # a constant group: variance 0, rstd 1 / sqrt(eps)
    t["x"] = torch.full_like(x, 3.25)
    y, mean, rstd = _forward(pa, t, torch.float32, case, "f32", "none")
    assert float(y.abs().max()) == 0.0 and float((rstd - 1e-5 ** -0.5).abs().max()) < 1e-3


def test_not_a_number_stays_in_its_group():
    import paper_1412_6249_amd as pa
    case = (2, 40, 16, 4)
    t, td = _inputs(case, "f32")
    clean, *_ = _forward(pa, t, td, case, "f32", "silu")
    for bad in (float("nan"), float("inf"), float("-inf")):
        for pos in (0, 17):
            t2 = dict(t, x=t["x"].clone())
            t2["x"][1, pos, 5] = bad
            y, mean, rstd = _forward(pa, t2, td, case, "f32", "silu")
            assert bool(torch.isnan(rstd[1, 1])) and bool(torch.isnan(y[1, :, 4:8]).all())
            keep = torch.ones_like(y, dtype=torch.bool)
            keep[1, :, 4:8] = False
            assert torch.equal(y[keep], clean[keep])


def test_gradient_against_differences():
    """The fp32 gradient along a direction, against the central difference of the 64-bit loss: curvature h^2 / 6 |f'''| and 64-bit
    rounding are below 1e-6 of the loss's scale at h = 1e-4."""
    import paper_1412_6249_amd as pa
    case = (3, 35, 18, 6)
    N, S, C, G = case
    for act in ("none", "silu", "gelu", "gelu_tanh"):
        t, td = _inputs(case, "f32", seed=5)
        y, mean, rstd = _forward(pa, t, td, case, "f32", act)
        dx, ds, db = torch.empty_like(t["x"]), torch.empty(C, device=DEV), torch.empty(C, device=DEV)
        pa.purine_group_norm_bwd(t["x"], t["scale"], t["shift"], mean, rstd, t["dy"], dx, ds, db, G, pa.ACTIVATIONS[act], ws=_ws(pa, 1, case, "f32"))
        d = {k: v.double() for k, v in t.items()}
        loss = lambda x, s, b: (ref.group_norm(x, s, b, G, 1e-5, act)[0] * d["dy"]).sum()  # noqa: E731
        g = torch.Generator().manual_seed(9)
        for which, grad in (("x", dx), ("scale", ds), ("shift", db)):
            u = torch.randn(d[which].shape, generator=g, dtype=torch.float64).to(DEV)
            at = lambda k: loss(*[d[n] + (k * u if n == which else 0) for n in ("x", "scale", "shift")])  # noqa: E731
            num = float(at(1e-4) - at(-1e-4)) / 2e-4
            got = float((grad.double() * u).sum())
            assert abs(got - num) <= 1e-5 * float(grad.double().norm() * u.norm()), (act, which)


def test_offsets_past_32_bits():
    import paper_1412_6249_amd as pa
    N, S, C, G = 2, 1 << 19, 1056, 33                     # 1.1e9 elements, 2.2 GB
    x = torch.empty(N, S, C, dtype=torch.bfloat16, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    for n in range(N):
        x[n] = torch.randn(S, C, generator=g, device=DEV)
    y = torch.empty_like(x)
    ws = _ws(pa, 1, (N, S, C, G), "bf16")
    mean, rstd = torch.empty(N, G, device=DEV), torch.empty(N, G, device=DEV)
    pa.purine_group_norm_fwd(x, None, None, y, mean, rstd, G, 1e-5, 0, ws=_ws(pa, 0, (N, S, C, G), "bf16"))
    per = C // G
    for n, k in ((0, 0), (1, G - 1)):
        part = x[n, :, k * per:(k + 1) * per].double()
        assert abs(float(mean[n, k]) - float(part.mean())) < 1e-6
        want = (part - part.mean()) * (part.var(unbiased=False) + 1e-5).rsqrt()
        _near(y[n, :, k * per:(k + 1) * per], want, 2 ** -8.5, "y")
    dx = y
    pa.purine_group_norm_bwd(x, None, None, mean, rstd, y, dx, None, None, G, 0, ws=ws)       # dy = xhat: its gradient is 0
    assert float(dx[-1, -1000:].float().abs().max()) < 0.05
