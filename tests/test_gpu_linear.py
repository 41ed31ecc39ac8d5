"""Matrix products with bias, activation and residual, their gradients and the gradient of an activation, against their definition in
64 bits: one row, one column, one product, ragged rows, columns and reductions, rows apart, all options, both types.

Bounds. Sums of C random products in fp32: 2e-8 sqrt(C) of the result's 2-norm (three quarters of an fp32 chain's), plus the
epilogue's few operations, 1e-6. A bf16 result is rounded once: 2^-8.5 with room in the 2-norm. What multiplies a bf16 operand that
an operator stored is given that operand, so that only its own roundings count."""
import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"

# rows, inputs, outputs
CASES = [(1, 1, 1), (1, 64, 8), (1, 4096, 1000), (2, 4104, 130), (3, 37, 501), (4, 256, 4096), (7, 333, 65), (15, 1024, 96), (16, 128, 264), (17, 72, 40),
         (31, 2048, 136), (33, 512, 33), (64, 1000, 250), (65, 64, 64), (100, 8, 300), (127, 129, 131), (128, 4096, 256), (128, 9216, 512), (200, 264, 776), (256, 256, 256),
         (257, 320, 520), (500, 1, 17), (777, 501, 333), (1000, 96, 96), (1024, 640, 512), (3000, 192, 96), (5000, 24, 12), (300, 6000, 8), (2048, 1032, 1288)]
IDS = ["x".join(map(str, c)) for c in CASES]
ACTS = ["none", "silu", "gelu", "gelu_tanh", "relu"]


def _td(dtype):
    return torch.float32 if dtype == "f32" else torch.bfloat16


def _inputs(case, dtype, seed=0):
    N, C, K = case
    g = torch.Generator().manual_seed(seed + N * 7 + C * 3 + K)
    rnd = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    t = {"x": rnd(N, C), "w": rnd(K, C) * C ** -0.5, "b": rnd(K), "r": rnd(N, K), "dy": rnd(N, K), "pre_x": rnd(N, C), "old_dx": rnd(N, C), "old_dw": rnd(K, C),
         "old_db": rnd(K)}
    return {k: v.to(_td(dtype)).to(DEV) for k, v in t.items()}


def _ws(pa, which, case, dtype):
    code = pa.PURINE_F32 if dtype == "f32" else pa.PURINE_BF16
    n = pa.purine_act_bwd_workspace_bytes(case[0], case[2]) if which == "act" else pa.purine_linear_workspace_bytes(which, *case, code)
    return torch.full((max(256, n),), 255, dtype=torch.uint8, device=DEV)


def _near(got, want, products, rounded, scale, what):
    tol = 2e-8 * products ** 0.5 + 1e-6 + (2 ** -8.5 if rounded else 0.0)
    got = got.double()
    assert bool(torch.isfinite(got).all()), what
    err = float((got - want).norm())
    assert err <= tol * float(scale), (what, err / float(scale), tol)


def _nan(*s, dt):
    return torch.full(s, float("nan"), dtype=dt, device=DEV)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_forward(case, dtype):
    import paper_1412_6249_amd as pa
    N, C, K = case
    t, td = _inputs(case, dtype), _td(dtype)
    d = {k: v.double() for k, v in t.items()}
    act = ACTS[(N + C + K) % 5]
    prod = d["x"] @ d["w"].t()
    for bias, res, keep in ((True, True, True), (False, False, False), (True, False, False)):
        y, pre = _nan(N, K, dt=td), _nan(N, K, dt=td) if keep else None
        pa.purine_linear_fwd(t["x"], t["w"], t["b"] if bias else None, t["r"] if res else None, y, pre, pa.ACTIVATIONS[act], ws=_ws(pa, 0, case, dtype))
        z = prod + (d["b"] if bias else 0.0)
        want = ref.act(z, act) + (d["r"] if res else 0.0)
        scale = prod.norm() + (d["b"].norm() * N ** 0.5 if bias else 0.0) + (d["r"].norm() if res else 0.0)
        _near(y, want, C, dtype == "bf16", scale, "y")
        if keep:
            _near(pre, z, C, dtype == "bf16", scale, "pre")
            again = t["r"].clone()                         # over the residual
            pa.purine_linear_fwd(t["x"], t["w"], t["b"], again, again, None, pa.ACTIVATIONS[act], ws=_ws(pa, 0, case, dtype))
            assert torch.equal(again, y)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=IDS)
def test_gradients(case, dtype):
    import paper_1412_6249_amd as pa
    N, C, K = case
    t, td = _inputs(case, dtype), _td(dtype)
    d = {k: v.double() for k, v in t.items()}
    act = ACTS[(N + C + K + 1) % 5]
    rounded = dtype == "bf16"
    prod = d["dy"] @ d["w"]
    for below, beta in ((False, 0.0), (True, 0.0), (True, 1.0), (False, 1.0)):
        dx = t["old_dx"].clone() if beta else _nan(N, C, dt=td)
        pa.purine_linear_bwd_data(t["dy"], t["w"], t["pre_x"] if below else None, dx, pa.ACTIVATIONS[act if below else "none"], beta, ws=_ws(pa, 1, case, dtype))
        want = prod * (ref.slope(d["pre_x"], act) if below else 1.0) + (d["old_dx"] if beta else 0.0)
        _near(dx, want, K, rounded, prod.norm() * 1.2 + beta * d["old_dx"].norm(), "dx")
    prod, sums = d["dy"].t().contiguous() @ d["x"], d["dy"].sum(0)
    for out, beta in ((torch.float32, 0.0), (td, 1.0), (td, 0.0)):
        dw, db = (t["old_dw"].to(out), t["old_db"].to(out)) if beta else (_nan(K, C, dt=out), _nan(K, dt=out))
        pa.purine_linear_bwd_weight(t["x"], t["dy"], dw, db, beta, ws=_ws(pa, 2, case, dtype))
        _near(dw, prod + beta * d["old_dw"], N, out == torch.bfloat16, prod.norm() + beta * d["old_dw"].norm(), "dw")
        _near(db, sums + beta * d["old_db"], N, out == torch.bfloat16, (N * K) ** 0.5 + beta * d["old_db"].norm(), "db")
        again = t["old_dw"].to(out) if beta else _nan(K, C, dt=out)
        pa.purine_linear_bwd_weight(t["x"], t["dy"], again, None, beta, ws=_ws(pa, 2, case, dtype))
        assert torch.equal(again, dw)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [c for c in CASES if c[0] * c[2] < 300000], ids=lambda c: "x".join(map(str, c)))
def test_gradient_of_an_activation(case, dtype):
    import paper_1412_6249_amd as pa
    N, C, K = case
    t, td = _inputs(case, dtype), _td(dtype)
    for act in ACTS:
        g, db = _nan(N, K, dt=td), _nan(K, dt=torch.float32)
        pa.purine_act_bwd(t["r"], t["dy"], g, db, pa.ACTIVATIONS[act], ws=_ws(pa, "act", case, dtype))
        want = t["dy"].double() * ref.slope(t["r"].double(), act)
        _near(g, want, 1, dtype == "bf16", t["dy"].double().norm(), act)
        _near(db, want.sum(0), N, False, (N * K) ** 0.5, act)
        over = t["dy"].clone()
        pa.purine_act_bwd(t["r"], over, over, None, pa.ACTIVATIONS[act])
        assert torch.equal(over, g)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [(1, 512, 96), (40, 72, 136), (300, 264, 520), (150, 33, 27)], ids=lambda c: "x".join(map(str, c)))
def test_rows_apart_on_a_stream(case, dtype):
    """Every matrix is columns of a wider one; what lies beside them stays."""
    import paper_1412_6249_amd as pa
    N, C, K = case
    t, td = _inputs(case, dtype), _td(dtype)

    def wide(m):
        rows, cols = m.shape
        big = torch.full((rows, (cols + 15) // 8 * 8 + 16), 3.0, dtype=td, device=DEV)
        big[:, 8:8 + cols] = m
        return big, big[:, 8:8 + cols]

    bx, x = wide(t["x"])
    bw, w = wide(t["w"])
    br, r = wide(t["r"])
    by, y = wide(torch.zeros(N, K, dtype=td, device=DEV))
    bp, pre = wide(torch.zeros(N, K, dtype=td, device=DEV))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    pa.purine_linear_fwd(x, w, t["b"], r, y, pre, pa.PURINE_ACT_SILU, ws=_ws(pa, 0, case, dtype), stream=side)
    side.synchronize()
    y2, pre2 = _nan(N, K, dt=td), _nan(N, K, dt=td)
    pa.purine_linear_fwd(t["x"], t["w"], t["b"], t["r"], y2, pre2, pa.PURINE_ACT_SILU, ws=_ws(pa, 0, case, dtype))
    assert torch.equal(y, y2) and torch.equal(pre, pre2)
    for big, inner in ((by, K), (bp, K)):
        assert bool((big[:, :8] == 3.0).all()) and bool((big[:, 8 + inner:] == 3.0).all())
    bd, dx = wide(torch.zeros(N, C, dtype=td, device=DEV))
    bg, dw = wide(torch.zeros(K, C, dtype=td, device=DEV))
    bdy, dy = wide(t["dy"])
    _, px = wide(t["pre_x"])
    pa.purine_linear_bwd_data(dy, w, px, dx, pa.PURINE_ACT_GELU, ws=_ws(pa, 1, case, dtype))
    pa.purine_linear_bwd_weight(x, dy, dw, None, ws=_ws(pa, 2, case, dtype))
    dx2, dw2 = _nan(N, C, dt=td), _nan(K, C, dt=td)
    pa.purine_linear_bwd_data(t["dy"], t["w"], t["pre_x"], dx2, pa.PURINE_ACT_GELU, ws=_ws(pa, 1, case, dtype))
    pa.purine_linear_bwd_weight(t["x"], t["dy"], dw2, None, ws=_ws(pa, 2, case, dtype))
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    for big, inner in ((bd, C), (bg, C)):
        assert bool((big[:, :8] == 3.0).all()) and bool((big[:, 8 + inner:] == 3.0).all())
    g = dy                                                 # in place in the wide buffer
    pa.purine_act_bwd(pre, dy, g, None, pa.PURINE_ACT_SILU)
    assert bool((bdy[:, :8] == 3.0).all()) and bool((bdy[:, 8 + K:] == 3.0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("case", [(1, 256, 64), (24, 100, 48), (260, 320, 264)], ids=lambda c: "x".join(map(str, c)))
def test_infinities_and_nan(case, dtype):
    """A row of x with one infinity or NaN makes its outputs what plain sums make them, and no others."""
    import paper_1412_6249_amd as pa
    N, C, K = case
    t, td = _inputs(case, dtype), _td(dtype)
    for bad in (float("inf"), float("nan")):
        x = t["x"].clone()
        x[N - 1, C // 2] = bad
        y = _nan(N, K, dt=td)
        pa.purine_linear_fwd(x, t["w"], t["b"], None, y, None, ws=_ws(pa, 0, case, dtype))
        want = x[N - 1].double() @ t["w"].double().t() + t["b"].double()
        got = y[N - 1].double()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~torch.isnan(got)], want[~torch.isnan(want)])
        clean = _nan(N, K, dt=td)
        pa.purine_linear_fwd(t["x"], t["w"], t["b"], None, clean, None, ws=_ws(pa, 0, case, dtype))
        assert torch.equal(y[:N - 1], clean[:N - 1])


def test_fp32_keeps_its_bits():
    """Operands of any size from 2^-100: an orthogonal choice of w copies x exactly."""
    import paper_1412_6249_amd as pa
    g = torch.Generator().manual_seed(2)
    for N in (1, 20, 150):
        C = 64
        x = (torch.randn(N, C, generator=g) * torch.exp2(torch.randint(-90, 90, (N, C), generator=g).float())).to(DEV)
        w = torch.eye(C, device=DEV)
        y = _nan(N, C, dt=torch.float32)
        pa.purine_linear_fwd(x, w, None, None, y, ws=_ws(pa, 0, (N, C, C), "f32"))
        assert torch.equal(y, x)


def test_gradient_against_differences():
    """fp32 gradients along a direction, against central differences of the 64-bit loss (as for the normalization)."""
    import paper_1412_6249_amd as pa
    case = (37, 50, 29)
    N, C, K = case
    for act in ("none", "silu", "gelu", "gelu_tanh"):
        t = _inputs(case, "f32", seed=4)
        y, pre, g, dx, dw, db = (_nan(*s, dt=torch.float32) for s in ((N, K), (N, K), (N, K), (N, C), (K, C), (K,)))
        a = pa.ACTIVATIONS[act]
        pa.purine_linear_fwd(t["x"], t["w"], t["b"], t["r"], y, pre, a, ws=_ws(pa, 0, case, "f32"))
        pa.purine_act_bwd(pre, t["dy"], g, db, a, ws=_ws(pa, "act", case, "f32"))
        pa.purine_linear_bwd_data(g, t["w"], None, dx, ws=_ws(pa, 1, case, "f32"))
        pa.purine_linear_bwd_weight(t["x"], g, dw, None, ws=_ws(pa, 2, case, "f32"))
        d = {k: v.double() for k, v in t.items()}
        loss = lambda x, w, b: ((ref.act(x @ w.t() + b, act) + d["r"]) * d["dy"]).sum()  # noqa: E731
        gen = torch.Generator().manual_seed(11)
        for which, grad in (("x", dx), ("w", dw), ("b", db)):
            u = torch.randn(d[which].shape, generator=gen, dtype=torch.float64).to(DEV)
            at = lambda k: loss(*[d[n] + (k * u if n == which else 0) for n in ("x", "w", "b")])  # noqa: E731
            num = float(at(1e-4) - at(-1e-4)) / 2e-4
            assert abs(float((grad.double() * u).sum()) - num) <= 1e-5 * float(grad.double().norm() * u.norm()), (act, which)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_offsets_past_32_bits(dtype):
    """A matrix of 2.2 GB (4.3 GB): its last rows, and both gradients of it."""
    import paper_1412_6249_amd as pa
    N, C, K = 270001, 4000, 16
    td = _td(dtype)
    x = torch.empty(N, C, dtype=td, device=DEV)
    g = torch.Generator(device=DEV).manual_seed(1)
    for i in range(0, N, 30000):
        x[i:i + 30000] = torch.randn(min(30000, N - i), C, generator=g, device=DEV)
    w = (torch.randn(K, C, generator=g, device=DEV) * C ** -0.5).to(td)
    y = _nan(N, K, dt=td)
    pa.purine_linear_fwd(x, w, None, None, y, ws=_ws(pa, 0, (N, C, K), dtype))
    want = x[-700:].double() @ w.double().t()
    _near(y[-700:], want, C, dtype == "bf16", want.norm(), "y")
    dy = torch.zeros(N, K, dtype=td, device=DEV)
    dy[-3:] = torch.randn(3, K, generator=g, device=DEV)
    dw = _nan(K, C, dt=torch.float32)
    pa.purine_linear_bwd_weight(x, dy, dw, None, ws=_ws(pa, 2, (N, C, K), dtype))
    want = dy[-3:].double().t().contiguous() @ x[-3:].double()
    _near(dw, want, 3, False, want.norm(), "dw")
    pa.purine_linear_bwd_data(dy, w, None, x, ws=_ws(pa, 1, (N, C, K), dtype))
    want = dy[-3:].double() @ w.double()
    _near(x[-3:], want, K, dtype == "bf16", want.norm(), "dx")
    assert float(x[:-3].abs().max()) == 0.0


def test_recorded_calls_replay():
    """A forward and backward pass in a HIP graph, replayed with other work in between, gives the eager bits."""
    import paper_1412_6249_amd as pa
    case = (200, 512, 264)
    N, C, K = case
    t, td = _inputs(case, "bf16"), torch.bfloat16
    y, pre, g, dx, dw, db = (_nan(*s, dt=td) for s in ((N, K), (N, K), (N, K), (N, C), (K, C), (K,)))
    ws = [_ws(pa, w, case, "bf16") for w in (0, 1, 2, "act")]

    def step():
        pa.purine_linear_fwd(t["x"], t["w"], t["b"], t["r"], y, pre, pa.PURINE_ACT_GELU, ws=ws[0])
        pa.purine_act_bwd(pre, t["dy"], g, db, pa.PURINE_ACT_GELU, ws=ws[3])
        pa.purine_linear_bwd_data(g, t["w"], None, dx, ws=ws[1])
        pa.purine_linear_bwd_weight(t["x"], g, dw, None, ws=ws[2])

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        t["x"].copy_(_inputs(case, "bf16", seed=k)["x"])
        step()
        torch.cuda.synchronize()
        eager = [v.clone() for v in (y, dx, dw, db)]
        for v in (y, pre, g, dx, dw, db):
            v.fill_(0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, (y, dx, dw, db)))
