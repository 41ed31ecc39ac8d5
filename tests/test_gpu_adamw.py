"""The AdamW step against its definition in 64 bits: fp32 states, 8-bit states (decoded, stepped and encoded in plain torch operations of the
same formulas), tensors of one element, of a block, of a workgroup and one beside them, more tensors than a launch holds, every type.

Bounds. fp32: about ten roundings of 2^-24 on w, three on the states: 16 eps. bf16 weights: one rounding, 2^-8 of the value. 8-bit codes: m
is known to 4 eps of the terms that it is made of, sqrt(v) to 4 eps of itself, so that a code may differ, by one place, only where the value
in steps of its codes plus the threshold is that near to a whole number (and 32 eps, the sum's own rounding). With bf16 gradients such ties are
common: 0.9 and 0.07 of small binary numbers add up to whole halves."""
import math

import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
DEV, EPS, BLOCK = "cuda:0", 2.0 ** -24, 256
SIZES = [1, 7, 8, 255, 256, 257, 2047, 2048, 2049, 5000, 100003]
H = {"lr": 3e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.05, "grad_scale": 0.7}


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def _tensors(sizes, w16, d16, seed=0):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda n: torch.randn(n, generator=g)  # noqa: E731
    td = lambda b: torch.bfloat16 if b else torch.float32  # noqa: E731
    w = [rnd(n).to(td(w16)).to(DEV) for n in sizes]
    dw = [(1e-3 * rnd(n)).to(td(d16)).to(DEV) for n in sizes]
    m = [(5e-4 * rnd(n)).to(DEV) for n in sizes]
    v = [(1e-6 * (0.2 + torch.rand(n, generator=g))).to(DEV) for n in sizes]
    return w, dw, m, v


@pytest.mark.parametrize("w16", [False, True], ids=["w32", "w16"])
@pytest.mark.parametrize("d16", [False, True], ids=["d32", "d16"])
@pytest.mark.parametrize("step", [1, 7, 20000])
def test_fp32_states(w16, d16, step):
    import paper_1412_6249_amd as pa
    sizes = SIZES * 4 + [3] * 3                             # 47 tensors: two launches
    w, dw, m, v = _tensors(sizes, w16, d16)
    copy = [torch.zeros(n, dtype=torch.bfloat16, device=DEV) if i % 2 else None for i, n in enumerate(sizes)]
    before = [[t.double().clone() for t in l] for l in (w, dw, m, v)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    pa.purine_adamw_step(pa.adamw_desc(step=step, **H), pa.adamw_params(w, dw, m, v, copy=copy), stream=side)
    side.synchronize()
    for i in range(len(sizes)):
        ww, wm, wv = ref.adamw(*(l[i] for l in before), step, **H)
        move = (ww - before[0][i]).abs() + before[0][i].abs()
        assert bool(((m[i].double() - wm).abs() <= 4 * EPS * (wm.abs() + before[1][i].abs())).all()), i
        assert bool(((v[i].double() - wv).abs() <= 4 * EPS * wv).all()), i
        assert bool(((w[i].double() - ww).abs() <= (2 ** -8 if w16 else 16 * EPS) * move).all()), i
        if copy[i] is not None:
            exact = w[i] if w16 else w[i].to(torch.bfloat16)
            assert torch.equal(copy[i], exact), i


# ---- 8-bit states: the formulas once more
def _mix(h):
    h = ((h ^ (h >> 16)) * 0x45D9F3B3) & 0xffffffff
    h = ((h ^ (h >> 15)) * 0x2C1B3C6D) & 0xffffffff
    return h ^ (h >> 16)


def _thresholds(n, tensor, seed, step):
    salt = _mix((_mix((seed + 0x9E3779B9 * step) & 0xffffffff) + 0x85EBCA6B * (tensor + 1)) & 0xffffffff)
    e = torch.arange(n, dtype=torch.int64)
    h = _mix((salt + (e >> 1)) & 0xffffffff) >> (16 * (e & 1))
    return [((b & 255).double() + 0.5) / 256 for b in (h, h >> 8)]


def _encode(x, d, floor, unsure=0.0):
    """Codes' values (in scales) and scales, in 64 bits on the CPU."""
    n = x.numel()
    pad = torch.zeros(_blocks(n) * BLOCK, dtype=torch.float64)
    pad[:n] = x.cpu()
    a = torch.where(torch.isfinite(pad), pad.abs(), torch.zeros_like(pad)).reshape(-1, BLOCK)
    top = a.amax(1)
    scale = torch.tensor([0.0 if t == 0 else 2.0 ** max(-100, math.ceil(math.log2(t / 448) - 1e-12)) for t in top.tolist()], dtype=torch.float64)
    assert bool((top <= 448 * scale).all())
    z = torch.where(scale[:, None] > 0, a / scale.clamp(min=2.0 ** -120)[:, None], torch.zeros_like(a)).reshape(-1)[:n]
    step = 2.0 ** (torch.floor(torch.log2(z.clamp(min=2.0 ** -30))).clamp(min=-6) - 3)
    place = z / step + d
    doubt = torch.as_tensor(unsure, dtype=torch.float64).cpu() / (scale.clamp(min=2.0 ** -120).repeat_interleave(BLOCK)[:n] * step)
    near = (place - place.round()).abs() <= doubt + 32 * EPS
    q = torch.floor(place) * step
    if floor:
        q = torch.where(z > 0, q.clamp(min=2.0 ** -9), q)
    q = torch.copysign(q, x.cpu().double())
    return torch.where(torch.isfinite(x.cpu()), q, torch.full_like(q, float("nan"))), scale, near


def _coded(sizes, seed=0, dither=None):
    w, dw, m, v = _tensors(sizes, False, False, seed)
    out = {"m": [], "m_scale": [], "v": [], "v_scale": []}
    for mm, vv in zip(m, v):
        for key, x, floor in (("m", mm.double(), False), ("v", vv.double().sqrt(), True)):
            q, s, _ = _encode(x, 0.5, floor)
            out[key].append(q.to(torch.float32).to(torch.float8_e4m3fn).to(DEV))
            out[key + "_scale"].append(s.float().to(DEV))
    return w, dw, out


def _values(code, scale):
    n = code.numel()
    return code.float().double() * scale.double().repeat_interleave(BLOCK)[:n]


@pytest.mark.parametrize("dither", [False, True], ids=["nearest", "dither"])
@pytest.mark.parametrize("types", ["w32d32", "w32d16", "w16d16"])
def test_8_bit_states(types, dither):
    import paper_1412_6249_amd as pa
    sizes = SIZES * 4
    w, dw, s = _coded(sizes)
    if "d16" in types:
        dw = [t.to(torch.bfloat16) for t in dw]
    if "w16" in types:
        w = [t.to(torch.bfloat16) for t in w]
    copy = [torch.zeros(n, dtype=torch.bfloat16, device=DEV) for n in sizes]
    w0 = [t.double().clone() for t in w]
    m0 = [_values(c, k) for c, k in zip(s["m"], s["m_scale"])]
    u0 = [_values(c, k) for c, k in zip(s["v"], s["v_scale"])]
    step, seed = 12, 0xDEADBEEF
    pa.purine_adamw_step(pa.adamw_desc(step=step, seed=seed, dither=dither, **H),
                         pa.adamw_params(w, dw, s["m"], s["v"], s["m_scale"], s["v_scale"], copy))
    torch.cuda.synchronize()
    for i, n in enumerate(sizes):
        ww, wm, wv = ref.adamw(w0[i], dw[i].double(), m0[i], u0[i] ** 2, step, **H)
        assert bool(((w[i].double() - ww).abs() <= (2 ** -8 if "w16" in types else 16 * EPS) * ((ww - w0[i]).abs() + w0[i].abs())).all()), i
        assert torch.equal(copy[i], w[i].to(torch.bfloat16))
        dm, dv = _thresholds(n, i, seed, step) if dither else (0.5, 0.5)
        for key, x, d, floor, terms in (("m", wm, dm, False, wm.abs() + m0[i].abs()), ("v", wv.sqrt(), dv, True, wv.sqrt())):
            q, scale, near = _encode(x, d, floor, 4 * EPS * terms)
            assert torch.equal(s[key + "_scale"][i].cpu().double(), scale), (key, i)
            off = (s[key][i].float().cpu().double() - q).abs()
            assert bool((off <= 0.1251 * q.abs() + 2.0 ** -9).all())
            assert bool(near[off > 0].all()), (key, i)


def test_dither_is_right_on_average_and_nearest_stalls():
    """500 steps of a constant gradient that should bring v from 1e-6 to 0.25e-6 + ...: with dither the mean of v follows the 64-bit
    recursion to a few per cent (its scatter, a tenth to a fifth per element, over 65536 elements); to nearest it stays where it was."""
    import paper_1412_6249_amd as pa
    n = 65536
    got = {}
    for dither in (False, True):
        w, dw = torch.zeros(n, device=DEV), torch.full((n,), 2e-4, device=DEV)
        x = torch.full((n,), 1e-3, dtype=torch.float64)
        q, sc, _ = _encode(x, 0.5, True)
        m, ms = torch.zeros(n, device=DEV).to(torch.float8_e4m3fn), torch.zeros(_blocks(n), device=DEV)
        # blocks keep their scale: one large element each
        v, vs = q.float().to(torch.float8_e4m3fn).to(DEV), sc.float().to(DEV)
        p = pa.adamw_params([w], [dw], [m], [v], [ms], [vs])
        for t in range(1, 501):
            pa.purine_adamw_step(pa.adamw_desc(lr=0.0, weight_decay=0.0, step=t, seed=3, dither=dither), p)
        got[dither] = float((_values(v, vs) ** 2).mean())
    start = float((q * sc.repeat_interleave(BLOCK)).pow(2).mean())
    want = start * 0.999 ** 500 + (1 - 0.999 ** 500) * 4e-8
    assert abs(got[True] / want - 1) < 0.05, (got, want)
    assert got[False] > 0.95 * start, (got, start)


def test_zeros_and_values_that_are_not_finite():
    import paper_1412_6249_amd as pa
    n = 1000
    w, dw = torch.ones(n, device=DEV), torch.zeros(n, device=DEV)
    new8 = lambda: torch.zeros(n, device=DEV).to(torch.float8_e4m3fn)  # noqa: E731
    m, v, ms, vs = new8(), new8(), torch.zeros(4, device=DEV), torch.zeros(4, device=DEV)
    p = pa.adamw_params([w], [dw], [m], [v], [ms], [vs])
    pa.purine_adamw_step(pa.adamw_desc(lr=0.1, weight_decay=0.0, dither=True), p)
    assert bool((w == 1).all()) and float(ms.abs().max()) == 0.0 and float(vs.abs().max()) == 0.0 and float(v.float().abs().max()) == 0.0
    dw[300], dw[301], dw[302] = float("nan"), float("inf"), 1e-3
    pa.purine_adamw_step(pa.adamw_desc(lr=0.1, weight_decay=0.0, step=2, dither=True), p)
    bad = ~torch.isfinite(w)
    assert sorted(bad.nonzero().flatten().tolist()) == [300, 301]
    assert sorted(torch.isnan(v.float()).nonzero().flatten().tolist()) == [300, 301]
    assert float(vs[1]) > 0 and float(v.float()[302]) > 0 and float(vs[[0, 2, 3]].abs().max()) == 0.0
    # the smallest second moments are not lost beside large ones
    dw.zero_()
    dw[0], dw[1:] = 1.0, 1e-9
    w2, m2, v2 = torch.ones(n, device=DEV), new8(), new8()
    pa.purine_adamw_step(pa.adamw_desc(lr=0.1, weight_decay=0.0), pa.adamw_params([w2], [dw], [m2], [v2], [torch.zeros(4, device=DEV)], [torch.zeros(4, device=DEV)]))
    assert float(v2.float().min()) > 0


@pytest.mark.parametrize("coded", [False, True], ids=["f32", "8bit"])
def test_counted_steps_replay(coded):
    """With `done` the call counts its steps: recorded once, replayed, it gives the bits of as many eager calls, which agree with
    calls that are told their step."""
    import paper_1412_6249_amd as pa
    sizes = [300, 5000, 17]

    def fresh():
        if coded:
            w, dw, s = _coded(sizes)
            return w, s["m"] + s["v"], pa.adamw_params(w, dw, s["m"], s["v"], s["m_scale"], s["v_scale"])
        w, dw, m, v = _tensors(sizes, False, False)
        return w, m + v, pa.adamw_params(w, dw, m, v)

    told, eager, rec = fresh(), fresh(), fresh()
    desc = pa.adamw_desc(seed=5, dither=True, **H)
    done_e, done_r = (torch.zeros(1, dtype=torch.int32, device=DEV) for _ in range(2))
    with torch.cuda.stream(torch.cuda.Stream()):
        pa.purine_adamw_step(desc, eager[2], done=done_e)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        pa.purine_adamw_step(desc, rec[2], done=done_r)
    for k in range(1, 5):
        graph.replay()
        torch.cuda.synchronize()
        if k > 1:
            pa.purine_adamw_step(desc, eager[2], done=done_e)
        pa.purine_adamw_step(pa.adamw_desc(step=k, seed=5, dither=True, **H), told[2])
        torch.cuda.synchronize()
        assert int(done_r) == int(done_e) == k
        for a, b, c in zip(rec[0], eager[0], told[0]):
            assert torch.equal(a, b) and float((b - c).abs().max()) <= 1e-6
        for a, b, c in zip(rec[1], eager[1], told[1]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)) and torch.equal(b.view(torch.uint8), c.view(torch.uint8))
