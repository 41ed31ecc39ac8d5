"""What the operators of a normalised residual block and its optimizer are measured on: group normalization with an
activation on channels-last tensors, the matrix product with bias, activation and residual in its epilogue, their
gradients, and the AdamW step over many tensors.

`listed()` holds the cases, `draw()` more of the same ranges. `run()` makes one pass: with `own` true through this
library's entry points, else in elementary torch operations in fp32, rounded once at the end.

* "norm":   y = act(group_norm(x)); with `train` also mean, rstd and the gradients of x, scale and shift;
* "linear": y = act(x w^T + b) + r; with `train` also the gradients of x, w and b;
* "adamw":  one step over all parameter tensors of a network, states in fp32 or in 8 bits (e4m3 with a power of two per
  256 elements: m as it is, v as its square root; both rounded by a dither that the seed, the step and the element give).

The optimizer's tensors lie in flat buffers, each at a multiple of 256 elements, as a training program keeps them; the
returned outputs are those buffers.
"""
import math
import zlib

import numpy as np
import torch

own = False
DEV = "cuda:0"
EPS = 1e-5                   # of the normalization
BLOCK = 256                  # elements that share a scale of the 8-bit states
MAX_BYTES, MAX_FLOPS = 2.0e9, 1.7e12

# parameter tensors (elements) of the networks of this repository: single layers, NIN's block, the inception module,
# AlexNet's layers with its fully-connected ones
CONV = [8 * 3 * 9, 8]
NIN = [96 * 3 * 121, 96, 96 * 96, 96, 96 * 96, 96]
INCEPTION = [64 * 192, 64, 96 * 192, 96, 128 * 96 * 9, 128, 16 * 192, 16, 32 * 16 * 25, 32, 32 * 192, 32]
ALEXNET = [96 * 363, 96, 256 * 96 * 25, 256, 384 * 256 * 9, 384, 384 * 384 * 9, 384, 256 * 384 * 9, 256,
           4096 * 9216, 4096, 4096 * 4096, 4096, 1000 * 4096, 1000]
NETS = {"conv": CONV, "nin": NIN, "inception": INCEPTION, "alexnet": ALEXNET}


def _norm(name, dtype, N, S, C, G, act, train):
    return {"name": name, "kind": "norm", "dtype": dtype, "N": N, "S": S, "C": C, "G": G, "act": act, "train": train}


def _linear(name, dtype, N, C, K, act, residual, train):
    return {"name": name, "kind": "linear", "dtype": dtype, "N": N, "C": C, "K": K, "act": act, "residual": residual,
            "train": train}


def _adamw(name, net, grads, states, step):
    return {"name": name, "kind": "adamw", "net": net, "times": 1, "grads": grads, "states": states, "step": step}


def listed():
    return [
        # one image's small feature map in a decoder: latency, few workgroups
        _norm("norm_small_f32", "f32", 1, 16 * 16, 64, 8, "silu", False),
        # training step behind the inception module's maps: 6 channels per group, planes that fit on the chip
        _norm("norm_28_bf16_train", "bf16", 128, 28 * 28, 192, 32, "silu", True),
        # the stem's maps: planes far larger than a compute unit's memory
        _norm("norm_112_bf16_train", "bf16", 64, 112 * 112, 64, 32, "gelu_tanh", True),
        # nothing is a multiple of anything: 10 channels per group, odd planes, fp32
        _norm("norm_odd_f32_train", "f32", 29, 29 * 31, 150, 15, "silu", True),
        # one token of a serving program: bound by the weight matrix
        _linear("linear_token_bf16", "bf16", 1, 4096, 4096, "silu", True, False),
        # fc6 of AlexNet at its batch, inference
        _linear("linear_fc6_bf16", "bf16", 128, 9216, 4096, "relu", False, False),
        # a 1x1 layer of the inception module as channels-last pixels, training: close to the memory roof
        _linear("linear_pixels_bf16_train", "bf16", 128 * 28 * 28, 192, 96, "gelu_tanh", False, True),
        # a wide layer at a large batch, training: bound by the matrix cores
        _linear("linear_wide_bf16_train", "bf16", 8192, 4096, 8192, "gelu", True, True),
        # odd everywhere, fp32, training
        _linear("linear_odd_f32_train", "f32", 777, 501, 333, "silu", True, True),
        # a few small tensors: launches and the host's part
        _adamw("adamw_inception_f32", "inception", "f32", "f32", 3),
        # AlexNet with fp32 states, and with 8-bit states, bf16 gradients and a bf16 copy of the weights
        _adamw("adamw_alexnet_f32", "alexnet", "f32", "f32", 1000),
        _adamw("adamw_alexnet_8bit", "alexnet", "bf16", "8bit", 1000),
    ]


# ------------------------------------------------------------------------------------------ drawn
def _spread(rng, lo, hi):
    """An integer of [lo, hi], spread over its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        kind = rng.choice(["norm", "norm", "linear", "linear", "linear", "adamw"])
        if kind == "norm":
            per, train = _spread(rng, 1, 48), rng.random() < 0.6
            G = _spread(rng, 1, 64)
            c = {"kind": "norm", "dtype": rng.choice(["f32", "bf16"]), "N": _spread(rng, 1, 128),
                 "S": _spread(rng, 1, 112 * 112), "C": G * per, "G": G,
                 "act": rng.choice(["none", "silu", "gelu", "gelu_tanh"]), "train": train}
            if per * c["S"] < 16:            # (statistics over a handful of values)
                continue
        elif kind == "linear":
            train = rng.random() < 0.5
            c = {"kind": "linear", "dtype": rng.choice(["f32", "bf16", "bf16"]), "N": _spread(rng, 1, 8192) if rng.random() < 0.8 else _spread(rng, 4096, 102400),
                 "C": _spread(rng, 16, 9216), "K": _spread(rng, 10, 8192),
                 "act": rng.choice(["none", "silu", "gelu", "gelu_tanh"]), "residual": rng.random() < 0.5, "train": train}
            if rng.random() < 0.6:           # layer widths are mostly multiples of 8
                c["C"], c["K"] = max(16, c["C"] // 8 * 8), max(16, c["K"] // 8 * 8)
            if 3072 in (c["N"], c["C"], c["K"]) or (c["dtype"] == "f32" and work(c)["flops"] > MAX_FLOPS / 4):
                continue
        else:
            c = {"kind": "adamw", "net": rng.choice(["conv", "nin", "inception", "alexnet"]), "times": 1,
                 "grads": rng.choice(["f32", "bf16"]), "states": rng.choice(["f32", "8bit"]), "step": _spread(rng, 1, 100000)}
            if c["net"] != "alexnet":
                c["times"] = _spread(rng, 1, 8)
        w = work(c)
        if w["flops"] <= MAX_FLOPS and w["bytes"] <= MAX_BYTES:
            return c


# ----------------------------------------------------------------------------------------- inputs
def _gen(seed, name):
    g = torch.Generator(device=DEV)
    g.manual_seed((int(seed) * 1000003 + zlib.crc32(name.encode())) % (1 << 62))
    return g


def _td(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def _randn(seed, name, *shape):
    return torch.randn(shape, generator=_gen(seed, name), device=DEV)


def _norm_inputs(case, seed):
    N, S, C, td = case["N"], case["S"], case["C"], _td(case["dtype"])
    # activations: every channel with a mean and a spread of its own
    x = _randn(seed, "x", N, S, C) * (0.5 + torch.rand(C, generator=_gen(seed, "xs"), device=DEV)) + _randn(seed, "xm", C)
    t = {"x": x.to(td), "scale": 1.0 + 0.2 * _randn(seed, "scale", C), "shift": 0.2 * _randn(seed, "shift", C)}
    if case["train"]:
        t["dy"] = (_randn(seed, "dy", N, S, C) * 1e-3).to(td)
    return t


def _linear_inputs(case, seed):
    N, C, K, td = case["N"], case["C"], case["K"], _td(case["dtype"])
    t = {"x": _randn(seed, "x", N, C).to(td), "w": (_randn(seed, "w", K, C) * C ** -0.5).to(td),
         "b": (_randn(seed, "b", K) * 0.1).to(td)}
    if case["residual"]:
        t["r"] = _randn(seed, "r", N, K).to(td)
    if case["train"]:
        t["dy"] = (_randn(seed, "dy", N, K) * 1e-3).to(td)
    return t


def _sizes(case):
    return NETS[case["net"]] * case["times"]


def _starts(case):
    """First elements of the tensors in the flat buffers, and the buffers' length."""
    at, total = [], 0
    for n in _sizes(case):
        at.append(total)
        total += (n + BLOCK - 1) // BLOCK * BLOCK
    return at, total


def _hyper(case):
    # the warm-up's end: step sizes, decay and clipping of ordinary training
    return {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01, "grad_scale": 0.5}


def _adamw_inputs(case, seed):
    at, total = _starts(case)
    live = torch.zeros(total, device=DEV)
    for a, n in zip(at, _sizes(case)):
        live[a:a + n] = 1.0
    flat = lambda name: _randn(seed, name, total) * live  # noqa: E731
    size = 1e-3 * torch.exp(0.7 * _randn(seed, "size", total // BLOCK)).repeat_interleave(BLOCK)
    w, dw = flat("w") * 0.05, flat("dw") * size
    m = 0.3 * flat("m") * size
    v = (size * live * (0.5 + torch.rand(total, generator=_gen(seed, "v"), device=DEV))).square()
    t = {"w": w, "dw": dw.to(_td(case["grads"]))}
    if case["states"] == "f32":
        t.update(m=m, v=v)
    else:
        (t["m"], t["m_scale"]), (t["v"], t["v_scale"]) = _encode(m, None), _encode(v.sqrt(), None)
        t["copy"] = w.to(torch.bfloat16)
    return t


def prepare(case, seed):
    if case["kind"] == "adamw":
        s = _adamw_inputs(case, seed)
        s.update(case=case, step=case["step"], seed=int(seed) & 0x7fffffff)
        if own:
            import paper_1412_6249_amd as pa
            at, n = _starts(case)[0], _sizes(case)
            part = lambda t: [t[a:a + k] for a, k in zip(at, n)]  # noqa: E731
            block = lambda t: [t[a // BLOCK:(a + k + BLOCK - 1) // BLOCK] for a, k in zip(at, n)]  # noqa: E731
            extra = {} if case["states"] == "f32" else {"m_scale": block(s["m_scale"]), "v_scale": block(s["v_scale"]), "copy": part(s["copy"])}
            s["params"] = pa.adamw_params(part(s["w"]), part(s["dw"]), part(s["m"]), part(s["v"]), **extra)
        return s
    norm = case["kind"] == "norm"
    s = (_norm_inputs if norm else _linear_inputs)(case, seed)
    s["case"] = case
    if own:                    # outputs and scratch that the program keeps
        import paper_1412_6249_amd as pa
        td, code = _td(case["dtype"]), pa.PURINE_BF16 if case["dtype"] == "bf16" else pa.PURINE_F32
        new = lambda *shape, dt=td: torch.empty(shape, dtype=dt, device=DEV)  # noqa: E731
        if norm:
            N, S, C, G = case["N"], case["S"], case["C"], case["G"]
            need = [pa.purine_group_norm_workspace_bytes(p, (N, S, C), G, code) for p in ((0, 1) if case["train"] else (0,))]
            s.update(y=new(N, S, C), mean=None, rstd=None)
            if case["train"]:
                f = torch.float32
                s.update(mean=new(N, G, dt=f), rstd=new(N, G, dt=f), dx=new(N, S, C), dscale=new(C, dt=f), dshift=new(C, dt=f))
        else:
            N, C, K = case["N"], case["C"], case["K"]
            need = [pa.purine_linear_workspace_bytes(p, N, C, K, code) for p in ((0, 1, 2) if case["train"] else (0,))]
            s.update(y=new(N, K), pre=None)
            if case["train"]:
                need.append(pa.purine_act_bwd_workspace_bytes(N, K))
                s.update(pre=new(N, K), g=new(N, K), dx=new(N, C), dw=new(K, C), db=new(K))
        s["ws"] = torch.empty(max(256, max(need)), dtype=torch.uint8, device=DEV)
    return s


# ------------------------------------------------------------------------------------- plain form
def _act(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def _norm_plain(s):
    case, f = s["case"], torch.float32
    N, S, C, G = case["N"], case["S"], case["C"], case["G"]
    x = s["x"].to(f).reshape(N, S, G, C // G)
    mean = x.sum((1, 3), keepdim=True) / (S * (C // G))
    xc = x - mean
    rstd = 1 / torch.sqrt((xc * xc).sum((1, 3), keepdim=True) / (S * (C // G)) + EPS)
    xhat = xc * rstd
    scale = s["scale"].reshape(1, 1, G, C // G)
    z = xhat * scale + s["shift"].reshape(1, 1, G, C // G)
    out = {"y": _act(z, case["act"]).reshape(N, S, C).to(s["x"].dtype)}
    if case["train"]:
        g = s["dy"].to(f).reshape(N, S, G, C // G) * _act_slope(z, case["act"])
        out.update(mean=mean.reshape(N, G), rstd=rstd.reshape(N, G), dshift=g.sum((0, 1)).reshape(C), dscale=(g * xhat).sum((0, 1)).reshape(C))
        g = g * scale
        n = S * (C // G)
        dx = rstd * (g - g.sum((1, 3), keepdim=True) / n - xhat * ((g * xhat).sum((1, 3), keepdim=True) / n))
        out["dx"] = dx.reshape(N, S, C).to(s["x"].dtype)
    return out


def _linear_plain(s):
    case, f, td = s["case"], torch.float32, s["x"].dtype
    x, w = s["x"].to(f), s["w"].to(f)
    pre = torch.matmul(x, w.t()) + s["b"].to(f)
    y = _act(pre, case["act"])
    if case["residual"]:
        y = y + s["r"].to(f)
    out = {"y": y.to(td)}
    if case["train"]:
        g = s["dy"].to(f) * _act_slope(pre, case["act"])
        out.update(dx=torch.matmul(g, w).to(td), dw=torch.matmul(g.t(), x).to(td), db=g.sum(0).to(td))
    return out


def _mix(h):
    """An integer mixer on 32-bit values held in int64."""
    h = ((h ^ (h >> 16)) * 0x45D9F3B3) & 0xffffffff
    h = ((h ^ (h >> 15)) * 0x2C1B3C6D) & 0xffffffff
    return h ^ (h >> 16)


def _mix_int(h):
    h = ((h ^ (h >> 16)) * 0x45D9F3B3) & 0xffffffff
    h = ((h ^ (h >> 15)) * 0x2C1B3C6D) & 0xffffffff
    return h ^ (h >> 16)


def _dither(case, seed, step):
    """Per element of the flat buffers the thresholds of m's and v's rounding: (byte + 0.5) / 256 of the mixer's output for
    the pair of elements, the tensor, the step and the seed."""
    at, total = _starts(case)
    base = _mix_int((seed + 0x9E3779B9 * (step & 0xffffffff)) & 0xffffffff)
    salts = torch.tensor([_mix_int((base + 0x85EBCA6B * (i + 1)) & 0xffffffff) for i in range(len(at))], device=DEV, dtype=torch.int64)
    starts = torch.tensor(at, device=DEV, dtype=torch.int64)
    i = torch.arange(total, device=DEV, dtype=torch.int64)
    t = torch.bucketize(i, starts, right=True) - 1
    e = i - starts[t]
    h = _mix((salts[t] + (e >> 1)) & 0xffffffff) >> (16 * (e & 1))
    return [((b & 255).to(torch.float32) + 0.5) / 256 for b in (h, h >> 8)]


def _decode(code, scale):
    return (code.to(torch.float32).reshape(-1, BLOCK) * scale.reshape(-1, 1)).reshape(-1)


def _pow2(e):
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _encode(x, dither, floor=False):
    """(e4m3 codes, scales): per block the smallest power of two (2^-100 at least) that brings its largest value to 448 or
    less; magnitudes between two codes go up where their place between them plus the dither (None: a half) reaches 1.
    `floor`: what is above zero stays above zero."""
    f = torch.float32
    a = x.abs().reshape(-1, BLOCK)
    most = a.amax(1, keepdim=True)
    frac, ex = torch.frexp(most)
    shift = (ex - 9 + (frac > 0.875).to(ex.dtype)).clamp(min=-100)
    scale = torch.where(most > 0, _pow2(shift), torch.zeros_like(most))
    z = torch.where(most > 0, a * _pow2(-shift), torch.zeros_like(a))
    step = _pow2((torch.frexp(z)[1] - 1).clamp(min=-6) - 3)
    d = 0.5 if dither is None else dither.to(f).reshape(-1, BLOCK)
    q = torch.floor(z / step + d) * step
    if floor:
        q = torch.where(a > 0, q.clamp(min=2.0 ** -9), q)
    q = torch.copysign(q, x.reshape(-1, BLOCK))
    return q.reshape(-1).to(torch.float8_e4m3fn), scale.reshape(-1)


def _adamw_plain(s):
    case, h, f = s["case"], _hyper(s["case"]), torch.float32
    b1, b2, t = h["beta1"], h["beta2"], s["step"]
    g = s["dw"].to(f) * h["grad_scale"]
    if case["states"] == "f32":
        m, v = s["m"], s["v"]
    else:
        m, v = _decode(s["m"], s["m_scale"]), _decode(s["v"], s["v_scale"]).square()
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * g * (1 - b2)
    s["w"] = s["w"] * (1 - h["lr"] * h["weight_decay"]) - (h["lr"] / (1 - b1 ** t)) * m / (torch.sqrt(v) * (1 / math.sqrt(1 - b2 ** t)) + h["eps"])
    out = {"w": s["w"]}
    if case["states"] == "f32":
        s["m"], s["v"] = m, v
    else:
        dm, dv = _dither(case, s["seed"], t)
        s["m"], s["m_scale"] = _encode(m, dm)
        s["v"], s["v_scale"] = _encode(torch.sqrt(v), dv, True)
        s["copy"] = s["w"].to(torch.bfloat16)
        out.update(copy=s["copy"], m_scale=s["m_scale"], v_scale=s["v_scale"])
    out.update(m=s["m"], v=s["v"])
    s["step"] = t + 1
    return out


# ------------------------------------------------------------------------------------------- run
def _norm_own(s):
    import paper_1412_6249_amd as pa
    case = s["case"]
    act, G = pa.ACTIVATIONS[case["act"]], case["G"]
    pa.purine_group_norm_fwd(s["x"], s["scale"], s["shift"], s["y"], s["mean"], s["rstd"], G, EPS, act, ws=s["ws"])
    if not case["train"]:
        return {"y": s["y"]}
    pa.purine_group_norm_bwd(s["x"], s["scale"], s["shift"], s["mean"], s["rstd"], s["dy"], s["dx"], s["dscale"], s["dshift"], G, act, ws=s["ws"])
    return {k: s[k] for k in ("y", "mean", "rstd", "dshift", "dscale", "dx")}


def _linear_own(s):
    import paper_1412_6249_amd as pa
    act = pa.ACTIVATIONS[s["case"]["act"]]
    pa.purine_linear_fwd(s["x"], s["w"], s["b"], s.get("r"), s["y"], s["pre"], act, ws=s["ws"])
    if not s["case"]["train"]:
        return {"y": s["y"]}
    pa.purine_act_bwd(s["pre"], s["dy"], s["g"], s["db"], act, ws=s["ws"])
    pa.purine_linear_bwd_data(s["g"], s["w"], None, s["dx"], ws=s["ws"])
    pa.purine_linear_bwd_weight(s["x"], s["g"], s["dw"], None, ws=s["ws"])
    return {k: s[k] for k in ("y", "dx", "dw", "db")}


def _adamw_own(s):
    import paper_1412_6249_amd as pa
    pa.purine_adamw_step(pa.adamw_desc(step=s["step"], seed=s["seed"], dither=True, **_hyper(s["case"])), s["params"])
    s["step"] += 1
    return {k: s[k] for k in (("w", "m", "v") if s["case"]["states"] == "f32" else ("w", "copy", "m_scale", "v_scale", "m", "v"))}


def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"norm": _norm_own, "linear": _linear_own, "adamw": _adamw_own}[kind](state)
    return {"norm": _norm_plain, "linear": _linear_plain, "adamw": _adamw_plain}[kind](state)


# ------------------------------------------------------------------------------------------ work
def work(case):
    if case["kind"] == "norm":
        n, e = case["N"] * case["S"] * case["C"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": n * e * (4 if case["train"] else 2) + case["C"] * (16 if case["train"] else 8), "flops": n * (30 if case["train"] else 10)}
    if case["kind"] == "linear":
        N, C, K, e = case["N"], case["C"], case["K"], 2 if case["dtype"] == "bf16" else 4
        rows = N * C + N * K * (2 if case["residual"] else 1)
        if case["train"]:                    # dy and dx besides, dw and db
            rows += N * C + N * K + C * K + K
        return {"bytes": e * (rows + C * K + K), "flops": 2 * N * C * K * (3 if case["train"] else 1)}
    n, g = sum(_sizes(case)), 2 if case["grads"] == "bf16" else 4
    # w and the states read and written, the gradient read, the bf16 copy written
    each = 8 + g + 16 if case["states"] == "f32" else 8 + g + 2 + 4 + 16 / BLOCK
    return {"bytes": n * each, "flops": n * 15}


# ----------------------------------------------------------------------------------------- exact
def _exact_norm(case, seed):
    t = {k: v.double() for k, v in _norm_inputs(case, seed).items()}
    N, S, C, G = case["N"], case["S"], case["C"], case["G"]
    out = {k: [] for k in ("y", "mean", "rstd", "dx")}
    dscale, dshift = 0.0, 0.0
    per = C // G
    spread = lambda u: u.repeat_interleave(per)  # noqa: E731  a value per group to its channels
    for i in range(N):
        x = t["x"][i]                                        # [S, C]
        mu = x.reshape(S, G, per).mean((0, 2))
        var = (x.reshape(S, G, per) - mu.reshape(1, G, 1)).pow(2).mean((0, 2))
        r = (var + EPS).rsqrt()
        xhat = (x - spread(mu)) * spread(r)
        z = xhat * t["scale"] + t["shift"]
        out["y"].append(_act(z, case["act"]))
        out["mean"].append(mu)
        out["rstd"].append(r)
        if case["train"]:
            dz = t["dy"][i] * _act_slope(z, case["act"])
            dshift, dscale = dshift + dz.sum(0), dscale + (dz * xhat).sum(0)
            h = dz * t["scale"]
            a, b = h.reshape(S, G, per).mean((0, 2)), (h * xhat).reshape(S, G, per).mean((0, 2))
            out["dx"].append(spread(r) * (h - spread(a) - xhat * spread(b)))
    if not case["train"]:
        return {"y": torch.stack(out["y"])}
    return {**{k: torch.stack(v) for k, v in out.items()}, "dscale": dscale, "dshift": dshift}


def _exact_linear(case, seed):
    t = {k: v.double() for k, v in _linear_inputs(case, seed).items()}
    z = torch.addmm(t["b"], t["x"], t["w"].t().contiguous())
    y = _act(z, case["act"]) + (t["r"] if case["residual"] else 0.0)
    if not case["train"]:
        return {"y": y}
    g = _act_slope(z, case["act"]).mul_(t["dy"])
    return {"y": y, "dx": g @ t["w"], "dw": g.t().contiguous() @ t["x"], "db": g.sum(0)}


def _exact_adamw(case, seed):
    t, h = _adamw_inputs(case, seed), _hyper(case)
    dec = lambda k: t[k].double() if case["states"] == "f32" else (t[k].double().view(-1, BLOCK) * t[k + "_scale"].double()[:, None]).view(-1)  # noqa: E731
    m, v = dec("m"), dec("v")
    v = v if case["states"] == "f32" else v * v
    g = t["dw"].double() * h["grad_scale"]
    m, v = torch.lerp(g, m, h["beta1"]), torch.lerp(g * g, v, h["beta2"])
    n = case["step"]
    up = (m / (1 - np.float64(h["beta1"]) ** n)) / ((v / (1 - np.float64(h["beta2"]) ** n)).sqrt() + h["eps"])
    w = t["w"].double() * (1 - h["lr"] * h["weight_decay"]) - h["lr"] * up
    if case["states"] == "f32":
        return {"w": w, "m": m, "v": v}
    return {"w": w, "copy": w, "m": None, "v": None, "m_scale": None, "v_scale": None}


def exact(case, seed):
    return {"norm": _exact_norm, "linear": _exact_linear, "adamw": _exact_adamw}[case["kind"]](case, seed)
