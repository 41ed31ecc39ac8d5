"""Block operators: what their entry points refuse (no launch happens, so none of it needs a GPU), their workspace queries, and
the 64-bit definitions that the GPU tests use, against differences and a second formulation."""
import ctypes
import os
import re

import pytest
import torch

import block_ref as ref
import paper_1412_6249_amd as pa
from paper_1412_6249_amd import binding

F32, BF16, I32, F8 = pa.PURINE_F32, pa.PURINE_BF16, pa.PURINE_I32, pa.PURINE_F8
NULL, SHAPE, DTYPE, LAYOUT, WORKSPACE, ARG = -1, -2, -3, -4, -5, -8
A = 0x10000000          # addresses of a made-up tensor each: never touched


def at(k, dims, dtype=F32, nstride=0, off=0):
    return pa.raw_desc(A + k * 0x4000000 + off, dtype, dims, nstride)


class WS:
    def __init__(self, n, ptr=A + 60 * 0x4000000):
        self.n, self.ptr = n, ptr

    def data_ptr(self):
        return self.ptr

    def numel(self):
        return self.n

    def element_size(self):
        return 1


def refused(status, f, *args, **kw):
    with pytest.raises(pa.PurineError) as e:
        f(*args, stream=0, **kw)
    assert e.value.status == status, e.value


def test_every_declared_symbol_is_exported_and_bound():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(root, "include", "purine_block.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(purine_[a-z_0-9]+)\s*\(", text))
    lib = ctypes.CDLL(binding.LIB_PATH)
    assert names == set(binding.EXPORTED_BLOCK) and all(hasattr(lib, n) and callable(getattr(pa, n)) for n in names)


def test_group_norm_refusals():
    N, S, C, G = 3, 10, 24, 4
    x, y, dy, dx = (at(k, (N, S, C)) for k in range(4))
    sc, sh, mean, rstd, ds, db = at(4, (C,)), at(5, (C,)), at(6, (N, G)), at(7, (N, G)), at(8, (C,)), at(9, (C,))
    fwd = lambda status, x=x, sc=sc, sh=sh, y=y, mean=mean, rstd=rstd, G=G, eps=1e-5, act=0, ws=WS(1 << 20): refused(  # noqa: E731
        status, pa.purine_group_norm_fwd, x, sc, sh, y, mean, rstd, G, eps, act, ws=ws)
    fwd(NULL, x=pa.raw_desc(0, F32, (N, S, C)))
    fwd(NULL, mean=None)
    fwd(SHAPE, G=5)
    fwd(ARG, G=0)
    fwd(ARG, act=5)
    fwd(ARG, act=-1)
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        fwd(ARG, eps=eps)
    fwd(SHAPE, x=at(0, (N,)), y=at(1, (N,)))
    fwd(SHAPE, y=at(1, (N, S, C + 4)))
    fwd(SHAPE, x=at(0, (0, S, C)))
    fwd(SHAPE, sc=at(4, (C + 1,)))
    fwd(DTYPE, sc=at(4, (C,), BF16))
    fwd(DTYPE, y=at(1, (N, S, C), BF16))
    fwd(DTYPE, x=at(0, (N, S, C), I32), y=at(1, (N, S, C), I32))
    fwd(DTYPE, x=at(0, (N, S, C), F8), y=at(1, (N, S, C), F8))
    fwd(SHAPE, mean=at(6, (N, G + 1)))
    fwd(LAYOUT, x=at(0, (N, S, C), off=4))
    fwd(LAYOUT, y=at(0, (N, S, C), off=16))
    fwd(LAYOUT, sc=at(1, (C,)))
    fwd(LAYOUT, rstd=mean)
    fwd(SHAPE, x=at(0, (N, S, C), nstride=S * C + 8))                    # only 4-axis tensors have images apart
    fwd(LAYOUT, x=at(0, (N, 2, 5, C), nstride=S * C + 2), y=at(1, (N, 2, 5, C)))
    need = pa.purine_group_norm_workspace_bytes(0, (N, S, C), G)
    assert need > 0
    fwd(WORKSPACE, ws=None)
    fwd(WORKSPACE, ws=WS(need - 1))
    fwd(LAYOUT, ws=WS(need, A))                                          # over x
    bwd = lambda status, x=x, mean=mean, rstd=rstd, dy=dy, dx=dx, ds=ds, db=db, beta=0.0, ws=WS(1 << 20): refused(  # noqa: E731
        status, pa.purine_group_norm_bwd, x, sc, sh, mean, rstd, dy, dx, ds, db, G, 2, beta, ws=ws)
    bwd(NULL, ds=None)
    bwd(ARG, beta=0.5)
    bwd(LAYOUT, dx=x)
    bwd(LAYOUT, dx=at(2, (N, S, C), off=16))
    bwd(DTYPE, dy=at(2, (N, S, C), BF16))
    bwd(SHAPE, rstd=at(7, (G, N)))
    bwd(LAYOUT, ds=db)
    bwd(WORKSPACE, ws=WS(pa.purine_group_norm_workspace_bytes(1, (N, S, C), G) - 1))
    for bad in (((0, 1, 8), 4), ((2, 3, 8), 3), ((1 << 16, 1 << 10, 32), 4), ((2, 8), 0)):
        assert pa.purine_group_norm_workspace_bytes(0, *bad) == 0


def test_linear_refusals():
    N, C, K = 33, 40, 24
    x, w, b, r, y, pre = at(0, (N, C)), at(1, (K, C)), at(2, (K,)), at(3, (N, K)), at(4, (N, K)), at(5, (N, K))
    big = WS(1 << 24)
    fwd = lambda status, x=x, w=w, b=b, r=r, y=y, pre=pre, act=0, ws=big: refused(status, pa.purine_linear_fwd, x, w, b, r, y, pre, act, ws=ws)  # noqa: E731
    fwd(NULL, w=pa.raw_desc(0, F32, (K, C)))
    fwd(SHAPE, w=at(1, (K, C + 1)))
    fwd(SHAPE, y=at(4, (K, N)))
    fwd(SHAPE, b=at(2, (N,)))
    fwd(SHAPE, x=at(0, (N, C, 1)))
    fwd(SHAPE, r=at(3, (1, K)))
    fwd(SHAPE, pre=at(5, (N, K + 1)))
    fwd(DTYPE, w=at(1, (K, C), BF16))
    fwd(DTYPE, b=at(2, (K,), BF16))
    fwd(DTYPE, y=at(4, (N, K), BF16))
    fwd(DTYPE, x=at(0, (N, C), I32))
    fwd(ARG, act=9)
    fwd(LAYOUT, y=at(0, (N, K)))
    fwd(LAYOUT, pre=y)
    fwd(LAYOUT, y=at(3, (N, K), off=32))
    fwd(LAYOUT, x=at(0, (N, C), off=8))
    fwd(LAYOUT, x=at(0, (N, C), nstride=C + 1))
    fwd(SHAPE, x=at(0, (N, C), nstride=C - 4))
    fwd(SHAPE, x=at(0, (N, C), nstride=1 << 31))
    fwd(LAYOUT, y=at(3, (N, K), nstride=K + 4))                          # r's first element, other rows
    data = lambda status, dy=at(0, (N, K)), w=w, pre=None, dx=at(4, (N, C)), act=0, beta=0.0, ws=big: refused(  # noqa: E731
        status, pa.purine_linear_bwd_data, dy, w, pre, dx, act, beta, ws=ws)
    data(ARG, act=2)                                                     # an activation and nothing it was applied to
    data(ARG, beta=2.0)
    data(SHAPE, dx=at(4, (N, K)))
    data(SHAPE, pre=at(5, (N, K)))
    data(LAYOUT, dx=at(0, (N, C)))
    data(LAYOUT, pre=at(4, (N, C)), beta=1.0)
    data(DTYPE, dx=at(4, (N, C), BF16))
    weight = lambda status, x=x, dy=at(3, (N, K)), dw=at(4, (K, C)), db=at(5, (K,)), beta=0.0, ws=big: refused(  # noqa: E731
        status, pa.purine_linear_bwd_weight, x, dy, dw, db, beta, ws=ws)
    weight(SHAPE, dy=at(3, (N + 1, K)))
    weight(SHAPE, dw=at(4, (C, K)))
    weight(DTYPE, dw=at(4, (K, C), BF16))
    weight(DTYPE, db=at(5, (K,), BF16))
    weight(SHAPE, db=at(5, (C,)))
    weight(ARG, beta=-1.0)
    weight(LAYOUT, dw=at(0, (K, C)))
    weight(LAYOUT, db=at(4, (K,)))
    weight(WORKSPACE, ws=None)
    act = lambda status, pre=pre, dy=r, g=y, db=None, a=2, ws=None: refused(status, pa.purine_act_bwd, pre, dy, g, db, a, ws=ws)  # noqa: E731
    act(SHAPE, g=at(4, (N, K + 4)))
    act(DTYPE, dy=at(3, (N, K), BF16))
    act(ARG, a=7)
    act(LAYOUT, g=at(3, (N, K), off=16))
    act(WORKSPACE, db=b)
    act(LAYOUT, db=at(4, (K,)), ws=big)
    for bad in ((3, 1, 1, 1), (0, 0, 4, 4), (0, 4, 4, -1), (0, 1 << 20, 1 << 11, 4), (1, 1, 1 << 31, 1)):
        assert pa.purine_linear_workspace_bytes(*bad) == 0
    assert pa.purine_act_bwd_workspace_bytes(0, 4) == 0 and pa.purine_act_bwd_workspace_bytes(5, 4) > 0


def test_adamw_refusals():
    n = 1000

    def step(status, desc=None, done=None, count=None, **change):
        t = {"w": at(0, (n,)), "dw": at(1, (n,)), "m": at(2, (n,)), "v": at(3, (n,)), "m_scale": None, "v_scale": None, "copy": None, **change}
        arr = (binding.purine_adamw_param * 1)()
        for k, v in t.items():
            if v is not None:
                setattr(arr[0], k, v)
        p = pa.AdamwParams(arr, None)
        refused(status, lambda stream: pa.purine_adamw_step(desc or pa.adamw_desc(1e-3), p, done, stream=stream))

    coded = {"m": at(2, (n,), F8), "v": at(3, (n,), F8), "m_scale": at(4, (4,)), "v_scale": at(5, (4,))}
    for bad in ({"lr": float("nan")}, {"lr": float("inf")}, {"lr": 1e39}, {"beta1": 1.0}, {"beta2": -0.1}, {"eps": 0.0}, {"eps": 1e-60}, {"weight_decay": float("inf")},
                {"grad_scale": float("nan")}, {"step": 0}):
        step(ARG, pa.adamw_desc(**{"lr": 1e-3, **bad}))
    step(NULL, dw=pa.raw_desc(0, F32, (n,)))
    step(SHAPE, dw=at(1, (n + 1,)))
    step(SHAPE, w=at(0, (0,)))
    step(DTYPE, w=at(0, (n,), I32))
    step(DTYPE, m=at(2, (n,), BF16))
    step(DTYPE, m=coded["m"], m_scale=coded["m_scale"], v_scale=coded["v_scale"])         # one state coded, the other not
    step(NULL, m=coded["m"], v=coded["v"])
    step(SHAPE, **{**coded, "m_scale": at(4, (3,))})
    step(DTYPE, **{**coded, "v_scale": at(5, (4,), BF16)})
    step(LAYOUT, **{**coded, "v_scale": at(5, (4,), off=2)})
    step(DTYPE, copy=at(6, (n,)))
    step(SHAPE, copy=at(6, (n - 1,), BF16))
    step(LAYOUT, w=at(0, (n,), off=4))
    step(LAYOUT, copy=at(0, (n,), BF16))
    step(LAYOUT, m=at(3, (n,), off=16))
    step(DTYPE, done=at(7, (1,)))
    step(SHAPE, done=at(7, (2,), I32))
    pa.purine_adamw_step(pa.adamw_desc(1e-3), pa.adamw_params([], [], [], []), stream=0)    # nothing to do
    two = pa.AdamwParams((binding.purine_adamw_param * 2)(), None)
    for i, dt in enumerate((F32, BF16)):
        for k, name in enumerate(("w", "dw", "m", "v")):
            setattr(two.array[i], name, at(8 * i + k, (n,), dt if name == "dw" else F32))
    refused(DTYPE, lambda stream: pa.purine_adamw_step(pa.adamw_desc(1e-3), two, stream=stream))
    with pytest.raises(ValueError):
        pa.adamw_params([None], [], [], [])


def test_binding_refuses_what_has_no_descriptor():
    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        pa.purine_linear_fwd(x, x, None, None, x, stream=0)                # not on the GPU
    for t in (torch.zeros(8, 4).t(), torch.zeros(4, 16)[:, ::2], torch.zeros(1, 8).expand(4, 8)):
        with pytest.raises(ValueError):
            pa.matrix_desc(t)
    with pytest.raises(ValueError):
        pa.adamw_params([torch.zeros(8)], [torch.zeros(8)], [torch.zeros(8)], [torch.zeros(8)])


@pytest.mark.parametrize("act", ["none", "silu", "gelu", "gelu_tanh"])
def test_definitions_against_differences(act):
    g = torch.Generator().manual_seed(1)
    rnd = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    z, h = rnd(200) * 3, 1e-5
    assert float(((ref.act(z + h, act) - ref.act(z - h, act)) / (2 * h) - ref.slope(z, act)).abs().max()) < 1e-8
    x, s, b, dy, u = rnd(2, 7, 12), rnd(12), rnd(12), rnd(2, 7, 12), rnd(2, 7, 12)
    loss = lambda t: float((ref.group_norm(t, s, b, 3, 1e-5, act)[0] * dy).sum())  # noqa: E731
    num = (loss(x + h * u) - loss(x - h * u)) / (2 * h)
    assert abs(num - float((ref.group_norm_grad(x, s, b, 3, 1e-5, act, dy)[0] * u).sum())) < 1e-7 * 100


def test_definitions_against_torch():
    g = torch.Generator().manual_seed(2)
    x, s, b = (torch.randn(sh, generator=g, dtype=torch.float64) for sh in ((2, 7, 12), (12,), (12,)))
    want = torch.nn.functional.silu(torch.nn.functional.group_norm(x.transpose(1, 2), 3, s, b, 1e-5)).transpose(1, 2)
    assert float((ref.group_norm(x, s, b, 3, 1e-5, "silu")[0] - want).abs().max()) < 1e-12
    w = torch.randn(50, generator=g, dtype=torch.float64)
    p = torch.nn.Parameter(w.clone())
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.8, 0.95), eps=1e-8, weight_decay=0.1)
    m, v = torch.zeros(50, dtype=torch.float64), torch.zeros(50, dtype=torch.float64)
    for t in range(1, 5):
        grad = torch.randn(50, generator=g, dtype=torch.float64)
        p.grad = grad.clone()
        opt.step()
        w, m, v = ref.adamw(w, grad, m, v, t, 1e-2, 0.8, 0.95, 1e-8, 0.1, 1.0)
        assert float((w - p.detach()).abs().max()) < 1e-12
