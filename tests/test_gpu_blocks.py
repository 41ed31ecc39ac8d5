"""A network of residual blocks trained with the block operators: gradients against the same network in 64 bits, differentiated by torch
there and by differences along a direction; recorded steps against eager ones; training with each kind of state.

Bounds, in the 2-norm. fp32: an operator is within 1e-6 of its result, a gradient passes some 8 per block and 4 more, and a normalization
or a product may put what it is given at up to a few times its size: 2e-5. bf16: every stored tensor carries 2^-9 / sqrt(3) = 1.1e-3 of
itself; a gradient has passed some 10 such roundings a block and 6 more, independent ones, which add as squares: 1.1e-3 sqrt(26) = 5.6e-3
with two blocks, and the few times of above: 2e-2."""
import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu

# images, positions, inputs, channels, outputs, hidden, blocks, groups
SHAPES = [(2, 49, 24, 64, 8, 128, 2, 8), (1, 1, 3, 8, 1, 12, 1, 2), (3, 35, 13, 30, 5, 41, 2, 5)]


def _net(shape, dtype, states="f32", act="gelu_tanh", seed=3):
    from paper_1412_6249_amd import blocks
    images, positions, inputs, channels, outputs, hidden, n, groups = shape
    net = blocks.ResidualNet(images, positions, inputs, channels, outputs, hidden, n, groups, act, dtype, states, seed=seed)
    g = torch.Generator().manual_seed(seed + 1)
    for w, c in zip(net.parameters.values, net.parameters.copies):       # biases and shifts off zero
        if w.dim() == 1:
            w.add_(0.1 * torch.randn(w.shape, generator=g).to(w.device))
            if c is not None:
                c.copy_(w)
    x = torch.randn(net.rows, inputs, generator=g).to(net.device, net.td)
    dout = torch.randn(net.rows, outputs, generator=g).to(net.device, net.td)
    return net, x, dout


def _forward64(net, x, params, act):
    it = iter(params)
    wi, bi = next(it), next(it)
    y = ref.act(x @ wi.T + bi, act)
    for _ in net.blocks:
        scale, shift, w1, b1, w2, b2 = (next(it) for _ in range(6))
        h = ref.group_norm(y.view(net.images, net.positions, -1), scale, shift, net.groups, net.eps, act)[0].reshape(net.rows, -1)
        y = y + ref.act(h @ w1.T + b1, act) @ w2.T + b2
    wo, bo = next(it), next(it)
    return y @ wo.T + bo


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=["x".join(map(str, s)) for s in SHAPES])
@pytest.mark.parametrize("act", ["gelu_tanh", "silu", "gelu"])
def test_gradients(shape, dtype, act):
    net, x, dout = _net(shape, dtype, act=act)
    out = net.forward(x)
    net.backward(dout)
    p = net.parameters
    params = [(w if c is None else c).double().cpu().requires_grad_() for w, c in zip(p.values, p.copies)]
    want = _forward64(net, x.double().cpu(), params, act)
    d64 = dout.double().cpu()
    grads = torch.autograd.grad((want * d64).sum(), params)
    tol = 2e-5 if dtype == "f32" else 2e-2
    assert float((out.double().cpu() - want).detach().norm()) <= tol * float(want.detach().norm())
    for i, (got, g) in enumerate(zip(p.grads, grads)):
        assert float((got.double().cpu() - g).norm()) <= tol * float(g.norm()) + 1e-30, (i, tuple(g.shape))
    # differences of the 64-bit network along a random direction: no derivative is taken
    gen = torch.Generator().manual_seed(9)
    u = [torch.randn(w.shape, generator=gen, dtype=torch.float64) * 0.1 for w in params]
    with torch.no_grad():
        f = lambda e: float((_forward64(net, x.double().cpu(), [w + e * d for w, d in zip(params, u)], act) * d64).sum())  # noqa: E731
        slope = (f(1e-5) - f(-1e-5)) / 2e-5
    along = sum(float((g.double().cpu() * d).sum()) for g, d in zip(p.grads, u))
    size = sum(float(g.norm() * d.norm()) for g, d in zip(p.grads, u))
    assert abs(along - slope) <= (tol + 1e-6) * size


@pytest.mark.parametrize("dtype,states", [("f32", "f32"), ("bf16", "f32"), ("bf16", "8bit"), ("f32", "8bit")])
def test_training(dtype, states):
    """30 steps towards a smooth function of the pixels more than halve the squared distance, recorded steps and eager ones give the same
    parameters, and the bf16 copies are those of the parameters."""
    shape = (2, 49, 24, 64, 8, 128, 2, 8)
    ends = []
    for recorded in (False, True):
        net, x, dout = _net(shape, dtype, states)
        target = torch.tanh(x.float()[:, :8])
        loss = torch.zeros((), device=net.device)

        def step():
            off = net.forward(x).float() - target
            loss.copy_(off.square().mean())
            dout.copy_(off * (2.0 / off.numel()))
            net.backward(dout)
            net.step(2e-3)

        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.synchronize()
        first = float(loss)
        graph = None
        if recorded:
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
        for _ in range(30):
            graph.replay() if recorded else step()
            torch.cuda.synchronize()
        assert float(loss) < 0.5 * first, (first, float(loss))
        for w, c in zip(net.parameters.values, net.parameters.copies):
            assert c is None or torch.equal(c, w.bfloat16())
        ends.append([w.clone() for w in net.parameters.values])
    assert all(torch.equal(a, b) for a, b in zip(*ends))


def test_refusals():
    from paper_1412_6249_amd import blocks
    with pytest.raises(ValueError):
        blocks.Parameters("f16", "f32", "cuda:0")
    net, x, dout = _net((2, 49, 24, 64, 8, 128, 1, 8), "f32")
    net.step(1e-3)
    with pytest.raises(ValueError):
        net.parameters.add(torch.zeros(3))


def test_command(capsys):
    from paper_1412_6249_amd import blocks
    blocks.main(["--images", "2", "--side", "7", "--channels", "64", "--hidden", "128", "--blocks", "1", "--groups", "8", "--steps", "5"])
    assert "ms a step" in capsys.readouterr().out
