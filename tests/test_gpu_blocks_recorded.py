"""The recorded training step of the residual network: what the graph holds, and replays against eager steps."""
import ctypes

import pytest
import torch

pytestmark = pytest.mark.gpu
KERNEL, COPY, MEMSET = 0, 1, 2                   # hipGraphNodeType


def _node_types(graph):
    hip = ctypes.CDLL("libamdhip64.so")
    raw, n = ctypes.c_void_p(graph.raw_cuda_graph()), ctypes.c_size_t(0)
    assert hip.hipGraphGetNodes(raw, None, ctypes.byref(n)) == 0
    nodes, types = (ctypes.c_void_p * n.value)(), []
    assert hip.hipGraphGetNodes(raw, nodes, ctypes.byref(n)) == 0
    for node in nodes:
        t = ctypes.c_int(-1)
        assert hip.hipGraphNodeGetType(ctypes.c_void_p(node), ctypes.byref(t)) == 0
        types.append(t.value)
    return types


def test_command_records_no_memset(monkeypatch, capsys):
    """Memset nodes have given wrong results in replays after the first. 12544 rows of 16 outputs: sizes at which a library reduction takes several blocks."""
    from paper_1412_6249_amd import blocks
    graphs, make = [], torch.cuda.CUDAGraph

    def keep():
        graphs.append(make(keep_graph=True))
        return graphs[-1]

    monkeypatch.setattr(torch.cuda, "CUDAGraph", keep)
    blocks.main(["--blocks", "1", "--steps", "3"])
    assert "ms a step" in capsys.readouterr().out
    types = _node_types(graphs[0])
    assert len(graphs) == 1 and KERNEL in types and MEMSET not in types, types


@pytest.mark.parametrize("dtype,states", [("bf16", "8bit"), ("f32", "f32")])
def test_replays_are_eager_steps(dtype, states):
    """Each replay's parameters are those of an eager step, with eager work and waits between the replays."""
    from paper_1412_6249_amd import blocks
    nets = [blocks.ResidualNet(2, 400, 24, 64, 8, 128, 2, 8, "gelu_tanh", dtype, states, seed=3) for _ in range(2)]
    g = torch.Generator(device=nets[0].device).manual_seed(1)
    x = torch.randn(nets[0].rows, 24, generator=g, device=nets[0].device).to(nets[0].td)
    target = torch.tanh(x.float()[:, :8])
    steps = []
    for net in nets:
        dout = torch.empty_like(net.out)

        def step(net=net, dout=dout):
            dout.copy_((net.forward(x).float() - target) * (2.0 / target.numel()))
            net.backward(dout)
            net.step(2e-3)
        steps.append(step)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for step in steps:
            step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        steps[0]()
    for i in range(6):
        graph.replay()
        steps[1]()
        torch.cuda.synchronize()
        for a, b in zip(nets[0].parameters.values, nets[1].parameters.values):
            assert torch.equal(a, b), i
        assert float((nets[0].out.float() - target).square().mean()) == float((nets[1].out.float() - target).square().mean())
