"""Normalised residual blocks on channels-last pixels, and a training step of a small network of them, out of the operators of
include/purine_block.h.

    y = x + W2 act(W1 act(norm(x)) + b1) + b2          per block, its 1x1 layers as products over all positions
    network: act(Wi x + bi), the blocks, Wo y + bo

    python -m paper_1412_6249_amd.blocks --images 16 --side 28 --channels 192 --blocks 4 --dtype bf16 --states 8bit

trains one on synthetic pixels and prints the loss and the time of a step, recorded as a HIP graph. Parameters are fp32, with bf16
copies that the products read in a bf16 network; gradients of parameters are fp32; AdamW states are fp32 or 8 bits. All buffers are
allocated once, one workspace serves every operator (they run on one stream), and a step makes no allocation.
"""
import argparse

import torch

from . import binding as B


class Parameters:
    """fp32 parameters with gradients, states and (in a bf16 network) bf16 copies. Vectors are not decayed."""

    def __init__(self, dtype, states, device):
        if dtype not in ("f32", "bf16") or states not in ("f32", "8bit"):
            raise ValueError("dtype: f32 or bf16; states: f32 or 8bit")
        self.dtype, self.states, self.device = dtype, states, device
        self.values, self.grads, self.copies = [], [], []
        self.groups = None

    def add(self, value, copied=True):
        """Returns the fp32 value, what the products read, and the gradient."""
        if self.groups is not None:
            raise ValueError("parameters are added before the first step")
        w = value.to(self.device, torch.float32).contiguous()
        copy = w.bfloat16() if copied and self.dtype == "bf16" else None
        self.values.append(w)
        self.copies.append(copy)
        self.grads.append(torch.zeros_like(w))
        return w, (w if copy is None else copy), self.grads[-1]

    def _group(self, members):
        w, dw, copy = ([l[i] for i in members] for l in (self.values, self.grads, self.copies))
        more = {}
        if self.states == "8bit":
            m, v = ([torch.zeros(t.shape, dtype=torch.float8_e4m3fn, device=self.device) for t in w] for _ in range(2))
            for name in ("m_scale", "v_scale"):
                more[name] = [torch.zeros(-(-t.numel() // B.PURINE_ADAMW_BLOCK), device=self.device) for t in w]
        else:
            m, v = ([torch.zeros_like(t) for t in w] for _ in range(2))
        return B.adamw_params(w, dw, m, v, copy=copy, **more), torch.zeros(1, dtype=torch.int32, device=self.device)

    def step(self, lr, weight_decay=0.01, grad_scale=1.0, seed=0, stream=None):
        """One AdamW step on everything; the step's number is counted on the device."""
        if self.groups is None:
            order = range(len(self.values))
            self.groups = [(self._group([i for i in order if (self.values[i].dim() > 1) == matrices]), matrices) for matrices in (True, False)]
        for (params, done), matrices in self.groups:
            desc = B.adamw_desc(lr, weight_decay=weight_decay if matrices else 0.0, grad_scale=grad_scale, seed=seed,
                                dither=self.states == "8bit")
            B.purine_adamw_step(desc, params, done, stream=stream)


class Block:
    """One block's parameters and what its backward pass needs of the forward pass."""

    def __init__(self, net, hidden, generator):
        self.net = net
        C, rows = net.channels, net.rows
        new = lambda *s: torch.empty(s, dtype=net.td, device=net.device)  # noqa: E731
        rnd = lambda *s: torch.randn(s, generator=generator) * s[1] ** -0.5  # noqa: E731
        p = net.parameters
        self.scale, _, self.dscale = p.add(torch.ones(C), copied=False)
        self.shift, _, self.dshift = p.add(torch.zeros(C), copied=False)
        _, self.w1, self.dw1 = p.add(rnd(hidden, C))
        _, self.b1, self.db1 = p.add(torch.zeros(hidden))
        _, self.w2, self.dw2 = p.add(rnd(C, hidden))
        _, self.b2, self.db2 = p.add(torch.zeros(C))
        self.normed, self.pre, self.hidden, self.y = new(rows, C), new(rows, hidden), new(rows, hidden), new(rows, C)
        self.mean, self.rstd = (torch.empty(net.images, net.groups, device=net.device) for _ in range(2))

    def forward(self, x, stream=None):
        n = self.net
        self.x = x
        B.purine_group_norm_fwd(n.pixels(x), self.scale, self.shift, n.pixels(self.normed), self.mean, self.rstd, n.groups, n.eps, n.act,
                                ws=n.ws, stream=stream)
        B.purine_linear_fwd(self.normed, self.w1, self.b1, None, self.hidden, self.pre, n.act, ws=n.ws, stream=stream)
        B.purine_linear_fwd(self.hidden, self.w2, self.b2, x, self.y, ws=n.ws, stream=stream)
        return self.y

    def backward(self, dy, stream=None):
        """dy becomes the gradient of the block's input."""
        n = self.net
        dpre, dnormed = n.dpre[:, :self.w1.shape[0]], n.dnormed
        B.purine_linear_bwd_weight(self.hidden, dy, self.dw2, self.db2, ws=n.ws, stream=stream)
        B.purine_linear_bwd_data(dy, self.w2, self.pre, dpre, n.act, ws=n.ws, stream=stream)
        B.purine_linear_bwd_weight(self.normed, dpre, self.dw1, self.db1, ws=n.ws, stream=stream)
        B.purine_linear_bwd_data(dpre, self.w1, None, dnormed, ws=n.ws, stream=stream)
        B.purine_group_norm_bwd(n.pixels(self.x), self.scale, self.shift, self.mean, self.rstd, n.pixels(dnormed), n.pixels(dy), self.dscale,
                                self.dshift, n.groups, n.act, beta=1.0, ws=n.ws, stream=stream)
        return dy


class ResidualNet:
    """inputs -> channels, blocks, channels -> outputs, on `images` images of `positions` pixels, rows of pixels throughout."""

    def __init__(self, images, positions, inputs, channels, outputs, hidden, blocks, groups=32, act="gelu_tanh", dtype="bf16", states="f32",
                 eps=1e-5, seed=0, device="cuda:0"):
        self.images, self.positions, self.rows, self.channels = images, positions, images * positions, channels
        self.groups, self.eps, self.act, self.dtype, self.device = groups, eps, B.ACTIVATIONS[act], dtype, torch.device(device)
        self.parameters = Parameters(dtype, states, self.device)
        self.td = torch.bfloat16 if dtype == "bf16" else torch.float32
        code = B.PURINE_BF16 if dtype == "bf16" else B.PURINE_F32
        g = torch.Generator().manual_seed(seed)
        new = lambda *s: torch.empty(s, dtype=self.td, device=self.device)  # noqa: E731
        rnd = lambda *s: torch.randn(s, generator=g) * s[1] ** -0.5  # noqa: E731
        rows = self.rows
        _, self.wi, self.dwi = self.parameters.add(rnd(channels, inputs))
        _, self.bi, self.dbi = self.parameters.add(torch.zeros(channels))
        self.blocks = [Block(self, hidden, g) for _ in range(blocks)]
        _, self.wo, self.dwo = self.parameters.add(rnd(outputs, channels))
        _, self.bo, self.dbo = self.parameters.add(torch.zeros(outputs))
        self.pre, self.first, self.out = new(rows, channels), new(rows, channels), new(rows, outputs)
        self.grad, self.dnormed, self.dpre = new(rows, channels), new(rows, channels), new(rows, hidden)
        shape = (images, positions, channels)
        need = [B.purine_group_norm_workspace_bytes(backward, shape, groups, code) for backward in (0, 1)]
        need.append(B.purine_act_bwd_workspace_bytes(rows, channels))
        for C, K in ((inputs, channels), (channels, hidden), (hidden, channels), (channels, outputs)):
            need += [B.purine_linear_workspace_bytes(which, rows, C, K, code) for which in (B.PURINE_CONV_FWD, B.PURINE_CONV_BWD_DATA,
                                                                                           B.PURINE_CONV_BWD_WEIGHT)]
        self.ws = torch.empty(max(256, *need), dtype=torch.uint8, device=self.device)

    def pixels(self, t):
        return t.view(self.images, self.positions, -1)

    def forward(self, x, stream=None):
        self.x = x
        B.purine_linear_fwd(x, self.wi, self.bi, None, self.first, self.pre, self.act, ws=self.ws, stream=stream)
        y = self.first
        for block in self.blocks:
            y = block.forward(y, stream)
        self.last = y
        B.purine_linear_fwd(y, self.wo, self.bo, None, self.out, ws=self.ws, stream=stream)
        return self.out

    def backward(self, dout, stream=None):
        """Gradients of all parameters, into parameters.grads."""
        B.purine_linear_bwd_weight(self.last, dout, self.dwo, self.dbo, ws=self.ws, stream=stream)
        B.purine_linear_bwd_data(dout, self.wo, None, self.grad, ws=self.ws, stream=stream)
        for block in reversed(self.blocks):
            block.backward(self.grad, stream)
        B.purine_act_bwd(self.pre, self.grad, self.grad, self.dbi, self.act, ws=self.ws, stream=stream)
        B.purine_linear_bwd_weight(self.x, self.grad, self.dwi, None, ws=self.ws, stream=stream)

    def step(self, lr, stream=None, **more):
        self.parameters.step(lr, stream=stream, **more)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("images", 16), ("side", 28), ("inputs", 64), ("channels", 192), ("outputs", 16), ("hidden", 768), ("blocks", 4),
                        ("groups", 32), ("steps", 100)):
        ap.add_argument("--" + name, type=int, default=value)
    ap.add_argument("--act", choices=sorted(B.ACTIVATIONS), default="gelu_tanh")
    ap.add_argument("--dtype", choices=["f32", "bf16"], default="bf16")
    ap.add_argument("--states", choices=["f32", "8bit"], default="8bit")
    ap.add_argument("--lr", type=float, default=1e-3)
    a = ap.parse_args(argv)
    net = ResidualNet(a.images, a.side * a.side, a.inputs, a.channels, a.outputs, a.hidden, a.blocks, a.groups, a.act, a.dtype, a.states)
    g = torch.Generator(device=net.device).manual_seed(1)
    x = torch.randn(net.rows, a.inputs, generator=g, device=net.device)
    target = torch.tanh(x @ torch.randn(a.inputs, a.outputs, generator=g, device=net.device) * a.inputs ** -0.5)
    x = x.to(net.td)
    dout = torch.empty_like(net.out)

    def step():                              # (recorded: no reductions of the library's, which fill their counters by memset nodes)
        dout.copy_((net.forward(x).float() - target) * (2.0 / target.numel()))
        net.backward(dout)
        net.step(a.lr)

    def loss():                              # before the last step's update
        return (net.out.float() - target).square().mean().item()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    first = loss()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    start, stop = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    start.record()
    for _ in range(a.steps):
        graph.replay()
    stop.record()
    torch.cuda.synchronize()
    print("loss %.5f after the first step, %.5f after %d more; %.3f ms a step" % (first, loss(), a.steps, start.elapsed_time(stop) / max(1, a.steps)))


if __name__ == "__main__":
    main()
