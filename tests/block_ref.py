"""The block operators' definitions in 64 bits (torch tensors of float64, on whatever device they are), for the tests."""
import math

import torch


def act(z, name):
    if name == "relu":
        return z.clamp(min=0)
    if name == "silu":
        return z * torch.sigmoid(z)
    if name == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2))
    if name == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)))
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    if name == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "gelu_tanh":
        k = math.sqrt(2 / math.pi)
        t = torch.tanh(k * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * k * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def group_norm(x, scale, shift, groups, eps, name):
    """x [N, S, C]. Returns y, mean, rstd [N, groups], xhat, z."""
    N, S, C = x.shape
    xg = x.reshape(N, S, groups, C // groups)
    mean = xg.mean((1, 3), keepdim=True)
    rstd = ((xg - mean).pow(2).mean((1, 3), keepdim=True) + eps).rsqrt()
    xhat = ((xg - mean) * rstd).reshape(N, S, C)
    z = xhat * scale + shift
    return act(z, name), mean.reshape(N, groups), rstd.reshape(N, groups), xhat, z


def group_norm_grad(x, scale, shift, groups, eps, name, dy):
    """dx, dscale, dshift and what their roundings are proportional to. A rounding of xhat is one of its group's spread, 1, however near 0
    xhat itself is, and one of the slope one of the activation's largest, 1: sums of (|dz| + |dy|) (|xhat| + 1) and of |dz| + |dy|."""
    N, S, C = x.shape
    _, _, rstd, xhat, z = group_norm(x, scale, shift, groups, eps, name)
    dz = dy * slope(z, name)
    h = dz * scale
    avg = lambda t: t.reshape(N, S, groups, -1).mean((1, 3)).repeat_interleave(C // groups, 1)[:, None]  # noqa: E731
    r = rstd.repeat_interleave(C // groups, 1)[:, None]
    dx = r * (h - avg(h) - xhat * avg(h * xhat))
    mag = dz.abs() + dy.abs()
    return dx, (dz * xhat).sum((0, 1)), dz.sum((0, 1)), (mag * (xhat.abs() + 1)).sum((0, 1)), mag.sum((0, 1)), (r * h).norm()


def adamw(w, g, m, v, t, lr, beta1, beta2, eps, weight_decay, grad_scale):
    g = g * grad_scale
    m, v = beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g
    return w * (1 - lr * weight_decay) - lr * (m / (1 - beta1 ** t)) / ((v / (1 - beta2 ** t)).sqrt() + eps), m, v
