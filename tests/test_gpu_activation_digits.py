"""How many digits activations have, from their small values in the tail on, against 64 bits: fp32 results and bf16 ones.

Bounds, of the value (eps = 2^-24). SiLU: exponential, sum, quotient, product, 10 eps. GELU: exponential with the square's lost part, quotient, a polynomial of eight
steps and its fit (0.6), three products: 24 eps. GELU by tanh: the same as SiLU and what its exponent's three roundings make, 12 + 4 |2 u| eps. bf16: one
rounding, 2^-8, with room for 1e-4 of the function. Slopes: the same of the magnitudes of their two terms."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
DEV = "cuda:0"


def _terms(z, act):
    """y, slope, and its two terms' magnitudes, |2 u| of GELU by tanh (else 0)."""
    if act == "gelu":
        s, d, u = 0.5 * torch.erfc(-z / math.sqrt(2)), torch.exp(-z * z / 2) / math.sqrt(2 * math.pi), 0 * z
    else:
        k = 2 * math.sqrt(2 / math.pi)
        u = z if act == "silu" else k * (z + 0.044715 * z ** 3)
        s = torch.sigmoid(u)
        d = s * torch.sigmoid(-u) * (1 if act == "silu" else k * (1 + 3 * 0.044715 * z * z))
        u = 0 * z if act == "silu" else u.abs()
    return z * s, s + z * d, s + (z * d).abs(), u


def _grid(act, td):
    reach = {"silu": 80.0, "gelu": 12.0, "gelu_tanh": 8.0}[act]
    z = torch.linspace(-reach, reach, 4096, dtype=torch.float64)
    return torch.cat([z, torch.logspace(-8, 0, 500, dtype=torch.float64), -torch.logspace(-8, 0, 500, dtype=torch.float64)]).to(td).to(DEV)


def _tolerance(act, u):
    return EPS * ({"silu": 10.0, "gelu": 24.0, "gelu_tanh": 12.0}[act] + 4 * u)


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_fp32(act):
    import paper_1412_6249_amd as pa
    z = _grid(act, torch.float32)
    n, code = z.numel(), pa.ACTIVATIONS[act]
    y, slope, size, u = _terms(z.double(), act)
    tol = _tolerance(act, u)
    near = lambda got: bool(((got.double() - y).abs() <= tol * y.abs() + 1e-37).all())  # noqa: E731
    for N, S in ((1, 6), (1, 20000)):                      # held, sliced: z is the shift where the scale is 0
        x, dx = torch.randn(N, S, n, device=DEV), torch.empty(N, S, n, device=DEV)
        got, zero = torch.empty_like(x), torch.zeros(n, device=DEV)
        mean, rstd = torch.empty(N, 1, device=DEV), torch.empty(N, 1, device=DEV)
        ds, db = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
        ws = torch.empty(max(pa.purine_group_norm_workspace_bytes(b, (N, S, n), 1) for b in (0, 1)), dtype=torch.uint8, device=DEV)
        pa.purine_group_norm_fwd(x, zero, z, got, mean, rstd, 1, 1e-5, code, ws=ws)
        assert near(got[0, 0]) and near(got[0, -1])
        dy = torch.zeros_like(x)
        dy[0, S // 2] = 1.0
        pa.purine_group_norm_bwd(x, zero, z, mean, rstd, dy, dx, ds, db, 1, code, ws=ws)
        assert bool(((db.double() - slope).abs() <= tol * size + 1e-37).all())
    for N in (1, 40, 700):                                 # products of zeros: z is the bias
        x, w = torch.zeros(N, 64, device=DEV), torch.zeros(n, 64, device=DEV)
        got, g = torch.empty(N, n, device=DEV), torch.empty(N, n, device=DEV)
        ws = torch.empty(max(256, pa.purine_linear_workspace_bytes(0, N, 64, n)), dtype=torch.uint8, device=DEV)
        pa.purine_linear_fwd(x, w, z, None, got, act=code, ws=ws)
        assert near(got[0]) and near(got[-1])
        pa.purine_act_bwd(z.expand(N, n).contiguous(), torch.ones(N, n, device=DEV), g, None, code)
        assert bool(((g[-1].double() - slope).abs() <= tol * size + 1e-37).all())


@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_bf16(act):
    import paper_1412_6249_amd as pa
    z = _grid(act, torch.bfloat16)
    z = z[: z.numel() // 8 * 8]
    n, code = z.numel(), pa.ACTIVATIONS[act]
    y, slope, size, _ = _terms(z.double(), act)
    for N in (1, 40, 700, 5000):                           # a row, few rows, tiles, streamed rows
        x, w = torch.zeros(N, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(n, 64, dtype=torch.bfloat16, device=DEV)
        got, g = (torch.empty(N, n, dtype=torch.bfloat16, device=DEV) for _ in range(2))
        ws = torch.empty(max(256, pa.purine_linear_workspace_bytes(0, N, 64, n, pa.PURINE_BF16)), dtype=torch.uint8, device=DEV)
        pa.purine_linear_fwd(x, w, z, None, got, act=code, ws=ws)
        assert bool(((got[-1].double() - y).abs() <= (2 ** -8 + 1e-4) * y.abs() + 1e-37).all()), N
        pa.purine_act_bwd(z.expand(N, n).contiguous(), torch.ones(N, n, dtype=torch.bfloat16, device=DEV), g, None, code)
        assert bool(((g[-1].double() - slope).abs() <= 2 ** -8 * slope.abs() + 1e-4 * size + 1e-37).all()), N
