"""Group normalization of more images than one launch can take a workgroup each of (2^32 threads), against 64 bits.

Bounds as in test_gpu_group_norm.py: results in bf16 are rounded once, 2^-8.5 in the 2-norm; fp32 statistics are within 32 eps."""
import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
EPS = 2.0 ** -24
DEV = "cuda:0"


def test_more_than_two_to_the_24():
    import paper_1412_6249_amd as pa
    N, C, G = (1 << 24) + 1001, 8, 2
    g = torch.Generator(device=DEV).manual_seed(1)
    x, dy = (torch.randn(N, C, generator=g, device=DEV).bfloat16() for _ in range(2))
    scale, shift = torch.linspace(0.5, 1.5, C, device=DEV), torch.linspace(-0.2, 0.2, C, device=DEV)
    ws = torch.empty(max(pa.purine_group_norm_workspace_bytes(b, (N, C), G, pa.PURINE_BF16) for b in (0, 1)), dtype=torch.uint8, device=DEV)
    y, dx = (torch.full_like(x, float("nan")) for _ in range(2))
    mean, rstd = (torch.full((N, G), float("nan"), device=DEV) for _ in range(2))
    pa.purine_group_norm_fwd(x, scale, shift, y, mean, rstd, G, 1e-2, pa.PURINE_ACT_SILU, ws=ws)
    pa.purine_group_norm_bwd(x, scale, shift, mean, rstd, dy, dx, None, None, G, pa.PURINE_ACT_SILU, ws=ws)
    for part in (slice(0, 1 << 20), slice((1 << 22) + 5, 5 << 20), slice((1 << 23) - 7, 9 << 20), slice(N - (1 << 20), N)):
        d = [t[part].double().reshape(-1, 1, C) for t in (x, dy)]
        s, b = scale.double(), shift.double()
        wy, wm, wr, _, _ = ref.group_norm(d[0], s, b, G, 1e-2, "silu")
        assert float((mean[part].double() - wm).abs().max()) <= 32 * EPS * float(d[0].abs().max())
        assert float((rstd[part].double() / wr - 1).abs().max()) <= 32 * EPS * (1 + float(wm.abs().max()))
        assert float((y[part].double() - wy[:, 0]).norm()) <= 2 ** -8.5 * float(wy.norm())
        wdx, *_, hnorm = ref.group_norm_grad(d[0], s, b, G, 1e-2, "silu", d[1])
        assert float((dx[part].double() - wdx[:, 0]).norm()) <= 2 ** -8.5 * float(hnorm)
