"""The activation gradient with column sums of many columns, whole packets and not, rows in few and many slices, against 64 bits.

Bounds. g: its few operations in fp32, 1e-6, and one rounding to bf16, 2^-8.5, of its 2-norm. db: sums of N products in fp32, each slope right to
1e-6 of 1: 2e-8 sqrt(N) + 2e-6 of the 2-norm of the columns' magnitudes, and the rounding of a bf16 result."""
import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", [(1, 4096), (3, 4099), (700, 4096), (517, 5001), (1024, 8192), (40, 70001), (5000, 4104)], ids=lambda c: "x".join(map(str, c)))
def test_column_sums(case, dtype):
    import paper_1412_6249_amd as pa
    N, K = case
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    gen = torch.Generator(device=DEV).manual_seed(N + K)
    pre, dy = (torch.randn(N, K, generator=gen, device=DEV).to(td) for _ in range(2))
    ws = torch.full((pa.purine_act_bwd_workspace_bytes(N, K),), 255, dtype=torch.uint8, device=DEV)
    for act in ("gelu", "silu"):
        want = dy.double() * ref.slope(pre.double(), act)
        ends = []
        for _ in range(2):
            g, db = torch.full((N, K), float("nan"), dtype=td, device=DEV), torch.full((K,), float("nan"), dtype=td, device=DEV)
            pa.purine_act_bwd(pre, dy, g, db, pa.ACTIVATIONS[act], ws=ws)
            ends.append((g, db))
        assert all(torch.equal(a, b) for a, b in zip(*ends))
        rounding = 2 ** -8.5 if dtype == "bf16" else 0.0
        assert float((g.double() - want).norm()) <= (1e-6 + rounding) * float(dy.double().norm())
        size = float(dy.double().abs().sum(0).norm())
        assert float((db.double() - want.sum(0)).norm()) <= (2e-8 * N ** 0.5 + 2e-6) * size + rounding * float(want.sum(0).norm())
