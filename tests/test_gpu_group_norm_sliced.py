"""Group normalization where an image's share of a few groups does not fit a workgroup's registers: slices of the positions, joined by the
kernel that writes the results."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ws(pa, backward, case, dtype):
    N, S, C, G = case
    n = pa.purine_group_norm_workspace_bytes(backward, (N, S, C), G, pa.PURINE_F32 if dtype == "f32" else pa.PURINE_BF16)
    return torch.full((max(256, n),), 255, dtype=torch.uint8, device=DEV)


# one group over all positions; 32 groups; a group over three tiles of channels and more workgroups than the card holds at once
SLICED = [(1, 12544, 32, 1), (64, 12544, 64, 32), (8, 8192, 4112, 1)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("case", SLICED, ids=["x".join(map(str, c)) for c in SLICED])
def test_sliced_in_place(case, dtype):
    """y = x and dx = dy where other workgroups read the statistics while a workgroup replaces its positions: the bits of separate tensors."""
    import paper_1412_6249_amd as pa
    N, S, C, G = case
    act = pa.PURINE_ACT_SILU
    td = torch.float32 if dtype == "f32" else torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(5)
    x = (torch.randn(N, S, C, generator=g, device=DEV) + 3.0).to(td)
    ws = _ws(pa, 0, case, dtype)
    new = lambda: [torch.full((N, G), float("nan"), device=DEV) for _ in range(2)]  # noqa: E731
    y, (mean, rstd) = torch.full_like(x, float("nan")), new()
    pa.purine_group_norm_fwd(x, None, None, y, mean, rstd, G, 1e-5, act, ws=ws)
    for _ in range(3):
        z, (m, r) = x.clone(), new()
        ws.fill_(255)
        pa.purine_group_norm_fwd(z, None, None, z, m, r, G, 1e-5, act, ws=ws)
        assert torch.equal(z, y) and torch.equal(m, mean) and torch.equal(r, rstd)
    ws = _ws(pa, 1, case, dtype)
    dx = torch.full_like(x, float("nan"))
    pa.purine_group_norm_bwd(x, None, None, mean, rstd, y, dx, None, None, G, act, ws=ws)
    ws.fill_(255)
    pa.purine_group_norm_bwd(x, None, None, mean, rstd, y, y, None, None, G, act, ws=ws)
    assert torch.equal(y, dx)
