"""An AdamW step whose tensors have more elements than a launch should take: their order, which the dither goes by, and their values."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV, BLOCK = "cuda:0", 256


def _states(n):
    codes = [torch.zeros(n, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2)]
    scales = [torch.zeros((n + BLOCK - 1) // BLOCK, device=DEV) for _ in range(2)]
    return codes + scales


def test_four_tensors_of_two_to_the_31():
    import paper_1412_6249_amd as pa
    desc = pa.adamw_desc(1e-2, step=3, seed=11, dither=True, weight_decay=0.0)
    g = torch.Generator(device=DEV).manual_seed(3)
    last_w, last_dw = (torch.randn(70000, generator=g, device=DEV).bfloat16() for _ in range(2))
    ends = []
    for n in ((1 << 31) - 1, 300):
        sizes = [n] * 4
        w = [torch.ones(k, dtype=torch.bfloat16, device=DEV) for k in sizes] + [last_w.clone()]
        dw = [torch.full((k,), 0.5, dtype=torch.bfloat16, device=DEV) for k in sizes] + [last_dw]
        m, v, ms, vs = (list(t) for t in zip(*(_states(t.numel()) for t in w)))
        pa.purine_adamw_step(desc, pa.adamw_params(w, dw, m, v, ms, vs))
        # one step from zero states: m = 0.1 g, v = 0.001 g^2; every element of the first tensors moves alike
        move = 1e-2 * (0.1 * 0.5 / (1 - 0.9 ** 3)) / ((0.001 * 0.25 / (1 - 0.999 ** 3)) ** 0.5 + 1e-8)
        want = float(torch.tensor(1.0 - move).bfloat16())
        for t in w[:4]:
            assert float(t.min()) == want and float(t.max()) == want
        ends.append([t[4].view(torch.uint8) if t[4].element_size() == 1 else t[4] for t in (w, m, v, ms, vs)])
        del w, dw, m, v, ms, vs
    assert all(torch.equal(a, b) for a, b in zip(*ends))
