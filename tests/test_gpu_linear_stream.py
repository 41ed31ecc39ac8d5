"""Matrix products of many rows with a small matrix, bf16: against their definition in 64 bits, with ragged rows, columns and reductions,
rows apart in buffers whose other columns hold NaN, all options, results over the residual.

Bounds as for the other products: sums of C random products in fp32, 2e-8 sqrt(C) of the result's 2-norm, 1e-6 for the epilogue, and one rounding
to bf16, 2^-8.5. Both gradients and results are also the same bits on two calls."""
import pytest
import torch

import block_ref as ref

pytestmark = pytest.mark.gpu
DEV, BF16 = "cuda:0", torch.bfloat16

# rows, inputs, outputs: forward, data gradient or both are streams
CASES = [(4096, 8, 8), (4097, 16, 40), (6001, 24, 24), (16383, 96, 96), (20000, 88, 104), (50177, 160, 160), (70000, 64, 256), (100352, 192, 96), (33000, 128, 72),
         (150001, 64, 64), (30000, 32, 320)]
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


def _apart(t, extra):
    """The matrix in the first columns of a wider one of NaN."""
    if not extra:
        return t.clone()
    wide = torch.full((t.shape[0], t.shape[1] + extra), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, :t.shape[1]] = t
    return wide[:, :t.shape[1]]


def _near(got, want, products, scale, what):
    got = got.double()
    assert bool(torch.isfinite(got).all()), what
    tol = 2e-8 * products ** 0.5 + 1e-6 + 2 ** -8.5
    err = float((got - want).norm())
    assert err <= tol * float(scale), (what, err / float(scale), tol)


def _ws(pa, which, case):
    return torch.full((max(256, pa.purine_linear_workspace_bytes(which, *case, pa.PURINE_BF16)),), 255, dtype=torch.uint8, device=DEV)


@pytest.mark.parametrize("extra", [0, 24], ids=["dense", "apart"])
@pytest.mark.parametrize("case", CASES, ids=["x".join(map(str, c)) for c in CASES])
def test_stream(case, extra):
    import paper_1412_6249_amd as pa
    N, C, K = case
    g = torch.Generator(device=DEV).manual_seed(N + 3 * C + 7 * K)
    rnd = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    x, w, b, r, dy, pre_x, old = (v.to(BF16) for v in (rnd(N, C), rnd(K, C) * C ** -0.5, rnd(K), rnd(N, K), rnd(N, K), rnd(N, C), rnd(N, C)))
    z = x.double() @ w.double().t()
    dz = dy.double() @ w.double()
    xs, ws_, rs, dys, ps = (_apart(v, extra) for v in (x, w, r, dy, pre_x))
    for n, act in enumerate(ACTS):
        y, pre = (_apart(torch.full((N, K), float("nan"), dtype=BF16, device=DEV), extra) for _ in range(2))
        code = pa.ACTIVATIONS[act]
        if n % 2:                            # everything
            for _ in range(2):
                before = y.clone()
                pa.purine_linear_fwd(xs, ws_, b, rs, y, pre, code, ws=_ws(pa, 0, case))
            assert torch.equal(before, y)
            zb = z + b.double()
            _near(pre, zb, C, zb.norm(), (act, "pre"))
            want = ref.act(zb, act)
            _near(y, want + r.double(), C, (want.norm() ** 2 + r.double().norm() ** 2) ** 0.5, (act, "y"))
        else:                                # the least, and the residual in place
            pa.purine_linear_fwd(xs, ws_, None, None, y, None, code, ws=_ws(pa, 0, case))
            _near(y, ref.act(z, act), C, z.norm(), (act, "y"))
            over = _apart(r, extra)
            pa.purine_linear_fwd(xs, ws_, b, over, over, None, code, ws=_ws(pa, 0, case))
            want = ref.act(z + b.double(), act)
            _near(over, want + r.double(), C, (want.norm() ** 2 + r.double().norm() ** 2) ** 0.5, (act, "over"))
        beta = float(n % 2)
        dx = _apart(old, extra)
        pa.purine_linear_bwd_data(dys, ws_, None if act == "none" else ps, dx, code, beta, ws=_ws(pa, 1, case))
        slope = ref.slope(pre_x.double(), act)
        want = dz * slope
        # (the slope is exact to 1e-6 of 1)
        _near(dx, want + beta * old.double(), K, (want.norm() ** 2 + beta * old.double().norm() ** 2 + (1e-3 * dz.norm()) ** 2) ** 0.5, (act, "dx"))
        if extra:                            # nothing was written beside the matrices
            for v in (y, pre, dx):
                wide = v.as_strided((N, v.shape[1] + extra), (v.stride(0), 1))
                assert bool(torch.isnan(wide[:, v.shape[1]:]).all())
