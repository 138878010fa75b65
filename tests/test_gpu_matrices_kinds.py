"""The kind of products that bfloat16 takes by default is each matrix's own: matrices of fewer than 64 rows keep float32's
accuracy whatever lies beside them in the vector."""

import numpy as np
import pytest

from tests.test_gpu_matrices import OPERAND_U, USUAL, _code, _dtype, _gradients, layout, reference, tolerance

pytestmark = pytest.mark.gpu

FEW = [(16, 700), (700, 24), (48, 1100), (63, 64)]
MANY = [(300, 520), (600, 530)]


def _few_and_many():
    """A vector with both, in turn: (matrices, elements)."""
    return layout([FEW[0], MANY[0], FEW[1], FEW[2], MANY[1], FEW[3]])


def test_few_rows_beside_many():
    """The same bits as handles of either kind alone, for both entry points."""
    import torch
    import paper_2312_02493_amd as lib

    mats, n = _few_and_many()
    x = torch.from_numpy(_gradients(np.random.default_rng(40), [m[1:3] for m in mats], n)).cuda()
    groups = [([m for m in mats if min(m[1:3]) < 64], lib.ARTOPK_PRODUCTS_SPLIT),
              ([m for m in mats if min(m[1:3]) >= 64], lib.ARTOPK_PRODUCTS_HALF)]
    b = torch.bfloat16

    def both(ctx):
        out, w, m = torch.full_like(x, 7.0).to(b), x.to(b), torch.ones_like(x)
        ctx.artopk_orthogonalize(x.to(b), out)
        ctx.artopk_muon_step(w, m, 2 * x, eta=0.1, decay=0.01, eta_rest=0.1)
        ctx.artopk_orthogonalize(x.to(b), out)
        return out, w, m

    out, w, m = both(lib.MatrixContext(mats, n, _code("bf16")))
    outside = torch.ones(n, dtype=torch.bool, device="cuda")
    for part, kind in groups:
        out1, w1, m1 = both(lib.MatrixContext(part, n, _code("bf16"), kind))
        assert torch.equal(m, m1)
        for at, r, c, _ in part:
            s = slice(at, at + r * c)
            outside[s] = False
            assert torch.equal(out[s], out1[s]) and torch.equal(w[s], w1[s]), (r, c)
    assert bool((out[outside] == 7.0).all())


def test_steps_from_zero_weights_of_few_rows():
    """New weights are the scaled direction itself: off by no more than SPLIT may be beyond what rounding the exact direction
    to bfloat16 leaves (a tenth more of it: over the 4000 elements and more of a matrix, the roundings of values a little off have
    the same mean square to within 2 %)."""
    import torch
    import paper_2312_02493_amd as lib

    mats, n = _few_and_many()
    u = _gradients(np.random.default_rng(41), [m[1:3] for m in mats], n)
    w = torch.zeros(n, dtype=_dtype("bf16"), device="cuda")
    lib.MatrixContext(mats, n, _code("bf16")).artopk_muon_step(w, torch.zeros(n, device="cuda"), torch.from_numpy(u).cuda(), eta=0.5,
                                                               mu=0.9, nesterov=False)
    got = w.cpu().double().numpy()
    for at, r, c, scale in mats:
        want, norms = reference(u[at:at + r * c].astype(np.float64).reshape(r, c))
        want *= -0.5 * scale
        own = np.linalg.norm(torch.from_numpy(want).bfloat16().double().numpy() - want)
        off = np.linalg.norm(got[at:at + r * c].reshape(r, c) - want)
        if min(r, c) < 64:
            assert off <= tolerance(norms, OPERAND_U[1]) * np.linalg.norm(want) + 1.1 * own, (r, c, off, own)


@pytest.mark.parametrize("steps", [0, 1, 4])
def test_steps_of_both_kinds_in_one_handle(steps):
    import torch
    import paper_2312_02493_amd as lib

    mats, n = _few_and_many()
    x = torch.from_numpy(_gradients(np.random.default_rng(42), [m[1:3] for m in mats], n)).cuda().to(torch.bfloat16)
    out = torch.full_like(x, 7.0)
    lib.MatrixContext(mats, n, _code("bf16")).artopk_orthogonalize(x, out, steps=steps)
    got, xs = out.cpu().double().numpy(), x.cpu().double().numpy()
    for at, r, c, scale in mats:
        want, norms = reference(xs[at:at + r * c].reshape(r, c), steps, USUAL)
        off = np.linalg.norm(got[at:at + r * c].reshape(r, c) - scale * want) / np.linalg.norm(scale * want)
        # HALF of 64 rows and more: some 2e-3 is what it is known to leave; twice that is taken
        kind = tolerance(norms, OPERAND_U[1]) if min(r, c) < 64 else 4e-3
        assert off <= kind + 2.0 ** -8, (r, c, off)
