"""Matrices whose norm lies far below eps, or that their coefficients shrink: X is small by definition, and keeps its bits.

The tolerance is that of tests/test_gpu_matrices.py; every matrix's scale brings its result back to a size that its element type
holds."""

import numpy as np
import pytest

from tests.test_gpu_matrices import OPERAND_U, OUT_U, USUAL, _code, _dtype, reference, tolerance

pytestmark = pytest.mark.gpu

# routes: one launch on one unit; launches of their own; two steps at once; tiles beyond 64
LAYOUTS = {"one-unit": [(64, 64), (30, 50), (70, 33)], "launches": [(200, 320), (320, 200), (65, 300)],
           "pairs": [(130, 2000), (2000, 130)], "large": [(1500, 700)]}
NORMS = [1.0, 1e-3, 1e-7, 1e-12, 1e-20, 1e-30]  # of a matrix, next to eps


def _run(t, products, shapes, norms, steps, co, seed):
    """(matrix, result and the definition's, iterates' norms) of every shape with every norm, all in one handle; eps is 100."""
    import torch
    import paper_2312_02493_amd as lib

    eps = 100.0
    rng = np.random.default_rng(seed)
    mats, values, at = [], [], 0
    for r, c in shapes:
        for size in norms:
            g = rng.standard_normal((r, c))
            g *= eps * size / np.linalg.norm(g)
            grown = 1.0
            for row in [co] * steps if np.ndim(co) == 1 else co:
                grown = min(1.0, grown * abs(row[0])) if size >= 1.0 else grown * abs(row[0])
            mats.append((at, r, c, float(np.float32(1.0 / min(1.0, size * grown)))))
            values.append(g.ravel())
            at += r * c
    x = torch.from_numpy(np.concatenate(values).astype(np.float32)).cuda().to(_dtype(t))
    out = torch.zeros_like(x)
    lib.MatrixContext(mats, at, _code(t), products).artopk_orthogonalize(x, out, steps=steps, coefficients=co, eps=eps)
    got, xs = out.cpu().double().numpy(), x.cpu().double().numpy()
    for at, r, c, scale in mats:
        want, iterates = reference(xs[at:at + r * c].reshape(r, c), steps, co, eps)
        yield (r, c, scale), got[at:at + r * c].reshape(r, c), scale * want, iterates


@pytest.mark.parametrize("t,products", [("f32", 1), ("f32", 0), ("bf16", 0), ("bf16", 1)])
@pytest.mark.parametrize("route", sorted(LAYOUTS))
def test_norms_below_eps(t, products, route):
    for what, got, want, iterates in _run(t, products, LAYOUTS[route], NORMS, 5, USUAL, 50):
        off = np.linalg.norm(got - want) / np.linalg.norm(want)
        # (two steps at once round a little more)
        assert off <= 2 * tolerance(iterates, OPERAND_U[products]) + 2 * OUT_U[t], (what, off)


@pytest.mark.parametrize("route", sorted(LAYOUTS))
def test_iterates_that_shrink(route):
    for co in ((0.01, 0.0, 0.0), (0.25, -0.1, 0.01)):
        for what, got, want, iterates in _run("f32", 1, LAYOUTS[route], [1.0, 1e-6], 5, co, 51):
            off = np.linalg.norm(got - want) / np.linalg.norm(want)
            assert off <= 2 * tolerance(iterates, OPERAND_U[1], co[0]) + 2 * OUT_U["f32"], (what, co, off)


@pytest.mark.parametrize("route", ["one-unit", "launches", "pairs"])
def test_from_far_below_eps_to_full_size(route):
    """So many steps that a norm of a thousandth of eps, and one of 1e-9, grow until the steps are no longer linear."""
    for size, steps in ((1e-3, 7), (1e-9, 18)):
        for what, got, want, iterates in _run("f32", 1, LAYOUTS[route], [size], steps, (1.875, -1.25, 0.375) if steps == 7 else USUAL, 52):
            off = np.linalg.norm(got - want) / np.linalg.norm(want)
            # up to full size every step keeps relative errors, then a handful of steps multiplies them by up to the slope
            slope = 1.875 if steps == 7 else USUAL[0]
            full = next((k for k, v in enumerate(iterates) if v > 0.1), steps)
            tol = 4 * (OPERAND_U[1] + 2.0 ** -22) * (steps + 1) * slope ** (steps - full) * max(iterates) / iterates[-1]
            assert off <= 2 * tol, (what, off, tol)


@pytest.mark.parametrize("route", sorted(LAYOUTS))
def test_polynomials_that_leave_nothing(route):
    import torch
    import paper_2312_02493_amd as lib

    mats, at = [], 0
    for r, c in LAYOUTS[route]:
        mats.append((at, r, c))
        at += r * c
    x, out = torch.randn(at, device="cuda"), torch.full((at,), 7.0, device="cuda")
    ctx = lib.MatrixContext(mats, at)
    for co in ((0.0, 0.0, 0.0), (1e-30, 0.0, 0.0)):
        for steps in (1, 2, 5):
            ctx.artopk_orthogonalize(x, out.fill_(7.0), steps=steps, coefficients=co)
            assert float(out.abs().max()) <= (0.0 if co[0] == 0.0 else 1e-29), (co, steps)
