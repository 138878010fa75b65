"""Layer norms of more rows than a launch has room for at once: every block takes several, and the weights' gradients gather
over them.  Against the definition in 64 bits on the GPU, within the bounds of tests/test_gpu_layernorm.py."""

import numpy as np
import pytest

from tests.test_gpu_layernorm import EPS, OUT_U, TINY, U, _depth, _dtype

pytestmark = pytest.mark.gpu

#: rows x columns of every shape of row (threads to a row and elements to a thread) that many rows take; 256 compute units
#: hold 2048 blocks of 256 threads forward and 1024 backward, four rows each where a wave holds one
SHAPES = [(9001, 40), (8301, 512), (8501, 1000), (4201, 1111), (2301, 2048), (2503, 3001), (4099, 2056), (2100, 4096), (1301, 6007),
          (1101, 8192), (1027, 10007), (1100, 16384), (519, 16400)]
#: distance beyond a row's length, and where it begins: x, dy, and what is written
PLACES = [((0, 0), (0, 0), (0, 0)), ((8, 0), (8, 0), (8, 0)), ((3, 1), (0, 0), (0, 0)), ((0, 0), (3, 1), (0, 0)), ((0, 0), (0, 0), (3, 1))]


def _rows(values, place):
    """(memory, view): the values as rows, with a marker around them."""
    import torch

    (pad, shift), (rows, cols) = place, values.shape
    mem = torch.full((shift + rows * (cols + pad) + 8,), 77.0, dtype=values.dtype, device="cuda")
    view = mem[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(values)
    return mem, view


def _marker_stays(mem, place, shape):
    (pad, shift), (rows, cols) = place, shape
    m = mem.clone()
    m[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = 77.0
    return bool((m == 77.0).all())


def _check(got, want, off, u, tiny, what):
    bad = ~((got.double() - want).abs() <= off + 1.01 * u * (want.abs() + off) + tiny)
    assert not bool(bad.any()), (what, int(bad.sum()), (got.double() - want).abs()[bad][:4].tolist())


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("place", [0, 1, 2, 4])
def test_forward(t, place):
    import torch
    import paper_2312_02493_amd as lib

    gen = torch.Generator(device="cuda").manual_seed(70 + place)
    at_x, _, at_y = PLACES[place]
    ctx = lib.NormContext(9100, 16400)
    for rows, cols in SHAPES:
        v = torch.randn(rows, cols, generator=gen, device="cuda") * (0.5 + 3.0 * torch.rand(rows, 1, generator=gen, device="cuda"))
        v += torch.randn(rows, 1, generator=gen, device="cuda")
        v[rows // 2] = 0.75
        _, x = _rows(v.to(_dtype(t)), at_x)
        mem, y = _rows(torch.zeros(rows, cols, dtype=_dtype(t), device="cuda"), at_y)
        gamma = 1.0 + 0.2 * torch.randn(cols, generator=gen, device="cuda")
        beta = 0.3 * torch.randn(cols, generator=gen, device="cuda")
        mo, ro = torch.full((rows,), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda")
        ctx.artopk_layernorm_forward(x, gamma, beta, y, mo, ro, eps=EPS)
        xd, g, b = x.double(), gamma.double(), beta.double()
        mean = xd.mean(1, keepdim=True)
        rstd = 1.0 / ((xd - mean).square().mean(1, keepdim=True) + EPS).sqrt()
        h = (xd - mean) * rstd
        d = _depth(cols)
        size = xd.abs().mean(1, keepdim=True)
        mean_off = (d + 2) * U * size
        h_off = (mean_off + 2 * U * (xd.abs() + mean.abs())) * rstd * (1 + h.abs()) + (d + 8) * U * h.abs()
        want = h * g + b
        _check(y, want, h_off * g.abs() + 2 * U * ((h * g).abs() + b.abs()), OUT_U[t], TINY[t], (t, rows, cols))
        _check(mo.view(-1, 1), mean, mean_off, U, 0.0, ("mean", t, rows, cols))
        rel = (d + 8) * U + (mean_off + 2 * U * (size + mean.abs())) * rstd * 2
        _check(ro.view(-1, 1), rstd, rel * rstd, U, 0.0, ("rstd", t, rows, cols))
        assert _marker_stays(mem, at_y, (rows, cols))


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("place", range(len(PLACES)))
def test_backward(t, place):
    import torch
    import paper_2312_02493_amd as lib

    gen = torch.Generator(device="cuda").manual_seed(80 + place)
    at_x, at_dy, at_dx = PLACES[place]
    ctx = lib.NormContext(9100, 16400)
    for at, (rows, cols) in enumerate(SHAPES):
        v = 1.5 * torch.randn(rows, cols, generator=gen, device="cuda") + torch.randn(rows, 1, generator=gen, device="cuda")
        _, x = _rows(v.to(_dtype(t)), at_x)
        _, dy = _rows(torch.randn(rows, cols, generator=gen, device="cuda").to(_dtype(t)), at_dy)
        mem, dx = _rows(torch.zeros(rows, cols, dtype=_dtype(t), device="cuda"), at_dx)
        gamma = 1.0 + 0.2 * torch.randn(cols, generator=gen, device="cuda")
        xd, dyd = x.double(), dy.double()
        mo = xd.mean(1).float()
        ro = (1.0 / ((xd - xd.mean(1, keepdim=True)).square().mean(1) + EPS).sqrt()).float()
        gt = ["f32", "bf16", "f16"][at % 3]
        flat = torch.full((2 * cols + 3,), 0.5, dtype=_dtype(gt), device="cuda")  # a worker's flat gradient vector
        dgamma, dbeta = flat[1:1 + cols], flat[2 + cols:2 + 2 * cols]
        mean, rstd = mo.double().view(-1, 1), ro.double().view(-1, 1)
        h = (xd - mean) * rstd
        h_off = 3 * U * (xd.abs() + mean.abs()) * rstd + U * h.abs()
        deep = rows + 8
        sums = (((dyd * h).sum(0), (dyd.abs() * h_off).sum(0) + deep * U * (dyd * h).abs().sum(0)),
                (dyd.sum(0), deep * U * dyd.abs().sum(0)))
        for accumulate in (False, True):
            before = flat.double()
            ctx.artopk_layernorm_backward(dy, x, gamma, mo, ro, dx, dgamma, dbeta, accumulate=accumulate)
            d = dyd * gamma.double()
            m1, m2 = d.mean(1, keepdim=True), (d * h).mean(1, keepdim=True)
            dep = _depth(cols)
            m1_off = (dep + 3) * U * d.abs().mean(1, keepdim=True)
            m2_off = (dep + 4) * U * (d * h).abs().mean(1, keepdim=True) + (d.abs() * h_off).mean(1, keepdim=True)
            off = rstd * (m1_off + h.abs() * m2_off + m2.abs() * h_off + 4 * U * (d.abs() + m1.abs() + (h * m2).abs()))
            _check(dx, rstd * (d - m1 - h * m2), off, OUT_U[t], TINY[t], ("dx", t, rows, cols))
            for got, s, (want, off) in zip((dgamma, dbeta), (slice(1, 1 + cols), slice(2 + cols, 2 + 2 * cols)), sums):
                if accumulate:
                    want = want + before[s]
                    off = off + U * (want.abs() + before[s].abs())
                _check(got, want, off, OUT_U[gt], TINY[gt], ("weights", gt, rows, cols))
            assert float(flat[0]) == float(flat[1 + cols]) == float(flat[-1]) == 0.5
        assert _marker_stays(mem, at_dx, (rows, cols))
        more = torch.zeros(2 * cols, device="cuda")  # the weights' gradients alone, one by one
        ctx.artopk_layernorm_backward(dy, x, None, mo, ro, None, more[:cols], None)
        ctx.artopk_layernorm_backward(dy, x, None, mo, ro, None, None, more[cols:])
        for got, (want, off) in zip((more[:cols], more[cols:]), sums):
            _check(got, want, off, U, 0.0, ("alone", t, rows, cols))


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_the_same_bits_from_the_same_places(t):
    """Same sizes, types and places in memory, to the sixteen bytes: the same bits, at whatever addresses."""
    import torch
    import paper_2312_02493_amd as lib

    gen = torch.Generator(device="cuda").manual_seed(90)
    for rows, cols in ((9, 1111), (4201, 1111), (2301, 2048), (700, 40)):
        ctx = lib.NormContext(rows, cols)
        v, d = (torch.randn(rows, cols, generator=gen, device="cuda").to(_dtype(t)) for _ in range(2))
        for place in ((0, 0), (3, 1)):
            found = []
            for _ in range(3):
                _, x = _rows(v, place)
                _, dy = _rows(d, place)
                _, y = _rows(torch.zeros_like(v), place)
                _, dx = _rows(torch.zeros_like(v), place)
                mean, rstd, dg, db = (torch.zeros(k, device="cuda") for k in (rows, rows, cols, cols))
                ctx.artopk_layernorm_forward(x, None, None, y, mean, rstd)
                ctx.artopk_layernorm_backward(dy, x, None, mean, rstd, dx, dg, db)
                found.append([a.clone() for a in (y, mean, rstd, dx, dg, db)])
            for other in found[1:]:
                assert all(torch.equal(a, b) for a, b in zip(found[0], other)), (rows, cols, place)
