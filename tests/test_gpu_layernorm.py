"""Layer norm forward and backward against the definition in 64 bits.

Tolerances, per element, follow from float32 sums of `cols` terms whose order is a tree over threads: a thread adds at
most `depth` terms one after the other, then at most ten halvings follow, so a sum is off by at most (depth + 10) u times
the sum of the terms' sizes, u = 2^-24.  Every other operation adds one u of its result, and the output type's own
rounding comes last.
"""

import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
OUT_U = {"f32": U, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}  # 24, 8 and 11 significant bits
TINY = {"f32": 0.0, "bf16": 0.0, "f16": 2.0 ** -25}  # half the smallest subnormal
EPS = 1e-5


def _dtype(t):
    import torch

    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[t]


def _strided(a, pad, dtype, shift=0):
    """The matrix on the GPU, rows `pad` apart, beginning `shift` elements into its memory; the rest is a marker."""
    import torch

    rows, cols = a.shape
    mem = torch.full((shift + rows * (cols + pad) + 8,), 77.0, dtype=dtype, device="cuda")
    view = mem[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    view.copy_(torch.from_numpy(a))
    return mem, view


def _f64(t):
    return t.detach().cpu().double().numpy()


def _depth(cols):
    return (16 if cols <= 16384 else -(-cols // 1024)) + 10


def _check(got, want, tol, what):
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (what, int(bad.sum()), np.abs(got - want)[bad][:4], tol[bad][:4], np.argwhere(bad)[:4])


def _stats(x):
    mean = x.mean(1, keepdims=True)
    var = ((x - mean) ** 2).mean(1, keepdims=True)
    return mean, 1.0 / np.sqrt(var + EPS)


SHAPES = [(1, 1), (3, 1), (1, 2), (5, 7), (4, 63), (9, 64), (7, 65), (130, 96), (6, 511), (6, 512), (5, 513), (3, 1000),
          (3, 1024), (2, 1025), (4, 2048), (3, 2056), (2, 4096), (2, 4097), (3, 8192), (2, 10007), (2, 16384), (2, 16385),
          (3, 40000), (1100, 24), (700, 160), (2500, 8)]


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
def test_forward(t, pad, shift):
    import torch
    import paper_2312_02493_amd as lib

    rng = np.random.default_rng(5 + pad)
    ctx = lib.NormContext(4096, 65536)
    for rows, cols in SHAPES:
        a = rng.standard_normal((rows, cols)) * (0.5 + rng.random((rows, 1)) * 3.0) + rng.standard_normal((rows, 1))
        if rows > 2:
            a[1] = 0.75  # a constant row
        mem_x, x = _strided(a.astype(np.float32), pad, _dtype(t), shift)
        mem_y, y = _strided(np.zeros((rows, cols), np.float32), pad, _dtype(t), shift)
        gamma_h = (1.0 + 0.2 * rng.standard_normal(cols)).astype(np.float32)
        beta_h = (0.3 * rng.standard_normal(cols)).astype(np.float32)
        flat = torch.zeros(2 * cols + 3, device="cuda")  # weights lie in a flat vector, off any boundary
        gamma, beta = flat[1:1 + cols], flat[2 + cols:2 + 2 * cols]
        gamma.copy_(torch.from_numpy(gamma_h))
        beta.copy_(torch.from_numpy(beta_h))
        xd = _f64(x)
        mean, rstd = _stats(xd)
        h = (xd - mean) * rstd
        d = _depth(cols)
        size = np.abs(xd).mean(1, keepdims=True)
        mean_off = (d + 2) * U * size
        h_off = (mean_off + 2 * U * (np.abs(xd) + np.abs(mean))) * rstd * (1 + np.abs(h)) + (d + 8) * U * np.abs(h)
        for use_gamma, use_beta in ((True, True), (False, False), (True, False)):
            mo, ro = torch.full((rows,), 9.0, device="cuda"), torch.full((rows,), 9.0, device="cuda")
            ctx.artopk_layernorm_forward(x, gamma if use_gamma else None, beta if use_beta else None, y,
                                         mo if use_beta else None, ro if use_beta else None, eps=EPS)
            g = gamma_h.astype(np.float64) if use_gamma else np.ones(cols)
            b = beta_h.astype(np.float64) if use_beta else np.zeros(cols)
            want = h * g + b
            tol = h_off * np.abs(g) + 2 * U * (np.abs(h * g) + np.abs(b)) + 1.01 * OUT_U[t] * np.abs(want) + TINY[t]
            tol = tol + 1.01 * OUT_U[t] * tol
            _check(_f64(y), want, tol, (t, rows, cols, pad, use_gamma))
            if use_beta:
                _check(_f64(mo)[:, None], mean, mean_off + U * np.abs(mean), ("mean", t, rows, cols))
                # rstd's relative error is half that of var + eps, whose terms are off by the differences' own errors
                rel = (d + 8) * U + (mean_off + 2 * U * (size + np.abs(mean))) * rstd * 2
                _check(_f64(ro)[:, None], rstd, rel * rstd, ("rstd", t, rows, cols))
        if pad:  # what lies between the rows
            m = mem_y.clone()
            m[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = 77.0
            assert bool((m == 77.0).all())


def _backward_reference(dy, x, gamma, mean, rstd):
    """(dx, dgamma, dbeta) and bounds of their errors before the outputs' roundings."""
    rows, cols = x.shape
    h = (x - mean) * rstd
    d = dy * gamma
    m1, m2 = d.mean(1, keepdims=True), (d * h).mean(1, keepdims=True)
    dx = rstd * (d - m1 - h * m2)
    dep = _depth(cols)
    h_off = 3 * U * (np.abs(x) + np.abs(mean)) * rstd + U * np.abs(h)
    m1_off = (dep + 3) * U * np.abs(d).mean(1, keepdims=True)
    m2_off = (dep + 4) * U * np.abs(d * h).mean(1, keepdims=True) + (np.abs(d) * h_off).mean(1, keepdims=True)
    dx_off = rstd * (m1_off + np.abs(h) * m2_off + np.abs(m2) * h_off + 4 * U * (np.abs(d) + np.abs(m1) + np.abs(h * m2)))
    # a column's sum is cut into shares, each added row by row
    dep = rows + 8
    return dx, (dy * h).sum(0), dy.sum(0), dx_off, (np.abs(dy) * h_off).sum(0) + dep * U * np.abs(dy * h).sum(0), \
        dep * U * np.abs(dy).sum(0)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad,shift", [(0, 0), (8, 0), (3, 1)])
def test_backward(t, pad, shift):
    import torch
    import paper_2312_02493_amd as lib

    rng = np.random.default_rng(11 + pad)
    ctx = lib.NormContext(4096, 65536)
    for at, (rows, cols) in enumerate(SHAPES):
        a = rng.standard_normal((rows, cols)) * 1.5 + rng.standard_normal((rows, 1))
        _, x = _strided(a.astype(np.float32), pad, _dtype(t), shift)
        _, dy = _strided(rng.standard_normal((rows, cols)).astype(np.float32), pad, _dtype(t), shift)
        mem_dx, dx = _strided(np.zeros((rows, cols), np.float32), pad, _dtype(t), shift)
        gamma_h = (1.0 + 0.2 * rng.standard_normal(cols)).astype(np.float32)
        xd, dyd = _f64(x), _f64(dy)
        mean, rstd = (v.astype(np.float32) for v in _stats(xd))
        mo, ro = torch.from_numpy(mean[:, 0].copy()).cuda(), torch.from_numpy(rstd[:, 0].copy()).cuda()
        gt = ["f32", "bf16", "f16"][at % 3]
        flat = torch.full((2 * cols + 3,), 0.5, dtype=_dtype(gt), device="cuda")  # a worker's flat gradient vector
        dgamma, dbeta = flat[1:1 + cols], flat[2 + cols:2 + 2 * cols]
        gamma = torch.from_numpy(gamma_h).cuda()
        for use_gamma, accumulate in ((True, False), (False, True)):
            before = _f64(flat).copy()
            ctx.artopk_layernorm_backward(dy, x, gamma if use_gamma else None, mo, ro, dx, dgamma, dbeta, accumulate=accumulate)
            g = gamma_h.astype(np.float64) if use_gamma else np.ones(cols)
            wx, wg, wb, ox, og, ob = _backward_reference(dyd, xd, g, mean.astype(np.float64), rstd.astype(np.float64))
            _check(_f64(dx), wx, ox + 1.01 * OUT_U[t] * (np.abs(wx) + ox) + TINY[t], ("dx", t, rows, cols))
            after = _f64(flat)
            for want, off, s in ((wg, og, slice(1, 1 + cols)), (wb, ob, slice(2 + cols, 2 + 2 * cols))):
                if accumulate:
                    want = want + before[s]
                    off = off + U * (np.abs(want) + np.abs(before[s]))
                _check(after[s], want, off + 1.01 * OUT_U[gt] * (np.abs(want) + off) + TINY[gt], ("weights", gt, rows, cols))
            assert after[0] == after[1 + cols] == after[-1] == 0.5
        if pad:
            m = mem_dx.clone()
            m[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = 77.0
            assert bool((m == 77.0).all())
        # each output by itself, and twice the same bits
        again, more = torch.zeros_like(dx), torch.zeros_like(flat)
        ctx.artopk_layernorm_backward(dy, x, None, mo, ro, again)
        assert torch.equal(again.view(rows, cols), dx)
        ctx.artopk_layernorm_backward(dy, x, None, mo, ro, None, more[1:1 + cols], None)
        first = more.clone()
        ctx.artopk_layernorm_backward(dy, x, None, mo, ro, None, more[1:1 + cols], None)
        assert torch.equal(first, more) and not bool(more[1 + cols:].any())
        ctx.artopk_layernorm_backward(dy, x, None, mo, ro, None, None, more[2 + cols:2 + 2 * cols])
        _check(_f64(more[2 + cols:2 + 2 * cols]), wb, ob + 1.01 * OUT_U[gt] * (np.abs(wb) + ob) + TINY[gt], ("dbeta", rows, cols))


def test_backward_against_differences():
    """The gradients of sum(w y) by central differences of the definition in 64 bits, eps included."""
    import torch
    import paper_2312_02493_amd as lib

    rng = np.random.default_rng(3)
    rows, cols = 3, 11
    x = rng.standard_normal((rows, cols)).astype(np.float32).astype(np.float64)
    w = rng.standard_normal((rows, cols)).astype(np.float32).astype(np.float64)
    gamma = (1.0 + 0.3 * rng.standard_normal(cols)).astype(np.float32).astype(np.float64)
    beta = np.zeros(cols)

    def loss(x, gamma, beta):
        mean, rstd = _stats(x)
        return float((w * ((x - mean) * rstd * gamma + beta)).sum())

    def differences(at, f, h=1e-5):
        out = np.zeros_like(at)
        for i in np.ndindex(at.shape):
            up, down = at.copy(), at.copy()
            up[i] += h
            down[i] -= h
            out[i] = (f(up) - f(down)) / (2 * h)
        return out

    ctx = lib.NormContext(rows, cols)
    xt, wt = (torch.from_numpy(v).float().cuda() for v in (x, w))
    gt, bt = (torch.from_numpy(v).float().cuda() for v in (gamma, beta))
    y, dx = torch.empty_like(xt), torch.empty_like(xt)
    mo, ro = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    dg, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    ctx.artopk_layernorm_forward(xt, gt, bt, y, mo, ro, eps=EPS)
    ctx.artopk_layernorm_backward(wt, xt, gt, mo, ro, dx, dg, db)
    # the differences' own error, h^2 and 2^-52 / h, is below 1e-8; the kernels' is some 30 u of values around 1
    for got, want in ((dx, differences(x, lambda v: loss(v, gamma, beta))), (dg, differences(gamma, lambda v: loss(x, v, beta))),
                      (db, differences(beta, lambda v: loss(x, gamma, v)))):
        np.testing.assert_allclose(_f64(got), want, rtol=0, atol=64 * U * 4)


def test_special_values_stay_in_their_row():
    import torch
    import paper_2312_02493_amd as lib

    ctx = lib.NormContext(8, 4096)
    for cols in (40, 4096):
        x = torch.randn(8, cols, device="cuda")
        x[2, 3], x[5, cols - 1] = float("inf"), float("nan")
        x[6] *= 1e18  # squares up to 1e37: still sums
        x[7] *= 1e-30
        y = torch.empty_like(x)
        mo, ro = torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
        ctx.artopk_layernorm_forward(x, None, None, y, mo, ro, eps=EPS)
        assert bool(torch.isnan(y[5]).all()) and bool(torch.isnan(y[2]).any())
        assert bool(torch.isfinite(y[[0, 1, 3, 4, 6, 7]]).all())
        dx = torch.empty_like(x)
        ctx.artopk_layernorm_backward(torch.ones_like(x), x, None, mo, ro, dx)
        assert bool(torch.isfinite(dx[[0, 1, 3, 4, 6, 7]]).all())


def test_rows_of_none():
    import torch
    import paper_2312_02493_amd as lib

    ctx = lib.NormContext(4, 33)
    x, y = torch.empty(0, 33, device="cuda"), torch.empty(0, 33, device="cuda")
    none = torch.empty(0, device="cuda")
    ctx.artopk_layernorm_forward(x, None, None, y)
    dg, db = torch.full((33,), 4.0, device="cuda"), torch.full((33,), 5.0, device="cuda")
    ctx.artopk_layernorm_backward(x, x, None, none, none, y, dg, db, accumulate=True)
    assert bool((dg == 4.0).all()) and bool((db == 5.0).all())
    ctx.artopk_layernorm_backward(x, x, None, none, none, y, dg, db)
    assert not bool(dg.any()) and not bool(db.any())


def test_refusals():
    import torch
    import paper_2312_02493_amd as lib

    ctx = lib.NormContext(8, 64)
    x, y = torch.ones(8, 64, device="cuda"), torch.zeros(8, 64, device="cuda")
    g, m = torch.ones(64, device="cuda"), torch.ones(8, device="cuda")

    def refused(text, f, *a, **k):
        with pytest.raises(lib.ArTopkError, match=text) as e:
            f(*a, **k)
        assert e.value.code == -1

    fwd, bwd = ctx.artopk_layernorm_forward, ctx.artopk_layernorm_backward
    refused("rows=9", fwd, torch.ones(9, 64, device="cuda"), None, None, torch.zeros(9, 64, device="cuda"))
    refused("cols=65", fwd, torch.ones(2, 65, device="cuda"), None, None, torch.zeros(2, 65, device="cuda"))
    refused("overlap", fwd, x, None, None, x)
    refused("overlap", fwd, x, g, None, y, m, m)
    refused("overlap", fwd, x, y.view(-1)[:64], None, y)
    refused("eps", fwd, x, None, None, y, eps=-1.0)
    refused("eps", fwd, x, None, None, y, eps=float("nan"))
    refused("shape or type", fwd, x, None, None, torch.zeros(8, 63, device="cuda"))
    refused("shape or type", fwd, x, None, None, y.half())
    refused("side by side", fwd, x.t()[:8, :8], None, None, y[:, :8])
    refused("not taken", fwd, x.double(), None, None, y.double())
    refused("gamma is not a contiguous", fwd, x, g[:63], None, y)
    refused("gamma is torch.float16", fwd, x, g.half(), None, y)
    refused("8 apart and 16 long", fwd, torch.as_strided(x, (4, 16), (8, 1)), None, None, torch.zeros(4, 16, device="cuda"))
    refused("all NULL", bwd, x, x, g, m, m, None)
    refused("mean or rstd", bwd, x, x, g, None, m, y)
    refused("overlap", bwd, x, x, g, m, m, x)
    refused("overlap", bwd, x, x, g, m, m, y, g)
    refused("different types", bwd, x, x, g, m, m, y, torch.ones(64, device="cuda"), torch.ones(64, device="cuda").half())
    assert bool((y == 0).all())
    raw = lib.load_library()
    p = lambda t: C.c_void_p(t.data_ptr())  # noqa: E731
    assert raw.artopk_layernorm_forward(None, p(x), 64, 0, 8, 64, None, None, 1e-5, p(y), 64, None, None) == -1
    assert raw.artopk_layernorm_forward(ctx._h, None, 64, 0, 8, 64, None, None, 1e-5, p(y), 64, None, None) == -1
    assert raw.artopk_layernorm_forward(ctx._h, p(x), 64, 3, 8, 64, None, None, 1e-5, p(y), 64, None, None) == -1
    assert raw.artopk_layernorm_forward(ctx._h, p(x), 64, 0, -1, 64, None, None, 1e-5, p(y), 64, None, None) == -1
    assert raw.artopk_layernorm_forward(ctx._h, C.c_void_p(x.data_ptr() + 2), 64, 0, 7, 64, None, None, 1e-5, p(y), 64, None,
                                        None) == -1
    for bad in ((0, 4), (4, 0), (1 << 31, 4), (4, 1 << 31)):
        with pytest.raises(lib.ArTopkError):
            lib.NormContext(*bad)
    fwd(x, g, None, y, m.clone(), m.clone())  # still works
    torch.cuda.synchronize()


def test_on_its_own_stream_and_in_a_graph():
    import torch
    import paper_2312_02493_amd as lib

    stream = torch.cuda.Stream()
    x = torch.randn(64, 768, device="cuda", dtype=torch.bfloat16)
    dy = torch.randn(64, 768, device="cuda", dtype=torch.bfloat16)
    y, dx = torch.zeros_like(x), torch.zeros_like(x)
    mo, ro, dg = torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda"), torch.zeros(768, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        ctx = lib.NormContext(64, 768)

        def go():
            ctx.artopk_layernorm_forward(x, None, None, y, mo, ro)
            ctx.artopk_layernorm_backward(dy, x, None, mo, ro, dx, dg, None, accumulate=True)

        go()
        stream.synchronize()
        want = [v.clone() for v in (y, dx, dg)]
        graph = torch.cuda.CUDAGraph()
        dg.zero_()
        stream.synchronize()
        with torch.cuda.graph(graph, stream=stream):
            go()
        for turn in range(3):
            y.zero_()
            dx.zero_()
            dg.zero_()
            graph.replay()
            stream.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, (y, dx, dg))), turn


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols", [(3, 9), (2, 515), (3, 1111), (2, 10001)])
def test_what_lies_between_rows_does_not_matter(t, rows, cols):
    """The same bits with NaN between the rows as with zeros."""
    import torch
    import paper_2312_02493_amd as lib

    rng = np.random.default_rng(9)
    ctx = lib.NormContext(rows, cols)
    a, d = (rng.standard_normal((rows, cols)).astype(np.float32) for _ in range(2))
    for pad in (1, 8, 23):
        found = []
        for between in (0.0, float("nan")):
            views = []
            for v in (a, d):
                mem, view = _strided(v, pad, _dtype(t))
                keep = view.clone()
                mem.fill_(between)
                view.copy_(keep)
                views.append(view)
            y, dx = torch.zeros(rows, cols, dtype=_dtype(t), device="cuda"), torch.zeros(rows, cols, dtype=_dtype(t), device="cuda")
            mean, rstd, dg, db = (torch.zeros(k, device="cuda") for k in (rows, rows, cols, cols))
            ctx.artopk_layernorm_forward(views[0], None, None, y, mean, rstd)
            ctx.artopk_layernorm_backward(views[1], views[0], None, mean, rstd, dx, dg, db)
            found.append((y, mean, rstd, dx, dg, db))
        for u, v in zip(*found):
            assert torch.equal(u, v) and not bool(u.isnan().any()), (pad, u.shape)


def test_tensors_of_the_host_are_refused():
    import torch
    import paper_2312_02493_amd as lib

    ctx = lib.NormContext(4, 8)
    x, y, v, w = torch.zeros(4, 8, device="cuda"), torch.zeros(4, 8, device="cuda"), torch.zeros(8, device="cuda"), torch.zeros(4, device="cuda")
    ctx.artopk_layernorm_forward(x, v, v, y, w, w.clone())
    for args in ((x.cpu(), v, v, y), (x, v.cpu(), v, y), (x, v, v.cpu(), y), (x, v, v, y.cpu()), (x, v, v, y, w.cpu()), (x, v, v, y, w, w.cpu())):
        with pytest.raises(lib.ArTopkError, match="cpu"):
            ctx.artopk_layernorm_forward(*args)
    good = [y, x, v, w, w.clone(), torch.zeros_like(x), v.clone(), v.clone()]
    ctx.artopk_layernorm_backward(*good)
    for i in range(len(good)):
        with pytest.raises(lib.ArTopkError, match="cpu"):
            ctx.artopk_layernorm_backward(*good[:i], good[i].cpu(), *good[i + 1:])
