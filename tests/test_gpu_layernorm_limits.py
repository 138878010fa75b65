"""Layer norm at the ends of what its arguments may be."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def test_every_finite_eps_is_taken():
    import torch
    import paper_2312_02493_amd as lib

    ctx = lib.NormContext(4, 100)
    x = torch.randn(4, 100, device="cuda")
    y, mean, rstd = torch.empty_like(x), torch.empty(4, device="cuda"), torch.empty(4, device="cuda")
    xd = x.cpu().double().numpy()
    for eps in (1e-45, 1e30, 1.1e30, 3.4e38):
        ctx.artopk_layernorm_forward(x, None, None, y, mean, rstd, eps=eps)
        want = 1.0 / np.sqrt(xd.var(1) + float(np.float32(eps)))
        # sums of 100 terms, a square root and a quotient
        assert (np.abs(rstd.cpu().double().numpy() - want) <= 40 * U * want).all(), eps
    for eps in (float("inf"), float("nan"), -1e-45):
        with pytest.raises(lib.ArTopkError, match="eps"):
            ctx.artopk_layernorm_forward(x, None, None, y, mean, rstd, eps=eps)


def test_more_columns_than_a_launch_has_threads_for_at_once():
    """2^28 and some columns: the joined weight gradients of one row, and those of none."""
    import torch
    import paper_2312_02493_amd as lib

    cols = (1 << 28) + 77
    ctx = lib.NormContext(1, cols)
    b = torch.bfloat16
    gen = torch.Generator(device="cuda").manual_seed(2)
    dy, x = (torch.randn(1, cols, generator=gen, device="cuda", dtype=b) for _ in range(2))
    mean, rstd = torch.full((1,), 0.25, device="cuda"), torch.full((1,), 1.5, device="cuda")
    dgamma, dbeta = torch.full((cols,), 7.0, device="cuda", dtype=b), torch.full((cols,), 7.0, device="cuda", dtype=b)
    ctx.artopk_layernorm_backward(dy, x, None, mean, rstd, None, dgamma, dbeta)
    assert torch.equal(dbeta, dy[0])
    for at in range(0, cols, 1 << 26):  # one row: a product, rounded to float32 and then to bfloat16
        s = slice(at, min(cols, at + (1 << 26)))
        assert torch.equal(dgamma[s], (dy[0, s].float() * ((x[0, s].float() - 0.25) * 1.5)).to(b)), at
    none = torch.empty(0, cols, device="cuda", dtype=b)
    ctx.artopk_layernorm_backward(none, none, None, mean[:0], rstd[:0], none, dgamma, dbeta)
    assert not bool(dgamma.any()) and not bool(dbeta.any())


def test_rows_that_reach_beyond_any_memory_are_refused():
    """2^20 rows and more at distances up to 2^40: refused on the host, before places pass 63 bits."""
    import ctypes as C

    import torch
    import paper_2312_02493_amd as lib

    rows = (1 << 31) - 1
    ctx = lib.NormContext(rows, 4)
    raw = lib.load_library()
    x, y, m = (torch.zeros(64, device="cuda") for _ in range(3))
    px, py, pm = (C.c_void_p(t.data_ptr()) for t in (x, y, m))
    for r, far in ((rows, (1 << 40) - 1), (rows, (1 << 33) + 4), (1 << 20, 1 << 39)):
        assert raw.artopk_layernorm_forward(ctx._h, px, far, 0, r, 4, None, None, 1e-5, py, 4, None, None) == -1
        assert b"2^46" in raw.artopk_norm_last_error(ctx._h)
        assert raw.artopk_layernorm_forward(ctx._h, px, 4, 0, r, 4, None, None, 1e-5, py, far, None, None) == -1
        for at in range(3):
            strides = [far if i == at else 4 for i in range(3)]
            assert raw.artopk_layernorm_backward(ctx._h, px, strides[0], px, strides[1], 0, r, 4, None, pm, pm, py, strides[2], None, None,
                                                 0, 0) == -1
            assert b"2^46" in raw.artopk_norm_last_error(ctx._h)
    ctx.artopk_layernorm_forward(x[:4].view(1, 4), None, None, y[:4].view(1, 4))
    torch.cuda.synchronize()
