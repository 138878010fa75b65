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
