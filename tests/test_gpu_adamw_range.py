"""AdamW's step over the whole range of eps, and of moments, against 64 bits from the moments that it stores.

Weights are 0, so a step is -rate m / (sqrt(v) root + eps): rate, root, the square root, the sum, the quotient or reciprocal and
products are some twelve roundings of u = 2^-24 (the hardware's root and reciprocal one each).  The quotient itself may lie below
float32's normal numbers: half a step there, 2^-150, times the rate, and another one of the result's own."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
TINY = 2.0 ** -150
EPS = [1e-45, 1e-38, 1e-30, 1e-8, 1.0, 1e30, 8e37, 8.6e37, 1.7e38, 3.4e38]


@pytest.mark.parametrize("eps", EPS)
@pytest.mark.parametrize("bits", [32, 8])
def test_eps(eps, bits):
    import torch
    import paper_2312_02493_amd as lib

    n = 1030
    g = torch.Generator().manual_seed(3)
    for size in (1e-44, 1e-38, 1e-30, 1e-22, 1e-15, 1.0, 1e15, 1e18):
        for beta1, beta2, step, eta in ((0.9, 0.999, 1, 1e-3), (0.0, 0.0, 5, 1.0), (0.5, 0.9, 7, 1e10)):
            ctx = lib.AdamWContext([(0, n)], n, state_bits=bits)
            first, second, scales = ctx.new_state()
            update = (size * torch.randn(n, generator=g)).float()
            if bits == 32:
                first[:n], second[:n] = (size * torch.randn(n, generator=g)).cuda(), (size * size * torch.rand(n, generator=g)).cuda()
            m0, v0 = first[:n].cpu().float(), second[:n].cpu().float()
            w = torch.zeros(n, device="cuda")
            ctx.artopk_adamw_step(w, update.cuda(), first, second, scales, step=step, eta=eta, beta1=beta1, beta2=beta2, eps=eps)
            f = np.float32
            # the moments before they are rounded to 8 bits, as float32 has them
            m = (m0.numpy() * f(beta1) + update.numpy() * f(1.0 - beta1)).astype(np.float64)
            with np.errstate(over="ignore"):
                v = (v0.numpy() * f(beta2) + (update.numpy() * update.numpy()) * f(1.0 - beta2)).astype(np.float64)
            assert np.isfinite(v).all()
            rate = float(f(eta)) / (1.0 - beta1 ** step)
            want = -rate * (m / (np.sqrt(v) / np.sqrt(1.0 - beta2 ** step) + float(f(eps))))
            got = w.cpu().numpy().astype(np.float64)
            tol = 12.0 * U * np.abs(want) + TINY * (1.0 + rate) * 1.001
            bad = np.abs(got - want) > tol
            assert not bad.any(), (size, beta1, int(bad.sum()), got[bad][:3], want[bad][:3])
