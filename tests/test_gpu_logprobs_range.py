"""Log probabilities of rows whose scaled logits lie far from zero, against the definition in 64 bits: by sixteen lanes, one wave,
four waves, and in parts.

Tolerances are those of test_gpu_logprobs (u = 2^-24).  What a row far from zero adds: an exponent is c (x - largest), the
difference and the product rounded once each, or c x less a reference that is at most 1/2 from c times the largest.  That distance
is exact (one fused operation); it is part of exponents and of where the reference moves, each rounded once, and taken out again
in the end: at most (6 |d| + 6) u more of an element, and 4 u more of the sum where the reference moves, which happens at most
once in 1024 elements.  Row64's `r`, `e1` and `e2` carry both.
"""

import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
SHAPES = [(7, 130), (7, 1000), (7, 2048), (7, 5003), (3, 140_001)]


def _check(x, t, top, scale=1.0):
    import torch
    from tests.test_gpu_logprobs import Row64, _dtype, _forward, _gen, _near

    x = x.to(_dtype(t))
    assert bool(torch.isfinite(x).any(1).all())
    rows, vocab = x.shape
    tok = torch.randint(0, vocab, (rows,), generator=_gen(vocab))
    tok[::3] = x.float().argmax(1)[::3]
    s = float(np.float32(scale))
    ref = Row64(x, s)
    more = U * ((6.0 + 4.0 * (vocab / 1024 + 2)) * ref.r + 6.0 * ref.e1)
    ref.tol_logsum = ref.tol_logsum + more / (1.0 + ref.r)
    ref.tol_entropy = ref.tol_entropy + (more * (2.0 + ref.e1 / (1.0 + ref.r)) + U * (6.0 + 4.0 * (vocab / 1024 + 2)) * ref.e1
                                         + 6.0 * U * ref.e2) / (1.0 + ref.r)
    _, _, _, logp, peak, logsum, entropy, ids, lps = _forward(x, tok, top, scale, 0, 0, t)
    assert torch.equal(peak.cpu().double(), ref.peak.view(-1))
    _near(logsum, ref.logsum, ref.tol_logsum, "logsum")
    _near(entropy, ref.entropy, ref.tol_entropy, "entropy")
    # (log p beyond float32 is -infinity there)
    below = lambda v: torch.where(v <= -(2.0 ** 128), torch.full_like(v, -math.inf), v)
    d = ref.d.gather(1, tok.view(-1, 1))
    _near(logp, below(d - ref.logsum.view(-1, 1)).view(-1), ref.tol_logp(d).view(-1), "logp")
    if top:
        order = torch.sort(x.float() + 0.0, dim=1, descending=True, stable=True).indices[:, :top]
        assert torch.equal(ids.cpu().long(), order)
        d = ref.d.gather(1, order)
        _near(lps, below(d - ref.logsum.view(-1, 1)), ref.tol_logp(d), "top_logp")


def _rows(rows, vocab, kind, far, seed=5):
    """kind: equal (nothing but `far`); peak (one `far` beside ordinary logits); half (half of the elements are `far`); near (all
    next to `far`); late (ordinary ones up to the last, which is `far`); early (the other way round)."""
    import torch

    g = torch.Generator().manual_seed(seed)
    x = 3.0 * torch.randn(rows, vocab, generator=g)
    if kind == "equal":
        return torch.full_like(x, far)
    if kind == "peak":
        x[torch.arange(rows), torch.randint(0, vocab, (rows,), generator=g)] = far
    if kind == "half":
        x[torch.rand(rows, vocab, generator=g) < 0.5] = far
    if kind == "near":
        x = (far * (1.0 + torch.randint(-3, 4, (rows, vocab), generator=g) * 2.0 ** -22)).float()
    if kind == "late":
        x[:, -1] = far
    if kind == "early":
        x[:, 1:] = far
    return x


@pytest.mark.parametrize("t", ["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("kind", ["equal", "peak", "half", "near", "late", "early"])
def test_logits_far_from_zero(t, rows, vocab, kind):
    for i, size in enumerate((1e7, 1e8, 1e9, 1e10, 1e12, 1e20, 1e30)):
        for far in (size, -size):
            _check(_rows(rows, vocab, kind, far), t, (0, 5)[i % 2])


@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("order", ["any", "rising", "falling"])
def test_logits_next_to_where_references_end(rows, vocab, sign, order):
    """Whole numbers next to those whose product with log2(e) is 2^22 to 2^26, so that elements before and behind are on either
    side while their differences are ordinary (steps of 1 to 4)."""
    import torch

    g = torch.Generator().manual_seed(9)
    for power in (22, 23, 24, 25, 26):
        step = max(1, 2 ** (power - 24))
        middle = math.floor(2.0 ** power / math.log2(math.e)) // step * step
        x = sign * middle + step * torch.randint(-15, 16, (rows, vocab), generator=g).double()
        if order != "any":
            x = torch.sort(x, 1, descending=order == "falling").values
        assert torch.equal(x.float().double(), x)
        _check(x.float(), "f32", 5)


@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_low_and_high_temperatures(rows, vocab, t):
    import torch

    g = torch.Generator().manual_seed(11)
    x = 10.0 + torch.randn(rows, vocab, generator=g)
    for scale in (1e8, 1e9, 1e12, 1e30):
        _check(x, t, 5, scale)
        _check(-x, t, 5, scale)
        _check(torch.full_like(x, 10.0), t, 5, scale)
    for size in (1e9, 1e20, 1e30):  # (ordinary logits, once they are scaled)
        _check(x * size, t, 5, 1.0 / size)


#: The scales that are taken: below, elements whose difference from the peak float32 does not hold would count; above, c is beyond it.
LEAST, MOST = 2.0 ** -120, 2.0 ** 127


@pytest.mark.parametrize("rows,vocab", SHAPES)
@pytest.mark.parametrize("t", ["f32", "bf16"])
def test_differences_beyond_float32(rows, vocab, t):
    """Logits at both ends of float32: their difference is not in it, scaled it is."""
    import torch

    g = torch.Generator().manual_seed(13)
    x = 3e38 * (2.0 * torch.rand(rows, vocab, generator=g) - 1.0)
    x[:, 5], x[:, 7] = 3.2e38, -3.2e38
    for scale in (LEAST, 1e-30, 1e-3, 0.4):
        _check(x, t, 5, scale)
        y = torch.full_like(x, -3.2e38)
        y[:, -3:] = 3.1e38
        _check(y, t, 5, scale)


@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_gradient_of_rows_far_from_zero(rows, vocab):
    """dlogits = scale dlogp ([index = token] - p): p is off by (6 |d| + 20) u of itself and its sum's share, the product by 4 u."""
    import torch
    import paper_2312_02493_amd as lib

    g = torch.Generator().manual_seed(14)
    for scale, far in ((1.0, 1e10), (1.0, -1e10), (1e9, 10.0), (1e-3, 3e38), (LEAST, 3e38)):
        for kind in ("equal", "peak", "half", "ends"):
            x = _rows(rows, vocab, kind, far)
            if kind == "ends":
                x = far * (2.0 * torch.rand(rows, vocab, generator=g) - 1.0)
            tok = torch.randint(0, vocab, (rows,), generator=g)
            s = float(np.float32(scale))
            d = s * (x.double() - x.double().amax(1, keepdim=True))
            logsum = torch.logsumexp(d, 1)
            out = [torch.empty(rows, device="cuda") for _ in range(2)]
            dx, one = torch.empty(rows, vocab, device="cuda"), torch.ones(rows, device="cuda")
            ctx = lib.TokenContext(rows, vocab)
            ctx.artopk_token_logprobs(x.cuda(), None, None, *out, scale=scale)
            ctx.artopk_token_logprobs_backward(x.cuda(), tok.cuda(), *out, dx, dlogp=one, scale=scale)
            lp = d - logsum.view(-1, 1)
            want = -torch.exp(lp)
            want[torch.arange(rows), tok] = -torch.expm1(lp[torch.arange(rows), tok])
            depth = 20.0 + 8.0 * (vocab / 2048 + 2) + 44 + 8 * (vocab / 1024 + 4)
            tol = s * U * torch.exp(lp) * (6.0 * d.abs().clamp(max=1e4) + 4.0 * logsum.view(-1, 1) + depth) + 4.0 * U * s * want.abs()
            got = dx.cpu().double()
            bad = (got - s * want).abs() > tol + 2.0 ** -126 * (1.0 + s)
            assert not bool(bad.any()), (scale, far, kind, got[bad][:4], (s * want)[bad][:4])


@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_ends_of_the_scales(rows, vocab):
    import torch
    import paper_2312_02493_amd as lib

    g = torch.Generator().manual_seed(15)
    for size in (1.0, 1e-30, 2.0 ** -127):
        x = size * torch.randint(-6, 7, (rows, vocab), generator=g).float()  # (many equal ones)
        _check(x, "f32", 5, MOST)
        _check(x, "f32", 5, LEAST)
    ctx = lib.TokenContext(rows, vocab)
    dev, out = x.cuda(), [torch.zeros(rows, device="cuda") for _ in range(2)]
    for scale in (float(np.nextafter(np.float32(LEAST), np.float32(0))), float(np.nextafter(np.float32(MOST), np.float32(np.inf))),
                  1e-45, 3e38):
        with pytest.raises(lib.ArTopkError) as e:
            ctx.artopk_token_logprobs(dev, None, None, *out, scale=scale)
        assert e.value.code == -1 and "scale" in str(e.value)
        with pytest.raises(lib.ArTopkError) as e:
            ctx.artopk_token_logprobs_backward(dev, None, *out, dev.clone(), dlse=out[0].clone(), scale=scale)
        assert e.value.code == -1 and "scale" in str(e.value)
    ctx.status()
