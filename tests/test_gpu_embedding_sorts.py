"""The embedding gradient by every number of passes of the sort (more than 8192 or 14336 tokens), with zeros beside them and
without.  Sums of small whole numbers, which are exact in float32 and compared bit for bit."""

import pytest

pytestmark = pytest.mark.gpu

#: Below, at and above the numbers of digits at which another pass begins (2^11, 2^22).
VOCABULARIES = [1, 2, 2046, 2047, 2048, 2049, 65535, 65536, (1 << 22) - 1, 1 << 22, 5_000_000]


def _tokens(count, vocab, how, seed):
    import torch

    g = torch.Generator().manual_seed(seed)
    tok = torch.randint(0, vocab, (count,), generator=g)
    if how == "mixed":
        tok[torch.rand(count, generator=g) < 0.4] = vocab - 1
        tok[torch.rand(count, generator=g) < 0.1] = -1
        tok[torch.rand(count, generator=g) < 0.1] = 0
    if how == "falling":
        tok = torch.sort(tok, descending=True).values
    if how == "upper":  # (other digits only in the last pass)
        tok = (tok >> 9) << 9
    return tok


def _check(count, vocab, width, how, accumulate, pad=0, t=None, grad=None, bad=False):
    import torch
    import paper_2312_02493_amd as lib

    t, grad = t or torch.float32, grad or torch.float32
    g = torch.Generator().manual_seed(count)
    tok = _tokens(count, vocab, how, vocab % 1000)
    if bad:
        tok[::7] = vocab + torch.arange(0, count, 7)[:tok[::7].numel()]
    dy = torch.randint(-3, 4, (count, width), generator=g).to(t)
    mem = torch.full((vocab, width + pad), 2.0, dtype=grad, device="cuda")
    out = mem[:, :width]
    total = torch.zeros(vocab, width, device="cuda")
    live = (tok >= 0) & (tok < vocab)
    total.index_add_(0, tok[live].cuda(), dy[live].float().cuda())
    if accumulate:
        total += 2.0
    want = total.to(grad)
    assert float(total.abs().max()) < (1 << 24)
    ctx = lib.TokenContext(count, vocab, width)
    dev_dy, dev_tok = dy.cuda(), tok.to("cuda", torch.int32 if count % 2 else torch.int64)
    for turn in range(2):
        ctx.artopk_embedding_backward(dev_dy, dev_tok, out, accumulate=accumulate)
        assert torch.equal(out, want), (turn, int((out != want).sum()))
        assert bool((mem[:, width:] == 2.0).all())
        out.fill_(2.0)
        if bad:
            with pytest.raises(lib.ArTopkError):
                ctx.status()
        ctx.status()


@pytest.mark.parametrize("vocab", VOCABULARIES)
@pytest.mark.parametrize("count", [8193, 14_337, 20_011])
@pytest.mark.parametrize("accumulate", [False, True])
def test_passes(vocab, count, accumulate):
    for how in ("mixed", "falling"):
        _check(count, vocab, 3, how, accumulate)


@pytest.mark.parametrize("vocab,width", [(70_000, 65), (1 << 22, 2), (4_200_000, 3), (33_000, 260)])
@pytest.mark.parametrize("count", [8193, 131_072, 131_073, 270_001])
@pytest.mark.parametrize("how", ["mixed", "upper"])
def test_zeros_beside_every_pass(vocab, width, count, how):
    """Tables above 16 MB, whose zeros are written by the launches of the sort."""
    import torch

    _check(count, vocab, width, how, False)
    _check(count, vocab, width, how, True, pad=1)
    _check(count, vocab, width, how, False, pad=3, t=torch.bfloat16, grad=torch.float32)


def test_one_pass_of_many_tokens():
    _check(300_001, 2000, 20, "mixed", False)
    _check(300_001, 2000, 20, "mixed", True, pad=1)


@pytest.mark.parametrize("count", [9000, 140_000])
def test_tokens_beyond_the_table(count):
    for vocab, width in ((2047, 5), (40_000, 110), (1 << 22, 1)):
        _check(count, vocab, width, "mixed", False, bad=True)
        _check(count, vocab, width, "mixed", True, bad=True)
