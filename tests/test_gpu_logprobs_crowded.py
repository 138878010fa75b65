"""Rows whose large elements crowd in few threads' pieces, so that more candidates for the alternatives are left than there is room
for on chip, and they are found one after the other."""

import math

import pytest

pytestmark = pytest.mark.gpu

ROOM_WAVE, ROOM_FOUR = 56 * 8 + 64, 128 * 8 + 64


def _dtype(t):
    import torch

    return {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[t]


def _order(x, top):
    """The `top` largest of each row, the lower index first among equal ones."""
    import torch

    bits = (x.float() + 0.0).view(torch.int32)
    key = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32
    key = key + (0x7FFFFFFF - torch.arange(x.shape[1], device=x.device))
    return 0x7FFFFFFF - (torch.topk(key, top, 1).values & 0xFFFFFFFF)


def _check(rows, vocab, t, top, threads, a_key, split, values):
    """Large elements in all pieces of the threads that have `top` - 1 of the keys, `a_key` threads to a key, in each part."""
    import torch
    import paper_2312_02493_amd as lib

    size = 16 // (4 if t == "f32" else 2)
    g = torch.Generator(device="cuda").manual_seed(vocab + top)
    pieces = -(-vocab // size)
    piece = torch.arange(vocab, device="cuda") // size
    crowd = torch.zeros(vocab, dtype=torch.bool, device="cuda")
    for part in range(split):
        q0, q1 = pieces * part // split, pieces * (part + 1) // split
        here = (piece >= q0) & (piece < q1)
        large = here & ((piece - q0) % threads < a_key * (top - 1))
        assert int(large.sum()) > (ROOM_WAVE if threads == 64 else ROOM_FOUR), int(large.sum())
        crowd |= large
    x = torch.randn(rows, vocab, generator=g, device="cuda")
    if values == "equal":
        x[:, crowd] = 9.0
        x[:, ~crowd] = -1.0
        x[::2, ~crowd] = -math.inf
    elif values == "some":
        x += 8.0 * crowd
        x[1::2] = torch.randn(rows // 2, vocab, generator=g, device="cuda")  # (ordinary rows in between)
    else:
        x = torch.where(crowd, 10.0 + torch.randint(0, 3, x.shape, generator=g, device="cuda"), x)
    x = x.to(_dtype(t))
    ids, lps = torch.full((rows, top), -9, dtype=torch.int32, device="cuda"), torch.full((rows, top), 9.0, device="cuda")
    logsum = torch.zeros(rows, device="cuda")
    ctx = lib.TokenContext(rows, vocab)
    ctx.artopk_token_logprobs(x, logsum_out=logsum, top_ids_out=ids, top_logp_out=lps)
    order = _order(x, top)
    assert torch.equal(ids.long(), order), (ids[:2], order[:2])
    z = x.double() - x.double().amax(1, keepdim=True)
    lse = torch.logsumexp(z, 1)
    # a sum of `vocab` terms, at most (20 + vocab / 128) steps one after the other
    u = 2.0 ** -24
    tol = (40.0 + vocab / 128) * u + 4.0 * u * lse.abs()
    assert bool(((logsum.double() - lse).abs() <= tol).all())
    want = z.gather(1, order) - lse.view(-1, 1)
    err = torch.where(want == lps.double(), torch.zeros_like(want), (want - lps.double()).abs())
    assert bool((err <= tol.view(-1, 1) + 6.0 * u * want.abs()).all())


# rows, columns, threads to a team and to a key (kernel's rules), parts
ONE_WAVE = [(7, 2048, "bf16", 30), (7, 2048, "f32", 56), (6, 2045, "f16", 40), (2048, 16_000, "bf16", 5)]
FOUR_WAVES = [(7, 5003, "bf16", 20, 4), (6, 5000, "f32", 32, 4), (6, 5003, "f16", 33, 2), (5, 6001, "bf16", 64, 2),
              (350, 128_000, "bf16", 2, 4)]


@pytest.mark.parametrize("values", ["some", "ties", "equal"])
@pytest.mark.parametrize("rows,vocab,t,top", ONE_WAVE)
def test_one_wave(rows, vocab, t, top, values):
    _check(rows, vocab, t, top, 64, 1, 1, values)


@pytest.mark.parametrize("values", ["some", "ties", "equal"])
@pytest.mark.parametrize("rows,vocab,t,top,a_key", FOUR_WAVES)
def test_four_waves(rows, vocab, t, top, a_key, values):
    _check(rows, vocab, t, top, 256, a_key, 1, values)


@pytest.mark.parametrize("values", ["some", "ties", "equal"])
@pytest.mark.parametrize("rows,split,vocab,t,top,a_key", [(100, 10, 131_001, "bf16", 20, 4), (100, 10, 80_000, "f32", 40, 2)])
def test_parts(rows, split, vocab, t, top, a_key, values):
    _check(rows, vocab, t, top, 256, a_key, split, values)
