"""Token and AdamW handles under another current device than their own: every call refuses.

There need not be a second device: a handle keeps the number of its device behind its stream, and here that number is changed."""

import ctypes

import pytest

pytestmark = pytest.mark.gpu


class Elsewhere:
    """The handle of a context as if it were another device's."""

    def __init__(self, ctx):
        import torch

        self.device = ctypes.c_int.from_address(ctx._h.value + ctypes.sizeof(ctypes.c_void_p))
        self.own = torch.cuda.current_device()
        assert self.device.value == self.own

    def __enter__(self):
        self.device.value = self.own + 1

    def __exit__(self, *_):
        self.device.value = self.own


def _refused(lib, f, *args, **kw):
    with pytest.raises(lib.ArTopkError) as e:
        f(*args, **kw)
    assert e.value.code == -1 and "device" in str(e.value), str(e.value)


def test_tokens():
    import torch
    import paper_2312_02493_amd as lib

    ctx = lib.TokenContext(8, 50, 16)
    table, y, tok = torch.ones(50, 16).cuda(), torch.zeros(8, 16).cuda(), torch.arange(8).cuda()
    x, v = torch.zeros(8, 50).cuda(), [torch.zeros(8).cuda() for _ in range(4)]
    tok[3] = 50
    ctx.artopk_embedding_forward(table, tok, y)
    torch.cuda.synchronize()
    with Elsewhere(ctx):
        _refused(lib, ctx.artopk_embedding_forward, table, tok, y)
        _refused(lib, ctx.artopk_embedding_backward, y, tok, table)
        _refused(lib, ctx.artopk_token_logprobs, x, tok, *v)
        _refused(lib, ctx.artopk_token_logprobs_backward, x, tok, v[1], v[2], x.clone(), dlogp=v[0])
        _refused(lib, ctx.status)
    with pytest.raises(lib.ArTopkError) as e:  # the report is still there
        ctx.status()
    assert e.value.code == -4
    ctx.status()


def test_adamw():
    import torch
    import paper_2312_02493_amd as lib

    ctx = lib.AdamWContext([(0, 300)], 300, state_bits=8)
    w, g, state = torch.ones(300).cuda(), torch.ones(300).cuda(), ctx.new_state()
    with Elsewhere(ctx):
        _refused(lib, ctx.set_step, 3)
        _refused(lib, ctx.artopk_adamw_step, w, g, *state, step=1)
        _refused(lib, ctx.artopk_adamw_values, *state, first_out=torch.zeros(512).cuda())
    torch.cuda.synchronize()
    assert bool((w == 1.0).all()) and not bool(state[0].any())
    ctx.artopk_adamw_step(w, g, *state, step=1)
    assert bool((w < 1.0).all())
