"""What the token and AdamW entry points answer without a GPU: sizes, limits, refusals, no fallback."""

import pytest

import paper_2312_02493_amd as lib


def test_tokens_scratch():
    q = lib.artopk_tokens_scratch_bytes
    for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (-1, 5, 5), (1 << 31, 1, 1), (1, 1 << 31, 1), (1, 1, 65537)):
        assert q(*bad) == -1, bad
    assert q(1, 1, 1) > 0
    assert q(1000, 5000) == q(1000, 5000, 1)
    assert q(4096, 32000, 512) < q(8192, 32000, 512) < q(8192, 32000, 1024)
    assert q((1 << 31) - 1, (1 << 31) - 1, 65536) > 1 << 40  # (no overflow)


def test_adamw_sizes():
    elems, q = lib.artopk_adamw_state_elems, lib.artopk_adamw_scratch_bytes
    assert elems([(0, 1)], 1) == 256 and elems([(0, 256)], 256) == 256 and elems([(0, 257)], 300) == 512
    assert elems([(5, 100, 0.5, 0.1), (105, 300)], 405) == 256 + 512
    assert 0 < q([(0, 1)], 1) < q([(0, 10_000_000)], 10_000_000)
    for tensors, n in (([], 4), ([(0, 5)], 4), ([(-1, 2)], 4), ([(0, 0)], 4), ([(0, 1)], 0), ([(0, 1)], 1 << 31), ([(3, 2)], 4),
                       ([(0, 1, float("nan"))], 1), ([(0, 1, 1.0, float("inf"))], 1), ([(0, 1 << 62)], 4), ([(1 << 62, 1)], 4)):
        assert elems(tensors, n) == q(tensors, n) == -1, (tensors, n)
    assert q([(0, 5), (4, 3)], 20) == -1  # overlapping
    raw = lib.load_library()
    assert b"overlap" in raw.artopk_last_error(None)
    assert raw.artopk_adamw_state_elems(None, 1, 1) == -1
    assert b"NULL" in raw.artopk_last_error(None)


def test_null_handles_are_refused():
    raw = lib.load_library()
    assert raw.artopk_tokens_destroy(None) == raw.artopk_adamw_destroy(None) == -1
    assert raw.artopk_tokens_status(None) == -1
    assert raw.artopk_embedding_forward(None, None, 1, 0, 1, 1, None, 64, 0, 1.0, None, 1, 0) == -1
    assert b"NULL" in raw.artopk_tokens_last_error(None)
    assert raw.artopk_embedding_backward(None, None, 1, 0, None, 64, 0, 1, 1.0, None, 1, 0, 1, 0) == -1
    assert raw.artopk_token_logprobs(None, None, 1, 0, 0, 1, None, 64, 1.0, None, None, None, None, 0, None, None) == -1
    assert raw.artopk_token_logprobs_backward(None, None, 1, 0, 0, 1, None, 64, 1.0, None, None, None, None, None, None, None,
                                              1) == -1
    assert raw.artopk_adamw_step(None, None, None, None, None, None, 1, 1.0, 0.1, 0.9, 0.99, 1e-8, 0) == -1
    assert raw.artopk_adamw_set_step(None, 0) == raw.artopk_adamw_values(None, None, None, None, 0, None, None) == -1
    assert b"NULL" in raw.artopk_adamw_last_error(None)


def test_no_cpu_fallback():
    import torch

    if torch.cuda.is_available():
        pytest.skip("GPU present")
    with pytest.raises(RuntimeError):
        lib.TokenContext(4, 4)
    with pytest.raises(RuntimeError):
        lib.AdamWContext([(0, 2)], 4)


def test_adamw_sizes_of_overlapping_tensors():
    for tensors, n in (([(0, 5), (4, 3)], 20), ([(4, 3), (0, 5)], 20), ([(0, 9), (3, 2)], 9), ([(2, 1), (2, 1)], 4)):
        assert lib.artopk_adamw_state_elems(tensors, n) == lib.artopk_adamw_scratch_bytes(tensors, n) == -1, tensors
        assert b"overlap" in lib.load_library().artopk_last_error(None)
    assert lib.artopk_adamw_state_elems([(5, 4), (0, 5)], 9) == 512  # side by side, in any order
