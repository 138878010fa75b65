"""What the operators around the step answer without a GPU: sizes of their scratch, limits, refusals, no fallback."""

import pytest

import paper_2312_02493_amd as lib


def test_norm_scratch():
    q = lib.artopk_norm_scratch_bytes
    for bad in ((0, 1), (1, 0), (-1, 5), (1 << 31, 1), (1, 1 << 31)):
        assert q(*bad) == -1
    assert q(1, 1) >= 8
    assert q(1, 4096) >= 2 * 4 * 4096
    assert q(100, 4096) <= q(100000, 4096) <= q(100000, 16384) <= 128 << 20
    assert q(1 << 20, 1 << 20) >= 2 * 4 << 20


def test_matrices_scratch():
    q = lib.artopk_matrices_scratch_bytes
    one = q([(0, 1024, 1024)], 1 << 20, lib.ARTOPK_G_BF16)
    two = q([(0, 1024, 1024)], 1 << 20, lib.ARTOPK_G_F32)
    assert one >= (2 + 2) * 2 << 20  # X before and after a step, A and Q
    assert 1.9 * one < two < 2.1 * one
    assert q([(0, 1024, 1024)], 1 << 20, lib.ARTOPK_G_F32, lib.ARTOPK_PRODUCTS_HALF) == one
    assert q([(0, 3, 5), (20, 5, 3)], 40) > 0
    for mats, n in (([], 4), ([(0, 2, 3)], 5), ([(0, 2, 3), (5, 1, 1)], 9), ([(0, 0, 3)], 5), ([(-1, 1, 1)], 5), ([(0, 1, 1)], 0),
                    ([(0, 1, 1)], 1 << 31), ([(0, 65537, 1)], 70000), ([(0, 1, 1, float("nan"))], 1)):
        assert q(mats, n) == -1, (mats, n)
    assert q([(0, 1, 1)], 1, 3) == -1
    assert q([(0, 1, 1)], 1, 0, 2) == -1
    raw = lib.load_library()
    assert raw.artopk_matrices_scratch_bytes(None, 1, 1, 0, 0) == -1
    assert b"NULL" in raw.artopk_last_error(None)


def test_null_handles_are_refused():
    raw = lib.load_library()
    assert raw.artopk_norm_destroy(None) == raw.artopk_matrices_destroy(None) == -1
    assert raw.artopk_layernorm_forward(None, None, 1, 0, 1, 1, None, None, 0.0, None, 1, None, None) == -1
    assert b"norm is NULL" in raw.artopk_norm_last_error(None)
    assert raw.artopk_muon_step(None, None, None, None, 1.0, 0.9, 0, 0.1, 0.0, 0.0, 5, None, 1e-7) == -1
    assert b"m is NULL" in raw.artopk_matrices_last_error(None)


def test_no_cpu_fallback():
    import torch

    if torch.cuda.is_available():
        pytest.skip("GPU present")
    with pytest.raises(RuntimeError):
        lib.NormContext(4, 4)
    with pytest.raises(RuntimeError):
        lib.MatrixContext([(0, 2, 2)], 4)


def test_matrices_scratch_of_both_kinds_of_products():
    q = lib.artopk_matrices_scratch_bytes
    mats, n = [(0, 512, 700)], 512 * 700
    half, split = (q(mats, n, lib.ARTOPK_G_F16, p) for p in (lib.ARTOPK_PRODUCTS_HALF, lib.ARTOPK_PRODUCTS_SPLIT))
    assert split <= q(mats, n, lib.ARTOPK_G_F16) < split + half // 4  # the iterates' memory serves one call at a time
    assert q(mats, n, lib.ARTOPK_G_BF16) == half
    assert q([(0, 64, 700)], n, lib.ARTOPK_G_BF16) > q([(0, 64, 700)], n, lib.ARTOPK_G_BF16, lib.ARTOPK_PRODUCTS_HALF)
    assert q(mats, n, lib.ARTOPK_G_F16, -2) == -1
