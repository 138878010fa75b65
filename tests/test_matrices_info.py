"""How handles of matrices work, as they say without a GPU; and that the layouts of the GPU tests reach every way."""

import ctypes as C

import pytest

import paper_2312_02493_amd as lib
from tests.matrices_layouts import HALF, SPLIT, routes


@pytest.mark.parametrize("kind", [HALF, SPLIT])
def test_layouts_reach_every_tile(kind):
    """A change of the table of costs that leaves a tile without a test shows here."""
    got = routes(kind)
    assert all(not g["one_launch"] and g["parts"] == kind + 1 for g in got.values())
    for key in ("gram_tile", "square_tile", "apply_tile"):
        assert {g[key] for g in got.values()} == {64, 128, 192, 256}, key
    assert {g["pairs"] for g in got.values()} == {0, 1}
    assert {g["square_tile"] for g in got.values() if g["pairs"]} >= {64, 128, 192, 256}
    assert {g["gram_tile"] for g in got.values() if g["shared_tiles"]} == {64, 128}


def test_groups_of_bfloat16():
    mats, n = [(0, 16, 700), (20000, 300, 520), (200000, 600, 530)], 600000
    q = lib.artopk_matrices_info
    for weights in (False, True):
        half, split = q(mats, n, lib.ARTOPK_G_BF16, weights=weights)
        assert (half["parts"], half["matrices"], split["parts"], split["matrices"]) == (1, 2, 2, 1)
    (one,) = q(mats, n, lib.ARTOPK_G_F32)
    assert (one["parts"], one["matrices"]) == (2, 3)
    (small,) = q([(0, 64, 64), (5000, 30, 100)], 9000, lib.ARTOPK_G_F16)
    assert small["one_launch"] and small["gram_tile"] == 0


def test_refusals():
    for mats, n in (([], 4), ([(0, 2, 3)], 5), ([(0, 2, 3), (5, 1, 1)], 9)):
        with pytest.raises(lib.ArTopkError):
            lib.artopk_matrices_info(mats, n)
    raw, out = lib.load_library(), (C.c_int32 * 17)()
    assert raw.artopk_matrices_info(None, 1, 1, 0, 0, 0, out, 17) == -1
    assert raw.artopk_matrices_info(None, 1, 1, 0, 0, 0, None, 17) == -1
    assert raw.artopk_matrices_info(None, 1, 1, 0, 0, 0, out, 16) == -1
    assert b"17" in raw.artopk_last_error(None)
