"""Limits that the operators around the step answer for without a GPU."""

import paper_2312_02493_amd as lib


def test_more_tiles_than_a_launch_holds():
    """Matrices of one row and 65536 columns are 1024 tiles each.  A launch has fewer than 2^32 threads, 512 a tile with SPLIT
    and 256 with HALF: 2^23 - 1 and 2^24 - 1 tiles are the most."""
    q = lib.artopk_matrices_scratch_bytes

    def of(count, products):
        return q([(i * 65536, 1, 65536) for i in range(count)], count * 65536, lib.ARTOPK_G_F32, products)

    assert of(8200, lib.ARTOPK_PRODUCTS_SPLIT) == of(16500, lib.ARTOPK_PRODUCTS_HALF) == -1
    raw = lib.load_library()
    assert b"tiles" in raw.artopk_last_error(None)
    assert of(500, lib.ARTOPK_PRODUCTS_SPLIT) > 500 * 64 * 65536 * 2 * 2 * 2
