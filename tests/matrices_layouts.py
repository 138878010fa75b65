"""Layouts of matrices that between them take every tile, with and without shares of the long sums, one step at once and two."""

import paper_2312_02493_amd as lib

HALF, SPLIT = lib.ARTOPK_PRODUCTS_HALF, lib.ARTOPK_PRODUCTS_SPLIT

#: name -> shapes
LAYOUTS = {
    "short-in-shares": [(2500, 129), (64, 1111)],
    "wide-in-shares": [(512, 16001)],
    "many-in-shares": [(1811, 870)] * 8 + [(769, 335)] * 8 + [(3061, 110)] * 16,
    "sixteen-641": [(641, 650)] * 16,
    "sixteen-618": [(1309, 618)] * 16,
    "eight-1391": [(1391, 1447)] * 8,
    "one-4001": [(4001, 4097)],
    "twenty-651": [(651, 1667)] * 20,
    "sixteen-1009": [(2366, 1009)] * 16,
}


def place(shapes, gap):
    """([(offset, rows, cols, scale)], elements) with `gap` loose elements before, between and behind; scales 1 and 0.75 in turn."""
    at, out = gap, []
    for i, (r, c) in enumerate(shapes):
        out.append((at, r, c, 0.75 if i % 2 else 1.0))
        at += r * c + gap
    return out, at


def routes(kind):
    """{layout: what artopk_matrices_info says of its one group}"""
    out = {}
    for name, shapes in LAYOUTS.items():
        (out[name],) = lib.artopk_matrices_info(*place(shapes, 3), lib.ARTOPK_G_F32, kind)
    return out
