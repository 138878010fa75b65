"""Which rows of a layer norm overlap: those that share an element, not those that lie between each other's."""

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,cols,pad", [(1, 5, 0), (4, 64, 0), (700, 40, 0), (6, 1111, 1), (300, 2048, 0), (3, 20000, 8), (520, 515, 2)])
def test_columns_of_one_matrix(t, rows, cols, pad):
    """x, dy and what is written side by side: the same bits as apart, and nothing else is touched."""
    import torch
    import paper_2312_02493_amd as lib

    dtype = getattr(torch, t)
    ctx = lib.NormContext(rows, cols)
    gen = torch.Generator(device="cuda").manual_seed(rows)
    width = 4 * cols + pad
    one = torch.randn(rows, width, generator=gen, device="cuda").to(dtype)
    gamma = torch.randn(cols, generator=gen, device="cuda")
    found = []
    for together in (True, False):
        bufs = [one.clone()] * 4 if together else [one.clone() for _ in range(4)]
        x, dy, y, dx = (b[:, i * cols:(i + 1) * cols] for i, b in enumerate(bufs))
        mean, rstd, dg, db = (torch.zeros(k, device="cuda") for k in (rows, rows, cols, cols))
        ctx.artopk_layernorm_forward(x, gamma, None, y, mean, rstd)
        ctx.artopk_layernorm_backward(dy, x, gamma, mean, rstd, dx, dg, db)
        assert torch.equal(x, one[:, :cols]) and torch.equal(dy, one[:, cols:2 * cols])
        if pad:
            assert all(torch.equal(b[:, 4 * cols:], one[:, 4 * cols:]) for b in bufs)
        found.append([v.clone() for v in (y, dx, mean, rstd, dg, db)])
    for a, b in zip(*found):
        assert torch.equal(a, b)


def test_vectors_between_rows():
    import torch
    import paper_2312_02493_amd as lib

    ctx = lib.NormContext(6, 16)
    buf = torch.randn(6, 64, device="cuda")
    x, y = buf[:, :16], buf[:, 16:32]
    gamma, mean, rstd = buf[2, 32:48], buf[0, 50:56], buf[5, 40:46]
    want = torch.layer_norm(x, (16,), gamma.clone(), None, 1e-5)
    ctx.artopk_layernorm_forward(x, gamma, None, y, mean, rstd)
    assert torch.allclose(y, want, atol=1e-4) and torch.allclose(mean, x.mean(1), atol=1e-5)
    with pytest.raises(lib.ArTopkError, match="overlap"):
        ctx.artopk_layernorm_forward(x, buf[2, 20:36], None, y)
    with pytest.raises(lib.ArTopkError, match="overlap"):
        ctx.artopk_layernorm_forward(x, None, None, y, torch.as_strided(buf, (6,), (1,), 60))  # ends in x's second row


def test_refused_exactly_where_an_element_is_shared():
    """Random places in one buffer, against the elements themselves."""
    import torch
    import paper_2312_02493_amd as lib

    rng = np.random.default_rng(5)
    ctx = lib.NormContext(8, 16)
    size = 200
    buf = torch.zeros(size, device="cuda")

    def rows_of(pitch):
        rows, cols = int(rng.integers(1, 7)), int(rng.integers(1, 9))
        pitch = max(pitch, cols)
        return int(rng.integers(0, size - (rows - 1) * pitch - cols + 1)), rows, cols, pitch

    taken = refused = careful = 0
    for _ in range(600):
        pitch = int(rng.integers(1, 30))
        a, rows, cols, pa = rows_of(pitch)
        pb = max(pitch if rng.random() < 0.8 else int(rng.integers(1, 30)), cols)
        b = int(rng.integers(0, size - (rows - 1) * pb - cols + 1))
        x, y = torch.as_strided(buf, (rows, cols), (pa, 1), a), torch.as_strided(buf, (rows, cols), (pb, 1), b)
        shared = bool({a + i * pa + j for i in range(rows) for j in range(cols)} &
                      {b + i * pb + j for i in range(rows) for j in range(cols)})
        try:
            ctx.artopk_layernorm_forward(x, None, None, y)
            assert not shared, (a, b, rows, cols, pa, pb)
            taken += 1
        except lib.ArTopkError as e:
            assert "overlap" in str(e)
            if not shared:
                assert rows > 1 and pa != pb, (a, b, rows, cols, pa, pb)
                careful += 1
            refused += 1
    torch.cuda.synchronize()
    assert taken > 150 and refused > 100 and careful < 60, (taken, refused, careful)
