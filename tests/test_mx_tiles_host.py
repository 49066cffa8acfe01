"""Which kernel a product takes, asked on the host: the shapes that the GPU tests
compare take every one of them."""

import pytest

import mx_tiles
from paper_2411_12692_amd import _lib


def tile(act, m, rows, n, gated):
    return _lib.load().si_linear_mxfp4_tile(int(act == "a4"), m, rows, n, int(gated))


@pytest.mark.parametrize("act,gated,want,shape", mx_tiles.EVERY)
def test_shape_takes_its_kernel(act, gated, want, shape):
    assert tile(act, *shape, gated) == want


@pytest.mark.parametrize("act", ["f16", "a4"])
@pytest.mark.parametrize("gated", [False, True])
def test_no_kernel_is_left_out(act, gated):
    """A grid of sizes over the whole range takes no kernel that the shapes lack."""
    taken = {tile(act, m, rows, 640, gated)
             for m in (1, 2, 3, 4, 5, 8, 16, 17, 32, 33, 48, 49, 64, 65, 100, 200, 400, 700, 1000, 2000, 4096, 5000, 8192, 20000)
             for rows in (1, 16, 32, 33, 64, 100, 300, 1000, 2048, 4096, 4097, 8192, 9000, 11008, 13824, 16384, 16385, 30000,
                          33000, 70000)}
    assert taken <= set((mx_tiles.MX if act == "a4" else mx_tiles.HALF)[gated])


@pytest.mark.parametrize("m,rows,n", mx_tiles.SPLIT)
@pytest.mark.parametrize("x", [16, None])
@pytest.mark.parametrize("gated", [0, 1])
def test_split_shapes(m, rows, n, x, gated):
    """Their workspace holds the parts: x needs no copy."""
    parts = _lib.load().si_linear_mxfp4_workspace_bytes(x, n, m, rows, n, gated) / ((1 + gated) * m * rows * 4)
    assert parts >= 2 and parts == int(parts)


def test_refused_shapes():
    for m, rows, n in ((0, 64, 128), (5, 0, 128), (5, 64, 0), (5, 64, (1 << 20) + 1), (-1, 64, 128), (5, -1, 128),
                       (1 << 24, 1 << 24, 128)):
        assert tile("f16", m, rows, n, False) == -2 and tile("a4", m, rows, n, True) == -2
