"""Nothing is written outside the outputs and the workspace: every output of the dense,
norm and FP8 calls lies between guard bytes, at sizes that end inside a piece, a tile
and a block, and the workspace is exactly as large as asked for."""

import pytest
import torch

from paper_2411_12692_amd import _lib

pytestmark = pytest.mark.gpu
DEV = "cuda"
GUARD = 4096
KINDS = {0: torch.float16, 1: torch.bfloat16, 2: torch.float32}


class Guarded:
    """Buffers between guard bytes."""

    def __init__(self):
        self.all = []

    def __call__(self, nbytes):
        raw = torch.full((GUARD + (nbytes + 15) // 16 * 16 + GUARD,), 0xA5, dtype=torch.uint8, device=DEV)
        self.all.append((raw, nbytes))
        return raw.data_ptr() + GUARD

    def check(self):
        torch.cuda.synchronize()
        for raw, nbytes in self.all:
            assert (raw[:GUARD] == 0xA5).all() and (raw[GUARD + nbytes:] == 0xA5).all()


def values(*shape, dtype=torch.float16):
    return torch.randn(*shape, device=DEV).to(dtype)


SHAPES = [(1, 1, 1), (1, 7, 9), (3, 129, 65), (5, 33, 200), (17, 31, 1001), (33, 100, 72), (70, 257, 130), (129, 77, 640),
          (300, 515, 259), (1025, 261, 67)]


@pytest.mark.parametrize("out", [0, 1, 2])
@pytest.mark.parametrize("m,rows,n", SHAPES)
def test_products(m, rows, n, out):
    lib, stream = _lib.load(), torch.cuda.current_stream().cuda_stream
    x, w, wu = values(m, n), values(rows, n), values(rows, n)
    wt = w.t().contiguous()
    size = m * rows * KINDS[out].itemsize
    for up in (None, wu.data_ptr()):
        g = Guarded()
        nb = lib.si_gated_linear_workspace_bytes(x.data_ptr(), n, m, n, w.data_ptr(), up, rows)
        keep = [g(4 * m * rows), g(4 * m * rows)] if up else [None, None]
        _lib.call("si_gated_linear", x.data_ptr(), 0, n, m, n, w.data_ptr(), up, rows, g(size), out, *keep,
                  g(nb) if nb else None, nb, stream)
        g.check()
        for want_dx, want_dw in ((1, 1), (1, 0), (0, 1)):
            g = Guarded()
            nb = lib.si_gated_linear_backward_workspace_bytes(x.data_ptr(), n, m, n, w.data_ptr(), up, rows, want_dx, want_dw)
            dh, gv, uv = values(m, rows, dtype=KINDS[out]), values(m, rows, dtype=KINDS[2]), values(m, rows, dtype=KINDS[2])
            _lib.call("si_gated_linear_backward", dh.data_ptr(), out, rows, gv.data_ptr(), 2, uv.data_ptr() if up else None,
                      x.data_ptr(), 0, n, m, n, w.data_ptr(), up, rows, g(2 * m * n) if want_dx else None,
                      g(2 * rows * n) if want_dw else None, g(2 * rows * n) if want_dw and up else None, g(nb) if nb else None,
                      nb, stream)
            g.check()
            dt = 2 if out == 2 else 0
            dy, h = values(m, n, dtype=KINDS[dt]), values(m, rows)
            for want_down in (1, 0):
                g = Guarded()
                nb = lib.si_mlp_backward_workspace_bytes(dy.data_ptr(), dt, n, x.data_ptr(), n, m, n, w.data_ptr(), up, wt.data_ptr(),
                                                         rows, want_dx, want_dw, want_down)
                _lib.call("si_mlp_backward", dy.data_ptr(), dt, n, x.data_ptr(), 0, n, m, n, w.data_ptr(), up, wt.data_ptr(), rows,
                          h.data_ptr(), gv.data_ptr() if up else None, uv.data_ptr() if up else None,
                          g(2 * m * n) if want_dx else None, g(2 * rows * n) if want_dw else None,
                          g(2 * rows * n) if want_dw and up else None, g(2 * rows * n) if want_down else None,
                          g(nb) if nb else None, nb, stream)
                g.check()
    for t, mat in ((0, w), (1, wt)):
        g = Guarded()
        nb = lib.si_linear_workspace_bytes(x.data_ptr(), n, m, n, mat.data_ptr(), rows, t)
        _lib.call("si_linear", x.data_ptr(), 0, n, m, n, mat.data_ptr(), rows, t, g(size), out, g(nb) if nb else None, nb, stream)
        g.check()
        dt = 2 if out == 2 else 0
        dy = values(m, rows, dtype=KINDS[dt])
        nb = lib.si_linear_backward_workspace_bytes(dy.data_ptr(), dt, rows, x.data_ptr(), n, m, n, mat.data_ptr(), rows, t, 1, 1)
        g = Guarded()
        _lib.call("si_linear_backward", dy.data_ptr(), dt, rows, x.data_ptr(), 0, n, m, n, mat.data_ptr(), rows, t,
                  g(2 * m * n), g(2 * rows * n), g(nb) if nb else None, nb, stream)
        g.check()


@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("m,rows,n", SHAPES)
def test_fp8(m, rows, n, dtype):
    lib, stream = _lib.load(), torch.cuda.current_stream().cuda_stream
    x, w = values(m, n, dtype=KINDS[dtype]), values(rows, n, dtype=KINDS[dtype])
    g = Guarded()
    xq, xs = g(lib.si_fp8_codes_bytes(m, n)), g(lib.si_fp8_scales_bytes(m, n))
    q, s = g(lib.si_fp8_codes_bytes(rows, n)), g(lib.si_fp8_block_scales_bytes(rows, n))
    _lib.call("si_quantize_rows_fp8", x.data_ptr(), dtype, n, m, n, xq, xs, stream)
    _lib.call("si_quantize_blocks_fp8", w.data_ptr(), dtype, n, rows, n, q, s, stream)
    _lib.call("si_dequantize_fp8", xq, xs, 1, m, n, g(m * n * KINDS[dtype].itemsize), dtype, stream)
    _lib.call("si_dequantize_fp8", q, s, 128, rows, n, g(rows * n * KINDS[dtype].itemsize), dtype, stream)
    size = m * rows * KINDS[dtype].itemsize
    for up in (None, q):
        nb = lib.si_linear_fp8_workspace_bytes(m, rows, n, up is not None)
        _lib.call("si_gated_linear_fp8", xq, xs, m, n, q, s, up, s if up else None, rows, g(size), dtype,
                  g(nb) if nb else None, nb, stream)
    nb = lib.si_linear_fp8_workspace_bytes(m, rows, n, 0)
    _lib.call("si_linear_fp8", xq, xs, m, n, q, s, rows, g(size), dtype, g(nb) if nb else None, nb, stream)
    g.check()


@pytest.mark.parametrize("w_dtype", [0, 2])
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("t,d", [(1, 1), (3, 7), (5, 511), (9, 513), (2, 4097), (7, 5120), (600, 129), (3, 16383)])
def test_norms(t, d, dtype, w_dtype):
    lib, stream = _lib.load(), torch.cuda.current_stream().cuda_stream
    e, ew = KINDS[dtype].itemsize, KINDS[w_dtype].itemsize
    x, dy = values(t, d, dtype=KINDS[dtype]), values(t, d, dtype=KINDS[dtype])
    w, b = values(d, dtype=KINDS[w_dtype]), values(d, dtype=KINDS[w_dtype])
    for center in (0, 1):
        g = Guarded()
        mean, rstd = g(4 * t), g(4 * t)
        _lib.call("si_layer_norm", x.data_ptr(), dtype, d, w.data_ptr(), b.data_ptr() if center else None, w_dtype, center, 1e-5,
                  g(t * d * e), mean, rstd, t, d, stream)
        nb = lib.si_layer_norm_backward_workspace_bytes(t, d)
        _lib.call("si_layer_norm_backward", dy.data_ptr(), d, x.data_ptr(), dtype, d, w.data_ptr(), w_dtype, center, mean, rstd,
                  g(t * d * e), g(d * ew), g(d * ew) if center else None, t, d, g(nb), nb, stream)
        g.check()
