"""A single row has no next one: its stride is not looked at, whatever it is."""

import pytest
import torch

import paper_2411_12692_amd as si
from paper_2411_12692_amd import _lib

pytestmark = pytest.mark.gpu

DEV = "cuda"
STRIDES = [0, 1, 255, 257, 1 << 22, (1 << 33) + 3, (1 << 63) + 5]


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("ld", STRIDES)
def test_product(ld):
    n, rows = 256, 40
    x = torch.randn(1, n, device=DEV).half()
    q, s = si.quantize_rows_mxfp4(torch.randn(rows, n, device=DEV))
    want = si.linear_mxfp4(x, q, s, torch.float32)
    y = torch.zeros(1, rows, device=DEV)
    need = _lib.load().si_linear_mxfp4_workspace_bytes(x.data_ptr(), ld, 1, rows, n, 0)
    ws = torch.empty(need + 16, dtype=torch.uint8, device=DEV)
    _lib.call("si_linear_mxfp4", x.data_ptr(), _lib.SI_F16, ld, 1, n, q.data_ptr(), s.data_ptr(), rows, y.data_ptr(),
              _lib.SI_F32, ws.data_ptr(), need, stream())
    assert torch.equal(y, want)


@pytest.mark.parametrize("ld", STRIDES)
def test_quantize(ld):
    w = torch.randn(1, 256, device=DEV)
    want = si.quantize_rows_mxfp4(w)
    q, s = torch.zeros_like(want[0]), torch.zeros_like(want[1])
    _lib.call("si_quantize_rows_mxfp4", w.data_ptr(), _lib.SI_F32, ld, 1, 256, q.data_ptr(), s.data_ptr(), stream())
    assert torch.equal(q, want[0]) and torch.equal(s, want[1])


@pytest.mark.parametrize("ld", STRIDES)
def test_norm(ld):
    d = 256
    h, b, out, x = torch.randn(4, 1, d, device=DEV)
    w = torch.rand(d, device=DEV)
    want, x_want = si.norm_residual(h, b, scale=0.5, pre_w=w, x_dtype=torch.float32)
    F32 = _lib.SI_F32
    _lib.call("si_norm_residual", h.data_ptr(), F32, ld, b.data_ptr(), F32, ld, None, None, 1, 0.5, out.data_ptr(), ld,
              w.data_ptr(), x.data_ptr(), F32, ld, 1, d, 1e-5, stream())
    # a stride that is not whole 16-byte pieces sums the row in another order: each
    # x within (d / 2 + 16) 2^-24 of its value
    assert torch.equal(out, want) and bool(((x - x_want).abs() <= (d + 32) * 2.0 ** -24 * x_want.abs()).all())
