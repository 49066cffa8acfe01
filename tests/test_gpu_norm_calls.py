"""Forms of the norm and block calls beside those of the values' tests."""

import pytest
import torch

import paper_2411_12692_amd as si
from paper_2411_12692_amd import _lib, synth

pytestmark = pytest.mark.gpu

DEV = "cuda"


@pytest.mark.parametrize("ldh,ldo", [(64, 64), (64, 0), (0, 64), (64, 1000)])
def test_one_token_in_place_at_any_stride(ldh, ldo):
    """A single row has no next one: h_out may be h whatever the two strides say."""
    d = 64
    h, b = torch.randn(2, 1, d, device=DEV)
    want, _ = si.norm_residual(h, b, scale=0.5)
    _lib.call("si_norm_residual", h.data_ptr(), _lib.SI_F32, ldh, b.data_ptr(), _lib.SI_F32, d, None, None, 1, 0.5,
              h.data_ptr(), ldo, None, None, _lib.SI_F32, d, 1, d, 1e-5, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(h, want)


@pytest.mark.parametrize("kind", ["fp16", "int8", "mxfp4"])
@pytest.mark.parametrize("shape", [(512,), (1, 512), (1, 1, 512)])
def test_block_returns_the_callers_y(kind, shape):
    """``block`` with a gate or a scale returns ``y`` itself, as the call without
    them does."""
    L = synth.planted_layer(512, 300, 0.5, config=1)
    make = {"fp16": si.MLPLayer, "int8": si.Int8MLPLayer, "mxfp4": si.MXFP4MLPLayer}[kind]
    layer = make(*(t.to(DEV) for t in (L.w_gate, L.w_up, L.w_down)))
    h, w = torch.randn(*shape, device=DEV), torch.ones(512, device=DEV)
    y = torch.empty(*shape, device=DEV)
    if kind == "fp16":
        assert layer.block(h, w, 1e-5, 1.0, y=y) is y
    assert layer.block(h, w, 1e-5, 1.0, y=y, scale=0.5) is y
    out, _ = layer.block(h, w, 1e-5, 1.0, y=y, scale=0.5, outputs=True)
    assert out is y
