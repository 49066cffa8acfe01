"""The MXFP4 calls and ``norm_residual`` run on the device of their tensors,
whichever is current.

Host tensors that say they are on device 1 go through the binding while device 0
is current; every call into the library has to be made with device 1 current and
on its stream.  Nothing is launched.
"""

import contextlib

import pytest
import torch

import paper_2411_12692_amd as si


class OnDevice1(torch.Tensor):
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 1


def on1(*shape, dtype=torch.float16):
    return torch.zeros(*shape, dtype=dtype).as_subclass(OnDevice1)


@pytest.fixture
def calls(monkeypatch):
    current, made = [0], []

    @contextlib.contextmanager
    def device(index):
        current.append(index)
        yield
        current.pop()

    real_empty = torch.empty
    monkeypatch.setattr(torch, "empty", lambda *a, **k: real_empty(*a, **k).as_subclass(OnDevice1))
    real_zeros = torch.zeros
    monkeypatch.setattr(torch, "zeros", lambda *a, **k: real_zeros(*a, **k).as_subclass(OnDevice1))
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[-1])
    monkeypatch.setattr(si, "_current_device", lambda: current[-1])
    monkeypatch.setattr(si, "_raw_stream", lambda index: 1000 + index)
    monkeypatch.setattr(si._lib, "call", lambda name, *args: made.append((name, current[-1], args[-1])))
    return made


def on_device_1(made, *names):
    assert sorted({name for name, _, _ in made}) == sorted(names)
    assert all(index == 1 and stream == 1001 for _, index, stream in made), made


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gated", [True, False])
def test_layer(calls, dtype, gated):
    k, d = 200, 256
    layer = si.MXFP4MLPLayer(on1(k, d, dtype=dtype), on1(k, d, dtype=dtype) if gated else None, on1(d, k, dtype=dtype),
                             max_batch=2, prompt=True)
    made = ["si_quantize_rows_mxfp4", "si_pack_signs_mxfp4"]
    on_device_1(calls, *made, *(["si_transpose_down"] if dtype != torch.float32 else []))
    calls.clear()
    layer(on1(2, d), 1.0)
    layer.sparse_mlp(on1(2, d), on1(k, dtype=torch.uint8))
    layer.block(on1(2, d, dtype=torch.float32), on1(d, dtype=torch.float32), 1e-5, 1.0, scale=0.5)
    layer.prompt_block(on1(9, d, dtype=torch.float32), on1(d, dtype=torch.float32), 1e-5)
    layer.prompt(on1(9, d), a4=True)
    on_device_1(calls, "si_predict_sparse_mlp_mxfp4", "si_sparse_mlp_mxfp4", "si_norm_residual", "si_gated_linear_mxfp4",
                "si_linear_mxfp4", "si_quantize_rows_mxfp4", "si_gated_linear_mxfp4_a4", "si_linear_mxfp4_a4")


def test_rows(calls):
    q, s = si.quantize_rows_mxfp4(on1(5, 100))
    si.dequantize_rows_mxfp4(q, s, 100)
    on_device_1(calls, "si_quantize_rows_mxfp4", "si_dequantize_rows_mxfp4")
