"""The scratch of a product belongs to the call until everything that uses it is
enqueued.

The library call releases Python's lock, so another thread can allocate while
the launches are made: a scratch tensor that is already free would be handed to
it.  Host tensors stand in for device ones; nothing is launched.
"""

import weakref

import pytest
import torch

import paper_2411_12692_amd as si

made = []


class Held(torch.Tensor):
    is_cuda = property(lambda self: True)

    def get_device(self):
        return 0

    def new_empty(self, *args, **kwargs):
        t = super().new_empty(*args, **kwargs)
        made.append((weakref.ref(t), t.data_ptr(), t.numel() * t.element_size()))
        return t


def held(*shape, dtype):
    return torch.zeros(*shape, dtype=dtype).as_subclass(Held)


@pytest.mark.parametrize("m,rows,n", [(3, 40, 100), (10, 100, 16384), (9, 72, 16500)])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("a4", [False, True])
def test_scratch_outlives_the_call(monkeypatch, m, rows, n, gated, a4):
    seen = []

    def call(name, *args):
        ws, nbytes = args[-3:-1]
        if nbytes:
            seen.append([r() is not None for r, p, size in made if p == ws and size == nbytes])

    monkeypatch.setattr(si, "_current_device", lambda: 0)
    monkeypatch.setattr(si, "_raw_stream", lambda index: 0)
    monkeypatch.setattr(si._lib, "call", call)
    made.clear()
    np = (n + 127) // 128 * 128
    w = [held(rows, np // 2, dtype=torch.uint8), held(rows, np // 32, dtype=torch.uint8)] * (2 if gated else 1)
    if a4:
        x = [held(m, np // 2, dtype=torch.uint8), held(m, np // 32, dtype=torch.uint8)]
        (si.gated_linear_mxfp4_a4 if gated else si.linear_mxfp4_a4)(*x, *w)
    else:
        (si.gated_linear_mxfp4 if gated else si.linear_mxfp4)(held(m, n, dtype=torch.float16), *w)
    need = si._lib.load().si_linear_mxfp4_workspace_bytes(None if a4 else 16, n, m, rows, np if a4 else n, gated)
    assert len(seen) == (1 if need else 0)
    assert all(alive and all(alive) for alive in seen)
