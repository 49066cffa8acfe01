"""Products that need scratch (a padded copy of x, partial sums of a split n),
from two Python threads on one stream, and with allocations while a call is
being made."""

import threading

import pytest
import torch

import paper_2411_12692_amd as si

pytestmark = pytest.mark.gpu

DEV = "cuda"
SHAPES = [(3, 40, 100), (10, 100, 16384), (300, 64, 8100)]  # padded, split, both


def operands(m, rows, n, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(m, n, generator=g).half().to(DEV)
    return x, *si.quantize_rows_mxfp4(torch.randn(rows, n, generator=g).to(DEV))


@pytest.mark.parametrize("m,rows,n", SHAPES)
def test_scratch_is_not_handed_out_during_the_call(monkeypatch, m, rows, n):
    x, q, s = operands(m, rows, n, 1)
    want = si.linear_mxfp4(x, q, s)
    real, taken = si._lib.call, []

    def call(name, *args):
        ws, nbytes = args[-3:-1]
        assert nbytes > 0
        others = [torch.full((nbytes,), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(3)]
        taken.append(all(t.data_ptr() + nbytes <= ws or ws + nbytes <= t.data_ptr() for t in others))
        real(name, *args)

    monkeypatch.setattr(si._lib, "call", call)
    assert torch.equal(si.linear_mxfp4(x, q, s), want)
    assert taken == [True]


def test_two_threads_on_one_stream():
    """Each thread's products agree with those made alone, bit for bit."""
    cases = [[operands(*shape, 10 * i + t) for i, shape in enumerate(SHAPES)] for t in range(2)]
    want = [[si.linear_mxfp4(*c) for c in mine] for mine in cases]
    torch.cuda.synchronize()
    wrong, start = [], threading.Barrier(2)

    def work(t):
        start.wait()
        for i in range(60):
            got = [si.linear_mxfp4(*c) for c in cases[t]]
            wrong.extend((t, i, j) for j, (a, b) in enumerate(zip(got, want[t])) if not torch.equal(a, b))

    threads = [threading.Thread(target=work, args=(t,)) for t in range(2)]
    for th in threads:
        th.start()
    for th in threads:
        th.join()
    assert wrong == []
