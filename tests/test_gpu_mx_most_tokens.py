"""The product's largest number of tokens."""

import pytest
import torch

import paper_2411_12692_amd as si

pytestmark = pytest.mark.gpu

DEV = "cuda"


def test_product_of_the_most_tokens():
    """2^24 tokens of 4096 4-bit values (34 GB), each compared: their x is one of 64
    rows, repeated in an order without a period of a tile."""
    m, rows, n = 1 << 24, 3, 4096
    g = torch.Generator(device=DEV).manual_seed(1)
    few = torch.randint(-1, 2, (64, n), generator=g, device=DEV)
    fq, fs = si.quantize_rows_mxfp4(few.half())
    q, s = si.quantize_rows_mxfp4(torch.randint(-3, 4, (rows, n), generator=g, device=DEV).half())
    want = si.linear_mxfp4_a4(fq, fs, q, s, torch.float32)
    pick = torch.randint(0, 64, (m,), generator=g, device=DEV)
    xq = torch.empty(m, n // 2, dtype=torch.uint8, device=DEV)
    for i in range(0, m, 1 << 20):
        xq[i:i + (1 << 20)] = fq[pick[i:i + (1 << 20)]]
    y = si.linear_mxfp4_a4(xq, fs[pick], q, s, torch.float32)
    assert torch.equal(y, want[pick])
