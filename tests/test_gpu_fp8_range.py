"""The range of the FP8 layer's hidden values, which lie in the tokens' type."""

import pytest
import torch

import paper_2411_12692_amd as si

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16, torch.float32])
def test_hidden_values_above_fp16(dtype, up):
    """Token 1's hidden value 0 is 12800^2 (without W_up 640 times 128): the token is NaN
    with fp16 tokens, its product with bf16 and float32 ones; the others are theirs
    either way.  All codes and scales are exact, so that each output is one product."""
    d, k, m = 128, 128, 5
    wg, wu, wd = (torch.zeros(s, device=DEV) for s in ((k, d), (k, d), (d, k)))
    wg[0], wu[0], wd[:, 0] = 1.0, 1.0, 0.5
    x = torch.ones(m, d, device=DEV)
    x[1] = 100.0 if up else 640.0
    h = x.sum(dim=1).square() if up else x.sum(dim=1)
    layer = si.FP8MLPLayer(wg, wu if up else None, wd)
    y = layer.prompt(x.to(dtype), out_dtype=torch.float32)
    others = [0, 2, 3, 4]
    # scales are largest / 448: the code of the largest value is 448, and what is left are
    # the scales' roundings and that of h, half a step of 2^-8 at most
    want = (0.5 * h)[:, None].expand(m, d)
    assert ((y - want).abs()[others] <= 2.0 ** -7 * want[others]).all()
    if dtype == torch.float16:
        assert y[1].isnan().all()
    else:
        assert ((y - want).abs()[1] <= 2.0 ** -7 * want[1]).all()
