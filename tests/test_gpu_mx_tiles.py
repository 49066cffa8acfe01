"""Every kernel of the MXFP4 products, for each kind of activations and number of
matrices, compared for equality (``test_gpu_mxfp4.test_product_exact``)."""

import pytest

import mx_tiles
import test_gpu_mxfp4

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act,gated,tile,shape", mx_tiles.EVERY)
def test_every_kernel(act, gated, tile, shape):
    test_gpu_mxfp4.test_product_exact(*shape, act, gated)


@pytest.mark.parametrize("m,rows,n", mx_tiles.SPLIT)
@pytest.mark.parametrize("act", ["f16", "bf16", "a4"])
@pytest.mark.parametrize("gated", [False, True])
def test_split_sums(m, rows, n, act, gated):
    test_gpu_mxfp4.test_product_exact(m, rows, n, act, gated)
