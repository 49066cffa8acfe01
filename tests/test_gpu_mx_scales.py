"""Scales at the ends of MXFP4's range in the products, on the GPU against NumPy
float64.

Sums are whole multiples of one power of two, below 2^24 of them, so float32 holds
them exactly in any order and the outputs are compared for equality.  Where the
sums lie below float32's normal numbers (2^-126) a product or a partial sum may be
flushed there: each of n products and n additions then errs by less than 2^-126.
Where a term's scale passes 2^103 nothing is asked: 2^24 quarters of it are past
float32's range, so a partial sum may be infinite, and two of them NaN, where the
whole sum (0, say) is not.
"""

import numpy as np
import pytest
import torch

import mx_ref as ref
import paper_2411_12692_amd as si

pytestmark = pytest.mark.gpu

DEV = "cuda"
# a few tokens and rows, small tiles, split sums, several tokens' and rows' tiles
SHAPES = [(1, 48, 256), (3, 33, 640), (9, 500, 384), (10, 40, 16384), (40, 700, 256), (70, 300, 640), (200, 1030, 256),
          (700, 1500, 384)]


def dev_mx(codes, scale):
    return torch.from_numpy(ref.pack(codes)).to(DEV), torch.from_numpy(scale).to(DEV)


def codes_of(rng, rows, n):
    return rng.integers(0, 16, (rows, n)).astype(np.uint8)


def unscaled(codes, n):
    return ref.values(codes, np.full((codes.shape[0], n // 32), 127, np.uint8), n)


def few(codes, n):
    """Of a long row every 8th value, so that its sum stays exact."""
    if n > 4096:
        codes[:, np.arange(n) % 8 != 0] = 0
    return codes


@pytest.mark.parametrize("m,rows,n", SHAPES)
@pytest.mark.parametrize("gated", [False, True])
def test_a4_scale_by_row_and_token(m, rows, n, gated):
    """Each row of W and each token at a scale of its own, from 2^-127 to 2^127."""
    rng = np.random.default_rng(m + rows)
    wc, xc = few(codes_of(rng, rows, n), n), codes_of(rng, m, n)
    we = rng.integers(0, 255, rows)
    we[:6] = [0, 254, 1, 253, 127, 126]
    xe = rng.integers(0, 255, m)
    xe[0] = 127 if m < 6 else 0
    if m >= 6:
        xe[1:6] = [254, 1, 253, 127, 128]
    S = unscaled(xc, n) @ unscaled(wc, n).T
    e = we[None, :] + xe[:, None] - 254
    with np.errstate(over="ignore", under="ignore"):
        want64 = np.ldexp(S, e)
    W = dev_mx(wc, np.repeat(we[:, None], n // 32, axis=1).astype(np.uint8))
    X = dev_mx(xc, np.repeat(xe[:, None], n // 32, axis=1).astype(np.uint8))
    if gated:
        # u from plain scales: the codes of W at 2^0, the tokens at theirs
        U = dev_mx(wc, np.full((rows, n // 32), 254 // 2, np.uint8))
        e_u = np.broadcast_to(xe[:, None] - 127, S.shape)
        y = si.gated_linear_mxfp4_a4(*X, *W, *U, out_dtype=torch.float32).cpu().numpy().astype(np.float64)
        u = np.ldexp(S, e_u)
        with np.errstate(over="ignore", invalid="ignore", under="ignore"):
            want = np.float64(np.float32(np.maximum(want64, 0)) * np.float32(u))
        # both sums within range, and their product too where it is not 0
        sums = (e > -120) & (e < 100) & (e_u > -120) & (e_u < 100)
        sure = sums & ((S == 0) | ((e + e_u > -120) & (e + e_u < 90)))
        assert sure.any() and np.array_equal(y[sure], want[sure])
        return
    y = si.linear_mxfp4_a4(*X, *W, out_dtype=torch.float32).cpu().numpy().astype(np.float64)
    normal = (e >= -124) & (e <= 127 - 24)  # a quarter of 2^e is normal, 2^24 of them finite
    assert normal.any() and np.array_equal(y[normal], want64[normal])
    small = e < -124
    assert (np.abs(y - want64)[small] <= 2 * n * 2.0 ** -126).all()


@pytest.mark.parametrize("m,rows,n", SHAPES)
def test_a4_scale_by_block(m, rows, n):
    """Every block of W at a scale from 2^-127 to 2^127, the tokens' blocks at its
    inverse: each product is of 4-bit values alone."""
    rng = np.random.default_rng(rows * 7 + n)
    wc, xc = few(codes_of(rng, rows, n), n), codes_of(rng, m, n)
    base = rng.integers(0, 255, n // 32)
    base[:4] = [0, 254, 1, 127]
    W = dev_mx(wc, np.repeat(base[None], rows, axis=0).astype(np.uint8))
    X = dev_mx(xc, np.repeat(254 - base[None], m, axis=0).astype(np.uint8))
    y = si.linear_mxfp4_a4(*X, *W, out_dtype=torch.float32).cpu().numpy()
    assert np.array_equal(y.astype(np.float64), unscaled(xc, n) @ unscaled(wc, n).T)


@pytest.mark.parametrize("m,rows,n", SHAPES)
@pytest.mark.parametrize("act", ["f16", "bf16", "a4"])
@pytest.mark.parametrize("gated", [False, True])
def test_nan_blocks_reach_their_row_and_token_alone(m, rows, n, act, gated):
    """The scale byte 255, whatever the codes: in the last and an inner row of W,
    and in the last and an inner token, where every tile repeats the last of each."""
    rng = np.random.default_rng(n + m)
    wc, xc = codes_of(rng, rows, n), codes_of(rng, m, n)
    wc[rows // 2] = 0
    ws, xs = np.full((rows, n // 32), 127, np.uint8), np.full((m, n // 32), 127, np.uint8)
    ws[rows - 1, n // 32 - 1] = ws[rows // 2, 1] = 255
    nan = np.zeros((m, rows), bool)
    nan[:, [rows - 1, rows // 2]] = True
    if act == "a4":
        xs[m - 1, n // 32 - 1] = xs[m // 2, 2] = 255
        nan[[m - 1, m // 2]] = True
        X = dev_mx(xc, xs)
        f = si.gated_linear_mxfp4_a4 if gated else si.linear_mxfp4_a4
    else:
        x = torch.from_numpy(unscaled(xc, n)).to(torch.float16 if act == "f16" else torch.bfloat16)
        x[m - 1, n - 1] = x[m // 2, 70] = float("nan")
        nan[[m - 1, m // 2]] = True
        X = (x.to(DEV),)
        f = si.gated_linear_mxfp4 if gated else si.linear_mxfp4
    W = dev_mx(wc, ws) * (2 if gated else 1)
    y = f(*X, *W, out_dtype=torch.float32).cpu().numpy()
    assert np.array_equal(np.isnan(y), nan)


@pytest.mark.parametrize("m,rows,n", SHAPES)
def test_bf16_smallest_and_largest_weights(m, rows, n):
    """bf16 activations meet weights of every scale as they are, those below bf16's
    normal numbers too: tokens at 2^40 and 2^-40 bring the sums into range."""
    rng = np.random.default_rng(m * 3 + n)
    wc = few(codes_of(rng, rows, n), n)
    x = rng.integers(-1, 2, (m, n)).astype(np.float64)
    for bytes_, shift in (((0, 1, 2, 3, 5, 20), 40), ((252, 251, 250, 240, 200, 238), -40)):
        we = rng.choice(bytes_, rows)
        y = si.linear_mxfp4(torch.from_numpy(np.ldexp(x, shift)).bfloat16().to(DEV),
                            *dev_mx(wc, np.repeat(we[:, None], n // 32, axis=1).astype(np.uint8)),
                            out_dtype=torch.float32).cpu().numpy().astype(np.float64)
        want = np.ldexp(x @ unscaled(wc, n).T, we[None, :] - 127 + shift)
        assert np.array_equal(y, want), bytes_
