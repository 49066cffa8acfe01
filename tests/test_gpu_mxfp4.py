"""MXFP4 rows and the products with them on the GPU against NumPy float64
(``mx_ref``).

Quantization is compared bit by bit.  Most products are built so that every
partial sum, in any order, is a whole multiple of one power of two below 2^24 of
them: the float32 sum is then exact and the outputs are compared for equality,
which a dropped, doubled or misplaced value cannot pass.  Products of Gaussian
values are compared within ``(n + 64) 2^-23 sum |x w|`` (one unit in the last
place for each addition) and half a step of the output's type.
"""

import numpy as np
import pytest
import torch

import mx_ref as ref
import paper_2411_12692_amd as si

pytestmark = pytest.mark.gpu

DEV = "cuda"
F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
HALF_STEP = {F16: 2.0 ** -11, BF16: 2.0 ** -8, F32: 2.0 ** -24}
SMALLEST = {F16: 2.0 ** -25, BF16: 2.0 ** -134, F32: 2.0 ** -150}  # half the smallest step


def f64(t):
    return t.detach().cpu().double().numpy()


def check_quantized(w, n=None):
    """Codes and scales of the device against the definition."""
    q, s = si.quantize_rows_mxfp4(w)
    codes, scale = ref.quantize(f64(w).reshape(-1, w.shape[-1]))
    assert np.array_equal(s.cpu().numpy(), scale)
    assert np.array_equal(ref.unpack(q.cpu().numpy()), codes)
    return q, s, codes, scale


# ---- quantization --------------------------------------------------------------

@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("rows,n", [(1, 1), (1, 31), (3, 32), (2, 33), (5, 100), (7, 128), (33, 129), (2, 1000),
                                    (257, 264), (19, 4096), (3, 11008), (1, 70001)])
def test_quantize_and_back(dtype, rows, n):
    g = torch.Generator().manual_seed(rows * 100003 + n)
    w = (torch.randn(rows, n, generator=g) * torch.exp2(torch.randint(-9, 9, (rows, 1), generator=g).float())).to(dtype)
    q, s, codes, scale = check_quantized(w.to(DEV))
    assert q.shape == (rows, ref.padded(n) // 2) and s.shape == (rows, ref.padded(n) // 32)
    for out in (F16, BF16, F32):
        back = si.dequantize_rows_mxfp4(q, s, n, out)
        assert back.dtype == out and back.shape == (rows, n)
        want = torch.from_numpy(ref.values(codes, scale, n)).to(out)  # one rounding, to nearest even
        assert torch.equal(back.cpu(), want)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_quantize_ties_and_signs(dtype):
    """Every midpoint between two codes, its neighbours, both zeros, and values
    above the largest code, at scales from the smallest to the largest."""
    mids = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0]
    eps = float(torch.finfo(dtype).eps)
    row = [0.0, 6.0, 5.5, 7.0] + mids + [m * (1 + eps) for m in mids] + [m * (1 - eps) for m in mids]
    row = (row + [0.5] * 32)[:32]
    base = torch.tensor(row, dtype=torch.float64)
    base = torch.stack([base, -base])
    lo, hi = {F16: (-10, 13), BF16: (-110, 125), F32: (-100, 125)}[dtype]
    w = torch.cat([base * 2.0 ** e for e in (lo, -3, 0, 1, hi)]).to(dtype)
    check_quantized(w.to(DEV))


def test_quantize_special_blocks():
    """Zeros of both signs, subnormals, the largest finite values, infinities and
    NaN: the block with one reads back as NaN, its neighbours as they are."""
    w = torch.zeros(8, 96)
    w[1] = -0.0
    w[2, 40] = float("inf")
    w[3, 40] = float("nan")
    w[4] = torch.arange(96) * 2.0 ** -149
    w[5] = torch.finfo(F32).max
    w[6] = torch.arange(96) * 2.0 ** -126
    w[7, 5], w[7, 95] = float("-inf"), 1.0
    w = w.to(DEV)
    q, s, codes, scale = check_quantized(w)
    back = si.dequantize_rows_mxfp4(q, s, 96, F32).cpu().numpy()
    want = ref.values(codes, scale, 96).astype(np.float32)
    assert np.array_equal(back, want, equal_nan=True)
    assert np.isnan(back[2, 32:64]).all() and not np.isnan(back[2, :32]).any()
    assert np.signbit(back[1]).all()
    h = torch.tensor([[65504.0, -65504.0, 2.0 ** -24, 0.0] * 8, [2.0 ** -24, 3 * 2.0 ** -24] * 16], dtype=F16)
    check_quantized(h.to(DEV))


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_quantize_strides_and_bounds(dtype):
    """Rows with a stride at an odd element, and nothing written behind the
    codes and scales."""
    wide = torch.randn(9, 300, generator=torch.Generator().manual_seed(5)).to(dtype).to(DEV)
    w = wide[:, 3:204]
    q, s = si.quantize_rows_mxfp4(w)
    q2, s2 = si.quantize_rows_mxfp4(w.contiguous())
    assert torch.equal(q, q2) and torch.equal(s, s2)
    from paper_2411_12692_amd import _lib
    qg = torch.full((9 * 128 + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    sg = torch.full((9 * 8 + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    _lib.call("si_quantize_rows_mxfp4", w.data_ptr(), si._DTYPE[dtype], 300, 9, 201, qg.data_ptr(), sg.data_ptr(),
              torch.cuda.current_stream().cuda_stream)
    assert torch.equal(qg[:9 * 128], q.flatten()) and bool((qg[9 * 128:] == 0xA5).all())
    assert torch.equal(sg[:9 * 8], s.flatten()) and bool((sg[9 * 8:] == 0xA5).all())


def test_no_rows():
    q, s = si.quantize_rows_mxfp4(torch.empty(0, 200, dtype=F16, device=DEV))
    assert q.shape == (0, 128) and s.shape == (0, 8)
    assert si.dequantize_rows_mxfp4(q, s, 200).shape == (0, 200)
    wq, ws = si.quantize_rows_mxfp4(torch.randn(5, 200, device=DEV))
    assert si.linear_mxfp4(torch.empty(0, 200, dtype=F16, device=DEV), wq, ws).shape == (0, 5)
    assert si.linear_mxfp4_a4(q, s, wq, ws).shape == (0, 5)


def test_pack_signs():
    w = torch.randn(100, 256, generator=torch.Generator().manual_seed(1))
    w[3] = 0.0
    w[4] = -0.0
    q, s, codes, _ = check_quantized(w.to(DEV))
    words = si.signs_to_canonical(si.pack_signs_mxfp4(q), 100, 256).cpu().numpy().view(np.uint32)
    assert np.array_equal(words, ref.pack_signs(codes))
    assert np.array_equal(words, ref.pack_signs((np.signbit(w.numpy()).astype(np.uint8) << 3)))


# ---- products ------------------------------------------------------------------

def exact_weights(rng, rows, n, top=4):
    """Codes and scales 2^0 .. 2^(top - 1), zeros behind the n-th value."""
    npad = ref.padded(n)
    codes = rng.integers(0, 16, (rows, npad)).astype(np.uint8)
    codes[:, n:] = 0
    scale = (127 + rng.integers(0, top, (rows, npad // 32))).astype(np.uint8)
    scale[:, -(-n // 32):] = 0
    return codes, scale


def dev_mx(codes, scale):
    return torch.from_numpy(ref.pack(codes)).to(DEV), torch.from_numpy(scale).to(DEV)


SHAPES = [(1, 1, 1), (1, 16, 128), (1, 100, 256), (2, 17, 384), (3, 33, 100), (16, 40, 1000), (17, 64, 128),
          (17, 65, 640), (40, 200, 1152), (64, 96, 2048), (65, 130, 513), (100, 33, 4096), (128, 256, 256),
          (130, 300, 384), (257, 520, 128), (1, 2000, 11008), (5, 4096, 896), (33, 13, 11008)]


@pytest.mark.parametrize("m,rows,n", SHAPES)
@pytest.mark.parametrize("act", ["f16", "bf16", "a4"])
@pytest.mark.parametrize("gated", [False, True])
def test_product_exact(m, rows, n, act, gated):
    """x in {-1, 0, 1} (or 4-bit values of scale 1 or 2): sums below 2^24 units
    of 0.5 (0.25), equal in any order."""
    rng = np.random.default_rng(m * 7919 + rows * 31 + n)
    a4 = act == "a4"
    top = 2 if a4 and n > 4096 else 4
    c, s = exact_weights(rng, rows, n, top)
    cu, su = exact_weights(rng, rows, n, top)
    if a4:
        xc, xs = exact_weights(rng, m, n, 2 if n <= 4096 else 1)
        x = ref.values(xc, xs, n)
    else:
        x = rng.integers(-1, 2, (m, n)).astype(np.float64)
    w, wu = ref.values(c, s, n), ref.values(cu, su, n)
    unit = 0.25 if a4 else 0.5
    assert max(np.abs(x).max() * np.abs(v).sum(axis=1).max() for v in (w, wu)) < 2 ** 24 * unit
    g, u = x @ w.T, x @ wu.T
    want = np.float32(np.maximum(g, 0)) * np.float32(u) if gated else np.float32(g)
    mats = dev_mx(c, s) + (dev_mx(cu, su) if gated else ())
    if a4:
        f = si.gated_linear_mxfp4_a4 if gated else si.linear_mxfp4_a4
        y = f(*dev_mx(xc, xs), *mats, out_dtype=F32)
    else:
        f = si.gated_linear_mxfp4 if gated else si.linear_mxfp4
        y = f(torch.from_numpy(x).to(F16 if act == "f16" else BF16).to(DEV), *mats, out_dtype=F32)
    assert np.array_equal(y.cpu().numpy(), want)


@pytest.mark.parametrize("m,rows,n", [(300, 1030, 640), (2048, 2048, 256), (1024, 3000, 384), (600, 8200, 128)])
@pytest.mark.parametrize("act", ["f16", "a4"])
@pytest.mark.parametrize("gated", [False, True])
def test_product_exact_large(m, rows, n, act, gated):
    """Grids of the large tiles, with rows and tokens that end inside one."""
    test_product_exact(m, rows, n, act, gated)


@pytest.mark.parametrize("m,rows,n", [(1, 64, 4096), (9, 48, 512), (50, 100, 700), (200, 80, 2048)])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("out", [F16, BF16, F32])
def test_product_gaussian(m, rows, n, dtype, out):
    g = torch.Generator().manual_seed(m + rows + n)
    w = torch.randn(rows, n, generator=g).half().to(DEV)
    x = torch.randn(m, n, generator=g).to(dtype).to(DEV)
    q, s, codes, scale = check_quantized(w)
    W, X = ref.values(codes, scale, n), f64(x)
    want, size = X @ W.T, np.abs(X) @ np.abs(W).T
    tol = (n + 64) * 2.0 ** -23 * size
    tol = tol + HALF_STEP[out] * (np.abs(want) + tol) + SMALLEST[out]
    y = si.linear_mxfp4(x, q, s, out_dtype=out)
    assert y.dtype == out
    assert (np.abs(f64(y) - want) <= tol).all()
    xq, xs, xcodes, xscale = check_quantized(x)
    XQ = ref.values(xcodes, xscale, n)
    want, size = XQ @ W.T, np.abs(XQ) @ np.abs(W).T
    tol = (n + 64) * 2.0 ** -23 * size
    tol = tol + HALF_STEP[out] * (np.abs(want) + tol) + SMALLEST[out]
    assert (np.abs(f64(si.linear_mxfp4_a4(xq, xs, q, s, out)) - want) <= tol).all()


@pytest.mark.parametrize("m", [3, 70])
@pytest.mark.parametrize("a4", [False, True])
def test_nongated_relu(m, a4):
    rng = np.random.default_rng(m)
    c, s = exact_weights(rng, 90, 300)
    x = rng.integers(-1, 2, (m, 300)).astype(np.float64)
    want = np.maximum(x @ ref.values(c, s, 300).T, 0).astype(np.float32)
    xt = torch.from_numpy(x).half().to(DEV)
    q, sc = dev_mx(c, s)
    y = si.gated_linear_mxfp4_a4(*si.quantize_rows_mxfp4(xt), q, sc, out_dtype=F32) if a4 else \
        si.gated_linear_mxfp4(xt, q, sc, out_dtype=F32)
    assert np.array_equal(y.cpu().numpy(), want)


@pytest.mark.parametrize("m", [2, 70, 300])
def test_product_strided_activations(m):
    """Rows of x at a stride and at an odd element; the row behind the last
    token's values is never read (it holds NaN)."""
    rng = np.random.default_rng(m)
    c, s = exact_weights(rng, 70, 256)
    q, sc = dev_mx(c, s)
    x = rng.integers(-1, 2, (m, 256)).astype(np.float32)
    want = (x.astype(np.float64) @ ref.values(c, s, 256).T).astype(np.float32)
    for off, ld in ((0, 264), (8, 272), (1, 257), (3, 300)):
        buf = torch.full((m, ld + 8), float("nan"), dtype=F16, device=DEV)
        view = buf[:, off:off + 256]
        view.copy_(torch.from_numpy(x))
        assert np.array_equal(si.linear_mxfp4(view, q, sc, out_dtype=F32).cpu().numpy(), want), (off, ld)


@pytest.mark.parametrize("m", [1, 20, 200])
def test_product_extreme_scales(m):
    """bf16 activations with weights from 2^-121 to 2^112; fp16 activations with
    the smallest and largest fp16 weights; a NaN block reaches its row alone."""
    n, rows = 256, 48
    rng = np.random.default_rng(m)
    codes = rng.integers(0, 16, (rows, n)).astype(np.uint8)
    x = rng.integers(-1, 2, (m, n)).astype(np.float64)
    for lo, hi, dtype in ((7, 237, BF16), (127 - 23, 127 + 13, F16)):
        scale = np.repeat(rng.integers(lo, hi + 1, (rows, 1)), n // 32, axis=1).astype(np.uint8)
        scale[0], scale[1] = lo, hi
        y = si.linear_mxfp4(torch.from_numpy(x).to(dtype).to(DEV), *dev_mx(codes, scale), out_dtype=F32)
        want = (x @ ref.values(codes, scale, n).T).astype(np.float32)
        assert np.array_equal(y.cpu().numpy(), want), dtype
    scale[5, 3] = 255
    y = si.linear_mxfp4(torch.from_numpy(x).half().to(DEV), *dev_mx(codes, scale), out_dtype=F32).cpu().numpy()
    assert np.isnan(y[:, 5]).all() and not np.isnan(np.delete(y, 5, axis=1)).any()


@pytest.mark.parametrize("a4", [False, True])
@pytest.mark.parametrize("m,rows,n,split", [(40, 72, 4096, False), (10, 100, 16384, True)])
def test_same_bits_and_bounds(a4, m, rows, n, split):
    """Runs of a product, split or not, agree bit for bit, and nothing is written
    behind y and the workspace."""
    from paper_2411_12692_amd import _lib
    g = torch.Generator().manual_seed(3)
    w, x = torch.randn(rows, n, generator=g).to(DEV), torch.randn(m, n, generator=g).half().to(DEV)
    q, s = si.quantize_rows_mxfp4(w)
    xq, xs = si.quantize_rows_mxfp4(x)
    first = si.linear_mxfp4_a4(xq, xs, q, s, F32) if a4 else si.linear_mxfp4(x, q, s, F32)
    need = _lib.load().si_linear_mxfp4_workspace_bytes(None if a4 else x.data_ptr(), n, m, rows, n, 0)
    assert (need > 0) == split
    ws = torch.full((need + 256,), 0xA5, dtype=torch.uint8, device=DEV)
    y = torch.full((m * rows + 64,), -7.0, device=DEV)
    st = torch.cuda.current_stream().cuda_stream
    for _ in range(3):
        if a4:
            _lib.call("si_linear_mxfp4_a4", xq.data_ptr(), xs.data_ptr(), m, n, q.data_ptr(), s.data_ptr(), rows,
                      y.data_ptr(), si._lib.SI_F32, ws.data_ptr(), need, st)
        else:
            _lib.call("si_linear_mxfp4", x.data_ptr(), si._lib.SI_F16, n, m, n, q.data_ptr(), s.data_ptr(), rows,
                      y.data_ptr(), si._lib.SI_F32, ws.data_ptr(), need, st)
        assert torch.equal(y[:m * rows].view(m, rows), first)
        assert bool((y[m * rows:] == -7.0).all()) and bool((ws[need:] == 0xA5).all())


def test_python_refusals():
    """Shapes, types and layouts that do not go together are refused on the host."""
    q, s = si.quantize_rows_mxfp4(torch.ones(4, 256, device=DEV))
    x = torch.ones(2, 256, dtype=F16, device=DEV)
    xq, xs = si.quantize_rows_mxfp4(x)
    for f in (lambda: si.linear_mxfp4(x[:, :100], q, s), lambda: si.linear_mxfp4(x.t(), q, s),
              lambda: si.linear_mxfp4(x, q, s[:, :4]), lambda: si.linear_mxfp4(x, q[:, :65], s),
              lambda: si.linear_mxfp4(x, q, s[:3]), lambda: si.linear_mxfp4(x[None], q, s),
              lambda: si.linear_mxfp4(x.expand(2, 256)[:1].expand(3, 256), q, s),
              lambda: si.gated_linear_mxfp4(x, q, s, q[:3].contiguous(), s[:3].contiguous()),
              lambda: si.linear_mxfp4_a4(xq, xs, *si.quantize_rows_mxfp4(torch.ones(4, 100, device=DEV))),
              lambda: si.dequantize_rows_mxfp4(q, s, 100), lambda: si.dequantize_rows_mxfp4(q, s, 257),
              lambda: si.linear_mxfp4(x.cpu(), q, s), lambda: si.linear_mxfp4(x, q.cpu(), s)):
        with pytest.raises(ValueError):
            f()
    for f in (lambda: si.linear_mxfp4(x.float(), q, s), lambda: si.linear_mxfp4(x, q.char(), s),
              lambda: si.quantize_rows_mxfp4(x.int()), lambda: si.linear_mxfp4(x, q, s, torch.float64),
              lambda: si.dequantize_rows_mxfp4(q, s, 256, torch.float64)):
        with pytest.raises(TypeError):
            f()
    h, w = torch.ones(4, 256, device=DEV), torch.ones(256, device=DEV)
    for f in (lambda: si.norm_residual(h), lambda: si.norm_residual(h, post_w=w, pre_w=w),
              lambda: si.norm_residual(h, h[:2]), lambda: si.norm_residual(h, h.clone(), gate=torch.ones(3, 256, device=DEV)),
              lambda: si.norm_residual(h, pre_w=w[:100]), lambda: si.norm_residual(h, h.clone(), out=h[:2]),
              lambda: si.norm_residual(h.t(), pre_w=w)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(si.SparseInferError):  # out over the branch
        b = h.clone()
        si.norm_residual(h, b, out=b)


# one shape for each tile of each kind of activations, and for the products larger
# than every tile's 256 blocks with few tokens
EVERY_TILE = [(9, 500, 640), (9, 9000, 384), (9, 18000, 256), (30, 8100, 640), (20, 20000, 256), (33, 32000, 256),
              (40, 25000, 128), (60, 20000, 384), (64, 40000, 128), (130, 30000, 128), (700, 3000, 640),
              (1100, 8100, 256), (5, 70000, 128), (3, 4097, 1152), (4, 1500, 13056)]


@pytest.mark.parametrize("m,rows,n", EVERY_TILE)
@pytest.mark.parametrize("act", ["f16", "a4"])
@pytest.mark.parametrize("gated", [False, True])
def test_product_exact_every_tile(m, rows, n, act, gated):
    """n of odd numbers of 128 values, so that the last ones do not fill a stage."""
    test_product_exact(m, rows, n, act, gated)


@pytest.mark.parametrize("m,rows,n", [(10, 100, 16384), (300, 64, 8192), (1, 64, 20000)])
@pytest.mark.parametrize("act", ["bf16", "a4"])
@pytest.mark.parametrize("gated", [False, True])
def test_product_exact_split(m, rows, n, act, gated):
    test_product_exact(m, rows, n, act, gated)
