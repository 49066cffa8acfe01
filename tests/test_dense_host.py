"""Host-side checks of the dense products, the norms with gradients and the FP8 calls
(no GPU, nothing is launched): the tests' reference against worked examples, sizes,
which kernel a product takes, and every refusal."""

import math

import pytest
import torch

import dense_ref as ref
import paper_2411_12692_amd as si
from paper_2411_12692_amd import _lib

A = 1 << 40  # a fake 16-byte-aligned address: validation fails before it is used
B, C, D, E, F, G, H, I, J, K, L, M = (A + (i << 36) for i in range(1, 13))  # far apart: no overlap
F16, BF16, F32 = _lib.SI_F16, _lib.SI_BF16, _lib.SI_F32
BIG = 1 << 50


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2411_12692_amd import build
        build.build()
    return _lib.load()


def refused(status, name, *args):
    assert _lib.status(name, *args) == status, (_lib.last_error(), args)


# ---- the reference ---------------------------------------------------------------

def test_reference_e4m3():
    v = ref.e4m3_values()
    assert v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[56] == 1.0 and v[126] == 448.0 and (v[1:] > v[:-1]).all()
    want = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    assert torch.equal(v, want)
    # midpoints go to the even code, everything above 448 to 448, signs of zeros stay
    mid = ((v[1:] + v[:-1]) / 2).float()
    assert (ref.e4m3_code(mid) % 2 == 0).all()
    assert ref.e4m3_code(torch.tensor([1e9, -1e9, 0.0, -0.0])).tolist() == [126, 254, 0, 128]
    x = torch.randn(4000) * 100
    assert torch.equal(ref.e4m3_code(x).to(torch.uint8), x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))


def test_reference_quantize_worked_example():
    """Largest 896: scale 2; 3 -> 1.5 (code 60), 0.7 -> 0.35: 0.34375 (43) or 0.375 (44),
    -896 -> -448 (254).  A block of zeros has scale 0, one with an infinity reads back NaN."""
    x = torch.zeros(3, 130)
    x[0, :3] = torch.tensor([3.0, 0.7, -896.0])
    x[1, 129] = 448.0 * 2.0 ** -20
    x[2, 5] = math.inf
    codes, scale = ref.quantize(x, 1)
    assert codes.shape == (3, 144) and codes[0, :3].tolist() == [60, 43, 254]
    assert scale[0].tolist() == [2.0, 0.0] and scale[1].tolist() == [0.0, 2.0 ** -20]
    v = ref.values(codes, scale, 130, 1)
    assert v[0, :3].tolist() == [3.0, 0.6875, -896.0] and v[1, 129] == x[1, 129]
    assert v[2, :128].isnan().all() and (v[2, 128:] == 0).all()


def test_reference_norm():
    x = torch.tensor([[1.0, 3.0]], dtype=torch.float64)
    w, b = torch.tensor([2.0, 2.0], dtype=torch.float64), torch.tensor([1.0, 0.0], dtype=torch.float64)
    assert torch.allclose(ref.norm(x, w, b, 0.0, True), torch.tensor([[-1.0, 2.0]], dtype=torch.float64))
    assert torch.allclose(ref.norm(x, w, None, 0.0, False), x * 2 / math.sqrt(5))
    for center in (True, False):  # against differences of the loss sum(y * dy)
        g = torch.Generator().manual_seed(1)
        x, w, dy = (torch.randn(s, generator=g, dtype=torch.float64) for s in ((3, 7), (7,), (3, 7)))
        dx, dw, db, *_ = ref.norm_grad(x, w, dy, 1e-3, center)
        loss = lambda x, w, b: float((ref.norm(x, w, b, 1e-3, center) * dy).sum())  # noqa: E731
        zero, h = torch.zeros(7, dtype=torch.float64), 1e-6
        for i in range(7):
            e = torch.zeros(7, dtype=torch.float64)
            e[i] = h
            assert abs((loss(x, w + e, zero) - loss(x, w - e, zero)) / (2 * h) - dw[i]) < 1e-6
            assert abs((loss(x, w, e) - loss(x, w, -e)) / (2 * h) - db[i]) < 1e-6
            step = torch.zeros(3, 7, dtype=torch.float64)
            step[1, i] = h
            assert abs((loss(x + step, w, zero) - loss(x - step, w, zero)) / (2 * h) - dx[1, i]) < 1e-6


# ---- sizes and kernels ---------------------------------------------------------------

def test_shapes_cover_every_kernel(lib):
    """The shapes that the GPU tests run take the kernels they are listed under, and
    every kernel of the kind is there."""
    for (kind, gated), tiles in ref.TILES.items():
        for tile, shapes in tiles.items():
            for m, rows, n in shapes:
                assert lib.si_dense_tile(ref.KIND[kind], m, rows, n, gated) == tile, (kind, gated, m, rows, n)
        found = {lib.si_dense_tile(ref.KIND[kind], m, rows, n, gated)
                 for m in (1, 7, 20, 64, 150, 257, 1500, 2050, 4100)
                 for rows in (64, 72, 328, 2056, 4100, 8200) for n in (64, 72, 200, 328, 2056, 4100)}
        assert found <= set(tiles), (kind, gated, found)
    f = lib.si_dense_tile
    assert f(0, 0, 5, 5, 0) == f(0, 5, 0, 5, 0) == f(7, 5, 5, 5, 0) == f(-1, 5, 5, 5, 0) == f(0, 5, 5, (1 << 20) + 1, 0) == -2


def test_workspace_sizes(lib):
    f = lib.si_linear_workspace_bytes
    assert f(A, 128, 1, 128, B, 64, 0) == 0                  # aligned, one part
    assert f(A + 2, 128, 3, 128, B, 64, 0) >= 3 * 128 * 2    # an unaligned x is copied
    assert f(A, 129, 3, 128, B, 64, 0) >= 3 * 128 * 2        # so are rows that are
    assert f(A, 129, 1, 128, B, 64, 0) == 0                  # a single row's stride leads nowhere
    assert f(A, 100, 3, 100, B, 64, 0) >= (3 + 64) * 104 * 2  # odd lengths: both
    assert f(A, 128, 3, 128, B, 63, 1) >= 128 * 64 * 2       # W^T [n][rows] by its own rows' length
    assert f(A, 128, 0, 128, B, 64, 0) == 0 and f(A, 128, 3, 128, B, 0, 0) == 0
    g = lib.si_gated_linear_workspace_bytes
    assert g(A, 100, 3, 100, B, C, 64) >= (3 + 128) * 104 * 2
    b = lib.si_linear_backward_workspace_bytes
    assert b(A, F16, 64, B, 128, 3, 128, C, 64, 0, 1, 1) == 0
    assert b(A, F32, 64, B, 128, 3, 128, C, 64, 0, 1, 1) >= 3 * 64 * 2   # a float32 dy is rounded
    assert b(A, F16, 64, B, 100, 3, 100, C, 64, 0, 0, 1) >= 3 * 104 * 2
    gb = lib.si_gated_linear_backward_workspace_bytes
    assert gb(A, 128, 3, 128, B, C, 63, 1, 1) >= 2 * 3 * 64 * 2          # dg and du
    assert gb(A, 128, 0, 128, B, C, 63, 1, 1) == 0
    mb = lib.si_mlp_backward_workspace_bytes
    assert mb(A, F16, 128, B, 128, 3, 128, C, D, E, 64, 0, 0, 1) == 0    # dw_down alone: operands as they are
    assert mb(A, F32, 128, B, 128, 3, 128, C, D, E, 64, 0, 0, 1) >= 3 * 128 * 2
    assert mb(A, F16, 128, B, 128, 3, 128, C, D, E, 64, 1, 0, 0) >= 2 * 3 * 64 * 2
    assert mb(A, F16, 128, B, 128, 3, 128, C, D, E + 2, 64, 1, 0, 0) >= 2 * 3 * 64 * 2 + 128 * 64 * 2
    assert mb(A, F16, 128, B, 128, 0, 128, C, D, E, 64, 1, 1, 1) == 0
    assert lib.si_layer_norm_backward_workspace_bytes(5, 100) == 2 * 2 * 100 * 4  # two blocks of four rows
    assert lib.si_layer_norm_backward_workspace_bytes(0, 100) == 0
    assert lib.si_layer_norm_backward_workspace_bytes(5, 16385) == 0
    assert lib.si_fp8_codes_bytes(3, 17) == 96 and lib.si_fp8_scales_bytes(3, 129) == 24
    assert lib.si_fp8_block_scales_bytes(129, 129) == 16 and lib.si_fp8_block_scales_bytes(0, 5) == 0
    assert lib.si_fp8_codes_bytes(-1, 5) == lib.si_fp8_codes_bytes(5, 0) == 0
    assert lib.si_linear_fp8_workspace_bytes(1, 64, 128, 0) == 0


# ---- refusals --------------------------------------------------------------------------

def linear(x=A, dtype=F16, ldx=128, m=3, n=128, w=B, rows=64, t=0, y=C, y_dtype=F16, ws=D, wb=BIG):
    return "si_linear", x, dtype, ldx, m, n, w, rows, t, y, y_dtype, ws, wb, None


def gated(x=A, dtype=F16, ldx=128, m=3, n=128, wg=B, wu=C, rows=64, h=D, h_dtype=F16, g=None, u=None, ws=E, wb=BIG):
    return "si_gated_linear", x, dtype, ldx, m, n, wg, wu, rows, h, h_dtype, g, u, ws, wb, None


@pytest.mark.parametrize("status,call", [
    (_lib.SI_ERR_ARG, linear(dtype=F32)), (_lib.SI_ERR_ARG, linear(dtype=7)), (_lib.SI_ERR_ARG, linear(y_dtype=3)),
    (_lib.SI_ERR_SHAPE, linear(m=-1)), (_lib.SI_ERR_SHAPE, linear(m=(1 << 24) + 1)), (_lib.SI_ERR_SHAPE, linear(n=0)),
    (_lib.SI_ERR_SHAPE, linear(n=(1 << 20) + 1)), (_lib.SI_ERR_SHAPE, linear(rows=0)),
    (_lib.SI_ERR_SHAPE, linear(rows=(1 << 20) + 1)), (_lib.SI_ERR_SHAPE, linear(ldx=127)),
    (_lib.SI_ERR_SHAPE, linear(ldx=(1 << 21) + 1)), (_lib.SI_ERR_SHAPE, linear(m=1 << 24, rows=1 << 20)),
    (_lib.SI_ERR_SHAPE, linear(n=1 << 18, ldx=1 << 18, rows=1 << 17)), (_lib.SI_ERR_SHAPE, linear(n=1 << 17, ldx=1 << 17, rows=1 << 18, t=1)),
    (_lib.SI_ERR_NULL, linear(x=None)), (_lib.SI_ERR_NULL, linear(w=None)), (_lib.SI_ERR_NULL, linear(y=None)),
    (_lib.SI_ERR_ALIGN, linear(x=A + 1)), (_lib.SI_ERR_ALIGN, linear(w=B + 1)), (_lib.SI_ERR_ALIGN, linear(y=C + 8)),
    (_lib.SI_ERR_ARG, linear(y=A + 256)), (_lib.SI_ERR_ARG, linear(y=B + 64 * 128 * 2 - 16)),
    (_lib.SI_ERR_NULL, linear(n=100, ldx=100, ws=None)), (_lib.SI_ERR_ALIGN, linear(n=100, ldx=100, ws=D + 8)),
    (_lib.SI_ERR_WORKSPACE, linear(n=100, ldx=100, wb=1000)),
    (_lib.SI_ERR_NULL, gated(wg=None)), (_lib.SI_ERR_NULL, gated(h=None)), (_lib.SI_ERR_ALIGN, gated(wu=C + 1)),
    (_lib.SI_ERR_NULL, gated(g=F)), (_lib.SI_ERR_NULL, gated(u=F)), (_lib.SI_ERR_ARG, gated(wu=None, g=F, u=G)),
    (_lib.SI_ERR_ALIGN, gated(g=F + 2, u=G)), (_lib.SI_ERR_ARG, gated(g=F, u=F)), (_lib.SI_ERR_ARG, gated(g=D, u=G)),
    (_lib.SI_ERR_ARG, gated(g=F, u=C)),
])
def test_products_refuse(status, call):
    refused(status, *call)


def backward(dy=A, dy_dtype=F16, lddy=64, x=B, dtype=F16, ldx=128, m=3, n=128, w=C, rows=64, t=0, dx=D, dw=E, ws=F, wb=BIG):
    return "si_linear_backward", dy, dy_dtype, lddy, x, dtype, ldx, m, n, w, rows, t, dx, dw, ws, wb, None


def gated_backward(dh=A, dh_dtype=F16, lddh=64, g=B, g_dtype=F32, u=C, x=D, dtype=F16, ldx=128, m=3, n=128, wg=E, wu=F,
                   rows=64, dx=G, dwg=H, dwu=I, ws=J, wb=BIG):
    return ("si_gated_linear_backward", dh, dh_dtype, lddh, g, g_dtype, u, x, dtype, ldx, m, n, wg, wu, rows, dx, dwg, dwu,
            ws, wb, None)


def mlp_backward(dy=A, dy_dtype=F16, lddy=128, x=B, dtype=F16, ldx=128, m=3, d=128, wg=C, wu=D, wd=E, k=64, h=F, g=G, u=H,
                 dx=I, dwg=J, dwu=K, dwd=L, ws=M, wb=BIG):
    return ("si_mlp_backward", dy, dy_dtype, lddy, x, dtype, ldx, m, d, wg, wu, wd, k, h, g, u, dx, dwg, dwu, dwd, ws, wb, None)


@pytest.mark.parametrize("status,call", [
    (_lib.SI_ERR_ARG, mlp_backward(dtype=F32, dy_dtype=F32)), (_lib.SI_ERR_ARG, mlp_backward(dy_dtype=BF16)),
    (_lib.SI_ERR_SHAPE, mlp_backward(m=-1)), (_lib.SI_ERR_SHAPE, mlp_backward(lddy=127)),
    (_lib.SI_ERR_SHAPE, mlp_backward(ldx=127)), (_lib.SI_ERR_SHAPE, mlp_backward(k=0)),
    (_lib.SI_ERR_SHAPE, mlp_backward(d=(1 << 20) + 1)), (_lib.SI_ERR_SHAPE, mlp_backward(m=1 << 24, k=1 << 20)),
    (_lib.SI_ERR_NULL, mlp_backward(dx=None, dwg=None, dwu=None, dwd=None)), (_lib.SI_ERR_NULL, mlp_backward(dy=None)),
    (_lib.SI_ERR_NULL, mlp_backward(x=None)), (_lib.SI_ERR_NULL, mlp_backward(wg=None)),
    (_lib.SI_ERR_NULL, mlp_backward(wd=None)), (_lib.SI_ERR_NULL, mlp_backward(h=None)),
    (_lib.SI_ERR_NULL, mlp_backward(g=None)), (_lib.SI_ERR_NULL, mlp_backward(u=None)),
    (_lib.SI_ERR_NULL, mlp_backward(wu=None, dwu=None, g=None, u=None, h=None)),
    (_lib.SI_ERR_ARG, mlp_backward(wu=None, dwu=None)), (_lib.SI_ERR_ARG, mlp_backward(wu=None, dwu=None, g=None)),
    (_lib.SI_ERR_ARG, mlp_backward(wu=None, g=None, u=None)),
    (_lib.SI_ERR_ALIGN, mlp_backward(dy=A + 1)), (_lib.SI_ERR_ALIGN, mlp_backward(wd=E + 1)),
    (_lib.SI_ERR_ALIGN, mlp_backward(h=F + 8)), (_lib.SI_ERR_ALIGN, mlp_backward(g=G + 4)),
    (_lib.SI_ERR_ALIGN, mlp_backward(u=H + 8)), (_lib.SI_ERR_ALIGN, mlp_backward(dwd=L + 2)),
    (_lib.SI_ERR_ARG, mlp_backward(dwd=A)), (_lib.SI_ERR_ARG, mlp_backward(dx=F)), (_lib.SI_ERR_ARG, mlp_backward(dwd=G + 752)),
    (_lib.SI_ERR_ARG, mlp_backward(dwu=L)), (_lib.SI_ERR_ARG, mlp_backward(dwg=E + 1024)),
    (_lib.SI_ERR_NULL, mlp_backward(ws=None)), (_lib.SI_ERR_WORKSPACE, mlp_backward(wb=2 * 3 * 64 * 2 - 1)),
    (_lib.SI_ERR_ALIGN, mlp_backward(ws=M + 4)),
])
def test_mlp_gradients_refuse(status, call):
    refused(status, *call)


@pytest.mark.parametrize("status,call", [
    (_lib.SI_ERR_ARG, gated_backward(g_dtype=F16)), (_lib.SI_ERR_ALIGN, gated_backward(g=B + 4)),
    (_lib.SI_ERR_ARG, backward(dtype=F32, dy_dtype=F32)), (_lib.SI_ERR_ARG, backward(dy_dtype=BF16)),
    (_lib.SI_ERR_SHAPE, backward(m=-1)), (_lib.SI_ERR_SHAPE, backward(lddy=63)), (_lib.SI_ERR_SHAPE, backward(ldx=127)),
    (_lib.SI_ERR_SHAPE, backward(lddy=(1 << 21) + 1)), (_lib.SI_ERR_NULL, backward(dx=None, dw=None)),
    (_lib.SI_ERR_NULL, backward(dy=None)), (_lib.SI_ERR_NULL, backward(x=None)), (_lib.SI_ERR_NULL, backward(w=None)),
    (_lib.SI_ERR_ALIGN, backward(dy=A + 1)), (_lib.SI_ERR_ALIGN, backward(dx=D + 8)), (_lib.SI_ERR_ALIGN, backward(dw=E + 8)),
    (_lib.SI_ERR_ARG, backward(dx=A)), (_lib.SI_ERR_ARG, backward(dw=C)), (_lib.SI_ERR_ARG, backward(dx=D, dw=D + 512)),
    (_lib.SI_ERR_NULL, backward(dy_dtype=F32, ws=None)), (_lib.SI_ERR_WORKSPACE, backward(dy_dtype=F32, wb=16)),
    (_lib.SI_ERR_NULL, gated_backward(g=None)), (_lib.SI_ERR_NULL, gated_backward(u=None)),
    (_lib.SI_ERR_ARG, gated_backward(wu=None, dwu=None)), (_lib.SI_ERR_ARG, gated_backward(wu=None, u=None)),
    (_lib.SI_ERR_ARG, gated_backward(dh_dtype=9)), (_lib.SI_ERR_ARG, gated_backward(g_dtype=9)),
    (_lib.SI_ERR_ALIGN, gated_backward(u=C + 1)), (_lib.SI_ERR_ALIGN, gated_backward(dwu=I + 8)),
    (_lib.SI_ERR_ARG, gated_backward(dwg=I, dwu=I)), (_lib.SI_ERR_ARG, gated_backward(dx=B)),
    (_lib.SI_ERR_WORKSPACE, gated_backward(wb=64)), (_lib.SI_ERR_NULL, gated_backward(ws=None)),
])
def test_gradients_refuse(status, call):
    refused(status, *call)


def fp8(xq=A, xs=B, m=3, n=128, q=C, s=D, rows=64, y=E, y_dtype=F16, ws=F, wb=BIG):
    return "si_linear_fp8", xq, xs, m, n, q, s, rows, y, y_dtype, ws, wb, None


def quant(name="si_quantize_rows_fp8", w=A, dt=F16, ld=100, rows=3, n=100, q=B, s=C):
    return name, w, dt, ld, rows, n, q, s, None


@pytest.mark.parametrize("status,call", [
    (_lib.SI_ERR_SHAPE, fp8(m=-1)), (_lib.SI_ERR_SHAPE, fp8(n=(1 << 20) + 1)), (_lib.SI_ERR_SHAPE, fp8(rows=0)),
    (_lib.SI_ERR_NULL, fp8(xq=None)), (_lib.SI_ERR_NULL, fp8(xs=None)), (_lib.SI_ERR_NULL, fp8(q=None)),
    (_lib.SI_ERR_NULL, fp8(s=None)), (_lib.SI_ERR_NULL, fp8(y=None)), (_lib.SI_ERR_ALIGN, fp8(xq=A + 8)),
    (_lib.SI_ERR_ALIGN, fp8(xs=B + 2)), (_lib.SI_ERR_ALIGN, fp8(q=C + 4)), (_lib.SI_ERR_ALIGN, fp8(y=E + 8)),
    (_lib.SI_ERR_ARG, fp8(y_dtype=4)), (_lib.SI_ERR_ARG, fp8(y=A)), (_lib.SI_ERR_ARG, fp8(y=C + 128)),
    (_lib.SI_ERR_ARG, fp8(y=D)),
    (_lib.SI_ERR_NULL, ("si_gated_linear_fp8", A, B, 3, 128, C, D, E, None, 64, F, F16, G, BIG, None)),
    (_lib.SI_ERR_ARG, quant(dt=5)), (_lib.SI_ERR_SHAPE, quant(rows=-1)), (_lib.SI_ERR_SHAPE, quant(n=0)),
    (_lib.SI_ERR_SHAPE, quant(ld=99)), (_lib.SI_ERR_SHAPE, quant(rows=1 << 24, n=1 << 24, ld=1 << 24)),
    (_lib.SI_ERR_NULL, quant(w=None)), (_lib.SI_ERR_NULL, quant(q=None)), (_lib.SI_ERR_NULL, quant(s=None)),
    (_lib.SI_ERR_ALIGN, quant(w=A + 1)), (_lib.SI_ERR_ALIGN, quant(q=B + 8)), (_lib.SI_ERR_ALIGN, quant(s=C + 4)),
    (_lib.SI_ERR_ARG, quant(q=A)), (_lib.SI_ERR_ARG, quant(s=B + 16)),
    (_lib.SI_ERR_NULL, quant(name="si_quantize_blocks_fp8", s=None)),
    (_lib.SI_ERR_ARG, ("si_dequantize_fp8", A, B, 2, 3, 100, C, F16, None)),
    (_lib.SI_ERR_NULL, ("si_dequantize_fp8", A, B, 1, 3, 100, None, F16, None)),
    (_lib.SI_ERR_ARG, ("si_dequantize_fp8", A, B, 1, 3, 100, A, F16, None)),
    (_lib.SI_ERR_ALIGN, ("si_dequantize_fp8", A, B, 128, 3, 100, C + 2, F32, None)),
])
def test_fp8_refuses(status, call):
    refused(status, *call)


def norm(x=A, dt=F16, ld=100, w=B, b=C, wt=F32, center=1, eps=1e-5, y=D, mean=E, rstd=F, tokens=3, d=100):
    return "si_layer_norm", x, dt, ld, w, b, wt, center, eps, y, mean, rstd, tokens, d, None


def norm_backward(dy=A, lddy=100, x=B, dt=F16, ldx=100, w=C, wt=F32, center=1, mean=D, rstd=E, dx=F, dw=G, db=H, tokens=3,
                  d=100, ws=I, wb=BIG):
    return "si_layer_norm_backward", dy, lddy, x, dt, ldx, w, wt, center, mean, rstd, dx, dw, db, tokens, d, ws, wb, None


@pytest.mark.parametrize("status,call", [
    (_lib.SI_ERR_ARG, norm(dt=3)), (_lib.SI_ERR_ARG, norm(wt=-1)), (_lib.SI_ERR_SHAPE, norm(tokens=-1)),
    (_lib.SI_ERR_SHAPE, norm(tokens=1 << 23)), (_lib.SI_ERR_SHAPE, norm(d=0)), (_lib.SI_ERR_SHAPE, norm(d=16385, ld=16385)),
    (_lib.SI_ERR_SHAPE, norm(ld=99)), (_lib.SI_ERR_ARG, norm(eps=-1.0)), (_lib.SI_ERR_ARG, norm(eps=math.nan)),
    (_lib.SI_ERR_ARG, norm(eps=math.inf)), (_lib.SI_ERR_NULL, norm(x=None)), (_lib.SI_ERR_NULL, norm(w=None)),
    (_lib.SI_ERR_NULL, norm(y=None)), (_lib.SI_ERR_NULL, norm(mean=None)), (_lib.SI_ERR_NULL, norm(rstd=None)),
    (_lib.SI_ERR_ALIGN, norm(x=A + 1)), (_lib.SI_ERR_ALIGN, norm(w=B + 2)), (_lib.SI_ERR_ALIGN, norm(y=D + 1)),
    (_lib.SI_ERR_ARG, norm(y=A)), (_lib.SI_ERR_ARG, norm(mean=D)), (_lib.SI_ERR_ARG, norm(rstd=B)),
    (_lib.SI_ERR_NULL, norm_backward(dx=None, dw=None, db=None)), (_lib.SI_ERR_NULL, norm_backward(dy=None)),
    (_lib.SI_ERR_NULL, norm_backward(x=None)), (_lib.SI_ERR_NULL, norm_backward(w=None)),
    (_lib.SI_ERR_NULL, norm_backward(mean=None)), (_lib.SI_ERR_NULL, norm_backward(rstd=None, center=0)),
    (_lib.SI_ERR_SHAPE, norm_backward(lddy=99)), (_lib.SI_ERR_SHAPE, norm_backward(ldx=99)),
    (_lib.SI_ERR_ALIGN, norm_backward(dw=G + 2)), (_lib.SI_ERR_ARG, norm_backward(dx=A)),
    (_lib.SI_ERR_ARG, norm_backward(dw=H, db=H)), (_lib.SI_ERR_NULL, norm_backward(ws=None)),
    (_lib.SI_ERR_WORKSPACE, norm_backward(wb=100)),
])
def test_norms_refuse(status, call):
    refused(status, *call)


def test_nothing_to_do():
    """No tokens: accepted without a launch (the weights' gradients, which are zeros
    then, are asked for on the GPU)."""
    for call in (linear(m=0, x=None), gated(m=0, x=None), quant(rows=0), fp8(m=0), norm(tokens=0, x=None),
                 backward(m=0, dw=None), mlp_backward(m=0, dwg=None, dwu=None, dwd=None), norm_backward(tokens=0, dw=None, db=None)):
        assert _lib.status(*call) == _lib.SI_OK, (call[0], _lib.last_error())


def test_no_tokens_and_no_gradient_of_a_weight():
    """The gradient with respect to x of no tokens has no address: with that alone asked
    for there is nothing to do, where with tokens it is a call without a gradient."""
    for call in (lambda m: backward(m=m, dx=None, dw=None), lambda m: backward(m=m, dx=None, dw=None, t=1),
                 lambda m: gated_backward(m=m, dx=None, dwg=None, dwu=None),
                 lambda m: mlp_backward(m=m, dx=None, dwg=None, dwu=None, dwd=None),
                 lambda m: norm_backward(tokens=m, dx=None, dw=None, db=None),
                 lambda m: norm_backward(tokens=m, dx=None, dw=None, db=None, center=0)):
        assert _lib.status(*call(0)) == _lib.SI_OK, (call(0)[0], _lib.last_error())
        refused(_lib.SI_ERR_NULL, *call(3))
    refused(_lib.SI_ERR_SHAPE, *backward(m=-1, dx=None, dw=None))
    refused(_lib.SI_ERR_ALIGN, *backward(m=0, dx=None, dw=None, w=C + 1))


def test_python_refuses_before_a_device_is_needed():
    x, w = torch.zeros(2, 8, dtype=torch.float16), torch.zeros(4, 8, dtype=torch.float16)
    for f in (lambda: si.linear(x, w), lambda: si.gated_linear(x, w, w), lambda: si.mlp(x, w, w, w.t()),
              lambda: si.layer_norm(x, x[0], x[0]), lambda: si.rms_norm(x, x[0]), lambda: si.quantize_rows_fp8(x),
              lambda: si.quantize_blocks_fp8(x), lambda: si.FP8MLPLayer(w, w, w)):
        with pytest.raises(ValueError, match="CUDA"):
            f()
    for f in (lambda: si.linear([1.0], w), lambda: si.layer_norm(None, x[0])):
        with pytest.raises(TypeError):
            f()
    with pytest.raises(ValueError):
        si.linear(torch.zeros((), dtype=torch.float16), w)
