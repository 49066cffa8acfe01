"""FP8 rows and blocks and the products with them on the GPU.

Codes and scales are compared bit by bit with the definition.  Most products are built so
that every partial sum is exact: codes that are small whole numbers and scales that are
powers of two.  Gaussian values are compared within ``(128 + 16) 2^-23`` of each block's
sum of magnitudes (a unit in the last place for each addition), a step for the scales'
product and for each block's addition, and half a step of the output's type.
"""

import math

import pytest
import torch

import dense_ref as ref
import paper_2411_12692_amd as si
from dense_ref import BF16, F16, F32, HALF_STEP, SMALLEST

pytestmark = pytest.mark.gpu
DEV = "cuda"
E4M3 = torch.float8_e4m3fn


def gen(*key):
    g = torch.Generator()
    g.manual_seed(hash(key) % (1 << 31))
    return g


def check_quantized(w, per):
    q, s = (si.quantize_rows_fp8 if per == 1 else si.quantize_blocks_fp8)(w)
    codes, scale = ref.quantize(w.float().cpu(), per)
    assert q.dtype == E4M3 and s.dtype == F32 and s.shape == scale.shape
    assert torch.equal(torch.nan_to_num(s.cpu(), nan=-1.0), torch.nan_to_num(scale, nan=-1.0))
    assert torch.equal(q.view(torch.uint8).cpu(), codes)
    return q, s, codes, scale


@pytest.mark.parametrize("per", [1, 128])
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("rows,n", [(1, 1), (1, 15), (3, 16), (2, 17), (5, 127), (7, 128), (130, 129), (128, 256), (257, 264),
                                    (19, 4096), (3, 11008), (129, 1000), (1, 70001)])
def test_quantize_and_back(rows, n, dtype, per):
    g = gen(0, rows, n)
    w = (torch.randn(rows, n, generator=g) * torch.exp2(torch.randint(-9, 9, (rows, 1), generator=g).float())).to(dtype)
    q, s, codes, scale = check_quantized(w.to(DEV), per)
    want = ref.values(codes, scale, n, per)
    assert torch.equal(si.dequantize_fp8(q, s, n, F32).cpu(), want.float())  # a product of 4 and 24 bits: one rounding
    for out in (F16, BF16):
        back = si.dequantize_fp8(q, s, n, out)
        assert back.dtype == out and torch.equal(back.cpu(), want.float().to(out))


@pytest.mark.parametrize("per", [1, 128])
def test_quantize_ties_signs_and_special_blocks(per):
    """Every midpoint of two codes and its neighbours at several scales; zeros of both
    signs; the largest and smallest values; infinities and NaN."""
    v = ref.e4m3_values()
    mid = ((v[1:] + v[:-1]) / 2).float()
    row = torch.cat([mid, torch.tensor([448.0])])[:127]
    row = torch.nn.functional.pad(row, (0, 1), value=448.0)
    base = torch.stack([row, -row, row * (1 + 2.0 ** -23), row * (1 - 2.0 ** -24)])
    base[2:, -2:] = 448.0
    rows = torch.cat([base * 2.0 ** e for e in (-60, -3, 0, 5, 100)])
    for part in (rows.split(4) if per == 128 else [rows]):
        check_quantized(part.contiguous().to(DEV), per)
    w = torch.zeros(8, 300)
    w[1] = -0.0
    w[2, 40], w[3, 140], w[4, 299] = math.inf, math.nan, -math.inf
    w[5] = torch.arange(300) * 2.0 ** -149
    w[6] = torch.finfo(F32).max
    w[7, 5] = 2.0 ** -149
    if per == 1:
        check_quantized(w.to(DEV), per)
        q, s = si.quantize_rows_fp8(w.to(DEV))
        back = si.dequantize_fp8(q, s, 300, F32)
        assert back[2, :128].isnan().all() and (back[2, 128:] == 0).all() and back[3, 128:256].isnan().all()
        assert back[4, 256:].isnan().all() and (back[0] == 0).all() and (back[6] == torch.finfo(F32).max).all()
    else:
        for i in range(8):
            check_quantized(w[i:i + 1].to(DEV), per)


def test_quantize_strides_and_no_rows():
    g = gen(1)
    big = torch.randn(40, 500, generator=g).half().to(DEV)
    for per in (1, 128):
        for w in (big[:, 3:259], big[::2, :264], big[5:6, 1:130], big[:0]):
            check_quantized(w, per) if w.shape[0] else None
    assert si.quantize_rows_fp8(big[:0])[0].shape == (0, 512)


# ---- products ----------------------------------------------------------------------

def whole_fp8(g, rows, n, per, most):
    """Codes that are whole numbers -most .. most, scales powers of two."""
    np_, nb = (n + 15) // 16 * 16, (n + 127) // 128
    v = torch.zeros(rows, np_)
    v[:, :n] = ref.whole(g, -most, most, rows, n).float()
    s = torch.exp2(ref.whole(g, -1, 1, (rows + per - 1) // per, nb).float())
    q = v.to(E4M3)
    assert torch.equal(q.float(), v)
    return q, s


def exact_values(q, s, per):
    """float64 values on the GPU."""
    v = q.float().double().to(DEV)
    scale = s.double().to(DEV).repeat_interleave(per, dim=0)[: q.shape[0]].repeat_interleave(128, dim=1)[:, : q.shape[1]]
    return v * scale


@pytest.mark.parametrize("m,rows,n", ref.shapes("fp8") + [(5, 200, 17), (6, 300, 4112), (2, 129, 100)])
def test_linear_exact(m, rows, n):
    g = gen(2, m, rows, n)
    xq, xs = whole_fp8(g, m, n, 1, 2)
    q, s = whole_fp8(g, rows, n, 128, 1)
    want = exact_values(xq, xs, 1) @ exact_values(q, s, 128).t().contiguous()
    assert want.abs().max() < 2 ** 20  # whole multiples of 1/4: exact in float32
    for out in (F16, BF16, F32):
        y = si.linear_fp8(xq.to(DEV), xs.to(DEV), q.to(DEV), s.to(DEV), out)
        assert y.dtype == out and torch.equal(y, want.float().to(out))


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("m,rows,n", ref.shapes("fp8", True) + [(5, 200, 17), (2, 129, 100)])
def test_gated_linear_exact(m, rows, n, up):
    g = gen(3, m, rows, n)
    xq, xs = whole_fp8(g, m, n, 1, 1)
    q, s = whole_fp8(g, rows, n, 128, 1)
    qu, su = whole_fp8(g, rows, n, 128, 1) if up else (None, None)
    X = exact_values(xq, xs, 1)
    gv = X @ exact_values(q, s, 128).t().contiguous()
    uv = X @ exact_values(qu, su, 128).t().contiguous() if up else None
    want = ref.gated(gv, uv)
    dev = [None if t is None else t.to(DEV) for t in (xq, xs, q, s, qu, su)]
    for out in (F16, BF16, F32):
        assert torch.equal(si.gated_linear_fp8(*dev, out_dtype=out), want.to(out))


@pytest.mark.parametrize("m,rows,n", [(1, 300, 11008), (3, 256, 4096), (20, 700, 4100), (200, 1000, 1371), (500, 3000, 2048)])
def test_gaussian_values(m, rows, n):
    g = gen(4, m, rows, n)
    x = torch.randn(m, n, generator=g).to(DEV)
    w, wu = (torch.randn(rows, n, generator=g).mul(n ** -0.5).to(DEV) for _ in range(2))
    xq, xs = si.quantize_rows_fp8(x)
    q, s = si.quantize_blocks_fp8(w)
    qu, su = si.quantize_blocks_fp8(wu)
    X, W, U = (exact_values(a.cpu(), b.cpu(), p) for a, b, p in ((xq, xs, 1), (q, s, 128), (qu, su, 128)))
    step = (128 + 16 + (n + 127) // 128 + 4) * 2.0 ** -23
    gv, gs, uv, us = X @ W.t(), X.abs() @ W.abs().t(), X @ U.t(), X.abs() @ U.abs().t()
    for out in (BF16, F32):
        y = si.linear_fp8(xq, xs, q, s, out).double()
        err = step * gs
        assert ((y - gv).abs() <= err + HALF_STEP[out] * 1.01 * (gv.abs() + err) + SMALLEST[out]).all()
        h = si.gated_linear_fp8(xq, xs, q, s, qu, su, out).double()
        want = torch.relu(gv) * uv
        err = step * gs * uv.abs() + gv.abs() * step * us + step * step * gs * us + 2.0 ** -23 * want.abs()
        assert ((h - want).abs() <= err + HALF_STEP[out] * 1.01 * (want.abs() + err) + SMALLEST[out]).all()


@pytest.mark.parametrize("m", [1, 9, 150])
def test_nan_scales_and_zero_scales(m):
    """A NaN scale of a token's block reaches that token, of W's block its 128 rows; a
    zero scale of a block of zeros does nothing; neighbours in a tile stay."""
    g = gen(5, m)
    n, rows = 640, 300
    x, w = torch.randn(m, n, generator=g).to(DEV), torch.randn(rows, n, generator=g).to(DEV)
    w[128:256, 256:384] = 0.0
    clean = si.linear_fp8(*si.quantize_rows_fp8(x), *si.quantize_blocks_fp8(w), out_dtype=F32)
    assert clean.isfinite().all()
    w[130, 130] = float("nan")
    y = si.linear_fp8(*si.quantize_rows_fp8(x), *si.quantize_blocks_fp8(w), out_dtype=F32)
    assert y[:, 128:256].isnan().all() and torch.equal(y[:, :128], clean[:, :128]) and torch.equal(y[:, 256:], clean[:, 256:])
    w[130, 130] = 0.5
    clean = si.linear_fp8(*si.quantize_rows_fp8(x), *si.quantize_blocks_fp8(w), out_dtype=F32)
    x[m - 1, 639] = float("inf")
    y = si.linear_fp8(*si.quantize_rows_fp8(x), *si.quantize_blocks_fp8(w), out_dtype=F32)
    assert y[m - 1].isnan().all() and torch.equal(y[:m - 1], clean[:m - 1])


def test_a_checkpoint_s_rows_that_end_inside_a_block():
    """n a multiple of 16 that is none of 128, codes as a checkpoint holds them, NaN codes
    behind other rows' ends and in other tensors must not be read."""
    g = gen(6)
    q, s = whole_fp8(g, 40, 144, 128, 1)
    xq, xs = whole_fp8(g, 33, 144, 1, 1)
    pool = torch.full((33 * 144 + 40 * 144 + 4096,), 0x7F, dtype=torch.uint8).view(E4M3).to(DEV)  # NaN everywhere
    a, b = pool[1024:1024 + 33 * 144].view(33, 144), pool[8192 - 1024 + 512:][: 40 * 144].view(40, 144)
    b = pool[1024 + 33 * 144 + 1024 - (33 * 144) % 16:][: 40 * 144].view(40, 144) if b.data_ptr() % 16 else b
    a.copy_(xq.to(DEV))
    b.copy_(q.to(DEV))
    want = exact_values(xq, xs, 1) @ exact_values(q, s, 128).t().contiguous()
    assert torch.equal(si.linear_fp8(a, xs.to(DEV), b, s.to(DEV), F32), want.float())


def test_longest_sum_and_offsets_past_32_bits():
    n = 1 << 20
    x = torch.ones(5, n, device=DEV)
    w = torch.ones(3, n, device=DEV)
    w[:, ::2] = 0.0
    xq, xs = si.quantize_rows_fp8(x)
    q, s = si.quantize_blocks_fp8(w)
    for m in (1, 5):
        y = si.linear_fp8(xq[:m], xs[:m], q, s, F32)
        # 2^19 products of 448^2 / 448^2, the scales 1/448 rounded twice
        assert ((y / (n / 2) - 1).abs() < 2.0 ** -22).all()
    m, rows = 70001, 32776  # more than 2^31 outputs
    xq = torch.zeros(m, 16, dtype=torch.uint8, device=DEV)
    xs = torch.ones(m, 1, device=DEV)
    xq[m - 1] = xq[0] = 0x38  # 1.0
    q = torch.full((rows, 16), 0x38, dtype=torch.uint8, device=DEV)
    s = torch.ones((rows + 127) // 128, 1, device=DEV)
    y = si.linear_fp8(xq.view(E4M3), xs, q.view(E4M3), s, F16)
    assert (y[0] == 16).all() and (y[m - 1] == 16).all() and not y[1:100].any() and not y[m - 100:m - 1].any()


def test_streams_and_graph():
    g = gen(7)
    x, w = torch.randn(37, 700, generator=g).half().to(DEV), torch.randn(400, 700, generator=g).half().to(DEV)
    q, s = si.quantize_blocks_fp8(w)
    f = lambda: si.gated_linear_fp8(*si.quantize_rows_fp8(x), q, s, q, s, F32)  # noqa: E731
    want = f()
    torch.cuda.synchronize()
    outs = []
    for st in [torch.cuda.Stream() for _ in range(3)]:
        with torch.cuda.stream(st):
            outs.append(f())
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = f()
    for scale in (1.0, -0.5, 3.0):
        x.copy_(torch.randn(37, 700, generator=g).half().mul(scale))
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        assert torch.equal(got, f())


def test_python_refuses():
    x, w = torch.randn(4, 64, device=DEV), torch.randn(130, 64, device=DEV)
    xq, xs = si.quantize_rows_fp8(x)
    q, s = si.quantize_blocks_fp8(w)
    for error, f in ((TypeError, lambda: si.linear_fp8(x, xs, q, s)), (ValueError, lambda: si.linear_fp8(xq, xs, q, s[:1])),
                     (ValueError, lambda: si.linear_fp8(xq, xs[:3], q, s)), (ValueError, lambda: si.linear_fp8(xq[:, :48].contiguous(), xs, q, s)),
                     (TypeError, lambda: si.linear_fp8(xq, xs, q, s, torch.int8)), (TypeError, lambda: si.linear_fp8(xq, xs.half(), q, s)),
                     (ValueError, lambda: si.gated_linear_fp8(xq, xs, q, s, q[:64], s[:1])), (ValueError, lambda: si.linear_fp8(xq, xs, q, s.cpu())),
                     (ValueError, lambda: si.dequantize_fp8(q, s, 80)), (TypeError, lambda: si.dequantize_fp8(q, s, 64, torch.int32)),
                     (ValueError, lambda: si.quantize_rows_fp8(x.t())), (TypeError, lambda: si.quantize_rows_fp8(x.int()))):
        with pytest.raises(error):
            f()


# ---- the layer, and a run from training to serving ------------------------------------

@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("m", [1, 3, 40, 300])
def test_layer(m, dtype, up):
    g = gen(8, m)
    d, k = 200, 328
    wg, wu, wd = (torch.randn(s, generator=g).mul(0.08).to(dtype).to(DEV) for s in ((k, d), (k, d), (d, k)))
    x = torch.randn(m, d, generator=g).to(dtype).to(DEV)
    layer = si.FP8MLPLayer(wg, wu if up else None, wd)
    y = layer.prompt(x)
    h = si.gated_linear_fp8(*si.quantize_rows_fp8(x), *si.quantize_blocks_fp8(wg), *(si.quantize_blocks_fp8(wu) if up else ()),
                            out_dtype=dtype)
    want = si.linear_fp8(*si.quantize_rows_fp8(h), *si.quantize_blocks_fp8(wd), out_dtype=dtype)
    assert torch.equal(y, want)
    same = si.FP8MLPLayer.from_blocks(si.quantize_blocks_fp8(wg), si.quantize_blocks_fp8(wu) if up else None,
                                      si.quantize_blocks_fp8(wd))
    assert torch.equal(same.prompt(x), want) and same.prompt(x, out_dtype=F32).dtype == F32
    hs = torch.randn(m, d, generator=g).to(DEV)
    out, nxt = layer.prompt_block(hs, torch.ones(d, device=DEV), 1e-5, next_norm_w=torch.ones(d, device=DEV))
    _, xn = si.norm_residual(hs, pre_w=torch.ones(d, device=DEV), x_dtype=BF16)
    o2, n2 = si.norm_residual(hs, layer.prompt(xn), pre_w=torch.ones(d, device=DEV), x_dtype=BF16)
    assert torch.equal(out, o2) and torch.equal(nxt, n2)
    with pytest.raises(ValueError):
        layer.prompt(x[:, :100].contiguous())
    with pytest.raises(ValueError):
        si.FP8MLPLayer.from_blocks(si.quantize_blocks_fp8(wg), None, si.quantize_blocks_fp8(wg))


@pytest.mark.parametrize("gated", [True, False])
def test_train_then_serve(gated):
    """The MLP half of a layer as a user has it: norm, MLP and residual forward and
    backward, an update of the weights, then the trained layer's prompts with fp16 and
    FP8 weights and its decode, each against float64 of the same weights."""
    g = gen(9)
    m, d, k = 48, 256, 704
    shapes = [(k, d), (k, d), (d, k)] if gated else [(k, d), (d, k)]
    weights = [torch.randn(s, generator=g).mul(s[1] ** -0.5).half().to(DEV).requires_grad_() for s in shapes]
    nw, nb = torch.ones(d, device=DEV).requires_grad_(), torch.zeros(d, device=DEV).requires_grad_()
    h = torch.randn(m, d, generator=g).half().to(DEV)
    target = torch.randn(m, d, generator=g).to(DEV)

    def unit(w):
        return si.rms_norm(h, nw) if gated else si.layer_norm(h, nw, nb)
    wg, wd = weights[0], weights[-1]
    wu = weights[1] if gated else None
    y = h + si.mlp(unit(h), wg, wu, wd)
    loss = (y.float() - target).square().mean()
    leaves = weights + ([nw] if gated else [nw, nb])
    grads = torch.autograd.grad(loss, leaves)
    # the same in float64, gradients by autograd
    L = [t.detach().double().requires_grad_() for t in leaves]
    X = h.double()
    c = X if gated else X - X.mean(dim=1, keepdim=True)
    n = c / torch.sqrt((c * c).mean(dim=1, keepdim=True) + 1e-5) * L[len(weights)]
    n = n if gated else n + L[-1]
    pre = n @ L[0].t()
    hid = torch.relu(pre) * (n @ L[1].t()) if gated else torch.relu(pre)
    Y = X + hid @ L[len(weights) - 1].t()
    want = torch.autograd.grad((Y - target.double()).square().mean(), L)
    # At most eight roundings of 2^-11 lie between the loss and any gradient, each of values
    # whose errors are independent of the sums they enter.  The loss is a mean over 12288
    # values, so dy, dh, dg and du (about 1e-4) lie around fp16's smallest normal number,
    # below which a rounding is off by up to 2^-25 whatever the value: those errors go
    # through the same sums as the values, with magnitudes in the matrices' places.
    tiny, W = 2.0 ** -25, [t.detach().abs() for t in L]
    pre_up = (n @ L[1].t()).detach().abs() if gated else torch.ones_like(pre)
    on, N = (pre.detach() > 0).double(), n.detach().abs()
    e_dy = torch.full_like(X, tiny)
    e_dh = e_dy @ W[len(weights) - 1] + tiny
    e_dg, e_du = e_dh * pre_up * on + tiny, e_dh * torch.relu(pre.detach()) + tiny
    e_dn = e_dg @ W[0] + (e_du @ W[1] if gated else 0.0) + tiny
    slack = [e_dg.t() @ N + tiny] + ([e_du.t() @ N + tiny] if gated else []) + [e_dy.t() @ hid.detach().abs() + tiny]
    slack += [(e_dn * N).sum(dim=0)] + ([] if gated else [e_dn.sum(dim=0)])
    for a, b, e in zip(grads, want, slack):
        assert (a.double() - b).norm() <= 8 * 2.0 ** -11 * b.norm() + e.norm()
    with torch.no_grad():
        for t, gr in zip(leaves, grads):
            t -= (0.1 * gr).to(t.dtype)
    x = unit(h).detach()
    wg, wd, wu = wg.detach(), wd.detach(), wu.detach() if gated else None
    P = x.double() @ wg.double().t()
    H = torch.relu(P) * (x.double() @ wu.double().t()) if gated else torch.relu(P)
    Y = H @ wd.double().t()
    fp16 = si.MLPLayer(wg, wu, wd)
    assert (fp16.prompt(x).double() - Y).norm() <= 4 * 2.0 ** -11 * Y.norm()
    assert (fp16(x[:1], float("inf")).double() - Y[:1]).norm() <= 4 * 2.0 ** -11 * Y[:1].norm()
    # FP8: weights, tokens and hidden values each off by at most half a step, 2^-4, of
    # themselves; independent errors of that size over three quarters of a uniform step
    fp8 = si.FP8MLPLayer(wg, wu, wd).prompt(x)
    assert (fp8.double() - Y).norm() <= 6 * 2.0 ** -4 * Y.norm()
