"""LayerNorm and RMSNorm with their gradients on the GPU against float64.

Bounds, relative to the magnitudes that are summed: a mean of d values in float32 is off
by at most ``(d + 64) 2^-24`` of the mean magnitude in any order (a half step for each
addition), the square root, division and products by a few half steps more; written
values by half a step of their type.
"""

import pytest
import torch

import dense_ref as ref
import paper_2411_12692_amd as si
from dense_ref import BF16, F16, F32, HALF_STEP, SMALLEST

pytestmark = pytest.mark.gpu
DEV = "cuda"
EPS = 1e-5


def gen(*key):
    g = torch.Generator()
    g.manual_seed(hash(key) % (1 << 31))
    return g


def call(x, w, b, center, eps=EPS):
    return si.layer_norm(x, w, b, eps=eps) if center else si.rms_norm(x, w, eps=eps)


def half(v, dtype):
    return HALF_STEP[dtype] * 1.01 * v.abs() + SMALLEST[dtype]


def check(x, w, b, dy, center, eps=EPS):
    """Forward and backward of given tensors; x, dy rows of any stride."""
    xr, wr = x.detach().requires_grad_(), w.detach().requires_grad_()
    br = b.detach().requires_grad_() if b is not None else None
    y = call(xr, wr, br, center, eps)
    leaves = [t for t in (xr, wr, br) if t is not None]
    got = torch.autograd.grad(y, leaves, dy)
    assert torch.equal(call(x, w, b, center, eps), y.detach())  # without a graph: the same bits
    X, W, DY = x.detach().double(), w.detach().double(), dy.double()
    B = None if b is None else b.detach().double()
    t, d = X.shape
    u = (d + 64) * 2.0 ** -24
    mean = X.mean(dim=1, keepdim=True) if center else torch.zeros(t, 1, dtype=torch.float64, device=DEV)
    # c = x - mean is off by the mean's error and half a step; r by c's error on it
    ec = (u * X.abs().mean(dim=1, keepdim=True) if center else 0.0) + 2.0 ** -24 * (X - mean).abs()
    c = X - mean
    var = (c * c).mean(dim=1, keepdim=True) + eps
    r = var.rsqrt()
    er = (u + 8 * 2.0 ** -24 + (c.abs() * ec).mean(dim=1, keepdim=True) / var) * 1.1  # relative
    n = c * r
    en = (ec * r + n.abs() * (er + 2 * 2.0 ** -24)) * 1.1
    want = ref.norm(X, W, B, eps, center)
    err = en * W.abs() + 3 * 2.0 ** -24 * ((n * W).abs() + (B.abs() if B is not None else 0.0))
    assert y.dtype == x.dtype
    assert ((y.detach().double() - want).abs() <= err + half(want.abs() + err, x.dtype)).all()
    dx, dw, db, size, aw, ab = ref.norm_grad(X, W, DY, eps, center)
    e = (DY * W).abs()
    edx = (u + 2 * er + 16 * 2.0 ** -24) * size + r * ((e * en).mean(dim=1, keepdim=True) * n.abs() + en * (e * n.abs()).mean(dim=1, keepdim=True))
    edx = 1.1 * edx
    assert got[0].dtype == x.dtype and ((got[0].double() - dx).abs() <= edx + half(dx.abs() + edx, x.dtype)).all()
    ut = (t + 64) * 2.0 ** -24
    ew = (DY.abs() * en).sum(dim=0) + ut * aw * 1.1
    assert got[1].dtype == w.dtype and ((got[1].double() - dw).abs() <= ew + half(dw.abs() + ew, w.dtype)).all()
    if b is not None:
        eb = ut * ab
        assert ((got[2].double() - db).abs() <= eb + half(db.abs() + eb, w.dtype)).all()


def inputs(g, t, d, dtype, w_dtype, bias):
    x = (torch.randn(t, d, generator=g) * 2 + 0.5).to(dtype).to(DEV)
    w = (1 + 0.1 * torch.randn(d, generator=g)).to(w_dtype).to(DEV)
    b = (0.1 * torch.randn(d, generator=g)).to(w_dtype).to(DEV) if bias else None
    return x, w, b, torch.randn(t, d, generator=g).to(dtype).to(DEV)


SIZES = [(1, 1), (1, 7), (3, 64), (5, 100), (2, 511), (9, 512), (4, 513), (33, 520), (1, 4096), (70, 5119), (130, 5120),
         (3, 8192), (2, 8200), (7, 16384), (5, 16383), (1999, 320), (2500, 96)]


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("dtype,w_dtype", [(F16, F32), (F16, F16), (BF16, BF16), (BF16, F32), (F32, F32), (F32, BF16)])
@pytest.mark.parametrize("t,d", SIZES)
def test_forward_and_backward(t, d, dtype, w_dtype, center):
    check(*inputs(gen(0, t, d), t, d, dtype, w_dtype, center), center)


@pytest.mark.parametrize("dtype", [F16, BF16, F32])
def test_layer_norm_without_bias(dtype):
    x, w, _, dy = inputs(gen(1), 40, 300, dtype, F32, False)
    check(x, w, None, dy, True)


@pytest.mark.parametrize("center", [True, False])
@pytest.mark.parametrize("dtype", [F16, BF16, F32])
@pytest.mark.parametrize("d", [256, 1000, 251])
def test_strides_and_unaligned_rows(dtype, center, d):
    g = gen(2, d)
    x, w, b, dy = inputs(g, 20, 2 * d + 5, dtype, F32, center)
    flat = torch.randn(d + 1, generator=g).to(DEV)
    b1 = b[1:d + 1] if b is not None else None
    check(x[:, 3:d + 3], flat[1:], b1, dy[:, 5:d + 5], center)
    check(x[::3, :d], flat[:d], b1, dy[1::3, :d], center)
    check(x[4:5, 1:d + 1], flat[:d], b1, dy[:1, :d], center)


@pytest.mark.parametrize("dtype", [F16, F32])
def test_large_mean_and_small_spread(dtype):
    """Values around 1000 that differ by a few steps: the variance is taken about the
    mean, not as a difference of squares."""
    g = gen(3)
    x = (1000 + torch.randint(-2, 3, (20, 768), generator=g) * float(torch.finfo(dtype).eps) * 512).to(dtype).to(DEV)
    w, dy = torch.ones(768, device=DEV), torch.randn(20, 768, generator=g).to(dtype).to(DEV)
    check(x, w, None, dy, True, eps=1e-12)


def test_zero_and_special_rows():
    """A row of zeros or of one value has y = b; a NaN or an infinity stays in its row
    (and in the columns' sums, whose terms it is)."""
    g = gen(4)
    x, w, b, dy = inputs(g, 9, 600, F16, F32, True)
    x[0] = 0.0
    x[1] = 3.0
    y = si.layer_norm(x, w, b)
    assert torch.equal(y[0], b.half()) and torch.equal(y[1], b.half())
    assert (si.rms_norm(x, w)[0] == 0).all()
    clean = si.layer_norm(x, w, b)
    x[2, 5] = float("nan")
    x[3, 599] = float("inf")
    y = si.layer_norm(x, w, b)
    assert y[2].isnan().all() and y[3].isnan().any() and torch.equal(y[4:], clean[4:])
    xr, wr = x.requires_grad_(), w.requires_grad_()
    dx, dw = torch.autograd.grad(si.layer_norm(xr, wr, b), (xr, wr), dy)
    assert dx[2].isnan().all() and dx[4:].isfinite().all() and dx[0].isfinite().all() and dw.isnan().any()


def test_eps_and_tiny_rows():
    """eps decides where the row is smaller than its root.  1e-40, the square, is a float32
    subnormal: a step of 2^-149 is 1.4e-5 of it, half a step in the sum and half of that
    in the root, 3.5e-6."""
    x = torch.full((3, 128), 1e-20, device=DEV)
    x[:, ::2] = -1e-20
    w = torch.ones(128, device=DEV)
    for eps in (1e-5, 0.0, 1.0):
        y = si.rms_norm(x, w, eps=eps)
        want = x.double() / torch.sqrt(x.double().square().mean(dim=1, keepdim=True) + eps)
        assert torch.allclose(y.double(), want, rtol=1e-5, atol=0)


@pytest.mark.parametrize("center", [True, False])
def test_incoming_gradients_of_any_layout(center):
    g = gen(5)
    x, w, b, dy = inputs(g, 33, 200, F16, F16, center)
    leaves = [t.requires_grad_() for t in (x, w, b) if t is not None]
    y = call(x, w, b, center)
    want = torch.autograd.grad(y, leaves, dy, retain_graph=True)
    for d in (dy.t().contiguous().t(), torch.cat([dy, dy], dim=1)[:, :200]):
        assert all(torch.equal(a, c) for a, c in zip(torch.autograd.grad(y, leaves, d, retain_graph=True), want))
    ones = torch.autograd.grad(y, leaves, torch.ones_like(y), retain_graph=True)
    assert all(torch.equal(a, c) for a, c in zip(torch.autograd.grad(y.sum(), leaves), ones))


def test_gradients_in_part_and_leading_dimensions():
    g = gen(6)
    x, w, b, dy = inputs(g, 30, 264, BF16, F32, True)
    full = [t.clone().requires_grad_() for t in (x, w, b)]
    want = torch.autograd.grad(si.layer_norm(*full), full, dy)
    for needs in ((1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (1, 0, 1), (0, 1, 1)):
        part = [t.clone().view(2, 15, 264).requires_grad_(bool(k)) if i == 0 else t.clone().requires_grad_(bool(k))
                for i, (t, k) in enumerate(zip((x, w, b), needs))]
        y = si.layer_norm(*part)
        assert y.shape == (2, 15, 264)
        leaves = [t for t in part if t.requires_grad]
        got = torch.autograd.grad(y, leaves, dy.view(2, 15, 264))
        assert all(torch.equal(a.flatten(), c.flatten()) for a, c in zip(got, [v for v, k in zip(want, needs) if k]))


def test_no_tokens():
    w, b = torch.ones(96, device=DEV).requires_grad_(), torch.zeros(96, device=DEV).requires_grad_()
    x = torch.zeros(0, 96, dtype=F16, device=DEV).requires_grad_()
    y = si.layer_norm(x, w, b)
    dx, dw, db = torch.autograd.grad(y, (x, w, b), torch.zeros_like(y))
    assert y.shape == dx.shape == (0, 96) and (dw == 0).all() and (db == 0).all()


def test_run_to_run_and_many_rows():
    """The columns' sums of more rows than blocks, the same bits each time."""
    x, w, b, dy = inputs(gen(7), 30011, 136, F16, F32, True)
    leaves = [t.requires_grad_() for t in (x, w, b)]
    runs = [torch.autograd.grad(si.layer_norm(*leaves), leaves, dy) for _ in range(3)]
    assert all(torch.equal(a, c) for r in runs[1:] for a, c in zip(r, runs[0]))
    check(x, w, b, dy, True)


def test_offsets_past_32_bits():
    """More than 2^31 values: the last rows as the first."""
    t, d = 140001, 16384
    x = torch.zeros(t, d, dtype=F16, device=DEV)
    row = torch.randn(d, generator=gen(8)).half().to(DEV)
    pick = [0, 131072, t - 1]
    x[pick] = row
    w = torch.ones(d, device=DEV)
    y = si.rms_norm(x, w)
    one = si.rms_norm(row.view(1, d), w)
    assert all(torch.equal(y[i], one[0]) for i in pick) and not y[1:1000].any()
    del y
    x.requires_grad_()
    dy = torch.zeros(t, d, dtype=F16, device=DEV)
    dy[pick] = 1.0
    dx, = torch.autograd.grad(si.rms_norm(x, w), x, dy)
    r1 = row.view(1, d).clone().requires_grad_()
    want, = torch.autograd.grad(si.rms_norm(r1, w), r1, torch.ones_like(r1))
    assert all(torch.equal(dx[i], want[0]) for i in pick) and not dx[1:1000].any()


def test_python_refuses():
    x, w = torch.zeros(4, 64, device=DEV), torch.ones(64, device=DEV)
    for error, f in ((ValueError, lambda: si.layer_norm(x, w[:60])), (ValueError, lambda: si.layer_norm(x, w, w[:60])),
                     (TypeError, lambda: si.layer_norm(x, w, w.half())), (TypeError, lambda: si.layer_norm(x.int(), w)),
                     (ValueError, lambda: si.layer_norm(x.t(), w[:4])), (ValueError, lambda: si.rms_norm(x, w.view(1, 64))),
                     (ValueError, lambda: si.rms_norm(x, w.cpu())), (ValueError, lambda: si.rms_norm(x[:1].expand(4, 64), w)),
                     (si.SparseInferError, lambda: si.rms_norm(x, w, eps=-1.0)),
                     (si.SparseInferError, lambda: si.rms_norm(torch.zeros(2, 16385, device=DEV), torch.ones(16385, device=DEV)))):
        with pytest.raises(error):
            f()


def test_agrees_with_norm_residual():
    """rms_norm is norm_residual's norm without the residual."""
    x, w, _, _ = inputs(gen(9), 21, 1024, F32, F32, False)
    _, want = si.norm_residual(x, pre_w=w, eps=EPS, x_dtype=F32)
    y = si.rms_norm(x, w)
    assert ((y - want).abs() <= (1024 + 64) * 2.0 ** -23 * want.abs() + 1e-30).all()
