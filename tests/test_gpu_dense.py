"""The dense products and their gradients on the GPU.

Most calls are of whole numbers, small enough that every partial sum, in any order, is
below 2^24 and every value that the kernels round to 16 bits (u, dg, du) has them: the
float32 sums are exact and the outputs are compared for equality with the same numbers
in float64, rounded once, which a dropped, doubled or misplaced value cannot pass.
Gaussian values are compared within ``(k + 64) 2^-23`` of the sum of magnitudes (a unit
in the last place for each addition of k products) and the roundings on the way, each
half a step of the type.
"""

import pytest
import torch

import dense_ref as ref
import paper_2411_12692_amd as si
from dense_ref import BF16, F16, F32, HALF_STEP, SMALLEST

pytestmark = pytest.mark.gpu
DEV = "cuda"


def gen(*key):
    g = torch.Generator()
    g.manual_seed(hash(key) % (1 << 31))
    return g


def same(got, want, dtype):
    """Equal to the float64 whole numbers ``want``, rounded once."""
    assert got.dtype == dtype and got.shape == want.shape
    assert want.abs().max() < 2 ** 24  # exact in float32: one rounding
    assert torch.equal(got.cpu(), want.float().to(dtype))


def sums(a, b):
    """a b^T of whole numbers, exactly (float64 on the GPU)."""
    return (a.double().to(DEV) @ b.double().to(DEV).t().contiguous()).cpu()


DTYPES = [F16, BF16]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,rows,n", ref.shapes("linear"))
def test_linear(dtype, m, rows, n):
    g = gen(0, m, rows, n)
    x, w = ref.whole(g, -2, 2, m, n), ref.whole(g, -1, 1, rows, n)
    want = sums(x, w)
    xd, wd = x.to(dtype).to(DEV), w.to(dtype).to(DEV)
    for out in (None, F32):
        same(si.linear(xd, wd, out_dtype=out), want, out or dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,rows,n", ref.shapes("transposed"))
def test_linear_transposed(dtype, m, rows, n):
    g = gen(1, m, rows, n)
    x, w = ref.whole(g, -2, 2, m, n), ref.whole(g, -1, 1, rows, n)
    y = si.linear(x.to(dtype).to(DEV), w.t().contiguous().to(dtype).to(DEV), transposed=True, out_dtype=F32)
    same(y, sums(x, w), F32)


def gated_values(x, wg, wu, dtype):
    """(g, u, h) as the kernel forms them: exact sums, one float32 product, one rounding."""
    g, u = sums(x, wg), None if wu is None else sums(x, wu)
    return g, u, ref.gated(g, u).to(dtype)


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,rows,n", ref.shapes("linear", True))
def test_gated_linear(dtype, m, rows, n, up):
    g = gen(2, m, rows, n)
    x, wg = ref.whole(g, -1, 1, m, n), ref.whole(g, -1, 1, rows, n)
    wu = ref.whole(g, -1, 1, rows, n) if up else None
    dev = [None if t is None else t.to(dtype).to(DEV) for t in (x, wg, wu)]
    want = gated_values(x, wg, wu, dtype)[2]
    assert torch.equal(si.gated_linear(*dev).cpu(), want)
    # with a graph the sums are kept as well; h is the same
    kept = [None if t is None else t.requires_grad_() for t in dev]
    assert torch.equal(si.gated_linear(*kept).detach().cpu(), want)


def exact_gradients(x, wg, wu, dh, dtype):
    """dx, dw_gate, dw_up in float64; asserts that what the kernels round to 16 bits is
    exact."""
    g, u = sums(x, wg), None if wu is None else sums(x, wu)
    dg = torch.where(g > 0, dh.double() * (u if wu is not None else 1.0), 0.0)
    du = dh.double() * torch.relu(g) if wu is not None else None
    for t in (g, u, dg, du):
        assert t is None or torch.equal(t.to(dtype).double(), t)
    dx = sums(dg, wg.t())
    if wu is None:
        return dx, sums(dg.t(), x.t()), None
    return dx + sums(du, wu.t()), sums(dg.t(), x.t()), sums(du.t(), x.t())


def sparse(g, *shape):
    """Whole numbers -1 .. 1, a few of them other than 0, so that sums stay small."""
    return ref.whole(g, -1, 1, *shape) * (torch.rand(*shape, generator=g) < 0.1)


GRAD_SHAPES = sorted(set(ref.shapes("dx", True) + ref.shapes("dw", True)) | {(33, 37, 29), (2, 1, 1), (5, 9, 200)})


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,rows,n", GRAD_SHAPES)
def test_gated_linear_backward(dtype, m, rows, n, up):
    g = gen(3, m, rows, n)
    x, wg, dh = sparse(g, m, n), sparse(g, rows, n), ref.whole(g, -1, 1, m, rows)
    wu = sparse(g, rows, n) if up else None
    want = [t for t in exact_gradients(x, wg, wu, dh, dtype) if t is not None]
    leaves = [t.to(dtype).to(DEV).requires_grad_() for t in (x, wg, wu) if t is not None]
    h = si.gated_linear(*leaves)
    for got, w in zip(torch.autograd.grad(h, leaves, dh.to(dtype).to(DEV)), want):
        same(got, w, dtype)


@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,rows,n", sorted(set(ref.shapes("transposed") + ref.shapes("dw transposed")) |
                                            {(33, 37, 29), (2, 1, 1), (5, 9, 200), (300, 204, 1000), (7, 63, 8200)}))
def test_mlp_backward(dtype, m, rows, n, up):
    """All four gradients of the whole MLP, and each alone, exact: dh = dy W_down goes
    into dg and du without a rounding."""
    g = gen(21, m, rows, n)
    few = min(1.0, 4.0 / n)  # of W_down's values are other than 0: dh stays small
    x, wg, dy = sparse(g, m, n), sparse(g, rows, n), ref.whole(g, -1, 1, m, n)
    wu = sparse(g, rows, n) if up else None
    wd = ref.whole(g, -1, 1, n, rows) * (torch.rand(n, rows, generator=g) < few)
    dh = sums(dy, wd.t())
    dx, dwg, dwu = exact_gradients(x, wg, wu, dh, dtype)
    pg, pu, h = gated_values(x, wg, wu, dtype)
    want = [t for t in (dx, dwg, dwu, sums(dy.t(), h.t())) if t is not None]
    leaves = [t.to(dtype).to(DEV).requires_grad_() if t is not None else None for t in (x, wg, wu, wd)]
    y, leaves = si.mlp(*leaves), [t for t in leaves if t is not None]
    dev = dy.to(dtype).to(DEV)
    got = torch.autograd.grad(y, leaves, dev, retain_graph=True)
    for a, w in zip(got, want):
        same(a, w, dtype)
    assert all(torch.equal(t, got[0]) for t in torch.autograd.grad(si.mlp(*(leaves if up else [*leaves[:2], None, leaves[2]]),
                                                                          out_dtype=F32), leaves[0], dev.float()))
    for i in range(len(leaves)):
        part = [t.detach().requires_grad_(i == j) for j, t in enumerate(leaves)]
        y = si.mlp(*(part if up else [*part[:2], None, part[2]]))
        assert torch.equal(torch.autograd.grad(y, part[i], dev)[0], got[i])


@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,rows,n", sorted(set(ref.shapes("dx") + ref.shapes("dw") + ref.shapes("dx transposed") +
                                                ref.shapes("dw transposed")) | {(33, 37, 29), (2, 1, 1)}))
def test_linear_backward(dtype, m, rows, n, transposed):
    g = gen(4, m, rows, n)
    x, w, dy = ref.whole(g, -1, 1, m, n), ref.whole(g, -1, 1, rows, n), ref.whole(g, -2, 2, m, rows)
    wd = (w.t().contiguous() if transposed else w).to(dtype).to(DEV).requires_grad_()
    xd = x.to(dtype).to(DEV).requires_grad_()
    dx, dw = sums(dy, w.t()), sums(dy.t(), x.t())
    for out in (None, F32):  # a float32 output's gradient is float32
        y = si.linear(xd, wd, transposed=transposed, out_dtype=out)
        got = torch.autograd.grad(y, (xd, wd), dy.to(y.dtype).to(DEV))
        same(got[0], dx, dtype)
        same(got[1], dw.t() if transposed else dw, dtype)


# ---- values, types, strides ---------------------------------------------------------

def bound(k, size, dtype, roundings=1):
    """Additions in float32 and roundings of half a step, relative to magnitudes."""
    return ((k + 64) * 2.0 ** -23 + roundings * HALF_STEP[dtype] * 1.01) * size + roundings * SMALLEST[dtype]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m,rows,n", [(1, 200, 4096), (3, 64, 11008), (37, 500, 1371), (333, 1371, 509)])
def test_gaussian_values(dtype, m, rows, n):
    """A whole MLP forward and backward against float64, with the roundings on the way:
    h; dg and du."""
    g = gen(5, m, rows, n)
    x, wg, wu = (torch.randn(s, generator=g).mul(f).to(dtype).to(DEV).requires_grad_()
                 for s, f in (((m, n), 1.0), ((rows, n), n ** -0.5), ((rows, n), n ** -0.5)))
    wd = torch.randn(n, rows, generator=g).mul(rows ** -0.5).to(dtype).to(DEV).requires_grad_()
    dy = torch.randn(m, n, generator=g).to(dtype).to(DEV)
    y = si.mlp(x, wg, wu, wd)
    got = torch.autograd.grad(y, (x, wg, wu, wd), dy)
    X, G, U, W, DY = (t.detach().double() for t in (x, wg, wu, wd, dy))
    pg, pu = X @ G.t(), X @ U.t()
    eg, eu = ((n + 64) * 2.0 ** -23 * (X.abs() @ t.abs().t()) for t in (G, U))
    h = torch.relu(pg) * pu
    eh = eg * pu.abs() + pg.abs() * eu + eg * eu + 2.0 ** -23 * h.abs() + HALF_STEP[dtype] * 1.01 * h.abs() + SMALLEST[dtype]
    size = h.abs() @ W.abs().t()
    assert ((y.detach().double() - h @ W.t()).abs() <= eh @ W.abs().t() + bound(rows, size + eh @ W.abs().t(), dtype)).all()
    # gradients: h's own error enters dW_down alone; the sums and dh stay in float32
    near = pg.abs() <= eg  # the sign of a sum that cancels is not decided
    dh = DY @ W
    edh = bound(n, DY.abs() @ W.abs(), F32)
    on = (pg > 0).double()
    dg, du = dh * pu * on, dh * torch.relu(pg)
    edg = edh * (pu.abs() + eu) + dh.abs() * eu
    edg = edg + HALF_STEP[dtype] * 1.01 * (dg.abs() + edg) + SMALLEST[dtype]
    edu = edh * (pg.abs() + eg) + dh.abs() * eg
    edu = edu + HALF_STEP[dtype] * 1.01 * (du.abs() + edu) + SMALLEST[dtype]
    edg = torch.where(near, (dh.abs() + edh) * (pu.abs() + eu) * 1.01, edg)
    dx, edx = dg @ G + du @ U, edg @ G.abs() + edu @ U.abs()
    size = dg.abs() @ G.abs() + du.abs() @ U.abs() + edx
    assert ((got[0].double() - dx).abs() <= edx + bound(2 * rows, size, dtype)).all()
    for have, d, e, v in ((got[1], dg, edg, X), (got[2], du, edu, X), (got[3], DY, torch.zeros_like(DY), h)):
        ev = eh if v is h else torch.zeros_like(v)
        err = e.t() @ (v.abs() + ev) + d.abs().t() @ ev
        assert ((have.double() - d.t() @ v).abs() <= err + bound(m, d.abs().t() @ v.abs() + err, dtype)).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_strides_and_unaligned_operands(dtype):
    """x at a stride and off 16 bytes, weights off 16 bytes, rows of odd length: the
    same bits as their contiguous copies give."""
    g = gen(6)
    big = ref.whole(g, -2, 2, 40, 300).to(dtype).to(DEV)
    flat = ref.whole(g, -1, 1, 70 * 97 + 1).to(dtype).to(DEV)
    for x, w in ((big[:, :96], flat[: 70 * 96].view(70, 96)), (big[::2, 3:100], flat[1: 1 + 70 * 97].view(70, 97)),
                 (big[5:, 8:104], flat[1: 1 + 70 * 96].view(70, 96)), (big[3:4, 1:98], flat[: 70 * 97].view(70, 97))):
        want = sums(x.float().cpu(), w.float().cpu())
        same(si.linear(x, w, out_dtype=F32), want, F32)
        xr, wr = x.detach().requires_grad_(), w.detach().requires_grad_()
        dh = ref.whole(g, -1, 1, x.shape[0], 70).to(dtype).to(DEV)
        a = torch.autograd.grad(si.gated_linear(xr, wr, wr), (xr, wr), dh)
        xc, wc = x.detach().clone().requires_grad_(), w.detach().clone().requires_grad_()
        b = torch.autograd.grad(si.gated_linear(xc, wc, wc), (xc, wc), dh)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_incoming_gradients_of_any_layout():
    """What autograd hands on: expanded (a sum's), transposed, at a stride, float32."""
    g = gen(7)
    x = ref.whole(g, -1, 1, 24, 64).half().to(DEV).requires_grad_()
    w = sparse(g, 40, 64).half().to(DEV).requires_grad_()
    wu = sparse(g, 40, 64).half().to(DEV).requires_grad_()
    for f in (lambda: si.linear(x, w), lambda: si.gated_linear(x, w, wu), lambda: si.gated_linear(x, w),
              lambda: si.linear(x, w, out_dtype=F32), lambda: si.gated_linear(x, w, wu, out_dtype=F32),
              lambda: si.gated_linear(x, w, wu, out_dtype=BF16), lambda: si.linear(x, w, out_dtype=BF16)):
        y = f()
        leaves = [t for t in (x, w, wu) if torch.autograd.grad(y.sum(), t, retain_graph=True, allow_unused=True)[0] is not None]
        dy = ref.whole(g, -1, 1, 24, 40).to(y.dtype).to(DEV)
        want = torch.autograd.grad(y, leaves, dy, retain_graph=True)
        wide = torch.zeros(24, 90, dtype=y.dtype, device=DEV)
        wide[:, 7:47] = dy
        for d in (dy.t().contiguous().t(), wide[:, 7:47]):
            for a, b in zip(torch.autograd.grad(y, leaves, d, retain_graph=True), want):
                assert torch.equal(a, b)
        ones = torch.autograd.grad(y, leaves, torch.ones_like(y), retain_graph=True)
        for a, b in zip(torch.autograd.grad(y.sum(), leaves), ones):
            assert torch.equal(a, b)


def test_leading_dimensions_and_single_rows():
    g = gen(8)
    x = ref.whole(g, -1, 1, 2, 3, 5, 64).half().to(DEV).requires_grad_()
    w, wd = sparse(g, 40, 64).half().to(DEV).requires_grad_(), sparse(g, 64, 40).half().to(DEV)
    y = si.mlp(x, w, w, wd)
    assert y.shape == (2, 3, 5, 64)
    (dx,) = torch.autograd.grad(y.float().sum(), x)
    flat = x.detach().view(30, 64).clone().requires_grad_()
    yf = si.mlp(flat, w, w, wd)
    assert dx.shape == x.shape and torch.equal(y.detach().view(30, 64), yf.detach())
    assert torch.equal(dx.view(30, 64), torch.autograd.grad(yf.float().sum(), flat)[0])
    row = si.linear(x.detach()[0, 0, 0], w.detach())
    assert row.shape == (40,) and torch.equal(row, si.linear(x.detach()[0, 0], w.detach())[0])


@pytest.mark.parametrize("n,k", [(64, 40), (37, 29)])
def test_no_tokens(n, k):
    """Nothing is computed; the weights' gradients are zeros.  At odd lengths there is
    nothing to copy either."""
    w, wt, wd = (torch.ones(*s, dtype=F16, device=DEV).requires_grad_() for s in ((k, n), (n, k), (n, k)))
    for x in (torch.zeros(0, n, dtype=F16, device=DEV), torch.zeros(2, 0, n, dtype=F16, device=DEV)):
        x.requires_grad_()
        for f, leaves in ((lambda: si.linear(x, w), (w,)), (lambda: si.linear(x, wt, transposed=True), (wt,)),
                          (lambda: si.linear(x, w, out_dtype=F32), (w,)), (lambda: si.gated_linear(x, w, w), (w,)),
                          (lambda: si.gated_linear(x, w), (w,)), (lambda: si.mlp(x, w, w, wd), (w, wd)),
                          (lambda: si.mlp(x, w, None, wd), (w, wd))):
            y = f()
            assert y.shape[:-1] == x.shape[:-1]
            dx, *dw = torch.autograd.grad(y, (x, *leaves), torch.zeros_like(y))
            assert dx.shape == x.shape and all(torch.equal(d, torch.zeros_like(d)) for d in dw)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("m", [1, 6, 140])
def test_special_values_stay_in_their_row(dtype, m):
    """An infinity or a NaN of a token reaches that token's outputs and gradients, of a
    row of W that row's; negative gate values stop both (relu), a NaN gate value is kept."""
    g = gen(9, m)
    x, wg, wu = torch.randn(m, 200, generator=g), torch.randn(70, 200, generator=g), torch.randn(70, 200, generator=g)
    x[0, 3] = float("nan")
    wg[5, 7] = float("inf")
    wu[6, 0] = float("nan")
    x, wg, wu = (t.to(dtype).to(DEV).requires_grad_() for t in (x, wg, wu))
    h = si.gated_linear(x, wg, wu)
    d = h.detach().float().cpu()
    assert d[0].isnan().all()
    if m > 1:
        pre = (x.detach().float() @ wg.detach().float().t()).cpu()
        assert (d[1:, 5].isinf() | (d[1:, 5] == 0)).all() and torch.equal(d[1:, 5].isinf(), pre[1:, 5] > 0)
        assert d[1:, 6].isnan().all()  # relu(g) * NaN, also where relu(g) is 0
        rest = [i for i in range(70) if i not in (5, 6)]
        assert d[1:, rest].isfinite().all()
        dh = torch.zeros(m, 70, dtype=dtype, device=DEV)
        dh[1:, rest] = 1.0
        dx, dwg, dwu = torch.autograd.grad(h, (x, wg, wu), dh)
        # token 0 has gradients of 0 * NaN, like its NaN values' products
        assert dwg[rest].isnan().any() and dwg[rest][:, 3].isnan().all()


@pytest.mark.parametrize("m", [1, 40])
def test_a_small_positive_gate_keeps_its_derivative(m):
    """g = 2^-40 rounds to 0 in fp16: u's product still passes its gradient."""
    x = torch.zeros(m, 64, dtype=F16, device=DEV)
    x[:, 0] = 2.0 ** -20
    x[:, 1] = 1.0
    wg, wu = (torch.zeros(8, 64, dtype=F16, device=DEV) for _ in range(2))
    wg[:, 0] = 2.0 ** -20
    wg[1, 0] = -2.0 ** -20
    wg[2, 0] = 0.0
    wu[:, 1] = 3.0
    leaves = [t.requires_grad_() for t in (x, wg, wu)]
    h = si.gated_linear(*leaves)
    assert (h == 0).all()
    dh = torch.ones_like(h)
    dwg = torch.autograd.grad(h, leaves, dh)[1]
    want = torch.full((8,), 3.0 * m, dtype=F16, device=DEV)  # sum over tokens of dh u x[1]
    want[1:3] = 0.0
    assert torch.equal(dwg[:, 1], want)


def test_overflow_becomes_infinite():
    x = torch.full((5, 64), 100.0, dtype=F16, device=DEV)
    w = torch.full((16, 64), 20.0, dtype=F16, device=DEV)
    assert si.linear(x, w).isinf().all() and (si.linear(x, w, out_dtype=F32) == 128000.0).all()
    assert (si.linear(x, -w) == -float("inf")).all() and (si.gated_linear(x, -w, w) == 0).all()


# ---- gradients asked for in part, differences, refusals -------------------------------

@pytest.mark.parametrize("needs", [(1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 0, 1), (0, 1, 1), (1, 1, 0)])
def test_gradients_in_part(needs):
    g = gen(10)
    vals = [sparse(g, 30, 100), sparse(g, 50, 100), sparse(g, 50, 100)]
    dh = ref.whole(g, -1, 1, 30, 50).half().to(DEV)
    full = [t.half().to(DEV).requires_grad_() for t in vals]
    want = torch.autograd.grad(si.gated_linear(*full), full, dh)
    part = [t.half().to(DEV).requires_grad_(bool(n)) for t, n in zip(vals, needs)]
    leaves = [t for t in part if t.requires_grad]
    got = torch.autograd.grad(si.gated_linear(*part), leaves, dh)
    assert all(torch.equal(a, b) for a, b in zip(got, [w for w, n in zip(want, needs) if n]))
    if needs[2] == 0:
        x, w = part[0], part[1]
        y = si.linear(x, w)
        ref_y = si.linear(full[0], full[1])
        want = torch.autograd.grad(ref_y, full[:2], dh)
        got = torch.autograd.grad(y, [t for t in (x, w) if t.requires_grad], dh)
        assert all(torch.equal(a, b) for a, b in zip(got, [v for v, n in zip(want, needs) if n]))


def test_same_tensor_twice():
    """W as W_gate and W_up, and y fed back: gradients add up."""
    g = gen(11)
    x, w = sparse(g, 20, 64).half().to(DEV).requires_grad_(), sparse(g, 64, 64).half().to(DEV).requires_grad_()
    h = si.gated_linear(x, w, w)
    dh = ref.whole(g, -1, 1, 20, 64).half().to(DEV)
    dw = torch.autograd.grad(h, w, dh)[0]
    w2 = w.detach().clone().requires_grad_()
    a, b = torch.autograd.grad(si.gated_linear(x, w, w2), (w, w2), dh)
    assert torch.equal(dw, a + b)


def test_against_differences():
    """The loss sum(y dy) in float64 of the plain MLP moves as dx and the weights'
    gradients say, in directions drawn at random: within the roundings of 16 bits."""
    g = gen(12)
    m, d, k = 12, 96, 160
    vals = [torch.randn(m, d, generator=g), torch.randn(k, d, generator=g) * d ** -0.5,
            torch.randn(k, d, generator=g) * d ** -0.5, torch.randn(d, k, generator=g) * k ** -0.5]
    leaves = [t.half().to(DEV).requires_grad_() for t in vals]
    dy = torch.randn(m, d, generator=g).half().to(DEV)
    grads = torch.autograd.grad(si.mlp(*leaves), leaves, dy)
    base = [t.detach().double() for t in leaves]

    def loss(x, wg, wu, wd):
        return float(((torch.relu(x @ wg.t()) * (x @ wu.t())) @ wd.t() * dy.double()).sum())
    for i, grad in enumerate(grads):
        way = torch.randn(base[i].shape, generator=g, dtype=torch.float64).to(DEV)
        eps = 1e-6
        up, down = ([t + s * eps * way if j == i else t for j, t in enumerate(base)] for s in (1, -1))
        slope = (loss(*up) - loss(*down)) / (2 * eps)
        # each gradient is a sum of values with up to four roundings of 2^-11; a sum of
        # products with random signs is off by that share of its magnitudes at most
        size = float((grad.double().abs() * way.abs()).sum())
        assert abs(float((grad.double() * way).sum()) - slope) <= 4 * 2.0 ** -11 * size * 4 + 1e-6


def test_second_order_is_refused():
    x = torch.randn(4, 64, device=DEV).half().requires_grad_()
    w = torch.randn(8, 64, device=DEV).half().requires_grad_()
    (dx,) = torch.autograd.grad(si.linear(x, w).float().square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        dx.float().sum().backward()


def test_python_refuses():
    x, w = torch.zeros(4, 64, dtype=F16, device=DEV), torch.zeros(8, 64, dtype=F16, device=DEV)
    for error, f in ((TypeError, lambda: si.linear(x, w.bfloat16())), (TypeError, lambda: si.linear(x.float(), w.float())),
                     (ValueError, lambda: si.linear(x, w[:, :60])), (ValueError, lambda: si.linear(x, w[:, ::2])),
                     (ValueError, lambda: si.linear(x[:, ::2], w[:, :32].contiguous())),
                     (ValueError, lambda: si.linear(x.t(), w[:, :4].contiguous())),
                     (ValueError, lambda: si.linear(x, w, transposed=True)), (TypeError, lambda: si.linear(x, w, out_dtype=torch.int8)),
                     (ValueError, lambda: si.gated_linear(x, w, w[:4])), (ValueError, lambda: si.gated_linear(x, w, w.cpu())),
                     (ValueError, lambda: si.linear(x[:1].expand(4, 64), w)), (ValueError, lambda: si.linear(x, w.view(2, 4, 64))),
                     (TypeError, lambda: si.linear(x, None)), (ValueError, lambda: si.mlp(x, w, w, w))):
        with pytest.raises(error):
            f()


# ---- longest sums, offsets past 32 bits, streams, graphs ------------------------------

def test_longest_sums():
    """n and rows at their limit of 2^20."""
    n = 1 << 20
    x = torch.ones(3, n, dtype=BF16, device=DEV)
    x[1] = -1.0
    w = torch.ones(4, n, dtype=BF16, device=DEV)
    w[:, ::2] = 0.0
    y = si.linear(x, w, out_dtype=F32)
    assert torch.equal(y, torch.tensor([[n / 2.0], [-n / 2.0], [n / 2.0]], device=DEV).expand(3, 4))
    x5 = x[:1].repeat(5, 1)
    assert (si.linear(x5, w, out_dtype=F32) == n / 2).all()  # tiles, the sum in parts
    wr = w[:1, :8].repeat(n, 1).requires_grad_()  # 2^20 rows of 8
    xr = torch.ones(5, 8, dtype=BF16, device=DEV).requires_grad_()
    y = si.linear(xr, wr)
    assert (y == 4.0).all()
    dx, dw = torch.autograd.grad(y, (xr, wr), torch.full_like(y, 2.0 ** -20))
    assert torch.equal(dx, wr.detach()[:1].expand(5, 8)) and torch.equal(dw, torch.full_like(dw, 5 * 2.0 ** -20))


def test_offsets_past_32_bits():
    """More than 2^31 elements of x and of y: the last tokens are as good as the first."""
    m, n, rows = 70001, 64, 32776
    x = torch.zeros(m, n, dtype=F16, device=DEV)
    pick = [0, 1, 65535, 65536, m - 2, m - 1]
    g = gen(13)
    vals = ref.whole(g, -2, 2, len(pick), n)
    x[pick] = vals.half().to(DEV)
    w = ref.whole(g, -1, 1, rows, n)
    y = si.linear(x, w.half().to(DEV))
    assert torch.equal(y[pick].cpu(), sums(vals, w).half())
    assert not y[2:65535].any() and not y[65537:m - 2].any()
    del y
    wide = torch.zeros(40, (1 << 21), dtype=F16, device=DEV)  # the largest stride
    wide[:, -64:] = x[:40]
    wide[39, -64:] = x[m - 1]
    y = si.linear(wide[:, -64:], w.half().to(DEV))
    assert torch.equal(y[39].cpu(), sums(vals, w).half()[-1])


def test_other_streams():
    g = gen(14)
    x, w = ref.whole(g, -2, 2, 300, 512).half().to(DEV), ref.whole(g, -1, 1, 400, 509 + 3).half().to(DEV)
    want = [si.linear(x, w), si.gated_linear(x[:, :509], w[:, :509].contiguous(), w[:, :509].contiguous())]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    out = []
    for s in streams:  # calls with scratch at once on several streams
        with torch.cuda.stream(s):
            out.append([si.linear(x, w), si.gated_linear(x[:, :509], w[:, :509].contiguous(), w[:, :509].contiguous())])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in out for a, b in zip(o, want))


def test_run_to_run():
    g = gen(15)
    x, w = torch.randn(600, 1024, generator=g).half().to(DEV).requires_grad_(), torch.randn(512, 1024, generator=g).half().to(DEV).requires_grad_()
    dh = torch.randn(600, 512, generator=g).half().to(DEV)
    runs = []
    for _ in range(3):
        h = si.gated_linear(x, w, w)
        runs.append([h.detach(), *torch.autograd.grad(h, (x, w), dh)])
    assert all(torch.equal(a, b) for r in runs[1:] for a, b in zip(r, runs[0]))


def test_mlp_gradients_on_several_streams():
    """Steps with scratch at once on several streams, odd lengths among the copies."""
    g = gen(22)
    leaves = [torch.randn(*s, generator=g).mul(0.1).half().to(DEV).requires_grad_() for s in ((70, 109), (203, 109), (203, 109), (109, 203))]
    dy = torch.randn(70, 109, generator=g).half().to(DEV)

    def step():
        y = si.mlp(*leaves)
        return [y.detach(), *torch.autograd.grad(y, leaves, dy)]
    want, out = step(), []
    torch.cuda.synchronize()
    for s in [torch.cuda.Stream() for _ in range(3)]:
        with torch.cuda.stream(s):
            out.append(step())
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for o in out for a, b in zip(o, want))


def test_captured_training_step():
    """Forward and backward of norm, MLP and residual in a graph, replayed with other
    inputs between eager work, against eager runs.  (The graph's leaves are its own.)"""
    g = gen(16)
    d, k, m = 192, 328, 37

    def step(x, nw, wg, wu, wd, dy):
        y = x + si.mlp(si.rms_norm(x, nw), wg, wu, wd)
        return [y.detach(), *torch.autograd.grad(y, (x, nw, wg, wu, wd), dy)]

    def inputs(seed):
        g = gen(17, seed)
        shapes = ((m, d), (d,), (k, d), (k, d), (d, k), (m, d))
        return [torch.randn(s, generator=g).mul(0.3).half().to(DEV) for s in shapes]
    static = [t.requires_grad_(i < 5) for i, t in enumerate(inputs(0))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*static)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(*static)
    for seed in (1, 2, 3):
        fresh = inputs(seed)
        with torch.no_grad():
            for s, f in zip(static, fresh):
                s.copy_(f)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in out]
        eager = step(*[t.requires_grad_(i < 5) for i, t in enumerate(fresh)])
        assert all(torch.equal(a, b) for a, b in zip(got, eager)), seed


# ---- the layers ---------------------------------------------------------------------

@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("m", [1, 4, 33, 300])
def test_prompt_of_the_fp16_layer(m, up):
    """MLPLayer.prompt, the dense MLP, against its decode call with every row kept, token
    by token, and against mlp with W_down."""
    g = gen(18, m)
    k, d = 328, 256
    wg, wu, wd = (torch.randn(s, generator=g).mul(0.05).half().to(DEV) for s in ((k, d), (k, d), (d, k)))
    x = torch.randn(m, d, generator=g).half().to(DEV)
    layer = si.MLPLayer(wg, wu if up else None, wd)
    y = layer.prompt(x, out_dtype=F32)
    h = si.gated_linear(x, wg, wu if up else None).double()
    size = h.abs() @ wd.double().abs().t()
    assert ((y.double() - h @ wd.double().t()).abs() <= (k + 64) * 2.0 ** -23 * size).all()
    dense = torch.cat([layer(x[t:t + 1], float("inf")) for t in range(min(m, 4))]).double()
    # decode keeps h in float32: half a step of fp16 and the two sums' additions
    assert ((y[:4].double() - dense).abs() <= (2.0 ** -11 * 1.01 + (k + d + 128) * 2.0 ** -22) * (size[:4] + 2.0 ** -14 * k)).all()
    assert torch.equal(layer.prompt(x), y.half()) and layer.prompt(x.view(1, m, d)).shape == (1, m, d)


# ---- the place in autograd's graph ------------------------------------------------------

def layer_of(g, m=40, d=96, k=130):
    vals = [torch.randn(*s, generator=g).mul(0.1).half().to(DEV).requires_grad_() for s in ((m, d), (d,), (k, d), (k, d), (d, k))]
    return vals, torch.randn(m, d, generator=g).half().to(DEV)


def block(x, nw, wg, wu, wd):
    return x + si.mlp(si.rms_norm(x, nw), wg, wu, wd) + si.linear(si.gated_linear(si.layer_norm(x, nw, nw), wg), wd)


def test_backward_accumulates_and_frees():
    leaves, dy = layer_of(gen(30))
    want = torch.autograd.grad(block(*leaves), leaves, dy)
    y = block(*leaves)
    y.backward(dy, retain_graph=True)
    assert all(torch.equal(t.grad, w) for t, w in zip(leaves, want))
    y.backward(dy)
    assert all(torch.equal(t.grad, w + w) for t, w in zip(leaves, want))
    with pytest.raises(RuntimeError, match="second time"):
        y.backward(dy)


@pytest.mark.parametrize("up", [True, False])
def test_a_saved_tensor_changed_in_place_is_refused(up):
    (x, _, wg, wu, wd), dy = layer_of(gen(31))
    for f in (lambda x: si.linear(x, wd, transposed=True), lambda x: si.gated_linear(x, wg, wu if up else None),
              lambda x: si.mlp(x, wg, wu if up else None, wd), lambda x: si.rms_norm(x, x.detach()[0].float())):
        own = x.detach().clone()
        y = f(own.requires_grad_())
        with torch.no_grad():
            own.add_(1)
        with pytest.raises(RuntimeError, match="inplace"):
            y.float().sum().backward()


def test_hooks_of_saved_tensors():
    """Checkpointing and saving to the host go through the same values."""
    from torch.utils.checkpoint import checkpoint
    leaves, dy = layer_of(gen(32))
    want = torch.autograd.grad(block(*leaves), leaves, dy)
    got = torch.autograd.grad(checkpoint(block, *leaves, use_reentrant=False), leaves, dy)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.autograd.graph.save_on_cpu():
        y = block(*leaves)
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(y, leaves, dy), want))


def test_gradients_on_this_thread_and_of_some_leaves():
    leaves, dy = layer_of(gen(33))
    want = torch.autograd.grad(block(*leaves), leaves, dy)
    with torch.autograd.set_multithreading_enabled(False):
        got = torch.autograd.grad(block(*leaves), leaves, dy)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    y = block(*leaves)
    for i in range(len(leaves)):  # only what is asked for is computed
        assert torch.equal(torch.autograd.grad(y, leaves[i], dy, retain_graph=True)[0], want[i])
    out = si.linear(leaves[0], leaves[2])
    unused = torch.autograd.grad(out[:0].sum() * 0 + leaves[1].sum(), (leaves[0], leaves[1]), allow_unused=True)
    assert unused[0] is None or not unused[0].any()


def test_a_graph_of_the_gradients_is_refused_where_it_is_used():
    leaves, dy = layer_of(gen(34))
    for f, of in ((lambda x, nw, wg, wu, wd: si.mlp(x, wg, wu, wd), (0, 2, 3, 4)), (lambda x, nw, *_: si.layer_norm(x, nw), (0, 1)),
                  (lambda x, nw, wg, wu, wd: si.gated_linear(x, wg, wu), (0, 2, 3))):
        y = f(*leaves)
        grads = torch.autograd.grad(y, [leaves[i] for i in of], torch.ones_like(y), create_graph=True)
        assert all(t.requires_grad for t in grads)
        with pytest.raises(RuntimeError, match="first order"):
            sum(t.float().sum() for t in grads).backward()


def test_capture_with_leaves_of_a_live_graph_is_refused():
    """Autograd would end the process in the backward pass; once the eager graph is gone
    the same capture goes through."""
    (x, nw, wg, wu, wd), dy = layer_of(gen(35))
    for f in (lambda: si.mlp(x, wg, wu, wd), lambda: si.rms_norm(x, nw), lambda: si.linear(x, wg), lambda: si.gated_linear(x, wg, wu)):
        alive = f()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with pytest.raises(RuntimeError, match="eager graph"):
            with torch.cuda.graph(graph):
                f()
        torch.cuda.synchronize()
        want = torch.autograd.grad(alive, x, torch.ones_like(alive))[0]
        del alive, graph
        graph = torch.cuda.CUDAGraph()
        ones = torch.ones_like(f())
        with torch.cuda.graph(graph):
            y = f()
            got = torch.autograd.grad(y, x, ones)[0]
        del y
        for _ in range(3):
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want)


def test_fp16_bits_and_graphs_of_one_gradient():
    """x as int16 (fp16 bits) has no gradient, W has; a graph of the gradients where only
    one is asked for."""
    (x, nw, wg, wu, wd), dy = layer_of(gen(36))
    bits = x.detach().view(torch.int16)
    with pytest.raises(TypeError, match="int16"):
        si.linear(bits, wg)
    with torch.no_grad():
        assert torch.equal(si.linear(bits, wg).view(F16), si.linear(x, wg))
    dh = torch.ones(40, 130, dtype=F16, device=DEV)
    for f in (lambda a: si.linear(a, wg, out_dtype=F16), lambda a: si.gated_linear(a, wg, wu, out_dtype=F16)):
        assert torch.equal(torch.autograd.grad(f(bits), wg, dh)[0], torch.autograd.grad(f(x), wg, dh)[0])
    assert torch.equal(torch.autograd.grad(si.mlp(bits, wg, wu, wd, out_dtype=F16), wd, dy)[0],
                       torch.autograd.grad(si.mlp(x, wg, wu, wd), wd, dy)[0])
    for f in (lambda: si.linear(x, wg.detach()), lambda: si.rms_norm(x, nw.detach()), lambda: si.mlp(x, wg.detach(), None, wd.detach())):
        y = f()
        (dx,) = torch.autograd.grad(y, x, torch.ones_like(y), create_graph=True)
        with pytest.raises(RuntimeError, match="first order"):
            dx.float().sum().backward()
