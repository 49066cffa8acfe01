"""Every element of every gradient against differences of the loss in float64, bounded by
the roundings that lie on its way alone, so that a wrong factor or a missing term shows.

The loss is ``sum(y dy)`` of the plain operator over the operands as they are after
rounding to 16 bits, on the CPU.  It is of second degree at most in each element of the
products' operands (no gate is near 0), so that a central difference is its derivative but
for float64's own rounding; the norms' differences are off by the third derivative times
``STEP^2``, far below the bound.

With e half a step of the type: an operand that is rounded (h, dg, du) adds e times the sum
of the magnitudes of the products it enters, the result e of itself.  The float32 sums, of
24 terms at most, three in a row, add 72 2^-24 < 2^-17 of the magnitudes.  Values near the
smallest normal number are off by half the smallest step whatever their size.
"""

import pytest
import torch

import paper_2411_12692_amd as si
from dense_ref import BF16, F16, F32, HALF_STEP, SMALLEST

pytestmark = pytest.mark.gpu
DEV = "cuda"
M, D, K = 6, 24, 20
STEP = 2.0 ** -20
SUMS = 2.0 ** -17


def gen(*key):
    g = torch.Generator()
    g.manual_seed(hash(key) % (1 << 31))
    return g


def slopes(loss, leaves):
    """The derivative of the loss by each element of each leaf, by central differences."""
    out = []
    for leaf in leaves:
        flat, slope = leaf.view(-1), torch.empty(leaf.numel(), dtype=torch.float64)
        for i in range(flat.numel()):
            at = flat[i].item()
            flat[i] = at + STEP
            up = loss(*leaves)
            flat[i] = at - STEP
            slope[i] = (up - loss(*leaves)) / (2 * STEP)
            flat[i] = at
        out.append(slope.view(leaf.shape))
    return out


def compare(grads, want, bounds):
    for i, (grad, slope, bound) in enumerate(zip(grads, want, bounds)):
        got = grad.double().cpu()
        off = (got - slope).abs()
        assert (off <= bound).all(), (i, float((off / bound).max()))
        for wrong in (0.5 * got, -got, torch.zeros_like(got)):  # what the bound would let pass
            assert ((wrong - slope).abs() > bound).float().mean() > 0.5, i


def operands(g, dtype, *shapes):
    return [(torch.randn(s, generator=g) * s[-1] ** -0.5).to(dtype) for s in shapes]


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("transposed", [False, True])
def test_linear(dtype, transposed):
    g = gen(0, transposed)
    x, w, dy = operands(g, dtype, (M, D), (D, K) if transposed else (K, D), (M, K))
    leaves = [x.to(DEV).requires_grad_(), w.to(DEV).requires_grad_()]
    grads = torch.autograd.grad(si.linear(*leaves, transposed=transposed), leaves, dy.to(DEV))
    X, W, DY = x.double(), w.double(), dy.double()
    want = slopes(lambda x, w: float((x @ (w if transposed else w.t()) * DY).sum()), [X, W])
    rows = W.t() if transposed else W
    size = [DY.abs() @ rows.abs(), DY.abs().t() @ X.abs()]
    if transposed:
        size[1] = size[1].t()
    e, tiny = HALF_STEP[dtype], SMALLEST[dtype]
    compare(grads, want, [e * s.abs() + SUMS * m + tiny + 1e-9 for s, m in zip(want, size)])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("up", [True, False])
@pytest.mark.parametrize("down", [True, False])
def test_gated_linear_and_mlp(dtype, up, down):
    g = gen(1, up, down)
    x, wg, wu, wd, dy = operands(g, dtype, (M, D), (K, D), (K, D), (D, K), (M, D if down else K))
    x, wg, wu = x * 4, wg * 2, wu * 2
    given = [x, wg] + ([wu] if up else []) + ([wd] if down else [])
    leaves = [t.to(DEV).requires_grad_() for t in given]
    args = (leaves[0], leaves[1], leaves[2] if up else None)
    y = si.mlp(*args, leaves[-1]) if down else si.gated_linear(*args)
    grads = torch.autograd.grad(y, leaves, dy.to(DEV))
    base = [t.double() for t in given]
    DY = dy.double()

    def loss(x, wg, *more):
        h = torch.relu(x @ wg.t())
        if up:
            h = h * (x @ more[0].t())
        return float(((h @ more[-1].t() if down else h) * DY).sum())
    X, G = base[0], base[1]
    gate = X @ G.t()
    assert gate.abs().min() > 1e-4  # on one side of ReLU's border in every arithmetic
    want = slopes(loss, base)
    e, tiny, on = HALF_STEP[dtype], SMALLEST[dtype], (gate > 0).double()
    U = base[2] if up else None
    lin = X @ U.t() if up else torch.ones_like(gate)
    h = gate * on * lin
    dh = DY @ base[-1] if down else DY
    # the magnitudes that sums and roundings are relative to
    m_dh = DY.abs() @ base[-1].abs() if down else DY.abs()
    m_gate, m_lin = X.abs() @ G.abs().t(), X.abs() @ U.abs().t() if up else torch.ones_like(gate)
    r_dg, r_du = e * (dh * lin * on).abs() + tiny, e * (dh * gate * on).abs() + tiny  # of dg and du
    s_dg, s_du = SUMS * m_dh * m_lin * on, SUMS * m_dh * m_gate * on
    d_dg, d_du = r_dg + s_dg, r_du + s_du
    d_x = d_dg @ G.abs() + (d_du @ U.abs() if up else 0.0)
    bounds = [d_x, d_dg.t() @ X.abs()] + ([d_du.t() @ X.abs()] if up else [])
    if down:
        bounds.append(DY.abs().t() @ ((e * h.abs() + tiny) + SUMS * m_gate * m_lin * on))
    # (1.01: products of two of these errors, below 2^-7 of one)
    compare(grads, want, [1.01 * b + e * s.abs() + tiny + 1e-9 for b, s in zip(bounds, want)])


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("center", [True, False])
def test_norms(dtype, center):
    g = gen(2, center)
    x, dy = (torch.randn(M, D, generator=g).to(dtype) for _ in range(2))
    w, b = 1.0 + 0.2 * torch.randn(D, generator=g), torch.randn(D, generator=g)
    given = [x, w] + ([b] if center else [])
    leaves = [t.to(DEV).requires_grad_() for t in given]
    grads = torch.autograd.grad(si.layer_norm(*leaves) if center else si.rms_norm(*leaves), leaves, dy.to(DEV))
    DY = dy.double()

    def unit(x):
        c = x - x.mean(dim=1, keepdim=True) if center else x
        return c / torch.sqrt((c * c).mean(dim=1, keepdim=True) + 1e-5)

    def loss(x, w, *b):
        return float(((unit(x) * w + (b[0] if b else 0.0)) * DY).sum())
    base = [t.double() for t in given]
    want = slopes(loss, base)
    n = unit(base[0])
    r = (n / (base[0] - (base[0].mean(dim=1, keepdim=True) if center else 0.0))).abs().amax(dim=1, keepdim=True)
    dn = (DY * base[1]).abs()
    size = r * (dn + dn.mean(dim=1, keepdim=True) + n.abs() * (dn * n.abs()).mean(dim=1, keepdim=True))
    sizes = [size, (DY * n).abs().sum(dim=0), DY.abs().sum(dim=0)]
    # dx is rounded to 16 bits, dw and db are float32
    parts = [HALF_STEP[dtype], HALF_STEP[F32], HALF_STEP[F32]]
    compare(grads, want, [p * s.abs() + SUMS * m + SMALLEST[dtype] + 1e-8 for p, s, m in zip(parts, want, sizes)])
