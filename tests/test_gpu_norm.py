"""``norm_residual`` on the GPU against NumPy float64 (``mx_ref``).

Bounds: a sum of d squares in float32 is within (d + 8) 2^-24 of its value (one
rounding a square and an addition each), so 1 / sqrt within half of that and 3
roundings; the products and the residual's fused multiply-add add at most 6
more.  An error of h' moves x by its own share and by that of the norm.  Then
half a step of the output's type.
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
SMALLEST = {F16: 2.0 ** -25, BF16: 2.0 ** -134, F32: 2.0 ** -150}


def f64(t):
    return t.detach().cpu().double().numpy() if t is not None else None


def rand(g, *shape):
    return torch.randn(*shape, generator=g)


def check(h, branch, post, gate, scale, pre, eps, x_dtype, out=None):
    h0 = f64(h)
    h_ref, x_ref = ref.norm_residual(h0, f64(branch), f64(post), f64(gate.view(-1, h.shape[-1])) if gate is not None else None,
                                     float(np.float32(scale)), f64(pre), float(np.float32(eps)))
    got_h, got_x = si.norm_residual(h, branch, post_w=post, gate=gate, scale=scale, pre_w=pre, eps=eps,
                                    x_dtype=x_dtype, out=out)
    d = h0.shape[1]
    unit = (d / 2 + 16) * 2.0 ** -24
    eh = np.zeros_like(h0)
    if branch is not None:
        eh = unit * np.abs(h_ref - h0) + 2.0 ** -24 * np.abs(h_ref)
        tol = eh + HALF_STEP[h.dtype] * (np.abs(h_ref) + eh) + SMALLEST[h.dtype]
        assert got_h.dtype == h.dtype and (np.abs(f64(got_h) - h_ref) <= tol).all()
    else:
        assert got_h is None
    if pre is not None:
        rms = np.sqrt((h_ref ** 2).mean(axis=1, keepdims=True) + eps)
        w = np.abs(f64(pre))
        ex = eh / rms * w + np.abs(x_ref) * (np.sqrt((eh ** 2).mean(axis=1, keepdims=True)) / rms + unit)
        tol = ex + HALF_STEP[x_dtype] * (np.abs(x_ref) + ex) + SMALLEST[x_dtype]
        assert got_x.dtype == x_dtype and (np.abs(f64(got_x) - x_ref) <= tol).all()
    else:
        assert got_x is None
    return got_h, got_x


SHAPES = [(1, 1), (1, 7), (3, 8), (2, 63), (5, 64), (9, 100), (1, 512), (7, 513), (4, 520), (33, 1447), (3, 2048),
          (2, 2056), (1, 4096), (5, 4100), (3, 5120), (2, 8192), (2, 8200), (3, 12287), (1, 16384), (1000, 24)]


@pytest.mark.parametrize("tokens,d", SHAPES)
@pytest.mark.parametrize("types", [(F32, F32, F16), (BF16, BF16, BF16), (F16, F32, F32), (F32, BF16, BF16),
                                   (F16, F16, F16)])
def test_parts(tokens, d, types):
    th, tb, tx = types
    g = torch.Generator().manual_seed(tokens * 1000 + d)
    h, b = rand(g, tokens, d).mul(4).to(th).to(DEV), rand(g, tokens, d).to(tb).to(DEV)
    post, pre = 1 + 0.1 * rand(g, d).to(DEV), 1 + 0.1 * rand(g, d).to(DEV)
    gate = rand(g, d).to(DEV)
    check(h, b, post, gate, 0.22, pre, 1e-5, tx)
    check(h, b, None, None, 1.0, pre, 1e-6, tx)
    check(h, b, post, None, -1.5, None, 0.0, tx)
    check(h, b, None, gate, 1.0, None, 1e-5, tx)
    check(h, None, None, None, 1.0, pre, 1e-5, tx)


@pytest.mark.parametrize("tokens,gates", [(6, 1), (6, 2), (6, 3), (6, 6), (500, 4)])
def test_gates_by_run_of_tokens(tokens, gates):
    g = torch.Generator().manual_seed(gates)
    for d in (96, 99, 2304):
        h, b = rand(g, tokens, d).to(DEV), rand(g, tokens, d).to(DEV)
        check(h, b, None, rand(g, gates, d).to(DEV), 0.5, 1 + 0.1 * rand(g, d).to(DEV), 1e-5, F16)


@pytest.mark.parametrize("d", [64, 67, 4096])
def test_in_place_and_strides(d):
    g = torch.Generator().manual_seed(d)
    tokens = 5
    pre = 1 + 0.1 * rand(g, d).to(DEV)
    for off, ld in ((0, d + 8), (1, d + 3), (8, d + 16)):
        buf = torch.full((tokens, ld + off), 9.0, dtype=F32, device=DEV)
        h = buf[:, off:off + d]
        h.copy_(rand(g, tokens, d))
        b = torch.empty(tokens, d + 2, dtype=BF16, device=DEV)[:, 1:1 + d]
        b.copy_(rand(g, tokens, d))
        keep = buf.clone()
        out, x = check(h.clone(), b, None, None, 0.5, pre, 1e-5, F16)
        got, x2 = si.norm_residual(h, b, scale=0.5, pre_w=pre, out=h)
        assert got is h and torch.equal(h, out) and torch.equal(x, x2)
        keep[:, off:off + d] = out
        assert torch.equal(buf, keep)  # nothing beside the rows
    both = torch.zeros(tokens, 2 * d, device=DEV)  # the result in the other columns of h's own matrix
    both[:, :d] = rand(g, tokens, d)
    out, _ = si.norm_residual(both[:, :d], b, scale=0.5, out=both[:, d:])
    want, _ = si.norm_residual(both[:, :d].contiguous(), b, scale=0.5)
    assert torch.equal(out, want)


def test_values_at_the_edges():
    """A row of zeros (eps holds the norm finite), one huge value, a row with an
    infinity or NaN: each row alone."""
    d = 256
    h = torch.ones(6, d, device=DEV)
    h[1] = 0
    h[2, 3] = 1e15
    h[3, 3] = float("inf")
    h[4, 3] = float("nan")
    _, x = si.norm_residual(h, pre_w=torch.ones(d, device=DEV), eps=1e-5, x_dtype=F32)
    assert torch.allclose(x[0], x[5]) and bool((x[1] == 0).all())
    assert abs(x[2, 3].item() - 16.0) < 1e-4 and bool((x[2, :3] < 1e-13).all())
    assert torch.isnan(x[3, 3]) and bool((x[3, :3] == 0).all()) and bool(torch.isnan(x[4]).all())
    _, z = si.norm_residual(h[:0], pre_w=torch.ones(d, device=DEV))
    assert z.shape == (0, d)


def test_graph_and_streams():
    g = torch.Generator().manual_seed(1)
    h, b = rand(g, 3, 1000).to(DEV), rand(g, 3, 1000).to(DEV)
    w = 1 + 0.1 * rand(g, 1000).to(DEV)
    out = torch.empty_like(h)
    si.norm_residual(h, b, post_w=w, pre_w=w, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _, x = si.norm_residual(h, b, post_w=w, pre_w=w, out=out)
    for i in range(3):
        b.copy_(rand(g, 3, 1000))
        graph.replay()
        torch.cuda.synchronize()
        want_h, want_x = si.norm_residual(h, b, post_w=w, pre_w=w)
        assert torch.equal(out, want_h) and torch.equal(x, want_x)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other, _ = si.norm_residual(h, b, post_w=w, pre_w=w)
    s.synchronize()
    assert torch.equal(other, want_h)
