"""The differentiable operators as nodes of PyTorch's graph: what hooks, streams, empty
batches and captures ask of them beyond the values of their gradients
(``test_gpu_dense.py``, ``test_gpu_norm_train.py``)."""

import pytest
import torch
import torch.autograd.forward_ad as fwAD

import paper_2411_12692_amd as si

pytestmark = pytest.mark.gpu
DEV = "cuda"
F16, F32 = torch.float16, torch.float32
M, N, K = 37, 96, 40


def gen(*key):
    g = torch.Generator()
    g.manual_seed(hash(key) % (1 << 31))
    return g


def values(g, *shape, dtype=F16):
    return torch.randn(*shape, generator=g).mul(0.3).to(dtype).to(DEV)


def operators(g):
    """Name, the call over x, its weights."""
    w, wt, wg, wu, wd = (values(g, *s).requires_grad_() for s in ((K, N), (N, K), (K, N), (K, N), (N, K)))
    nw, nb = values(g, N, dtype=F32).requires_grad_(), values(g, N, dtype=F32).requires_grad_()
    return [("linear", lambda x: si.linear(x, w), (w,)),
            ("linear, W^T", lambda x: si.linear(x, wt, transposed=True), (wt,)),
            ("gated_linear", lambda x: si.gated_linear(x, wg, wu), (wg, wu)),
            ("gated_linear, no W_up", lambda x: si.gated_linear(x, wg), (wg,)),
            ("mlp", lambda x: si.mlp(x, wg, wu, wd), (wg, wu, wd)),
            ("mlp, no W_up", lambda x: si.mlp(x, wg, None, wd), (wg, wd)),
            ("layer_norm", lambda x: si.layer_norm(x, nw, nb), (nw, nb)),
            ("rms_norm", lambda x: si.rms_norm(x, nw), (nw,))]


NAMES = ["linear", "linear, W^T", "gated_linear", "gated_linear, no W_up", "mlp", "mlp, no W_up", "layer_norm", "rms_norm"]


def pick(name, g):
    return next((f, leaves) for n, f, leaves in operators(g) if n == name)


class Wider(torch.autograd.graph.saved_tensors_hooks):
    """Hands matrices back as column ranges of wider ones."""

    def __init__(self):
        def unpack(t):
            return t if t.dim() != 2 else torch.nn.functional.pad(t, (16, 24))[:, 16:16 + t.shape[1]]
        super().__init__(lambda t: t, unpack)


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("width", [304, 300])
def test_slices_and_hooks_of_saved_tensors(name, width):
    """x is a column range; hooks hand it back contiguous (``save_on_cpu``) or in rows of
    yet another stride: the same gradients, bit for bit.  (A norm of rows that do not
    start on 16 bytes adds in another order, and only those that do are compared.)"""
    if "norm" in name and width % 8:
        width += 8 - width % 8
    f, leaves = pick(name, gen(1))
    x = values(gen(2), M, width)[:, 8:8 + N].detach().requires_grad_()
    assert x.stride(0) == width
    dy = values(gen(3), *f(x).shape)
    want = torch.autograd.grad(f(x), (x, *leaves), dy)
    for hooks in (torch.autograd.graph.save_on_cpu, Wider):
        with hooks():
            y = f(x)
        got = torch.autograd.grad(y, (x, *leaves), dy)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), hooks


@pytest.mark.parametrize("name", NAMES)
def test_tangents_are_refused(name):
    """A tensor with a tangent: every operand is looked at, with and without reverse mode.
    Inside a ``dual_level`` tensors without one are taken."""
    f, leaves = pick(name, gen(4))
    x = values(gen(5), M, N)
    want = f(x)
    with fwAD.dual_level():
        assert torch.equal(f(x), want)
        dual = fwAD.make_dual(x, torch.ones_like(x))
        for call in (lambda: f(dual), lambda: f(dual.view(1, M, N))):
            with pytest.raises(NotImplementedError, match="forward-mode"):
                call()
            with torch.no_grad(), pytest.raises(NotImplementedError, match="forward-mode"):
                call()


def test_tangents_of_weights_are_refused():
    g = gen(6)
    x, w, wt, nw = values(g, M, N), values(g, K, N), values(g, N, K), values(g, N, dtype=F32)
    with fwAD.dual_level():
        d, dt, dn = (fwAD.make_dual(t, torch.ones_like(t)) for t in (w, wt, nw))
        for call in (lambda: si.linear(x, d), lambda: si.gated_linear(x, d, w), lambda: si.gated_linear(x, w, d),
                     lambda: si.gated_linear(x, d), lambda: si.mlp(x, d, w, wt), lambda: si.mlp(x, w, d, wt),
                     lambda: si.mlp(x, w, w, dt), lambda: si.mlp(x, w, None, dt), lambda: si.layer_norm(x, dn, nw),
                     lambda: si.layer_norm(x, nw, dn), lambda: si.rms_norm(x, dn)):
            with pytest.raises(NotImplementedError, match="forward-mode"):
                call()


@pytest.mark.parametrize("name", NAMES)
def test_no_tokens_and_frozen_weights(name):
    """The gradient with respect to x alone, of no tokens: asked for alone, or with
    weights that have none."""
    f, leaves = pick(name, gen(7))
    for shape in ((0, N), (2, 0, N)):
        x = torch.zeros(shape, dtype=F16, device=DEV).requires_grad_()
        y = f(x)
        (dx,) = torch.autograd.grad(y, x, torch.zeros_like(y))
        assert dx.shape == x.shape and dx.dtype == F16
        for t in leaves:
            t.requires_grad_(False)
        f(x).float().sum().backward()
        assert x.grad.shape == x.shape
        for t in leaves:
            t.requires_grad_(True)
        dw = torch.autograd.grad(f(x), leaves, torch.zeros_like(y))
        assert all(torch.equal(d, torch.zeros_like(t)) for d, t in zip(dw, leaves))


def leaf_cases():
    """What of a leaf a call is given: the leaf itself is another test's."""
    return [("3-D", (3, 13, N), lambda t: t), ("3-D, copied rows", (13, 3, N), lambda t: t.transpose(0, 1)),
            ("slice", (M, 304), lambda t: t[:, 8:8 + N]), ("slice of 3-D", (4, 13, N), lambda t: t[1:]),
            ("one row", (N,), lambda t: t)]


@pytest.mark.parametrize("case", range(5))
def test_capture_with_views_of_a_leaf_of_a_live_graph_is_refused(case):
    """The refusal comes in the forward call, before any captured backward pass.  Once the
    eager graph is gone the same capture goes through."""
    kind, shape, part = leaf_cases()[case]
    x = values(gen(8), *shape).requires_grad_()
    for name in NAMES:
        f, leaves = pick(name, gen(9))
        for t in leaves:
            t.requires_grad_(False)
        alive = f(part(x))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with pytest.raises(RuntimeError, match="eager graph"):
            with torch.cuda.graph(graph):
                f(part(x))
        torch.cuda.synchronize()
        ones = torch.ones_like(alive)
        want = torch.autograd.grad(alive, x, ones)[0]
        del alive, graph
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            y = f(part(x))
            got = torch.autograd.grad(y, x, ones)[0]
        del y
        for _ in range(3):
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(got, want), (kind, name)


def test_capture_with_weights_that_are_views_of_a_leaf_of_a_live_graph_is_refused():
    g = gen(10)
    both = values(g, 2 * K, N).requires_grad_()  # W_gate over W_up
    down, norm = values(g, N, 2 * K).requires_grad_(), values(g, 2, N, dtype=F32).requires_grad_()
    x, w, wt = values(g, M, N), values(g, K, N), values(g, N, K)
    for f, leaf in ((lambda: si.linear(x, both[K:]), both), (lambda: si.gated_linear(x, both[:K], w), both),
                    (lambda: si.gated_linear(x, w, both[K:]), both), (lambda: si.mlp(x, w, both[:K], wt), both),
                    (lambda: si.mlp(x, w, w, down.view(2, N, K)[1]), down), (lambda: si.layer_norm(x, norm[0], norm[1]), norm),
                    (lambda: si.layer_norm(x, norm[0].detach(), norm[1]), norm), (lambda: si.rms_norm(x, norm[0]), norm)):
        alive = f()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with pytest.raises(RuntimeError, match="eager graph"):
            with torch.cuda.graph(graph):
                f()
        torch.cuda.synchronize()
        assert torch.autograd.grad(alive, leaf, torch.ones_like(alive))[0].shape == leaf.shape
        del alive, graph


@pytest.mark.parametrize("name", NAMES)
def test_a_node_called_by_itself(name):
    """On the stream of the forward call: as in a backward pass.  On another one, where
    its memory and launches would not be in order: refused before any launch."""
    f, leaves = pick(name, gen(11))
    x = values(gen(12), M, N).requires_grad_()
    y = f(x)
    dy = values(gen(13), *y.shape)
    want = torch.autograd.grad(y, (x, *leaves), dy, retain_graph=True)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        with pytest.raises(RuntimeError, match="another stream"):
            y.grad_fn(dy)
        # autograd changes to the forward call's stream
        other = torch.autograd.grad(y, (x, *leaves), dy, retain_graph=True)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(other, want))
    got = [t for t in y.grad_fn(dy) if t is not None]
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and len(got) == len(want)
