"""The autograd nodes on the CPU: which arguments a backward pass hands to the library.

The nodes run over CPU tensors in a process of their own, with ``autograd_calls.cpp`` in
the library's place: it computes nothing and writes each call's arguments, which are
compared with the tensors that the saved tensors' hooks handed back."""

import os
import shutil
import subprocess
import sys

import pytest
import torch
import torch.autograd.forward_ad as fwAD

import paper_2411_12692_amd as si
from paper_2411_12692_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def calls(tmp_path_factory):
    """The library of recording calls."""
    if shutil.which(build.CXX) is None:
        pytest.skip("no C++ compiler")
    if not os.path.exists(build.AUTOGRAD_LIB):
        build.build()
    lib = str(tmp_path_factory.mktemp("calls") / "calls.so")
    subprocess.run([build.CXX, "-shared", "-fPIC", f"-I{os.path.join(build.ROOT, 'include')}",
                    os.path.join(HERE, "autograd_calls.cpp"), "-o", lib], check=True)
    return lib


PRELUDE = r'''
import ctypes, os, sys
calls = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
sys.path.insert(0, sys.argv[2])
import torch
from paper_2411_12692_amd import _lib
nodes = _lib.autograd()
F16, F32 = torch.float16, torch.float32
M, N, K = 6, 96, 40
NODES = ("linear", "linear_t", "gated", "relu", "mlp", "mlp_relu", "layer_norm", "rms_norm")


def tensor(*shape, dtype=F16):
    return torch.rand(*shape).to(dtype)


def make(name, x, leaves=True):
    """A call of the node over x [M][N]: the output and its leaves."""
    M = x.shape[0]
    def leaf(t):
        return t.requires_grad_(leaves)
    if name in ("linear", "linear_t"):
        w = leaf(tensor(N, K) if name == "linear_t" else tensor(K, N))
        y = tensor(M, K)
        nodes.linear(y, x, w, M, N, K, name == "linear_t", 0)
        return y, [w]
    if name in ("gated", "relu"):
        up = name == "gated"
        wg, wu = leaf(tensor(K, N)), leaf(tensor(K, N)) if up else None
        h = tensor(M, K)
        g, u = (tensor(M, K, dtype=F32), tensor(M, K, dtype=F32)) if up else (None, None)
        nodes.gated_linear(h, x, wg, wu, g, u, M, N, K, 0)
        return h, [wg, wu][:1 + up]
    if name in ("mlp", "mlp_relu"):
        up = name == "mlp"
        wg, wu, wd = leaf(tensor(K, N)), leaf(tensor(K, N)) if up else None, leaf(tensor(N, K))
        y, h = tensor(M, N), tensor(M, K)
        g, u = (tensor(M, K, dtype=F32), tensor(M, K, dtype=F32)) if up else (None, None)
        nodes.mlp(y, x, wg, wu, wd, h, g, u, M, N, K, 0)
        return y, [t for t in (wg, wu, wd) if t is not None]
    layer = name == "layer_norm"
    w, b = leaf(tensor(N, dtype=F32)), leaf(tensor(N, dtype=F32)) if layer else None
    y = tensor(M, N)
    nodes.norm(y, x, w, b, tensor(M, dtype=F32) if layer else None, tensor(M, dtype=F32), M, N, layer, 0)
    return y, [t for t in (w, b) if t is not None]


def capture(f):
    """What f's calls write."""
    out = os.dup(1)
    r, w = os.pipe()
    libc = ctypes.CDLL(None)
    sys.stdout.flush()
    libc.fflush(None)
    os.dup2(w, 1)
    try:
        f()
    finally:
        libc.fflush(None)
        os.dup2(out, 1)
        os.close(w)
        os.close(out)
    with os.fdopen(r) as lines:
        return [{k: int(v) for k, v in (p.split("=") for p in l.split()[1:])} | {"call": l.split()[0]} for l in lines]


def of(text):
    """The arguments of the library's call, and the strides that workspaces were asked for."""
    made = [c for c in text if c["call"] != "workspace"]
    assert len(made) == 1, text
    for c in text:
        if c["call"] == "workspace":
            assert c["ldx"] == made[0]["ldx"] and c.get("lddy", made[0].get("lddy")) == made[0].get("lddy"), text
    return made[0]
'''


EACH = """

for name in NODES:
    print(name, flush=True)
    check(name)
"""


def run(calls, script):
    p = subprocess.run([sys.executable, "-c", PRELUDE + script + EACH, calls, build.ROOT], capture_output=True, text=True,
                       timeout=300)
    assert p.returncode == 0, p.stdout + p.stderr
    return p.stdout


def test_strides_are_those_of_the_tensors_that_hooks_hand_back(calls):
    """x is a slice of wider rows.  A hook hands back a contiguous copy, rows at another
    stride, or rows that the library does not take (transposed, overlapping): each is read
    with its own stride, and never past its own end."""
    run(calls, r'''
def check(name):
    wide = tensor(M, 300)

    def wider(t):
        return torch.cat([t, t], dim=1)[:, :t.shape[1]]

    def transposed(t):
        return t.t().contiguous().t()

    for layout, ld in ((lambda t: t.contiguous(), N), (wider, 2 * N), (transposed, N), (lambda t: t, 300)):
        back = []

        def unpack(t):
            if t.dim() == 2 and tuple(t.shape) == (M, N):
                t = layout(t)
                back.append(t)
            return t
        x = wide[:, :N].requires_grad_()
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, unpack):
            y, leaves = make(name, x)
        grads = []
        c = of(capture(lambda: grads.extend(torch.autograd.grad(y, [x, *leaves], torch.ones_like(y)))))
        assert c["ldx"] == ld, (c, ld)
        xs = [t for t in back if t.data_ptr() == c["x"]]
        if layout is transposed:
            assert not xs, c  # a copy that the node made
        else:
            assert xs and xs[0].stride(0) == c["ldx"], c
            # the last element that is read lies in the tensor's own memory
            t = xs[0]
            assert (M - 1) * c["ldx"] + N <= t.untyped_storage().nbytes() // t.element_size() - t.storage_offset()
        assert [g.shape for g in grads] == [t.shape for t in (x, *leaves)]
''')


def test_strides_without_hooks(calls):
    """As the forward call had them; a single row's stride leads nowhere."""
    run(calls, r'''
def check(name):
    for x, ld in ((tensor(M, 300)[:, :N], 300), (tensor(M, N), N)):
        x.requires_grad_()
        y, leaves = make(name, x)
        c = of(capture(lambda: torch.autograd.grad(y, [x, *leaves], torch.ones_like(y))))
        assert c["ldx"] == ld and c["x"] == x.data_ptr(), c
    x = tensor(1, 300)[:, :N].requires_grad_()
    y, leaves = make(name, x)
    assert of(capture(lambda: torch.autograd.grad(y, [x, *leaves], torch.ones_like(y))))["ldx"] == N
''')


def test_saved_tensors_of_another_type_size_or_device_are_refused(calls):
    """Whatever is saved and handed back as something else: an error, no call."""
    run(calls, r'''
def check(name):
    count = [0]

    def counted(t):
        count[0] += 1
        return t

    with torch.autograd.graph.saved_tensors_hooks(counted, lambda t: t):
        make(name, tensor(M, N).requires_grad_())
    assert count[0] >= 2
    for i in range(count[0]):
        for change in (lambda t: t.double(), lambda t: t.bfloat16(), lambda t: t.flatten()[:-1], lambda t: t[:0],
                       lambda t: t.unsqueeze(0), lambda t: t.to("meta")):
            seen = [0]

            def pack(t):
                seen[0] += 1
                return (seen[0] - 1, t)
            x = tensor(M, N).requires_grad_()
            with torch.autograd.graph.saved_tensors_hooks(pack, lambda p: change(p[1]) if p[0] == i else p[1]):
                y, leaves = make(name, x)
            error = []

            def backward():
                try:
                    torch.autograd.grad(y, [x, *leaves], torch.ones_like(y))
                except RuntimeError as e:
                    error.append(str(e))
            text = capture(backward)
            assert error and ("handed back" in error[0] or "backward pass" in error[0]), (i, error)
            assert not [c for c in text if c["call"] != "workspace"], (i, text)
''')


def test_other_saved_tensors_may_change_their_strides(calls):
    """Weights, sums and statistics handed back with other strides are made whole."""
    run(calls, r'''
def check(name):
    def strided(t):
        wide = t.new_zeros(*t.shape[:-1], 2 * t.shape[-1])
        wide[..., ::2] = t
        return wide[..., ::2]

    x = tensor(M, N).requires_grad_()
    back = []
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t, lambda t: back.append(strided(t)) or back[-1]):
        y, leaves = make(name, x)
    c = of(capture(lambda: torch.autograd.grad(y, [x, *leaves], torch.ones_like(y))))
    read = {k: c[k] for k in ("x", "w", "w_up", "w_down", "g", "u", "h", "mean", "r") if c.get(k)}
    assert len(read) == len(back) and not {t.data_ptr() for t in back} & set(read.values()), c
    assert c["ldx"] == N
''')


def test_tangents_are_refused():
    """Forward-mode: outputs have no tangents, so inputs with one are not taken, with or
    without reverse mode; inputs without one are, inside a ``dual_level`` too."""
    x, w = torch.ones(2, 4), torch.ones(3, 4).requires_grad_()
    with fwAD.dual_level():
        dual = fwAD.make_dual(x, torch.ones_like(x))
        for tensors in ((dual, None, w), (x, dual), (dual,)):
            with pytest.raises(NotImplementedError, match="forward-mode"):
                si._wants_grad(*tensors)
            with torch.no_grad(), pytest.raises(NotImplementedError, match="forward-mode"):
                si._wants_grad(*tensors)
        assert si._wants_grad(x, None, w) and not si._wants_grad(x)
    assert si._wants_grad(x, w) and not si._wants_grad(x)


def test_gradients_of_another_size_type_or_device(calls):
    """A node's own call and hooks in front of it are not looked at by autograd: another
    type is y's first, as autograd makes it; another size or device is refused."""
    run(calls, r'''
def check(name):
    x = tensor(M, N).requires_grad_()
    y, leaves = make(name, x)
    good = of(capture(lambda: y.grad_fn(torch.ones_like(y))))
    for other in (torch.ones(y.shape).double(), torch.ones(y.shape).bfloat16(), torch.ones(y.shape)):
        c = of(capture(lambda: y.grad_fn(other)))
        assert c["dy"] != other.data_ptr() and c.get("dy_dtype") == good.get("dy_dtype") and c["lddy"] == good["lddy"], c
    bad = (tensor(M - 1, y.shape[1]), tensor(M, y.shape[1] - 1), tensor(y.shape[1]), tensor(1, *y.shape), tensor(0, y.shape[1]),
           torch.empty(y.shape, dtype=F16, device="meta"))
    for other in bad:
        text = []

        def refused(f):
            try:
                f()
            except RuntimeError as e:
                text.append(str(e))
        assert not capture(lambda: refused(lambda: y.grad_fn(other))) and "a gradient" in text[-1], (other.shape, text)
        hook = y.grad_fn.register_prehook(lambda grads: (other,))
        lines = capture(lambda: refused(lambda: torch.autograd.grad(y, x, torch.ones_like(y), retain_graph=True)))
        assert not lines and len(text) == 2, (other.shape, lines, text)
        hook.remove()
''')


def test_lazily_negated_gradients(calls):
    """The sign of an imaginary part of a conjugate is a bit of the tensor, not of its
    values: the library is given values."""
    run(calls, r'''
def check(name):
    x = tensor(M, N).requires_grad_()
    y, leaves = make(name, x)
    dy = torch._neg_view(torch.ones_like(y))
    assert dy.is_neg()
    c = of(capture(lambda: torch.autograd.grad(y, x, dy)))
    assert c["dy"] != dy.data_ptr(), c
''')
