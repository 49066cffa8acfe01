"""One workspace under calls of different kinds and numbers of tokens.

A single-launch call takes a 64-bit word of the workspace as published when its
high half is the call's tag, ``0x80000000 | call counter``.  Whatever other
calls leave there must never read as one: a 64-bit word whose top bit is clear
cannot, whatever the counter is.
"""

import itertools

import numpy as np
import pytest
import torch

import paper_2411_12692_amd as si
from paper_2411_12692_amd import _lib, synth

pytestmark = pytest.mark.gpu

DEV = "cuda"


def tokens(d, b, seed):
    g = torch.Generator().manual_seed(seed)
    return torch.randn(b, d, generator=g).half().to(DEV)


def layer_weights(d, k, s=0.5, seed=1):
    L = synth.planted_layer(d, k, s, config=seed)
    return [t.to(DEV) for t in (L.w_gate, L.w_up, L.w_down)]


def counter(ws):
    return int(ws[:4].view(torch.int32).item()) & 0xffffffff


def assert_no_tag(ws, what):
    words = ws[:ws.numel() // 8 * 8].view(torch.int64)
    assert not bool((words < 0).any()), what


@pytest.mark.parametrize("gated", [True, False])
@pytest.mark.parametrize("d,k", [(512, 1376), (640, 65), (128, 1)])
def test_mxfp4_calls_leave_no_tags(d, k, gated):
    wg, wu, wd = layer_weights(d, k)
    layer = si.MXFP4MLPLayer(wg, wu if gated else None, wd, max_batch=8)
    every = torch.ones(k, dtype=torch.uint8, device=DEV)
    for b in range(1, 9):
        for mask in (None, every):
            layer.workspace.zero_()
            x = tokens(d, b, b)
            if mask is None:
                layer(x, 1.0, outputs=True)
            else:
                layer.sparse_mlp(x, mask, counters=True)
            torch.cuda.synchronize()
            assert_no_tag(layer.workspace, (b, mask is None))


def layers(d, k):
    wg, wu, wd = layer_weights(d, k)
    made = {"fp16": si.MLPLayer(wg, wu, wd, 8), "int8": si.Int8MLPLayer(wg, wu, wd, 8),
            "mxfp4": si.MXFP4MLPLayer(wg, wu, wd, 8)}
    ws = si.new_workspace_mxfp4(k, d, 8)
    return made, ws


@pytest.mark.parametrize("mx_b,b", [(p, q) for p in (1, 2, 3, 5, 8) for q in (1, 2, 3, 4, 6, 8)])
@pytest.mark.parametrize("kind", ["fp16", "int8"])
def test_row_sets_are_not_taken_for_h3(kind, mx_b, b):
    """MXFP4 calls whose kept rows, as a number, are the next single-launch call's
    tag (row 31 and the counter's bits of every 32 rows): that call's y is the one
    of a workspace of its own."""
    d, k = 512, 1376
    made, ws = layers(d, k)
    every = torch.ones(k, dtype=torch.uint8, device=DEV)
    lay, mx = made[kind], made["mxfp4"]
    x = tokens(d, b, 7)
    want = lay.sparse_mlp(x, every)
    scale = want.abs().max()
    lay.workspace = mx.workspace = ws
    for _ in range(3):
        now = counter(ws)
        bits = torch.tensor([(now >> i) & 1 for i in range(31)] + [1], dtype=torch.uint8, device=DEV)
        mx.sparse_mlp(tokens(d, mx_b, 9), bits.repeat(k // 32))
        y = lay.sparse_mlp(x, every)
        assert counter(ws) == now + 1
        assert bool(((y - want).abs() <= 1e-4 * scale).all())
        h3 = si.read_h3(ws, k, d, b, every)
        assert not torch.isnan(h3).any()


def test_calls_of_every_kind_in_turn():
    """fp16, INT8 and MXFP4 calls of 1 to 8 tokens, each after each: y, and h3 read
    back, as from a workspace of the call's own."""
    d, k = 640, 1000
    made, ws = layers(d, k)
    every = torch.ones(k, dtype=torch.uint8, device=DEV)
    want = {}
    for (name, lay), b in itertools.product(made.items(), range(1, 9)):
        y, (mask, *_) = lay(tokens(d, b, b), 1.0, outputs=True)
        want[name, b] = (y, mask, si.read_h3(lay.workspace, k, d, b, mask))
    for lay in made.values():
        lay.workspace = ws
    order = list(want)
    rng = np.random.default_rng(5)
    for _ in range(6):
        rng.shuffle(order)
        for name, b in order:
            b = int(b)
            y, (mask, *_) = made[name](tokens(d, b, b), 1.0, outputs=True)
            y0, mask0, h30 = want[name, b]
            assert torch.equal(mask, mask0), (name, b)
            assert torch.equal(si.read_h3(ws, k, d, b, mask), h30), (name, b)
            assert bool(((y - y0).abs() <= 1e-4 * y0.abs().max()).all()), (name, b)
            assert _lib.status("si_workspace_check", ws.data_ptr(), ws.numel(), 0) == 0


def test_layers_of_different_sizes_in_turn():
    """Layers of other k and d, whose regions lie over each other's, on one
    workspace that holds the largest."""
    sizes = [(640, 1000), (512, 1376), (1152, 300), (128, 4000)]
    calls, want = {}, {}
    for d, k in sizes:
        made, _ = layers(d, k)
        for (name, lay), b in itertools.product(made.items(), (1, 2, 4, 7)):
            y, (mask, *_) = lay(tokens(d, b, b), 1.0, outputs=True)
            calls[d, name, b] = lay
            want[d, name, b] = (y, mask)
    ws = torch.zeros(max(si.workspace_bytes(k, d, 8) for d, k in sizes), dtype=torch.uint8, device=DEV)
    for lay in calls.values():
        lay.workspace = ws
    order = list(calls)
    rng = np.random.default_rng(6)
    for _ in range(5):
        for i in rng.permutation(len(order)):
            d, name, b = order[i]
            y, (mask, *_) = calls[order[i]](tokens(d, b, b), 1.0, outputs=True)
            y0, mask0 = want[order[i]]
            assert torch.equal(mask, mask0), order[i]
            assert bool(((y - y0).abs() <= 1e-4 * y0.abs().max()).all()), order[i]
    assert _lib.status("si_workspace_check", ws.data_ptr(), ws.numel(), 0) == 0


class TestTwoLaunches:
    """A layer with more rows than the single-launch kernel takes, except from a
    list: the calls of two launches leave h3 of either sign in the workspace."""

    d, k = 1152, 65400

    @pytest.fixture(scope="class")
    def big(self):
        g = torch.Generator(device=DEV).manual_seed(3)
        return [0.05 * torch.randn(*shape, generator=g, device=DEV) for shape in ((self.k, self.d),) * 3]

    @pytest.fixture(scope="class")
    def weights(self, big):
        return [w.half() for w in big]

    @pytest.mark.parametrize("b", [1, 2, 5, 8])
    @pytest.mark.parametrize("form", ["mask", "predict", "relu"])
    def test_calls_leave_no_tags(self, weights, form, b):
        wg, wu, wdt = weights
        assert _lib.load().si_single_launch(self.k, self.d, b) == 0
        ws = si.new_workspace(self.k, self.d, 8)
        x = tokens(self.d, b, b)
        if form == "predict":
            si.predict_sparse_mlp(si.pack_signs(wg), wg, wu, wdt, x, 1.0, ws, outputs=True)
            status = 256 + (self.k + 63) // 64 * 8  # look-back words, tagged: the header and they come first
            assert_no_tag(ws[(status + 255) // 256 * 256:], b)
        else:
            every = torch.ones(self.k, dtype=torch.uint8, device=DEV)
            si.sparse_mlp(wg, wu if form == "mask" else None, wdt, x, ws, mask=every, counters=True)
            assert_no_tag(ws, b)

    @pytest.mark.parametrize("b", [1, 2, 4])
    def test_list_call_after_a_mask_call(self, weights, b):
        """The list call is a single launch on the same workspace, with its counter
        still 0: h3 of the tokens whose gate value is 0 must not be its tag."""
        every = torch.ones(self.k, dtype=torch.uint8, device=DEV)
        idx = torch.arange(self.k, dtype=torch.int32, device=DEV)
        n = torch.tensor([self.k], dtype=torch.int32, device=DEV)
        x = tokens(self.d, b, 11)
        want = si.sparse_mlp(*weights, x, si.new_workspace(self.k, self.d, b), active_idx=idx, n_active=n)
        ws = si.new_workspace(self.k, self.d, 8)
        si.sparse_mlp(*weights, tokens(self.d, 8, 12), ws, mask=every)
        assert counter(ws) == 0
        got = si.sparse_mlp(*weights, x, ws, active_idx=idx, n_active=n)
        assert counter(ws) == 1 and bool(((got - want).abs() <= 1e-4 * want.abs().max()).all())
        h3 = si.read_h3(ws, self.k, self.d, b, every)
        assert not torch.isnan(h3).any()
