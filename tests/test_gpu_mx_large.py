"""The MXFP4 operators and ``norm_residual`` where offsets pass 32 bits, at their
longest sums, and captured together into a graph.

The large cases compare whole rows at both ends and around the 2^32-byte mark with
the same rows alone, or with exact sums (see ``test_gpu_mxfp4``)."""

import numpy as np
import pytest
import torch

import mx_ref as ref
import paper_2411_12692_amd as si

pytestmark = pytest.mark.gpu

DEV = "cuda"


def f64(t):
    return t.detach().cpu().double().numpy()


def test_quantize_past_32_bits():
    rows, n = 40000, 65536  # 5.2 GB of fp16
    w = torch.empty(rows, n, dtype=torch.float16, device=DEV)
    for i in range(0, rows, 5000):
        w[i:i + 5000].normal_(generator=torch.Generator(device=DEV).manual_seed(i))
    q, s = si.quantize_rows_mxfp4(w)
    back = si.dequantize_rows_mxfp4(q, s, n)
    for r in (0, 1, 16383, 16384, 32767, 32768, 39999):
        q1, s1 = si.quantize_rows_mxfp4(w[r:r + 1].clone())
        assert torch.equal(q[r], q1[0]) and torch.equal(s[r], s1[0])
        assert torch.equal(back[r], si.dequantize_rows_mxfp4(q1, s1, n)[0])


@pytest.mark.parametrize("m", [2, 20, 70])
@pytest.mark.parametrize("a4", [False, True])
def test_product_past_32_bits(m, a4):
    rows, n = 600000, 16384  # 4.9 GB of codes
    g = torch.Generator(device=DEV).manual_seed(m)
    q = torch.empty(rows, n // 2, dtype=torch.uint8, device=DEV)
    for i in range(0, rows, 100000):
        q[i:i + 100000] = torch.randint(0, 256, (100000, n // 2), generator=g, dtype=torch.uint8, device=DEV)
    s = torch.full((rows, n // 32), 127, dtype=torch.uint8, device=DEV)
    x = torch.randint(-1, 2, (m, n), generator=g, device=DEV).half()
    y = si.linear_mxfp4_a4(*si.quantize_rows_mxfp4(x), q, s, torch.float32) if a4 else \
        si.linear_mxfp4(x, q, s, torch.float32)
    pick = [0, 1, 262143, 262144, 524287, 524288, 599998, 599999]
    # |sums| at most 6 n units of 0.5: below 2^24
    w = ref.values(ref.unpack(q[pick].cpu().numpy()), np.full((len(pick), n // 32), 127, np.uint8), n)
    assert np.array_equal(y[:, pick].cpu().numpy(), (f64(x) @ w.T).astype(np.float32))


@pytest.mark.parametrize("m,rows", [(1, 40), (5, 40)])
def test_product_longest_sum(m, rows):
    n = 1 << 20  # |sums| at most 6 n units of 0.5: below 2^24
    g = torch.Generator(device=DEV).manual_seed(m)
    q = torch.randint(0, 256, (rows, n // 2), generator=g, dtype=torch.uint8, device=DEV)
    s = torch.full((rows, n // 32), 127, dtype=torch.uint8, device=DEV)
    x = torch.randint(-1, 2, (m, n), generator=g, device=DEV)
    w = ref.values(ref.unpack(q.cpu().numpy()), s.cpu().numpy(), n)
    want = (f64(x) @ w.T).astype(np.float32)
    for dtype in (torch.float16, torch.bfloat16):
        assert np.array_equal(si.linear_mxfp4(x.to(dtype), q, s, torch.float32).cpu().numpy(), want)
    y = si.linear_mxfp4_a4(*si.quantize_rows_mxfp4(x.half()), q, s, torch.float32)
    assert np.array_equal(y.cpu().numpy(), want)


@pytest.mark.parametrize("b", [1, 6])
def test_sparse_past_32_bits(b):
    k, d = 1050000, 8192  # 4.3 GB of codes a matrix
    g = torch.Generator(device=DEV).manual_seed(b)
    mats = []
    for _ in range(3):
        q = torch.empty(k, d // 2, dtype=torch.uint8, device=DEV)
        for i in range(0, k, 150000):
            q[i:i + 150000] = torch.randint(0, 256, (150000, d // 2), generator=g, dtype=torch.uint8, device=DEV)
        mats += [q, torch.full((k, d // 32), 120, dtype=torch.uint8, device=DEV)]
    x = torch.randn(b, d, generator=g, device=DEV).half()
    pick = [0, 31, 32, 524287, 524288, 1048575, 1048576, 1049998, 1049999]
    mask = torch.zeros(k, dtype=torch.uint8, device=DEV)
    mask[pick] = 1
    y, cnt = si.sparse_mlp_mxfp4(*mats, x, si.new_workspace_mxfp4(k, d, b), mask, counters=True)
    wg, wu, wd = (ref.values(ref.unpack(mats[i][pick].cpu().numpy()), mats[i + 1][pick].cpu().numpy(), d)
                  for i in (0, 2, 4))
    want, h3, _, _ = ref.mlp(wg, wu, wd, f64(x), np.ones(len(pick)))
    assert cnt[0].item() == len(pick) and np.abs(want).max() > 0
    # g and u each within (d + 66) 2^-24 of their absolute sums, here about 4e-3 of an h3's typical size at most
    size = (np.abs(f64(x)) @ np.abs(wg).T) * (np.abs(f64(x)) @ np.abs(wu).T)
    tol = 3 * (d + 66) * 2.0 ** -24 * size @ np.abs(wd)
    assert (np.abs(f64(y) - want) <= tol).all()
    assert np.linalg.norm(f64(y) - want) <= 1e-5 * np.linalg.norm(want)


def test_norm_past_32_bits():
    rows, ld, d = 4100, 1 << 20, 300  # 8.6 GB from the first row to the last
    buf = torch.zeros(rows, ld, dtype=torch.float16, device=DEV)
    h = buf[:, 5:5 + d]
    small = torch.randn(rows, d, generator=torch.Generator().manual_seed(1)).half().to(DEV)
    h.copy_(small)
    branch = small.flip(0).contiguous()
    w = torch.rand(d, device=DEV)
    want, x_want = si.norm_residual(small, branch, post_w=w, pre_w=w)
    out, x = si.norm_residual(h, branch, post_w=w, pre_w=w, out=h)
    assert out is h and torch.equal(h, want) and torch.equal(x, x_want)
    assert not buf[:, :5].any() and not buf[:, 5 + d:5 + d + 64].any()


def test_int16_patterns():
    """fp16 values given as int16 bit patterns, as the other calls take them."""
    g = torch.Generator(device=DEV).manual_seed(1)
    w, x = torch.randn(40, 256, generator=g, device=DEV).half(), torch.randn(3, 256, generator=g, device=DEV).half()
    q, s = si.quantize_rows_mxfp4(w)
    q2, s2 = si.quantize_rows_mxfp4(w.view(torch.int16))
    assert torch.equal(q, q2) and torch.equal(s, s2)
    y = si.linear_mxfp4(x, q, s)
    assert torch.equal(si.linear_mxfp4(x.view(torch.int16), q, s).view(torch.float16), y)
    assert torch.equal(si.dequantize_rows_mxfp4(q, s, 256, torch.int16).view(torch.float16),
                       si.dequantize_rows_mxfp4(q, s, 256))


@pytest.mark.parametrize("m", [1, 12, 300])
def test_products_captured(m):
    """Quantization and every product in one graph (among them one whose n is
    split), replayed with new activations and eager work between the replays."""
    g = torch.Generator(device=DEV).manual_seed(m)
    n, rows = 8192, 130
    q, s = si.quantize_rows_mxfp4(torch.randn(rows, n, generator=g, device=DEV))
    qu, su = si.quantize_rows_mxfp4(torch.randn(rows, n, generator=g, device=DEV))
    x = torch.randn(m, n, generator=g, device=DEV).half()

    def run(x):
        xq, xs = si.quantize_rows_mxfp4(x)
        return [si.linear_mxfp4(x, q, s), si.gated_linear_mxfp4(x, q, s, qu, su), si.linear_mxfp4_a4(xq, xs, q, s),
                si.gated_linear_mxfp4_a4(xq, xs, q, s, qu, su, torch.float32), si.linear_mxfp4(x[:, 1:4002], *short),
                si.dequantize_rows_mxfp4(xq, xs, n)]

    short = si.quantize_rows_mxfp4(torch.randn(rows, 4001, generator=g, device=DEV))
    run(x)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run(x)
    for i in range(3):
        x.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        seen = [t.clone() for t in got]
        for a, b in zip(seen, run(x)):
            assert torch.equal(a, b)
