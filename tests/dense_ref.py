"""Plain float64 forms of the dense products, the norms and FP8, for the tests, and
the sizes at which the products' tests run."""

import torch

F16, BF16, F32 = torch.float16, torch.bfloat16, torch.float32
HALF_STEP = {F16: 2.0 ** -11, BF16: 2.0 ** -8, F32: 2.0 ** -24}   # of a rounding, relative
SMALLEST = {F16: 2.0 ** -25, BF16: 2.0 ** -134, F32: 2.0 ** -150}  # half the smallest step

# (m, rows, n) by the kernel that each kind of product takes there (si_dense_tile)
TILES = {
    ("linear", False): {100: [(1, 65, 72), (4, 130, 520)], 0: [(7, 64, 64), (16, 100, 1000)], 1: [(2050, 72, 64)],
                        2: [(33, 8200, 72)], 3: [(100, 8200, 64)], 4: [(100, 8200, 520)], 5: [(2050, 4100, 328)]},
    ("linear", True): {100: [(1, 65, 72), (3, 130, 520)], 0: [(7, 64, 64), (16, 100, 1000)], 1: [(20, 4100, 64)],
                       2: [(33, 4100, 72)], 3: [(7, 8200, 64)], 4: [(33, 8200, 520)], 5: [(2050, 2056, 328)]},
    ("transposed", False): {0: [(1, 64, 64), (16, 100, 1000)], 1: [(2050, 72, 64)], 2: [(33, 8200, 72)],
                            3: [(100, 8200, 64)], 4: [(100, 8200, 520)], 5: [(2050, 4100, 328)]},
    ("dx", False): {0: [(1, 64, 64), (16, 1000, 100)], 1: [(2050, 64, 72)], 2: [(4100, 64, 72)],
                    3: [(4100, 64, 200)], 4: [(4100, 520, 200)], 5: [(2050, 328, 4100)]},
    ("dx", True): {0: [(1, 64, 64), (16, 1000, 100)], 1: [(2050, 64, 72)], 2: [(4100, 64, 72)],
                   3: [(4100, 64, 200)], 4: [(4100, 328, 200)], 5: [(2050, 136, 4100)]},
    ("dx transposed", False): {100: [(1, 64, 64), (4, 200, 130)], 0: [(7, 64, 64)], 1: [(2050, 64, 72)], 2: [(4100, 64, 72)],
                               3: [(4100, 64, 200)], 4: [(4100, 520, 200)], 5: [(2050, 328, 4100)]},
    ("dw", False): {2: [(1, 64, 64), (1000, 100, 72)], 3: [(1, 8200, 72)], 4: [(520, 8200, 72)], 5: [(257, 2056, 4100)]},
    ("dw", True): {2: [(1, 64, 64), (1000, 100, 72)], 3: [(3, 72, 4100)], 4: [(520, 72, 4100)], 5: [(257, 2056, 2056)]},
    ("dw transposed", False): {2: [(1, 64, 64), (1000, 100, 72)], 3: [(1, 8200, 72)], 4: [(520, 8200, 72)],
                               5: [(257, 2056, 4100)]},
    ("fp8", False): {100: [(1, 65, 72), (4, 130, 1040)], 0: [(7, 64, 64), (16, 100, 1000)], 1: [(2050, 72, 64)],
                     2: [(33, 8200, 64)], 3: [(100, 8200, 64)], 4: [(100, 8200, 1032)], 5: [(2050, 4100, 520)]},
    ("fp8", True): {100: [(1, 65, 72), (3, 130, 1040)], 0: [(7, 64, 64), (16, 100, 1000)], 1: [(20, 4100, 64)],
                    2: [(33, 4100, 72)], 3: [(7, 8200, 64)], 4: [(33, 8200, 1032)], 5: [(2050, 2056, 520)]},
}
KIND = {"linear": 0, "transposed": 1, "dx": 2, "dx transposed": 3, "dw": 4, "dw transposed": 5, "fp8": 6}


def shapes(kind, gated=False):
    return [s for tile in TILES[kind, gated].values() for s in tile]


def whole(g, lo, hi, *shape):
    """Whole numbers lo .. hi."""
    return torch.randint(lo, hi + 1, shape, generator=g)


def gated(g, u):
    """relu(g) * u as the kernels form it: one float32 product."""
    h = torch.relu(g.to(F32))
    return h if u is None else h * u.to(F32)


# ---- norms ------------------------------------------------------------------------

def norm(x, w, b, eps, center):
    c = x - x.mean(dim=1, keepdim=True) if center else x
    r = 1.0 / torch.sqrt((c * c).mean(dim=1, keepdim=True) + eps)
    y = c * r * w
    return y if b is None else y + b


def norm_grad(x, w, dy, eps, center):
    """(dx, dw, db) and the sums of magnitudes that bound their rounding."""
    c = x - x.mean(dim=1, keepdim=True) if center else x
    r = 1.0 / torch.sqrt((c * c).mean(dim=1, keepdim=True) + eps)
    n, e = c * r, dy * w
    me = e.mean(dim=1, keepdim=True) if center else 0.0
    dx = r * (e - me - n * (e * n).mean(dim=1, keepdim=True))
    size = r * (e.abs() + e.abs().mean(dim=1, keepdim=True) + n.abs() * (e * n).abs().mean(dim=1, keepdim=True))
    return dx, (dy * n).sum(dim=0), dy.sum(dim=0), size, (dy * n).abs().sum(dim=0), dy.abs().sum(dim=0)


# ---- e4m3 -----------------------------------------------------------------------------

def e4m3_values():
    """Magnitudes of codes 0 .. 126."""
    code = torch.arange(127, dtype=torch.float64)
    e, f = torch.floor(code / 8), code % 8
    return torch.where(e == 0, f * 2.0 ** -9, (8 + f) * torch.exp2(e - 10))


def e4m3_code(v):
    """The code (with its sign bit) of the e4m3 value nearest to float32 v, ties to even."""
    table = e4m3_values()
    a = v.double().abs().clamp(max=448.0)
    i = torch.bucketize(a, table).clamp(max=126)       # first value >= a
    lo = (i - 1).clamp(min=0)
    below, above = a - table[lo], table[i] - a
    take = torch.where(below < above, lo, i)
    take = torch.where((below == above) & (lo % 2 == 0), lo, take)
    return take + 128 * torch.signbit(v).long()


def quantize(v, rows_per_scale):
    """(codes [rows][n rounded up to 16], scales) of float32 v on the CPU."""
    rows, n = v.shape
    p = torch.nn.functional.pad(v, (0, -n % 128, 0, -rows % rows_per_scale))
    b = p.view(p.shape[0] // rows_per_scale, rows_per_scale, p.shape[1] // 128, 128)
    top = torch.where(b.isnan(), torch.inf, b.abs()).amax(dim=(1, 3), keepdim=True)
    scale = torch.where(torch.isinf(top), torch.nan, top * (torch.ones(()) / 448))
    ok = scale > 0
    q = torch.where(ok, e4m3_code(torch.where(ok, b / scale, torch.zeros(()))), 0)
    codes = q.reshape(p.shape)[:rows, : (n + 15) // 16 * 16]
    return codes.to(torch.uint8), scale[:, 0, :, 0].contiguous()


def values(codes, scale, n, rows_per_scale):
    """float64 values of stored rows."""
    table = torch.cat([e4m3_values(), torch.full((1,), torch.nan, dtype=torch.float64)])
    c = codes[:, :n].long()
    v = table[c & 127] * torch.where(c > 127, -1.0, 1.0)
    s = scale.double().repeat_interleave(rows_per_scale, dim=0)[: codes.shape[0]].repeat_interleave(128, dim=1)[:, :n]
    return v * s
