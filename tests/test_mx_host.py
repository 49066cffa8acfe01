"""Host-side checks of the MXFP4 operators and ``norm_residual`` (no GPU, nothing
is launched): the tests' own reference against worked examples, sizes, and every
refusal."""

import ctypes
import math

import numpy as np
import pytest
import torch

import mx_ref as ref
import paper_2411_12692_amd as si
from paper_2411_12692_amd import _lib

A = 1 << 40  # a fake 16-byte-aligned address: validation fails before it is used
B, C, D, E, F, G, H = (A + (i << 34) for i in range(1, 8))  # far apart: no overlap
F16, BF16, F32 = _lib.SI_F16, _lib.SI_BF16, _lib.SI_F32


@pytest.fixture(scope="module", autouse=True)
def lib():
    import os
    if not os.path.exists(_lib.LIB_PATH):
        from paper_2411_12692_amd import build
        build.build()
    return _lib.load()


# ---- the reference ---------------------------------------------------------------

def test_reference_worked_example():
    """max 5.5: X = floor(log2 5.5) - 2 = 0, so the codes are the values rounded to
    e2m1; max 0.3 in the second block: X = -2 - 2 = -4, scale 1/16."""
    row = np.zeros(64)
    row[:10] = [5.5, -0.25, 0.26, -0.75, 1.25, 2.5, -3.5, 5.0, 0.0, -0.0]
    row[32:36] = [0.3, 0.0625, -0.03125, 0.04]
    codes, scale = ref.quantize(row[None])
    assert scale.tolist() == [[127, 123, 0, 0]]
    # 5.5 -> 6 (7), -0.25 -> -0 (8), 0.26 -> 0.5 (1), -0.75 -> -1 (10), 1.25 -> 1 (2), 2.5 -> 2 (4),
    # -3.5 -> -4 (14), 5 -> 4 (6), 0 -> 0, -0 -> 8
    assert codes[0, :10].tolist() == [7, 8, 1, 10, 2, 4, 14, 6, 0, 8]
    # 4.8 -> 4 (6), 1 (2), -0.5 (9), 0.64 -> 0.5 (1)
    assert codes[0, 32:36].tolist() == [6, 2, 9, 1]
    assert ref.values(codes, scale, 64)[0, 32:36].tolist() == [0.25, 0.0625, -0.03125, 0.03125]
    packed = ref.pack(codes)
    assert packed[0, 0] == 7 | 8 << 4 and np.array_equal(ref.unpack(packed), codes)
    assert ref.pack_signs(codes)[0].tolist() == [1 << 1 | 1 << 3 | 1 << 6 | 1 << 9, 1 << 2, 0, 0]


def test_reference_rounds_to_the_nearest():
    """Every code is at least as near as its neighbours, and 6 takes what lies
    above (up to 8)."""
    rng = np.random.default_rng(0)
    w = rng.standard_normal((50, 96)) * np.exp2(rng.integers(-20, 20, (50, 1)))
    codes, scale = ref.quantize(w)
    v = ref.values(codes, scale, 96)
    unit = np.exp2(np.repeat(scale.astype(float) - 127, 32, axis=1)[:, :96])
    err = np.abs(v - w) / unit
    a = np.abs(w) / unit
    assert (a < 8).all() and (a.reshape(50, 3, 32).max(axis=2) >= 4).all()
    assert (err <= np.where(a < 2, 0.25, np.where(a < 4, 0.5, np.where(a < 6, 1.0, a - 6 + 1e-12)))).all()


def test_reference_special_blocks():
    w = np.zeros((1, 128))
    w[0, 0], w[0, 1], w[0, 33], w[0, 70] = np.inf, -1.0, np.nan, 2.0 ** -149
    codes, scale = ref.quantize(w)
    assert scale.tolist() == [[255, 255, 0, 0]]
    assert codes[0, 1] == 8 and codes[0, 70] == 0
    assert np.isnan(ref.values(codes, scale, 128)[0, :64]).all()
    big = np.full((1, 32), float(np.finfo(np.float32).max))
    codes, scale = ref.quantize(big)
    assert scale[0, 0] == 127 + 125 and (codes[0, :32] == 7).all()


def test_reference_norm():
    h, _ = ref.norm_residual(np.array([[1.0, 2.0]]), np.array([[3.0, 4.0]]), None, None, 2.0, None, 0.0)
    assert h.tolist() == [[7.0, 10.0]]
    _, x = ref.norm_residual(np.array([[3.0, 4.0]]), None, None, None, 1.0, np.array([1.0, 2.0]), 0.0)
    assert np.allclose(x, np.array([[3.0, 8.0]]) / math.sqrt(12.5))
    h, _ = ref.norm_residual(np.zeros((2, 2)), np.array([[3.0, 4.0]] * 2), np.array([1.0, 1.0]),
                             np.array([[1.0, 0.0], [0.0, 1.0]]), 1.0, None, 0.0)
    assert np.allclose(h, np.array([[3.0, 0.0], [0.0, 4.0]]) / math.sqrt(12.5))


# ---- sizes -------------------------------------------------------------------------

@pytest.mark.parametrize("rows,n,codes,scales", [(1, 1, 64, 4), (3, 128, 192, 12), (3, 129, 384, 24),
                                                 (11008, 4096, 11008 * 2048, 11008 * 128), (0, 5, 0, 0),
                                                 (1 << 24, 1 << 24, 1 << 47, 1 << 43), (-1, 5, 0, 0), (5, 0, 0, 0),
                                                 (1, (1 << 24) + 1, 0, 0)])
def test_mxfp4_bytes(lib, rows, n, codes, scales):
    assert lib.si_mxfp4_codes_bytes(rows, n) == codes and lib.si_mxfp4_scales_bytes(rows, n) == scales


def test_workspace_sizes(lib):
    for k, d, b in ((11008, 4096, 1), (1, 128, 8), (1 << 24, 8192, 8)):
        assert lib.si_mxfp4_workspace_bytes(k, d, b) >= lib.si_workspace_bytes(k, d, b) > 0
    for k, d, b in ((0, 128, 1), (5, 100, 1), (5, 128, 9), (5, 128, 0)):
        assert lib.si_mxfp4_workspace_bytes(k, d, b) == 0
    f = lib.si_linear_mxfp4_workspace_bytes
    assert f(A, 128, 1, 64, 128, 0) == 0                 # one token, aligned: nothing
    assert f(A, 100, 1, 64, 100, 0) >= 128 * 2           # rows that end inside 128 values are copied
    assert f(A + 2, 128, 1, 64, 128, 0) >= 128 * 2       # so are unaligned ones
    assert f(A, 129, 3, 64, 128, 0) >= 3 * 128 * 2
    assert f(None, 0, 1, 64, 100, 0) == 0                # MXFP4 activations never are
    assert f(A, 128, 0, 64, 128, 0) == 0 and f(A, 128, 1, 64, (1 << 20) + 1, 0) == 0


# ---- refusals of the C ABI -----------------------------------------------------------

def refused(name, args, want):
    st = _lib.status(name, *(ctypes.c_void_p(a) if isinstance(a, int) and a >= A else a for a in args))
    assert st == want, (name, args, st, _lib.last_error())
    assert _lib.last_error() != ""


def test_quantize_refusals():
    ok = [A, F16, 64, 4, 64, B, C, None]

    def bad(want, **kw):
        args = list(ok)
        for i, v in kw.items():
            args[int(i[1:])] = v
        refused("si_quantize_rows_mxfp4", args, want)

    bad(_lib.SI_ERR_NULL, _0=None)
    bad(_lib.SI_ERR_NULL, _5=None)
    bad(_lib.SI_ERR_NULL, _6=None)
    bad(_lib.SI_ERR_ARG, _1=3)
    bad(_lib.SI_ERR_ARG, _1=-1)
    bad(_lib.SI_ERR_SHAPE, _2=63)
    bad(_lib.SI_ERR_SHAPE, _3=-1)
    bad(_lib.SI_ERR_SHAPE, _3=(1 << 24) + 1)
    bad(_lib.SI_ERR_SHAPE, _4=0)
    bad(_lib.SI_ERR_ALIGN, _0=A + 1)
    bad(_lib.SI_ERR_ALIGN, _0=A + 2, _1=F32)
    bad(_lib.SI_ERR_ALIGN, _5=B + 8)
    bad(_lib.SI_ERR_ALIGN, _6=C + 4)
    bad(_lib.SI_ERR_ARG, _5=A + 64)
    bad(_lib.SI_ERR_ARG, _6=A + 16)
    bad(_lib.SI_ERR_ARG, _6=B + 16)
    bad(_lib.SI_ERR_SHAPE, _2=1 << 20, _3=1 << 24, _4=1 << 20)  # more threads than a launch holds
    assert _lib.status("si_quantize_rows_mxfp4", None, F16, 64, 0, 64, None, None, None) == _lib.SI_OK


def test_dequantize_and_signs_refusals():
    for args, want in (((None, B, 4, 64, C, F16, None), _lib.SI_ERR_NULL),
                       ((A, None, 4, 64, C, F16, None), _lib.SI_ERR_NULL),
                       ((A, B, 4, 64, None, F16, None), _lib.SI_ERR_NULL),
                       ((A, B, 4, 64, C, 7, None), _lib.SI_ERR_ARG),
                       ((A, B, 4, 0, C, F16, None), _lib.SI_ERR_SHAPE),
                       ((A, B, -4, 64, C, F16, None), _lib.SI_ERR_SHAPE),
                       ((A + 4, B, 4, 64, C, F16, None), _lib.SI_ERR_ALIGN),
                       ((A, B, 4, 64, C + 1, F16, None), _lib.SI_ERR_ALIGN),
                       ((A, B, 4, 64, C + 2, F32, None), _lib.SI_ERR_ALIGN),
                       ((A, B, 4, 64, A + 64, F16, None), _lib.SI_ERR_ARG),
                       ((A, B, 4, 64, B - 16, F32, None), _lib.SI_ERR_ARG)):
        refused("si_dequantize_rows_mxfp4", args, want)
    for args, want in (((None, 128, 256, B, None), _lib.SI_ERR_NULL), ((A, 128, 200, B, None), _lib.SI_ERR_SHAPE),
                       ((A, 0, 256, B, None), _lib.SI_ERR_SHAPE), ((A + 8, 128, 256, B, None), _lib.SI_ERR_ALIGN)):
        refused("si_pack_signs_mxfp4", args, want)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("a4", [False, True])
def test_product_refusals(gated, a4):
    x = [A, B] if a4 else [A, F16, 256]
    w = [C, D, E, F] if gated else [C, D]
    ok = x + [2, 256] + w + [64, G, F32, H, 1 << 20, None]
    name = "si_" + ("gated_" if gated else "") + "linear_mxfp4" + ("_a4" if a4 else "")
    m, n, q, rows = len(x), len(x) + 1, len(x) + 2, len(x) + 2 + len(w)
    y, yt, ws = rows + 1, rows + 2, rows + 3

    def bad(want, **kw):
        args = list(ok)
        for i, v in kw.items():
            args[int(i[1:])] = v
        refused(name, args, want)

    for i in [0, q, q + 1, y] + ([1] if a4 else []):
        bad(_lib.SI_ERR_NULL, **{f"_{i}": None})
    bad(_lib.SI_ERR_SHAPE, **{f"_{m}": -1})
    bad(_lib.SI_ERR_SHAPE, **{f"_{n}": 0})
    bad(_lib.SI_ERR_SHAPE, **{f"_{n}": (1 << 20) + 1})
    bad(_lib.SI_ERR_SHAPE, **{f"_{rows}": 0})
    bad(_lib.SI_ERR_SHAPE, **{f"_{m}": 1 << 24, f"_{rows}": 1 << 24})
    bad(_lib.SI_ERR_ARG, **{f"_{yt}": 5})
    for i in [q, q + 1, y] + ([0, 1] if a4 else []):
        bad(_lib.SI_ERR_ALIGN, **{f"_{i}": ok[i] + 8})
    for i in [0, q, q + 1]:
        bad(_lib.SI_ERR_ARG, **{f"_{y}": ok[i]})  # y over an input
    if gated:
        bad(_lib.SI_ERR_NULL, **{f"_{q + 3}": None})
        bad(_lib.SI_ERR_NULL, **{f"_{q + 2}": None})
        bad(_lib.SI_ERR_ARG, **{f"_{y}": E})
    if not a4:
        bad(_lib.SI_ERR_ARG, _1=F32)
        bad(_lib.SI_ERR_ALIGN, _0=A + 1)
        bad(_lib.SI_ERR_SHAPE, _2=255)
        bad(_lib.SI_ERR_SHAPE, _2=1 << 22)
        bad(_lib.SI_ERR_NULL, **{f"_{n}": 200, f"_{ws}": None})  # the padded copy needs a workspace
        bad(_lib.SI_ERR_WORKSPACE, **{f"_{n}": 200, f"_{ws + 1}": 16})
        bad(_lib.SI_ERR_ALIGN, **{f"_{n}": 200, f"_{ws}": H + 8})
    none = list(ok)
    none[m] = 0
    none[0] = none[y] = None
    assert _lib.status(name, *(ctypes.c_void_p(a) if isinstance(a, int) and a >= A else a for a in none)) == _lib.SI_OK


@pytest.mark.parametrize("predict", [False, True])
def test_sparse_refusals(lib, predict):
    k, d, b = 128, 256, 2
    need = lib.si_mxfp4_workspace_bytes(k, d, b)
    w = [A, B, C, D, E, F]
    if predict:
        name = "si_predict_sparse_mlp_mxfp4"
        ok = [G] + w + [k, d, H, b, 1.0, None, None, None, A + (9 << 34), A + (10 << 34), need, 0, None, None]
        at = dict(w=1, k=7, d=8, x=9, b=10, y=15, ws=16, n=17, flags=18, cnt=19, sel=0)
    else:
        name = "si_sparse_mlp_mxfp4"
        ok = w + [k, d, H, b, G, A + (9 << 34), A + (10 << 34), need, 0, None, None]
        at = dict(w=0, k=6, d=7, x=8, b=9, sel=10, y=11, ws=12, n=13, flags=14, cnt=15)

    def bad(want, **kw):
        args = list(ok)
        for key, v in kw.items():
            args[at[key] if key in at else int(key[1:])] = v
        refused(name, args, want)

    for key in ("sel", "x", "y", "ws"):
        bad(_lib.SI_ERR_NULL, **{key: None})
    for i in range(6):
        bad(_lib.SI_ERR_NULL, **{f"_{at['w'] + i}": None})
        bad(_lib.SI_ERR_ALIGN, **{f"_{at['w'] + i}": ok[at["w"] + i] + 8})
    for key in ("sel", "x", "y", "ws", "cnt"):
        bad(_lib.SI_ERR_ALIGN, **{key: H + 4})
    bad(_lib.SI_ERR_SHAPE, k=0)
    bad(_lib.SI_ERR_SHAPE, d=200)
    bad(_lib.SI_ERR_SHAPE, d=8320)
    bad(_lib.SI_ERR_SHAPE, b=9)
    bad(_lib.SI_ERR_SHAPE, b=0)
    bad(_lib.SI_ERR_FLAGS, flags=4)
    bad(_lib.SI_ERR_WORKSPACE, n=need - 1)
    bad(_lib.SI_ERR_ARG, y=H)
    if predict:
        bad(_lib.SI_ERR_ALPHA, _11=math.nan)
        bad(_lib.SI_ERR_ALPHA, _11=-1.0)


def test_norm_refusals():
    # h, type, ldh, branch, type, ldb, post_w, gate, rows_per_gate, scale, h_out, ldo, pre_w, x, type, ldx, tokens, d, eps
    ok = [A, F32, 64, B, F16, 64, C, D, 1, 1.0, E, 64, F, G, F16, 64, 4, 64, 1e-5, None]

    def bad(want, **kw):
        args = list(ok)
        for i, v in kw.items():
            args[int(i[1:])] = v
        refused("si_norm_residual", args, want)

    bad(_lib.SI_ERR_NULL, _0=None)
    bad(_lib.SI_ERR_NULL, _3=None)                          # post_w, gate, h_out without a branch
    bad(_lib.SI_ERR_NULL, _12=None)
    bad(_lib.SI_ERR_NULL, _13=None)
    bad(_lib.SI_ERR_NULL, _10=None, _12=None, _13=None)     # nothing to write
    for i in (1, 4, 14):
        bad(_lib.SI_ERR_ARG, **{f"_{i}": 4})
    for i in (2, 5, 11, 15):
        bad(_lib.SI_ERR_SHAPE, **{f"_{i}": 63})
    bad(_lib.SI_ERR_SHAPE, _16=-1)
    bad(_lib.SI_ERR_SHAPE, _16=1 << 23)
    bad(_lib.SI_ERR_SHAPE, _17=0)
    bad(_lib.SI_ERR_SHAPE, _17=16385, _2=16385, _5=16385, _11=16385, _15=16385)
    bad(_lib.SI_ERR_SHAPE, _8=0)
    for v in (math.nan, math.inf, -1e-6):
        bad(_lib.SI_ERR_ARG, _18=v)
    for v in (math.nan, math.inf):
        bad(_lib.SI_ERR_ARG, _9=v)
    for i, off in ((0, 2), (3, 1), (6, 2), (7, 2), (10, 2), (12, 2), (13, 1)):
        bad(_lib.SI_ERR_ALIGN, **{f"_{i}": ok[i] + off})
    bad(_lib.SI_ERR_ARG, _10=A + 4)                         # h_out one value behind h
    bad(_lib.SI_ERR_ARG, _10=A, _11=65)                     # h itself at another stride
    bad(_lib.SI_ERR_ARG, _10=B)
    bad(_lib.SI_ERR_ARG, _13=A)
    bad(_lib.SI_ERR_ARG, _13=B)
    bad(_lib.SI_ERR_ARG, _13=E)
    bad(_lib.SI_ERR_ARG, _13=C)
    bad(_lib.SI_ERR_ARG, _10=D)
    # columns that cross into h's, before and behind
    bad(_lib.SI_ERR_ARG, _2=128, _11=128, _10=A + 4 * 63)
    bad(_lib.SI_ERR_ARG, _2=128, _11=128, _10=A + 4 * 65)
    args = list(ok)
    args[16] = 0
    assert _lib.status("si_norm_residual", *(ctypes.c_void_p(a) if isinstance(a, int) and a >= A else a
                                             for a in args)) == _lib.SI_OK


# ---- refusals of the Python calls --------------------------------------------------

def test_python_calls_refuse_host_tensors():
    f = torch.zeros(4, 256)
    u, s = torch.zeros(4, 128, dtype=torch.uint8), torch.zeros(4, 8, dtype=torch.uint8)
    for call in (lambda: si.quantize_rows_mxfp4(f), lambda: si.dequantize_rows_mxfp4(u, s, 256),
                 lambda: si.pack_signs_mxfp4(u), lambda: si.linear_mxfp4(f.half(), u, s),
                 lambda: si.gated_linear_mxfp4(f.half(), u, s, u, s), lambda: si.linear_mxfp4_a4(u, s, u, s),
                 lambda: si.norm_residual(f, pre_w=torch.ones(256)),
                 lambda: si.predict_sparse_mlp_mxfp4(torch.zeros(1, dtype=torch.int32), u, s, u, s, u, s, f.half(), 1.0,
                                                     torch.zeros(1, dtype=torch.uint8))):
        with pytest.raises(ValueError, match="CUDA tensor"):
            call()
    with pytest.raises(TypeError):
        si.norm_residual(None)
    with pytest.raises(ValueError, match="unsupported shape"):
        si.new_workspace_mxfp4(5, 100)
