"""MXFP4 and the norms around a block in NumPy float64, written from their
definitions (no code of the package): the reference of the tests."""

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def padded(n: int) -> int:
    return -(-n // 128) * 128


def quantize(w: np.ndarray):
    """float64 rows -> (codes uint8 [rows][np], scale bytes uint8 [rows][np / 32])."""
    rows, n = w.shape
    v = np.zeros((rows, padded(n)))
    v[:, :n] = w
    b = v.reshape(rows, -1, 32)
    finite = np.isfinite(b).all(axis=2)
    top = np.where(finite, np.abs(np.where(np.isfinite(b), b, 0.0)).max(axis=2), 1.0)
    _, e = np.frexp(top)  # top = f 2^e, f in [0.5, 1)
    x = np.maximum(np.where(top > 0, e - 3, -127), -127)
    a = np.ldexp(np.abs(np.where(finite[:, :, None], b, 0.0)), -x[:, :, None])
    dist = np.abs(a[..., None] - LEVELS)
    best = dist.min(axis=-1, keepdims=True)
    # of two levels equally near, the even code
    even = np.arange(8) % 2 == 0
    code = np.where((dist == best) & even, 1, np.where(dist == best, 0, -1)).argmax(axis=-1)
    code = np.where(a >= 6, 7, code)
    code = code + 8 * np.signbit(b)
    scale = np.where(finite, x + 127, 255)
    return code.reshape(rows, -1).astype(np.uint8), scale.astype(np.uint8)


def pack(codes: np.ndarray) -> np.ndarray:
    return (codes[:, 0::2] | (codes[:, 1::2] << 4)).astype(np.uint8)


def unpack(q: np.ndarray) -> np.ndarray:
    out = np.empty((q.shape[0], 2 * q.shape[1]), dtype=np.uint8)
    out[:, 0::2] = q & 15
    out[:, 1::2] = q >> 4
    return out


def values(codes: np.ndarray, scale: np.ndarray, n: int) -> np.ndarray:
    """float64 values of unpacked codes."""
    v = np.where(codes & 8, -1.0, 1.0) * LEVELS[codes & 7]
    s = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127.0))
    with np.errstate(invalid="ignore"):
        return (v * np.repeat(s, 32, axis=1))[:, :n]


def pack_signs(codes: np.ndarray) -> np.ndarray:
    """[k][d / 32] words, bit j of word w the sign of element 32 w + j."""
    bits = (codes >> 3).reshape(codes.shape[0], -1, 32).astype(np.uint64)
    return (bits << np.arange(32, dtype=np.uint64)).sum(axis=2).astype(np.uint32)


def mlp(wg, wu, wd_t, x, mask):
    """Eq. (1) over the rows of ``mask``: ``wd_t`` is W_down^T [k][d].  Returns
    (y, h3, g, u)."""
    g = x @ wg.T
    u = x @ wu.T if wu is not None else np.ones_like(g)
    h3 = np.where(mask[None, :] != 0, np.maximum(g, 0) * u, 0.0)
    return h3 @ wd_t, h3, g, u


def norm_residual(h, branch, post_w, gate, scale, pre_w, eps):
    def rms(v):
        return v / np.sqrt((v * v).mean(axis=1, keepdims=True) + eps)

    if branch is not None:
        p = branch if post_w is None else rms(branch) * post_w
        if gate is not None:
            p = p * np.repeat(gate, h.shape[0] // gate.shape[0], axis=0)
        h = h + scale * p
    return h, (rms(h) * pre_w if pre_w is not None else None)
