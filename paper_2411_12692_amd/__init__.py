"""MI355X-native SparseInfer decode path (arXiv 2411.12692).

Thin PyTorch-facing binding of ``libsparseinfer.so`` (see
``include/sparseinfer.h``).  PyTorch only provides device memory and the
current stream; every step of the path runs in the library's HIP kernels.
The functions take contiguous CUDA tensors: fp16 weights/inputs (``float16``
or ``int16`` bit patterns), and return new tensors.  The MXFP4, FP8 and dense
products and the norms also take bf16 and float32 and rows with a stride, and run
on the device of their tensors.  ``linear``, ``gated_linear``, ``mlp``,
``layer_norm`` and ``rms_norm`` have gradients.
"""

from __future__ import annotations

import functools

import torch
import torch.autograd.forward_ad as _forward_ad

from . import _lib
from ._lib import SI_NO_AS, SI_NO_SPECULATION, SparseInferError

__all__ = [
    "SI_NO_AS", "SI_NO_SPECULATION", "SparseInferError", "signs_bytes", "alpha_threshold", "workspace_bytes",
    "new_workspace", "workspace_check", "read_h3", "pack_signs", "signs_to_canonical", "transpose_down", "predict",
    "sparse_mlp", "predict_sparse_mlp", "mlp_block", "MLPLayer",
    "quantize_rows_i8", "pack_signs_i8", "transpose_down_i8", "sparse_mlp_i8", "predict_sparse_mlp_i8",
    "Int8MLPLayer",
    "quantize_rows_mxfp4", "dequantize_rows_mxfp4", "pack_signs_mxfp4", "linear_mxfp4", "gated_linear_mxfp4",
    "linear_mxfp4_a4", "gated_linear_mxfp4_a4", "mxfp4_workspace_bytes", "new_workspace_mxfp4", "sparse_mlp_mxfp4",
    "predict_sparse_mlp_mxfp4", "MXFP4MLPLayer", "norm_residual",
    "linear", "gated_linear", "mlp", "layer_norm", "rms_norm", "quantize_rows_fp8", "quantize_blocks_fp8",
    "dequantize_fp8", "linear_fp8", "gated_linear_fp8", "FP8MLPLayer",
]


def _vp(t):
    """Device pointer of a tensor as an argument of the library (an int: ctypes
    converts it to ``void *`` itself, without an object of its own)."""
    return None if t is None else t.data_ptr()


# The current stream's handle without a torch.cuda.Stream object (which takes
# about 3 us to make, a third of a call made from Python).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _dev(t: torch.Tensor, name: str, dtypes, ndim=None):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor (got {t.device})")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {dtypes}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if ndim is not None and t.dim() != ndim:
        raise ValueError(f"{name} must have {ndim} dims, got {tuple(t.shape)}")
    return t


_F16 = (torch.float16, torch.int16)


def signs_bytes(k: int, d: int) -> int:
    return int(_lib.load().si_signs_bytes(k, d))


def alpha_threshold(alpha: float, d: int) -> int:
    """Integer form of Eq. (2): rows are kept iff N_neg < T (host only)."""
    return int(_lib.load().si_alpha_threshold(alpha, d))


def workspace_bytes(k: int, d: int, b: int = 1) -> int:
    return int(_lib.load().si_workspace_bytes(k, d, b))


def new_workspace(k: int, d: int, b: int = 1, device=None) -> torch.Tensor:
    """Zero-filled workspace for calls with up to ``b`` tokens."""
    n = workspace_bytes(k, d, b)
    if n == 0:
        raise ValueError(f"unsupported shape k={k} d={d} b={b}")
    return torch.zeros(n, dtype=torch.uint8, device=device or "cuda")


def workspace_check(workspace: torch.Tensor, stream=None) -> int:
    """``si_workspace_check``: waits for the stream, returns the status of the
    workspace's sticky device error word (``SI_OK``, ``SI_ERR_TIMEOUT`` or
    ``SI_ERR_LIST``) and resets the workspace when it is not ``SI_OK``."""
    st = stream if stream is not None else _stream()
    return int(_lib.status("si_workspace_check", _vp(workspace), workspace.numel(), st))


def read_h3(workspace: torch.Tensor, k: int, d: int, b: int, mask: torch.Tensor) -> torch.Tensor:
    """``si_read_h3``: the per-row h3 (Eq. (1) step 3) of the last MLP call
    made with ``workspace``, ``[k][b]`` float32 (0 off ``mask``, NaN for a
    kept row the call left no value for)."""
    _dev(mask, "mask", (torch.uint8,), 1)
    out = torch.empty(k, b, dtype=torch.float32, device=mask.device)
    _lib.call("si_read_h3", _vp(workspace), workspace.numel(), k, d, b, _vp(mask), _vp(out), _stream())
    return out


def pack_signs(w_gate: torch.Tensor) -> torch.Tensor:
    """Packed sign bits of ``W_gate [k][d]`` (private layout, int32 words)."""
    _dev(w_gate, "w_gate", _F16, 2)
    k, d = w_gate.shape
    nbytes = signs_bytes(k, d)
    if nbytes == 0:
        raise ValueError(f"unsupported shape k={k} d={d}")
    out = torch.empty(nbytes // 4, dtype=torch.int32, device=w_gate.device)
    _lib.call("si_pack_signs", _vp(w_gate), k, d, _vp(out), _stream())
    return out


def signs_to_canonical(signs: torch.Tensor, k: int, d: int) -> torch.Tensor:
    """``[k][d/32]`` int32 words, bit j of word w = sign of element 32w+j."""
    _dev(signs, "signs", (torch.int32,))
    out = torch.empty(k, d // 32, dtype=torch.int32, device=signs.device)
    _lib.call("si_signs_to_canonical", _vp(signs), k, d, _vp(out), _stream())
    return out


def transpose_down(w_down: torch.Tensor) -> torch.Tensor:
    """``W_down [d][k]`` -> ``W_down^T [k][d]`` (fp16), on ``w_down``'s device."""
    _dev(w_down, "w_down", _F16, 2)
    d, k = w_down.shape
    out = torch.empty(k, d, dtype=w_down.dtype, device=w_down.device)
    _call_on(w_down.get_device(), "si_transpose_down", _vp(w_down), d, k, _vp(out))
    return out


def _x2(x: torch.Tensor, d: int):
    _dev(x, "x", _F16)
    if x.dim() == 1:
        x = x.view(1, -1)
    if x.dim() != 2 or x.shape[1] != d:
        raise ValueError(f"x must be [b][{d}], got {tuple(x.shape)}")
    return x


def predict(signs: torch.Tensor, x: torch.Tensor, alpha: float, k: int, workspace: torch.Tensor):
    """Eq. (2) for every row: returns ``(mask [k] uint8, active_idx [k] int32,
    n_active [1] int32)``; entries ``n..k-1`` of ``active_idx`` are undefined."""
    _dev(signs, "signs", (torch.int32,))
    d = x.shape[-1]
    x = _x2(x, d)
    b = x.shape[0]
    mask = torch.empty(k, dtype=torch.uint8, device=x.device)
    idx = torch.empty(k, dtype=torch.int32, device=x.device)
    n = torch.empty(1, dtype=torch.int32, device=x.device)
    _lib.call("si_predict", _vp(signs), k, d, _vp(x), b, float(alpha), _vp(mask), _vp(idx), _vp(n),
              _vp(workspace), workspace.numel(), _stream())
    return mask, idx, n


def sparse_mlp(w_gate, w_up, w_down_t, x, workspace, mask=None, active_idx=None, n_active=None,
               flags: int = 0, counters: bool = False):
    """Eq. (1) over the kept rows; returns ``y [b][d]`` float32 (and the
    ``[3]`` work counters when ``counters``).  ``w_up=None`` runs the
    non-gated ReLU MLP ``ReLU(x W_fc1) W_down^T`` with ``w_gate`` as
    ``W_fc1`` (``si_sparse_relu_mlp``)."""
    for t, nm in ((w_gate, "w_gate"), (w_up, "w_up"), (w_down_t, "w_down_t")):
        if t is not None or nm != "w_up":
            _dev(t, nm, _F16, 2)
    k, d = w_gate.shape
    x = _x2(x, d)
    b = x.shape[0]
    y = torch.empty(b, d, dtype=torch.float32, device=x.device)
    cnt = torch.zeros(3, dtype=torch.int32, device=x.device) if counters else None
    tail = (k, d, _vp(x), b, _vp(mask), _vp(active_idx), _vp(n_active), _vp(y), _vp(workspace),
            workspace.numel(), flags, _vp(cnt), _stream())
    if w_up is None:
        _lib.call("si_sparse_relu_mlp", _vp(w_gate), _vp(w_down_t), *tail)
    else:
        _lib.call("si_sparse_mlp", _vp(w_gate), _vp(w_up), _vp(w_down_t), *tail)
    return (y, cnt) if counters else y


def predict_sparse_mlp(signs, w_gate, w_up, w_down_t, x, alpha, workspace, flags: int = 0,
                       outputs: bool = False, y: torch.Tensor = None):
    """The whole per-token path.  Returns ``y`` (written into ``y`` when
    given); with ``outputs`` also ``(mask, active_idx, n_active, counters)``.
    ``w_up=None``: the non-gated ReLU MLP (``si_predict_sparse_relu_mlp``)."""
    k, d = w_gate.shape
    x = _x2(x, d)
    b = x.shape[0]
    if y is None:
        y = torch.empty(b, d, dtype=torch.float32, device=x.device)
    else:
        _dev(y, "y", (torch.float32,))
        if y.numel() != b * d:
            raise ValueError(f"y must hold [{b}][{d}] floats")
    if outputs:
        mask = torch.empty(k, dtype=torch.uint8, device=x.device)
        idx = torch.empty(k, dtype=torch.int32, device=x.device)
        n = torch.empty(1, dtype=torch.int32, device=x.device)
        cnt = torch.zeros(3, dtype=torch.int32, device=x.device)
    else:
        mask = idx = n = cnt = None
    tail = (k, d, _vp(x), b, float(alpha), _vp(mask), _vp(idx), _vp(n), _vp(y), _vp(workspace),
            workspace.numel(), flags, _vp(cnt), _stream())
    if w_up is None:  # the non-gated ReLU MLP, w_gate as W_fc1
        _lib.call("si_predict_sparse_relu_mlp", _vp(signs), _vp(w_gate), _vp(w_down_t), *tail)
    else:
        _lib.call("si_predict_sparse_mlp", _vp(signs), _vp(w_gate), _vp(w_up), _vp(w_down_t), *tail)
    return (y, (mask, idx, n, cnt)) if outputs else y


def mlp_block(h, norm_w, eps, signs, w_gate, w_up, w_down_t, alpha, workspace, flags: int = 0,
              outputs: bool = False, y: torch.Tensor = None):
    """The MLP half of a decoder layer with its neighbours fused
    (``si_rmsnorm_predict_sparse_mlp``): ``y = h + MLP(fp16(RMSNorm(h) *
    norm_w))``; ``h`` ``[b][d]`` and ``norm_w`` ``[d]`` float32.  Returns
    ``y`` (and ``(mask, active_idx, n_active, counters)`` with ``outputs``);
    ``w_up=None``: the non-gated ReLU MLP."""
    _dev(h, "h", (torch.float32,))
    _dev(norm_w, "norm_w", (torch.float32,), 1)
    k, d = w_gate.shape
    h2 = h.view(-1, d)
    b = h2.shape[0]
    if y is None:
        y = torch.empty(b, d, dtype=torch.float32, device=h.device)
    else:
        _dev(y, "y", (torch.float32,))
        if y.numel() != b * d:
            raise ValueError(f"y must hold [{b}][{d}] floats")
    if outputs:
        mask = torch.empty(k, dtype=torch.uint8, device=h.device)
        idx = torch.empty(k, dtype=torch.int32, device=h.device)
        n = torch.empty(1, dtype=torch.int32, device=h.device)
        cnt = torch.zeros(3, dtype=torch.int32, device=h.device)
    else:
        mask = idx = n = cnt = None
    _lib.call("si_rmsnorm_predict_sparse_mlp", _vp(h2), _vp(norm_w), float(eps), _vp(signs), _vp(w_gate),
              _vp(w_up), _vp(w_down_t), k, d, b, float(alpha), _vp(mask), _vp(idx), _vp(n), _vp(y),
              _vp(workspace), workspace.numel(), flags, _vp(cnt), _stream())
    return (y, (mask, idx, n, cnt)) if outputs else y


class MLPLayer:
    """One layer's device-resident state: weights, packed signs and
    ``W_down^T`` (both made once at load), plus a workspace.  With
    ``w_up=None`` the layer is a non-gated ReLU MLP and ``w_gate`` is its
    ``W_fc1``."""

    def __init__(self, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, max_batch: int = 1,
                 keep_w_down: bool = False):
        self.k, self.d = w_gate.shape
        self.w_gate = w_gate
        self.w_up = w_up
        self.signs = pack_signs(w_gate)
        self.w_down_t = transpose_down(w_down)
        self.w_down = w_down if keep_w_down else None
        self.workspace = new_workspace(self.k, self.d, max_batch, w_gate.device)

    def __call__(self, x, alpha: float, flags: int = 0, outputs: bool = False, y: torch.Tensor = None):
        return predict_sparse_mlp(self.signs, self.w_gate, self.w_up, self.w_down_t, x, alpha, self.workspace,
                                  flags=flags, outputs=outputs, y=y)

    def block(self, h, norm_w, eps: float, alpha: float, flags: int = 0, outputs: bool = False,
              y: torch.Tensor = None, post_norm_w=None, gate=None, scale: float = 1.0):
        """``h + MLP(RMSNorm(h) * norm_w)`` in one launch (see ``mlp_block``).
        With a norm behind the MLP, a gate or a residual scale
        (``h + scale * gate * RMSNorm(MLP(..)) * post_norm_w``) the call is
        ``norm_residual`` in front of and behind the MLP."""
        if post_norm_w is not None or gate is not None or scale != 1.0:
            return _block(self, h, norm_w, eps, alpha, flags, outputs, y, post_norm_w, gate, scale)
        return mlp_block(h, norm_w, eps, self.signs, self.w_gate, self.w_up, self.w_down_t, alpha, self.workspace,
                         flags=flags, outputs=outputs, y=y)

    def predict(self, x, alpha: float):
        return predict(self.signs, x, alpha, self.k, self.workspace)

    def sparse_mlp(self, x, mask=None, active_idx=None, n_active=None, flags: int = 0, counters: bool = False):
        return sparse_mlp(self.w_gate, self.w_up, self.w_down_t, x, self.workspace, mask, active_idx, n_active,
                          flags, counters)

    def prompt(self, x, out_dtype=None):
        """The dense MLP of a prompt, ``x [..., d]`` fp16: ``ReLU(x W_gate^T) * (x
        W_up^T)`` in fp16, then the product with ``W_down^T``; returns ``[..., d]`` in
        ``out_dtype`` (``x``'s type).  A hidden value above 65504 becomes infinite,
        which in decode, where it is float32, it does not."""
        h = gated_linear(x, self.w_gate, self.w_up)
        return linear(h, self.w_down_t, transposed=True, out_dtype=out_dtype or x.dtype)


# ---- INT8 weights ---------------------------------------------------------

def quantize_rows_i8(w: torch.Tensor):
    """Symmetric per-row INT8 quantization of fp16 ``w [rows][n]``: returns
    ``(q int8 [rows][n], scale float32 [rows])`` (``si_quantize_rows_i8``)."""
    _dev(w, "w", _F16, 2)
    rows, n = w.shape
    q = torch.empty(rows, n, dtype=torch.int8, device=w.device)
    scale = torch.empty(rows, dtype=torch.float32, device=w.device)
    _lib.call("si_quantize_rows_i8", _vp(w), rows, n, _vp(q), _vp(scale), _stream())
    return q, scale


def pack_signs_i8(q_gate: torch.Tensor) -> torch.Tensor:
    """Packed MSBs of INT8 ``W_gate [k][d]`` (the layout of ``pack_signs``)."""
    _dev(q_gate, "q_gate", (torch.int8,), 2)
    k, d = q_gate.shape
    nbytes = signs_bytes(k, d)
    if nbytes == 0:
        raise ValueError(f"unsupported shape k={k} d={d}")
    out = torch.empty(nbytes // 4, dtype=torch.int32, device=q_gate.device)
    _lib.call("si_pack_signs_i8", _vp(q_gate), k, d, _vp(out), _stream())
    return out


def transpose_down_i8(q_down: torch.Tensor) -> torch.Tensor:
    """INT8 ``W_down [d][k]`` -> ``W_down^T [k][d]``."""
    _dev(q_down, "q_down", (torch.int8,), 2)
    d, k = q_down.shape
    out = torch.empty(k, d, dtype=torch.int8, device=q_down.device)
    _lib.call("si_transpose_down_i8", _vp(q_down), d, k, _vp(out), _stream())
    return out


def _i8_weights(q_gate, s_gate, q_up, s_up, q_down_t, s_down):
    _dev(q_gate, "q_gate", (torch.int8,), 2)
    _dev(q_down_t, "q_down_t", (torch.int8,), 2)
    k, d = q_gate.shape
    _dev(s_gate, "s_gate", (torch.float32,), 1)
    _dev(s_down, "s_down", (torch.float32,), 1)
    if q_up is not None:
        _dev(q_up, "q_up", (torch.int8,), 2)
        _dev(s_up, "s_up", (torch.float32,), 1)
        if tuple(q_up.shape) != (k, d) or s_up.numel() != k:
            raise ValueError("q_up / s_up do not match q_gate")
    if tuple(q_down_t.shape) != (k, d) or s_gate.numel() != k or s_down.numel() != d:
        raise ValueError("q_down_t [k][d], s_gate [k] and s_down [d] expected")
    return k, d


def sparse_mlp_i8(q_gate, s_gate, q_up, s_up, q_down_t, s_down, x, workspace, mask, flags: int = 0,
                  counters: bool = False):
    """Eq. (1) over the rows kept by ``mask`` with INT8 weights
    (``si_sparse_mlp_i8``); ``q_up=None``: the non-gated ReLU MLP.  Returns
    ``y [b][d]`` float32 (and the ``[3]`` work counters with ``counters``)."""
    k, d = _i8_weights(q_gate, s_gate, q_up, s_up, q_down_t, s_down)
    x = _x2(x, d)
    b = x.shape[0]
    y = torch.empty(b, d, dtype=torch.float32, device=x.device)
    cnt = torch.zeros(3, dtype=torch.int32, device=x.device) if counters else None
    _lib.call("si_sparse_mlp_i8", _vp(q_gate), _vp(s_gate), _vp(q_up), _vp(s_up if q_up is not None else None),
              _vp(q_down_t), _vp(s_down), k, d, _vp(x), b, _vp(mask), _vp(y), _vp(workspace), workspace.numel(),
              flags, _vp(cnt), _stream())
    return (y, cnt) if counters else y


def predict_sparse_mlp_i8(signs, q_gate, s_gate, q_up, s_up, q_down_t, s_down, x, alpha, workspace,
                          flags: int = 0, outputs: bool = False, y: torch.Tensor = None):
    """The whole per-token path with INT8 weights
    (``si_predict_sparse_mlp_i8``); ``signs`` from ``pack_signs_i8``.
    Returns ``y`` (and ``(mask, active_idx, n_active, counters)`` with
    ``outputs``)."""
    k, d = _i8_weights(q_gate, s_gate, q_up, s_up, q_down_t, s_down)
    _dev(signs, "signs", (torch.int32,))
    x = _x2(x, d)
    b = x.shape[0]
    if y is None:
        y = torch.empty(b, d, dtype=torch.float32, device=x.device)
    else:
        _dev(y, "y", (torch.float32,))
        if y.numel() != b * d:
            raise ValueError(f"y must hold [{b}][{d}] floats")
    if outputs:
        mask = torch.empty(k, dtype=torch.uint8, device=x.device)
        idx = torch.empty(k, dtype=torch.int32, device=x.device)
        n = torch.empty(1, dtype=torch.int32, device=x.device)
        cnt = torch.zeros(3, dtype=torch.int32, device=x.device)
    else:
        mask = idx = n = cnt = None
    _lib.call("si_predict_sparse_mlp_i8", _vp(signs), _vp(q_gate), _vp(s_gate), _vp(q_up),
              _vp(s_up if q_up is not None else None), _vp(q_down_t), _vp(s_down), k, d, _vp(x), b, float(alpha),
              _vp(mask), _vp(idx), _vp(n), _vp(y), _vp(workspace), workspace.numel(), flags, _vp(cnt), _stream())
    return (y, (mask, idx, n, cnt)) if outputs else y


class Int8MLPLayer:
    """One layer with INT8 weights, made on the device at load from fp16
    weights: per-row quantization of ``W_gate``, ``W_up`` (``[k][d]``) and
    ``W_down`` (``[d][k]``), the packed MSBs of the INT8 ``W_gate`` and the
    INT8 ``W_down^T``.  ``w_up=None``: a non-gated ReLU MLP."""

    def __init__(self, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, max_batch: int = 1):
        self.k, self.d = w_gate.shape
        self.q_gate, self.s_gate = quantize_rows_i8(w_gate)
        self.q_up, self.s_up = quantize_rows_i8(w_up) if w_up is not None else (None, None)
        q_down, self.s_down = quantize_rows_i8(w_down)
        self.q_down_t = transpose_down_i8(q_down)
        self.signs = pack_signs_i8(self.q_gate)
        self.workspace = new_workspace(self.k, self.d, max_batch, w_gate.device)

    def __call__(self, x, alpha: float, flags: int = 0, outputs: bool = False, y: torch.Tensor = None):
        return predict_sparse_mlp_i8(self.signs, self.q_gate, self.s_gate, self.q_up, self.s_up, self.q_down_t,
                                     self.s_down, x, alpha, self.workspace, flags=flags, outputs=outputs, y=y)

    def block(self, h, norm_w, eps: float, alpha: float, flags: int = 0, outputs: bool = False,
              y: torch.Tensor = None, post_norm_w=None, gate=None, scale: float = 1.0):
        """``h + scale * gate * [RMSNorm](MLP(RMSNorm(h) * norm_w))`` (see
        ``MLPLayer.block``): ``norm_residual`` in front of and behind the MLP."""
        return _block(self, h, norm_w, eps, alpha, flags, outputs, y, post_norm_w, gate, scale)

    def sparse_mlp(self, x, mask, flags: int = 0, counters: bool = False):
        return sparse_mlp_i8(self.q_gate, self.s_gate, self.q_up, self.s_up, self.q_down_t, self.s_down, x,
                             self.workspace, mask, flags, counters)


# ---- MXFP4 weights and the norms around a block -----------------------------

_DTYPE = {torch.float16: _lib.SI_F16, torch.int16: _lib.SI_F16, torch.bfloat16: _lib.SI_BF16,
          torch.float32: _lib.SI_F32}
_HALF = frozenset((torch.float16, torch.int16, torch.bfloat16))
_ANY = _HALF | {torch.float32}
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


# These calls take a few microseconds each, so what is checked on every call is
# checked in few steps, and what is wrong is named afterwards.

def _call_on(index: int, name: str, *args) -> None:
    """``name(*args, stream)`` on the current stream of device ``index``, which
    need not be the current one."""
    if index == _current_device():
        _lib.call(name, *args, _raw_stream(index) if _raw_stream is not None else _stream())
    else:
        with torch.cuda.device(index):
            _lib.call(name, *args, _stream())


@functools.lru_cache(maxsize=4096)
def _product_workspace(aligned, ldx: int, m: int, rows: int, n: int, gated: bool) -> int:
    """``si_linear_mxfp4_workspace_bytes`` for activations at an address that is a
    multiple of 16 or not (None: MXFP4 activations)."""
    address = None if aligned is None else 16 if aligned else 18
    return int(_lib.load().si_linear_mxfp4_workspace_bytes(address, ldx, m, rows, n, gated))


def _same_device(*tensors) -> int:
    """The index of the device that all of the tensors (None: none) are on."""
    index = tensors[0].get_device()
    for t in tensors:
        if t is not None and t.get_device() != index:
            raise ValueError(f"tensors on {tensors[0].device} and {t.device}")
    return index


def _rows(t, name: str, dtypes):
    """A ``[rows][n]`` tensor (or one row ``[n]``) whose rows are contiguous, with
    any stride between them: returns ``(rows, n, stride)``."""
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if not t.is_cuda:
        raise ValueError(f"{name} must be a CUDA tensor (got {t.device})")
    if t.dtype not in dtypes:
        raise TypeError(f"{name} has dtype {t.dtype}, expected one of {sorted(map(str, dtypes))}")
    shape, stride = t.shape, t.stride()
    if len(shape) == 2:
        rows, n = shape
        ld = stride[0] if rows > 1 else n
    elif len(shape) == 1:
        rows, n = 1, shape[0]
        ld = n
    else:
        raise ValueError(f"{name} must be [rows][n], got {tuple(shape)}")
    if stride[-1] != 1 and n > 1:
        raise ValueError(f"{name} must have contiguous rows")
    if ld < n:
        raise ValueError(f"{name}'s rows overlap")
    return rows, n, ld


def _mx(q, scale, name: str, n: int = None) -> int:
    """The number of the MXFP4 rows ``q, scale``; of ``n`` values each when
    given."""
    try:
        rows, width = q.shape
        if (q.is_cuda and scale.is_cuda and q.dtype is torch.uint8 and scale.dtype is torch.uint8
                and q.is_contiguous() and scale.is_contiguous() and width & 63 == 0
                and scale.shape == (rows, width >> 4) and (n is None or width == (n + 127) // 128 * 64)):
            return rows
    except (AttributeError, ValueError):
        pass
    _dev(q, name, (torch.uint8,), 2)
    _dev(scale, f"{name}'s scales", (torch.uint8,), 2)
    if width & 63 or tuple(scale.shape) != (rows, width // 16):
        raise ValueError(f"{name} {tuple(q.shape)} and its scales {tuple(scale.shape)} are not MXFP4 rows")
    raise ValueError(f"{name} has rows of {2 * width} stored values, {n} do not take that many")


def _floats(t, shape, name: str) -> int:
    """The address of a contiguous float32 tensor of that shape, or None."""
    if t is None:
        return None
    if (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype is torch.float32 and t.is_contiguous()
            and t.shape == shape):
        return t.data_ptr()
    _dev(t, name, (torch.float32,))
    raise ValueError(f"{name} must be {list(shape)}, got {tuple(t.shape)}")


def quantize_rows_mxfp4(w: torch.Tensor):
    """Rows ``w [rows][n]`` (fp16, bf16 or float32, any row stride) to MXFP4
    (``si_quantize_rows_mxfp4``): returns the codes, uint8 ``[rows][np / 2]``, and
    scales, uint8 ``[rows][np / 32]``, with ``np`` = ``n`` rounded up to 128."""
    rows, n, ld = _rows(w, "w", _ANY)
    pieces = (n + 127) // 128
    q = w.new_empty((rows, pieces * 64), dtype=torch.uint8)
    scale = w.new_empty((rows, pieces * 4), dtype=torch.uint8)
    _call_on(w.get_device(), "si_quantize_rows_mxfp4", w.data_ptr(), _DTYPE[w.dtype], ld, rows, n, q.data_ptr(),
             scale.data_ptr())
    return q, scale


def dequantize_rows_mxfp4(q: torch.Tensor, scale: torch.Tensor, n: int, dtype=torch.float16) -> torch.Tensor:
    """MXFP4 rows of ``n`` values as ``[rows][n]`` of ``dtype``
    (``si_dequantize_rows_mxfp4``)."""
    rows = _mx(q, scale, "q", n)
    if dtype not in _ANY:
        raise TypeError(f"dtype {dtype}, expected one of {sorted(map(str, _ANY))}")
    w = q.new_empty((rows, n), dtype=dtype)
    _call_on(_same_device(q, scale), "si_dequantize_rows_mxfp4", q.data_ptr(), scale.data_ptr(), rows, n, w.data_ptr(),
             _DTYPE[dtype])
    return w


def pack_signs_mxfp4(q_gate: torch.Tensor) -> torch.Tensor:
    """Packed signs of MXFP4 ``W_gate`` codes (the layout of ``pack_signs``)."""
    _dev(q_gate, "q_gate", (torch.uint8,), 2)
    k, d = q_gate.shape[0], 2 * q_gate.shape[1]
    nbytes = signs_bytes(k, d)
    if nbytes == 0:
        raise ValueError(f"unsupported shape k={k} d={d}")
    out = torch.empty(nbytes // 4, dtype=torch.int32, device=q_gate.device)
    _call_on(q_gate.get_device(), "si_pack_signs_mxfp4", _vp(q_gate), k, d, _vp(out))
    return out


def _product(name, x, x_args, ldx, m, n, weights, out_dtype, *more):
    """One of the four products; ``weights`` is ``q, scale`` or ``q_gate,
    s_gate, q_up, s_up``, ``more`` further tensors that have to be on ``x``'s
    device.  Scratch comes from torch's allocator, in the stream's order like any
    tensor, and is held until the call returns: another thread may allocate while
    the call makes its launches."""
    gated = len(weights) == 4
    rows = _mx(weights[0], weights[1], "q_gate" if gated else "q", n)
    up = gated and weights[2] is not None
    if up and _mx(weights[2], weights[3], "q_up", n) != rows:
        raise ValueError("q_up does not match q_gate")
    if out_dtype not in _ANY:
        raise TypeError(f"out_dtype {out_dtype}, expected one of {sorted(map(str, _ANY))}")
    index = _same_device(x, *weights, *more)
    y = x.new_empty((m, rows), dtype=out_dtype)
    nbytes = _product_workspace(x_args[0] & 15 == 0 if len(x_args) == 3 else None, ldx, m, rows, n, up)
    ws = x.new_empty((nbytes,), dtype=torch.uint8) if nbytes else None
    _call_on(index, name, *x_args, m, n, *(None if t is None else t.data_ptr() for t in weights), rows, y.data_ptr(),
             _DTYPE[out_dtype], _vp(ws), nbytes)
    return y


def linear_mxfp4(x: torch.Tensor, q: torch.Tensor, scale: torch.Tensor, out_dtype=None) -> torch.Tensor:
    """``x W^T`` with MXFP4 weights ``q, scale`` of ``[rows][n]``
    (``si_linear_mxfp4``); ``x [m][n]`` fp16 or bf16, any row stride.  Returns
    ``[m][rows]`` in ``out_dtype`` (``x``'s type)."""
    m, n, ld = _rows(x, "x", _HALF)
    return _product("si_linear_mxfp4", x, (x.data_ptr(), _DTYPE[x.dtype], ld), ld, m, n, (q, scale),
                    out_dtype or x.dtype)


def gated_linear_mxfp4(x: torch.Tensor, q_gate, s_gate, q_up=None, s_up=None, out_dtype=None) -> torch.Tensor:
    """``ReLU(x W_gate^T) * (x W_up^T)`` over every row, Eq. (1) steps 1-3 of a
    prompt (``si_gated_linear_mxfp4``); ``q_up=None``: ``ReLU(x W_fc1^T)``."""
    m, n, ld = _rows(x, "x", _HALF)
    return _product("si_gated_linear_mxfp4", x, (x.data_ptr(), _DTYPE[x.dtype], ld), ld, m, n,
                    (q_gate, s_gate, q_up, s_up), out_dtype or x.dtype)


def linear_mxfp4_a4(xq: torch.Tensor, x_scale: torch.Tensor, q: torch.Tensor, scale: torch.Tensor,
                    out_dtype=torch.float16) -> torch.Tensor:
    """``linear_mxfp4`` with the activations in MXFP4 too
    (``quantize_rows_mxfp4``), on the 4-bit matrix instructions."""
    m = _mx(xq, x_scale, "xq")
    return _product("si_linear_mxfp4_a4", xq, (xq.data_ptr(), x_scale.data_ptr()), 0, m, 2 * xq.shape[1], (q, scale),
                    out_dtype, x_scale)


def gated_linear_mxfp4_a4(xq: torch.Tensor, x_scale: torch.Tensor, q_gate, s_gate, q_up=None, s_up=None,
                          out_dtype=torch.float16) -> torch.Tensor:
    """``gated_linear_mxfp4`` with the activations in MXFP4 too."""
    m = _mx(xq, x_scale, "xq")
    return _product("si_gated_linear_mxfp4_a4", xq, (xq.data_ptr(), x_scale.data_ptr()), 0, m, 2 * xq.shape[1],
                    (q_gate, s_gate, q_up, s_up), out_dtype, x_scale)


def mxfp4_workspace_bytes(k: int, d: int, b: int = 1) -> int:
    return int(_lib.load().si_mxfp4_workspace_bytes(k, d, b))


def new_workspace_mxfp4(k: int, d: int, b: int = 1, device=None) -> torch.Tensor:
    """Zero-filled workspace for MXFP4 sparse MLP calls with up to ``b`` tokens."""
    n = mxfp4_workspace_bytes(k, d, b)
    if n == 0:
        raise ValueError(f"unsupported shape k={k} d={d} b={b}")
    return torch.zeros(n, dtype=torch.uint8, device=device or "cuda")


def _mx_mlp(q_gate, s_gate, q_up, s_up, q_down_t, s_down_t, x, y, workspace, *more):
    """Checks of the two MXFP4 MLP calls: returns ``(k, d, b, device index,
    y)`` and the addresses of the weights."""
    k = _mx(q_gate, s_gate, "q_gate")
    shape, s_shape = q_gate.shape, s_gate.shape
    d = 2 * shape[1]
    weights = [q_gate.data_ptr(), s_gate.data_ptr(), None, None, q_down_t.data_ptr(), s_down_t.data_ptr()]
    for q, s, name in ((q_up, s_up, "q_up"), (q_down_t, s_down_t, "q_down_t")):
        if q is None:
            continue
        if s is None or not (q.shape == shape and s.shape == s_shape and q.dtype is torch.uint8 and s.dtype is torch.uint8
                and q.is_contiguous() and s.is_contiguous()):
            _mx(q, s, name, d)
            raise ValueError(f"{name} does not match q_gate")
    if q_up is not None:
        weights[2], weights[3] = q_up.data_ptr(), s_up.data_ptr()
    if not (isinstance(x, torch.Tensor) and x.dim() == 2 and x.shape[1] == d and x.dtype in _F16
            and x.is_contiguous()):
        x = _x2(x, d)
    b = x.shape[0]
    if y is None:
        y = torch.empty_like(x, dtype=torch.float32)
    else:
        _dev(y, "y", (torch.float32,))
        if y.numel() != b * d:
            raise ValueError(f"y must hold [{b}][{d}] floats")
    index = _same_device(q_gate, x, s_gate, q_up, s_up, q_down_t, s_down_t, y, workspace, *more)
    return k, d, b, index, y, weights


def sparse_mlp_mxfp4(q_gate, s_gate, q_up, s_up, q_down_t, s_down_t, x, workspace, mask, flags: int = 0,
                     counters: bool = False, y: torch.Tensor = None):
    """Eq. (1) over the rows kept by ``mask`` with MXFP4 weights
    (``si_sparse_mlp_mxfp4``); ``q_up=None``: the non-gated ReLU MLP.  Returns
    ``y [b][d]`` float32 (and the ``[3]`` work counters with ``counters``)."""
    _dev(mask, "mask", (torch.uint8,), 1)
    k, d, b, index, y, weights = _mx_mlp(q_gate, s_gate, q_up, s_up, q_down_t, s_down_t, x, y, workspace, mask)
    if mask.numel() != k:
        raise ValueError(f"mask must hold {k} rows")
    cnt = x.new_empty((3,), dtype=torch.int32) if counters else None
    _call_on(index, "si_sparse_mlp_mxfp4", *weights, k, d, x.data_ptr(), b, mask.data_ptr(), y.data_ptr(),
             workspace.data_ptr(), workspace.numel(), flags, _vp(cnt))
    return (y, cnt) if counters else y


def predict_sparse_mlp_mxfp4(signs, q_gate, s_gate, q_up, s_up, q_down_t, s_down_t, x, alpha, workspace,
                             flags: int = 0, outputs: bool = False, y: torch.Tensor = None):
    """The whole per-token path with MXFP4 weights
    (``si_predict_sparse_mlp_mxfp4``); ``signs`` from ``pack_signs_mxfp4``.
    Returns ``y`` (and ``(mask, active_idx, n_active, counters)`` with
    ``outputs``)."""
    _dev(signs, "signs", (torch.int32,))
    k, d, b, index, y, weights = _mx_mlp(q_gate, s_gate, q_up, s_up, q_down_t, s_down_t, x, y, workspace, signs)
    if signs.numel() * 32 != (k + 63) // 64 * 64 * d:
        raise ValueError(f"signs do not belong to [{k}][{d}]")
    if outputs:
        mask = x.new_empty((k,), dtype=torch.uint8)
        idx = x.new_empty((k,), dtype=torch.int32)
        n = x.new_empty((1,), dtype=torch.int32)
        cnt = x.new_empty((3,), dtype=torch.int32)
        out = (mask.data_ptr(), idx.data_ptr(), n.data_ptr())
    else:
        out, cnt = (None, None, None), None
    _call_on(index, "si_predict_sparse_mlp_mxfp4", signs.data_ptr(), *weights, k, d, x.data_ptr(), b, float(alpha), *out,
             y.data_ptr(), workspace.data_ptr(), workspace.numel(), flags, _vp(cnt))
    return (y, (mask, idx, n, cnt)) if outputs else y


def norm_residual(h: torch.Tensor, branch: torch.Tensor = None, post_w: torch.Tensor = None,
                  gate: torch.Tensor = None, scale: float = 1.0, pre_w: torch.Tensor = None, eps: float = 1e-5,
                  x_dtype=torch.float16, out: torch.Tensor = None):
    """What stands between the products of two blocks, in one launch
    (``si_norm_residual``)::

        h' = h + scale * gate * (RMSNorm(branch) * post_w)   # post_w None: branch itself
        x  = RMSNorm(h') * pre_w

    ``h`` and ``branch`` are ``[tokens][d]`` (or ``[d]``) in fp16, bf16 or
    float32, with any row stride; ``gate`` float32 ``[d]`` or ``[g][d]``, each row
    for ``tokens / g`` consecutive tokens; ``post_w`` and ``pre_w`` float32
    ``[d]``.  Returns ``(h', x)``: ``h'`` in ``h``'s type (in ``out`` when given,
    which may be ``h``; None without a branch), ``x`` in ``x_dtype`` (None without
    ``pre_w``)."""
    tokens, d, ldh = _rows(h, "h", _ANY)
    if x_dtype not in _ANY:
        raise TypeError(f"x_dtype {x_dtype}, expected one of {sorted(map(str, _ANY))}")
    index = _same_device(h, branch, post_w, gate, pre_w, out)
    hp, ht = h.data_ptr(), _DTYPE[h.dtype]
    bp, bt, ldb, op, ldo, gp, per = None, ht, 0, None, 0, None, 1
    if branch is not None:
        bt_, bd, ldb = _rows(branch, "branch", _ANY)
        if bt_ != tokens or bd != d:
            raise ValueError(f"branch {tuple(branch.shape)} does not match h {tuple(h.shape)}")
        bp, bt = branch.data_ptr(), _DTYPE[branch.dtype]
        if out is None:
            out = torch.empty_like(h, memory_format=torch.contiguous_format)
            ldo = d
        else:
            ot, od, ldo = _rows(out, "out", (h.dtype,))
            if ot != tokens or od != d:
                raise ValueError(f"out {tuple(out.shape)} does not match h {tuple(h.shape)}")
        op = out.data_ptr()
        if gate is not None:
            g = gate.shape[0] if gate.dim() == 2 else 1
            gp = _floats(gate, (g, d) if gate.dim() == 2 else (d,), "gate")
            if g < 1 or tokens % g:
                raise ValueError(f"gate has {g} rows, which do not divide {tokens} tokens")
            per = max(tokens // g, 1)
    elif post_w is not None or gate is not None or out is not None:
        raise ValueError("post_w, gate and out need a branch")
    elif pre_w is None:
        raise ValueError("nothing to compute: neither branch nor pre_w")
    x = xp = None
    wp = _floats(pre_w, (d,), "pre_w")
    if wp is not None:
        x = torch.empty_like(h, dtype=x_dtype, memory_format=torch.contiguous_format)
        xp = x.data_ptr()
    _call_on(index, "si_norm_residual", hp, ht, ldh, bp, bt, ldb, _floats(post_w, (d,), "post_w"), gp, per, float(scale), op,
             ldo, wp, xp, _DTYPE[x_dtype], d, tokens, d, float(eps))
    return out, x


def _block(layer, h, norm_w, eps, alpha, flags, outputs, y, post_norm_w, gate, scale):
    """The MLP half of a decoder layer around ``layer``'s call: ``h`` float32
    ``[b][d]``; the result in ``y`` when given."""
    _dev(h, "h", (torch.float32,))
    h2 = h.view(-1, layer.d)
    _, x = norm_residual(h2, pre_w=norm_w, eps=eps)
    res = layer(x, alpha, flags=flags, outputs=outputs)
    branch = res[0] if outputs else res
    if y is not None:
        _dev(y, "y", (torch.float32,))
        if y.numel() != h2.numel():
            raise ValueError(f"y must hold [{h2.shape[0]}][{layer.d}] floats")
    out, _ = norm_residual(h2, branch, post_w=post_norm_w, gate=gate, scale=scale, eps=eps,
                           out=None if y is None else y.view(h2.shape))
    if y is not None:
        out = y
    return (out, res[1]) if outputs else out


class MXFP4MLPLayer:
    """One layer with MXFP4 weights, made on the device at load from fp16, bf16
    or float32 weights ``W_gate``, ``W_up`` (``[k][d]``) and ``W_down``
    (``[d][k]``): the quantized ``W_gate``, ``W_up`` and ``W_down^T``, and the
    packed signs.  ``prompt=True`` keeps ``W_down`` quantized along ``k`` as
    well, for ``prompt`` (its scales cover other values than ``W_down^T``'s).
    ``w_up=None``: a non-gated ReLU MLP."""

    def __init__(self, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, max_batch: int = 1,
                 prompt: bool = False):
        self.k, self.d = w_gate.shape
        self.q_gate, self.s_gate = quantize_rows_mxfp4(w_gate)
        self.q_up, self.s_up = quantize_rows_mxfp4(w_up) if w_up is not None else (None, None)
        if w_down.dtype == torch.float32:
            w_down_t = w_down.t().contiguous()
        else:
            w_down_t = transpose_down(w_down.view(torch.int16)).view(w_down.dtype)
        self.q_down_t, self.s_down_t = quantize_rows_mxfp4(w_down_t)
        self.q_down, self.s_down = quantize_rows_mxfp4(w_down) if prompt else (None, None)
        self.signs = pack_signs_mxfp4(self.q_gate)
        self.workspace = new_workspace_mxfp4(self.k, self.d, max_batch, w_gate.device)

    def __call__(self, x, alpha: float, flags: int = 0, outputs: bool = False, y: torch.Tensor = None):
        return predict_sparse_mlp_mxfp4(self.signs, self.q_gate, self.s_gate, self.q_up, self.s_up, self.q_down_t,
                                        self.s_down_t, x, alpha, self.workspace, flags=flags, outputs=outputs, y=y)

    def sparse_mlp(self, x, mask, flags: int = 0, counters: bool = False):
        return sparse_mlp_mxfp4(self.q_gate, self.s_gate, self.q_up, self.s_up, self.q_down_t, self.s_down_t, x,
                                self.workspace, mask, flags, counters)

    def block(self, h, norm_w, eps: float, alpha: float, flags: int = 0, outputs: bool = False,
              y: torch.Tensor = None, post_norm_w=None, gate=None, scale: float = 1.0):
        """``h + scale * gate * [RMSNorm](MLP(RMSNorm(h) * norm_w))`` of 1 to 8
        tokens (see ``MLPLayer.block``)."""
        return _block(self, h, norm_w, eps, alpha, flags, outputs, y, post_norm_w, gate, scale)

    def prompt(self, x, out_dtype=None, a4: bool = False):
        """The dense MLP of a prompt, ``x [m][d]`` fp16 or bf16: ``ReLU(x
        W_gate^T) * (x W_up^T)`` in ``x``'s type, then the product with
        ``W_down^T``; returns ``[m][d]`` in ``out_dtype`` (``x``'s type).
        With fp16 tokens a hidden value above 65504 becomes infinite, which in
        decode, where it is float32, it does not; bf16 holds it.
        ``a4``: both products take their activations in MXFP4."""
        if self.q_down is None:
            raise ValueError("the layer was made without prompt=True")
        out_dtype = out_dtype or x.dtype
        if a4:
            h = gated_linear_mxfp4_a4(*quantize_rows_mxfp4(x), self.q_gate, self.s_gate, self.q_up, self.s_up,
                                      out_dtype=x.dtype)
            return linear_mxfp4_a4(*quantize_rows_mxfp4(h), self.q_down, self.s_down, out_dtype)
        h = gated_linear_mxfp4(x, self.q_gate, self.s_gate, self.q_up, self.s_up)
        return linear_mxfp4(h, self.q_down, self.s_down, out_dtype)

    def prompt_block(self, h, norm_w, eps: float, x_dtype=torch.bfloat16, a4: bool = False, post_norm_w=None, gate=None,
                     scale: float = 1.0, next_norm_w=None, out: torch.Tensor = None):
        """The MLP half of a decoder layer of a prompt: ``norm_residual``,
        ``prompt``, ``norm_residual``.  Returns ``(h', x')`` with ``x' =
        RMSNorm(h') * next_norm_w`` for what follows (None without it)."""
        _, x = norm_residual(h, pre_w=norm_w, eps=eps, x_dtype=x_dtype)
        branch = self.prompt(x, a4=a4)
        return norm_residual(h, branch.view(h.shape), post_w=post_norm_w, gate=gate, scale=scale, pre_w=next_norm_w,
                             eps=eps, x_dtype=x_dtype, out=out)


# ---- dense products with their gradients --------------------------------------

@functools.lru_cache(maxsize=4096)
def _dense_workspace(name: str, *args) -> int:
    """Workspace bytes of a dense call: ``args`` as the C function takes them, with
    ``_like`` addresses."""
    return int(getattr(_lib.load(), name)(*args))


def _like(t):
    """An address that is a multiple of 16 where ``t``'s is, as the workspaces'
    sizes ask; None for None."""
    return None if t is None else 16 if t.data_ptr() & 15 == 0 else 18


def _scratch(x, nbytes: int):
    return x.new_empty((nbytes,), dtype=torch.uint8) if nbytes else None


def _flat(x, name: str, dtypes):
    """``x [..., n]`` as rows: returns ``(x2, rows, n, stride)``."""
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"{name} must be a tensor")
    if x.dim() == 0:
        raise ValueError(f"{name} must be [..., n]")
    x2 = x if x.dim() == 2 else x.reshape(-1, x.shape[-1])
    return (x2, *_rows(x2, name, dtypes))


def _weight(w, name: str, x, shape=None):
    """A contiguous matrix of ``x``'s type."""
    _dev(w, name, _HALF, 2)
    if _DTYPE[w.dtype] != _DTYPE[x.dtype]:
        raise TypeError(f"{name} has dtype {w.dtype}, x {x.dtype}")
    if shape is not None and tuple(w.shape) != shape:
        raise ValueError(f"{name} must be {list(shape)}, got {list(w.shape)}")
    return w.shape


def _out_type(dtype, x):
    dtype = x.dtype if dtype is None else dtype
    if dtype not in _ANY:
        raise TypeError(f"out_dtype {dtype}, expected one of {sorted(map(str, _ANY))}")
    return dtype


def _wants_grad(*tensors) -> bool:
    """Whether a call has gradients to give.  A tangent (forward-mode
    differentiation) would be lost in its output, and is refused."""
    if getattr(_forward_ad, "_current_level", 0) >= 0:  # within a dual_level
        for t in tensors:
            if t is not None and _forward_ad.unpack_dual(t).tangent is not None:
                raise NotImplementedError("this operator has gradients in reverse mode alone: a tensor with a tangent "
                                          "(forward-mode differentiation) is not taken")
    return torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors)


def _linear_forward(x2, m, n, ld, w, rows, transposed, out_dtype):
    index = _same_device(x2, w)
    y = x2.new_empty((m, rows), dtype=out_dtype)
    nbytes = _dense_workspace("si_linear_workspace_bytes", _like(x2), ld, m, n, _like(w), rows, transposed)
    ws = _scratch(x2, nbytes)
    _call_on(index, "si_linear", x2.data_ptr(), _DTYPE[x2.dtype], ld, m, n, w.data_ptr(), rows, transposed, y.data_ptr(),
             _DTYPE[out_dtype], _vp(ws), nbytes)
    return y


_nodes = None


def _graph(y, x):
    """The module that places a call of ``x`` with output ``y`` in autograd's graph
    (``csrc/autograd.cpp``), and the stream of the call."""
    global _nodes
    if _nodes is None:
        _nodes = _lib.autograd()
    if y.dtype == torch.int16:
        raise TypeError("an output of int16 (fp16 bits) has no gradient: ask for another out_dtype")
    if x.dim() != 2:  # its rows, which the node is given, may be a copy
        _nodes.refuse_foreign_leaf(x)
    index = y.get_device()
    if _raw_stream is not None:
        return _nodes, _raw_stream(index)
    return _nodes, torch.cuda.current_stream(index).cuda_stream


def linear(x: torch.Tensor, w: torch.Tensor, transposed: bool = False, out_dtype=None) -> torch.Tensor:
    """``x W^T`` (``si_linear``) with ``x [..., n]`` and ``W [rows][n]`` (``[n][rows]``
    when ``transposed``) in fp16 or bf16; ``[..., rows]`` in ``out_dtype`` (``x``'s
    type).  Differentiable with respect to both."""
    x2, m, n, ld = _flat(x, "x", _HALF)
    shape = _weight(w, "w", x)
    rows = shape[1] if transposed else shape[0]
    if shape[0 if transposed else 1] != n:
        raise ValueError(f"w {tuple(shape)} does not take rows of {n} values")
    out_dtype = _out_type(out_dtype, x)
    keep = _wants_grad(x, w)
    y = _linear_forward(x2, m, n, ld, w, rows, bool(transposed), out_dtype)
    if keep:
        graph, stream = _graph(y, x)
        graph.linear(y, x2, w, m, n, rows, bool(transposed), stream)
    return y if x.dim() == 2 else y.view(*x.shape[:-1], rows)


def _gated_forward(x2, m, n, ld, w_gate, w_up, rows, out_dtype, keep):
    """``(h, g, u)``; g and u (with ``keep`` and ``w_up``) the two sums, float32."""
    index = _same_device(x2, w_gate, w_up)
    h = x2.new_empty((m, rows), dtype=out_dtype)
    g = u = None
    if keep and w_up is not None:
        g, u = x2.new_empty((m, rows), dtype=torch.float32), x2.new_empty((m, rows), dtype=torch.float32)
    nbytes = _dense_workspace("si_gated_linear_workspace_bytes", _like(x2), ld, m, n, _like(w_gate), _like(w_up), rows)
    ws = _scratch(x2, nbytes)
    _call_on(index, "si_gated_linear", x2.data_ptr(), _DTYPE[x2.dtype], ld, m, n, w_gate.data_ptr(), _vp(w_up), rows,
             h.data_ptr(), _DTYPE[out_dtype], _vp(g), _vp(u), _vp(ws), nbytes)
    return h, g, u


def gated_linear(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor = None, out_dtype=None) -> torch.Tensor:
    """``ReLU(x W_gate^T) * (x W_up^T)`` over every row, Eq. (1) steps 1-3, in one
    launch (``si_gated_linear``); ``w_up=None``: ``ReLU(x W_fc1^T)``.  ``x [..., n]``
    and the weights ``[rows][n]`` in fp16 or bf16; returns ``[..., rows]`` in
    ``out_dtype`` (``x``'s type).  Differentiable with respect to all; both sums
    are kept for the backward pass in float32."""
    x2, m, n, ld = _flat(x, "x", _HALF)
    shape = _weight(w_gate, "w_gate", x)
    rows = shape[0]
    if shape[1] != n:
        raise ValueError(f"w_gate {tuple(shape)} does not take rows of {n} values")
    if w_up is not None:
        _weight(w_up, "w_up", x, (rows, n))
    out_dtype = _out_type(out_dtype, x)
    keep = _wants_grad(x, w_gate, w_up)
    h, g, u = _gated_forward(x2, m, n, ld, w_gate, w_up, rows, out_dtype, keep)
    if keep:
        graph, stream = _graph(h, x)
        graph.gated_linear(h, x2, w_gate, w_up, g, u, m, n, rows, stream)
    return h if x.dim() == 2 else h.view(*x.shape[:-1], rows)


def mlp(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor, out_dtype=None) -> torch.Tensor:
    """The dense MLP of Eq. (1), ``(ReLU(x W_gate^T) * (x W_up^T)) W_down^T``, with
    ``W_gate, W_up [k][d]`` and ``W_down [d][k]`` (``w_up=None``: the non-gated one):
    ``gated_linear`` and ``linear``, differentiable with respect to all; the backward
    pass is one call (``si_mlp_backward``).  The hidden values are rounded to ``x``'s
    type; where gradients are asked for they and both sums (float32) are kept."""
    x2, m, n, ld = _flat(x, "x", _HALF)
    rows = _weight(w_gate, "w_gate", x)[0]
    if w_gate.shape[1] != n:
        raise ValueError(f"w_gate {tuple(w_gate.shape)} does not take rows of {n} values")
    if w_up is not None:
        _weight(w_up, "w_up", x, (rows, n))
    _weight(w_down, "w_down", x, (n, rows))
    out_dtype = _out_type(out_dtype, x)
    keep = _wants_grad(x, w_gate, w_up, w_down)
    h, g, u = _gated_forward(x2, m, n, ld, w_gate, w_up, rows, x2.dtype, keep)
    y = _linear_forward(h, m, rows, rows, w_down, n, False, out_dtype)
    if keep:
        graph, stream = _graph(y, x)
        graph.mlp(y, x2, w_gate, w_up, w_down, h, g, u, m, n, rows, stream)
    return y if x.dim() == 2 else y.view(x.shape)


# ---- norms with their gradients -------------------------------------------------

def _norm_forward(x2, tokens, d, ld, w, b, center, eps, keep):
    """``(y, mean, rstd)``, the last two with ``keep``."""
    index = _same_device(x2, w, b)
    y = x2.new_empty((tokens, d))
    mean = x2.new_empty((tokens,), dtype=torch.float32) if keep and center else None
    rstd = x2.new_empty((tokens,), dtype=torch.float32) if keep else None
    _call_on(index, "si_layer_norm", x2.data_ptr(), _DTYPE[x2.dtype], ld, w.data_ptr(), _vp(b), _DTYPE[w.dtype], center, eps,
             y.data_ptr(), _vp(mean), _vp(rstd), tokens, d)
    return y, mean, rstd


_FLOATS = frozenset((torch.float16, torch.bfloat16, torch.float32))


def _norm(x, w, b, eps, center):
    x2, tokens, d, ld = _flat(x, "x", _FLOATS)
    for t, name in ((w, "w"), (b, "b")):
        if t is None and name == "b":
            continue
        _dev(t, name, _FLOATS, 1)
        if t.shape[0] != d:
            raise ValueError(f"{name} must be [{d}], got {list(t.shape)}")
    if b is not None and b.dtype != w.dtype:
        raise TypeError(f"b has dtype {b.dtype}, w {w.dtype}")
    keep = _wants_grad(x, w, b)
    y, mean, rstd = _norm_forward(x2, tokens, d, ld, w, b, center, float(eps), keep)
    if keep:
        graph, stream = _graph(y, x)
        graph.norm(y, x2, w, b, mean, rstd, tokens, d, center, stream)
    return y if x.dim() == 2 else y.view(x.shape)


def layer_norm(x: torch.Tensor, w: torch.Tensor, b: torch.Tensor = None, eps: float = 1e-5) -> torch.Tensor:
    """``(x - mean) / sqrt(var + eps) * w + b`` over the last dimension
    (``si_layer_norm``), the norm in front of a non-gated MLP: ``x [..., d]`` in fp16,
    bf16 or float32, ``w`` and ``b`` ``[d]`` of one of these types, in ``x``'s type.
    Differentiable with respect to all."""
    return _norm(x, w, b, eps, True)


def rms_norm(x: torch.Tensor, w: torch.Tensor, eps: float = 1e-5) -> torch.Tensor:
    """``x / sqrt(mean(x^2) + eps) * w`` over the last dimension (``si_layer_norm``),
    differentiable; types as ``layer_norm``.  ``norm_residual`` is its form for
    inference, with the residual."""
    return _norm(x, w, None, eps, False)


# ---- FP8 weights -----------------------------------------------------------------

_E4M3 = torch.float8_e4m3fn


def _quantize_fp8(name, w, arg, rows_per_scale):
    rows, n, ld = _rows(w, arg, _ANY)
    q = w.new_empty((rows, (n + 15) // 16 * 16), dtype=_E4M3)
    scale = w.new_empty(((rows + rows_per_scale - 1) // rows_per_scale, (n + 127) // 128), dtype=torch.float32)
    _call_on(w.get_device(), name, w.data_ptr(), _DTYPE[w.dtype], ld, rows, n, q.data_ptr(), scale.data_ptr())
    return q, scale


def quantize_rows_fp8(x: torch.Tensor):
    """Tokens ``x [rows][n]`` (fp16, bf16 or float32, any row stride) to e4m3 with a
    scale for each 128 values of a row (``si_quantize_rows_fp8``): returns the codes,
    ``float8_e4m3fn [rows][n rounded up to 16]``, and scales, float32
    ``[rows][ceil(n / 128)]``."""
    return _quantize_fp8("si_quantize_rows_fp8", x, "x", 1)


def quantize_blocks_fp8(w: torch.Tensor):
    """Weights ``w [rows][n]`` to e4m3 with a scale for each 128 x 128 block
    (``si_quantize_blocks_fp8``): the codes as ``quantize_rows_fp8``, the scales
    float32 ``[ceil(rows / 128)][ceil(n / 128)]``."""
    return _quantize_fp8("si_quantize_blocks_fp8", w, "w", 128)


def _fp8(q, scale, name: str, rows_per_scale: int):
    """Rows and stored values a row of FP8 rows or blocks."""
    _dev(q, name, (_E4M3,), 2)
    _dev(scale, f"{name}'s scales", (torch.float32,), 2)
    rows, width = q.shape
    if width % 16 or width == 0:
        raise ValueError(f"{name} must hold rows of a multiple of 16 codes, got {width}")
    want = ((rows + rows_per_scale - 1) // rows_per_scale, (width + 127) // 128)
    if tuple(scale.shape) != want:
        raise ValueError(f"{name}'s scales must be {list(want)}, got {list(scale.shape)}")
    return rows, width


def dequantize_fp8(q: torch.Tensor, scale: torch.Tensor, n: int, dtype=torch.float16) -> torch.Tensor:
    """FP8 tokens (a scale row for each row) or weights (one for each 128) of ``n``
    values as ``[rows][n]`` of ``dtype`` (``si_dequantize_fp8``)."""
    per = 1 if isinstance(scale, torch.Tensor) and scale.dim() == 2 and scale.shape[0] == q.shape[0] else 128
    rows, width = _fp8(q, scale, "q", per)
    if width != (n + 15) // 16 * 16:
        raise ValueError(f"q has rows of {width} codes, {n} values do not take that many")
    if dtype not in _ANY:
        raise TypeError(f"dtype {dtype}, expected one of {sorted(map(str, _ANY))}")
    w = q.new_empty((rows, n), dtype=dtype)
    _call_on(_same_device(q, scale), "si_dequantize_fp8", q.data_ptr(), scale.data_ptr(), per, rows, n, w.data_ptr(),
             _DTYPE[dtype])
    return w


def _fp8_product(name, xq, x_scale, weights, out_dtype):
    m, n = _fp8(xq, x_scale, "xq", 1)
    gated = len(weights) == 4
    rows, width = _fp8(weights[0], weights[1], "q_gate" if gated else "q", 128)
    up = gated and weights[2] is not None
    if up and _fp8(weights[2], weights[3], "q_up", 128) != (rows, width):
        raise ValueError("q_up does not match q_gate")
    if width != n:
        raise ValueError(f"weights of {width} codes a row, tokens of {n}")
    if out_dtype not in _ANY:
        raise TypeError(f"out_dtype {out_dtype}, expected one of {sorted(map(str, _ANY))}")
    index = _same_device(xq, x_scale, *weights)
    y = xq.new_empty((m, rows), dtype=out_dtype)
    nbytes = _dense_workspace("si_linear_fp8_workspace_bytes", m, rows, n, up)
    ws = _scratch(xq, nbytes)
    _call_on(index, name, xq.data_ptr(), x_scale.data_ptr(), m, n, *(_vp(t) for t in weights), rows, y.data_ptr(),
             _DTYPE[out_dtype], _vp(ws), nbytes)
    return y


def linear_fp8(xq: torch.Tensor, x_scale: torch.Tensor, q: torch.Tensor, scale: torch.Tensor,
               out_dtype=torch.float16) -> torch.Tensor:
    """``x W^T`` of FP8 tokens (``quantize_rows_fp8``) and FP8 weights
    (``quantize_blocks_fp8``, or a checkpoint's of that form) on the matrix cores
    (``si_linear_fp8``): ``[m][rows]`` in ``out_dtype``."""
    return _fp8_product("si_linear_fp8", xq, x_scale, (q, scale), out_dtype)


def gated_linear_fp8(xq: torch.Tensor, x_scale: torch.Tensor, q_gate, s_gate, q_up=None, s_up=None,
                     out_dtype=torch.float16) -> torch.Tensor:
    """``gated_linear`` of FP8 tokens and weights (``si_gated_linear_fp8``);
    ``q_up=None``: ``ReLU(x W_fc1^T)``."""
    return _fp8_product("si_gated_linear_fp8", xq, x_scale, (q_gate, s_gate, q_up, s_up), out_dtype)


class FP8MLPLayer:
    """One layer's dense MLP with FP8 weights, made on the device at load from fp16,
    bf16 or float32 ``W_gate``, ``W_up`` (``[k][d]``) and ``W_down`` (``[d][k]``), or
    (``from_blocks``) from a checkpoint's codes and block scales.  ``w_up=None``: a
    non-gated ReLU MLP."""

    def __init__(self, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor):
        self._set(quantize_blocks_fp8(w_gate), None if w_up is None else quantize_blocks_fp8(w_up),
                  quantize_blocks_fp8(w_down))
        self.d = w_gate.shape[1]

    @classmethod
    def from_blocks(cls, gate, up, down):
        """From ``(codes, scales)`` pairs of the three matrices (``up=None``: non-gated)."""
        layer = cls.__new__(cls)
        layer._set(gate, up, down)
        layer.d = layer.q_down.shape[0]
        return layer

    def _set(self, gate, up, down):
        self.q_gate, self.s_gate = gate
        self.q_up, self.s_up = up if up is not None else (None, None)
        self.q_down, self.s_down = down
        self.k, width = _fp8(self.q_gate, self.s_gate, "gate", 128)
        if up is not None and _fp8(self.q_up, self.s_up, "up", 128) != (self.k, width):
            raise ValueError("up does not match gate")
        d, width_down = _fp8(self.q_down, self.s_down, "down", 128)
        if (d + 15) // 16 * 16 != width or (self.k + 15) // 16 * 16 != width_down:
            raise ValueError(f"down has {d} rows of {width_down} codes, gate {self.k} of {width}")

    def prompt(self, x, out_dtype=None):
        """The MLP of any number of tokens, ``x [m][d]`` fp16, bf16 or float32: tokens
        to FP8, ``ReLU(x W_gate^T) * (x W_up^T)`` in ``x``'s type, that to FP8, the
        product with ``W_down^T``; ``[m][d]`` in ``out_dtype`` (``x``'s type).  With fp16
        tokens a hidden value above 65504 becomes infinite, its block's scale NaN and
        that token's output NaN; with bf16 or float32 tokens it does not."""
        if x.shape[-1] != self.d:
            raise ValueError(f"x has rows of {x.shape[-1]} values, the layer takes {self.d}")
        h = gated_linear_fp8(*quantize_rows_fp8(x), self.q_gate, self.s_gate, self.q_up, self.s_up, out_dtype=x.dtype)
        return linear_fp8(*quantize_rows_fp8(h), self.q_down, self.s_down, out_dtype or x.dtype)

    def prompt_block(self, h, norm_w, eps: float, x_dtype=torch.bfloat16, post_norm_w=None, gate=None, scale: float = 1.0,
                     next_norm_w=None, out: torch.Tensor = None):
        """The MLP half of a decoder layer: ``norm_residual``, ``prompt``,
        ``norm_residual`` (see ``MXFP4MLPLayer.prompt_block``)."""
        _, x = norm_residual(h, pre_w=norm_w, eps=eps, x_dtype=x_dtype)
        branch = self.prompt(x.view(-1, self.d))
        return norm_residual(h, branch.view(h.shape), post_w=post_norm_w, gate=gate, scale=scale, pre_w=next_norm_w,
                             eps=eps, x_dtype=x_dtype, out=out)
