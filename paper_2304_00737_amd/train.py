"""Thin Python binding of libspardl_train.so (argument marshalling only): the
training operators of include/spardl_train.h, whose weight gradients the calls
of spardl.py synchronise.

Every function takes torch tensors for device buffers, outputs included, all on
the current device, and raises SpardlError on failure.  Matrices are 2-d with contiguous rows (any row
stride); types are bfloat16, float16 and, except for the feed-forward block,
float32.  All compute runs in the HIP kernels of the library; there is no
fallback: if it is missing, importing this module fails.
"""

from __future__ import annotations

import ctypes
import os

import torch

from .spardl import EINVAL, OK, SpardlError, _stream

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libspardl_train.so")

BF16, FP16, FP32 = 0, 1, 2
ACT = {"silu": 0, "gelu": 1}
NORM_MAX_DIM = 16384
DISTILL_MAX_TOP = 1024

if not os.path.exists(LIB_PATH):
    raise ImportError(f"{LIB_PATH} is not built (run __graft_entry__.build()); "
                      "there is no fallback implementation")

_lib = ctypes.CDLL(LIB_PATH)
_p, _i32, _i64, _sz, _f = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float

_lib.spardl_rms_norm.argtypes = [_p, _i64, _p, _i64, _p, _p, _i64, _p, _i64, _p, _i64, _i32, _f, _i32, _p]
_lib.spardl_rms_norm_workspace_bytes.argtypes = [_i64, _i32]
_lib.spardl_rms_norm_backward.argtypes = [_p, _i64, _p, _i64, _p, _p, _p, _i64, _p, _i64, _p, _i64, _i32, _i32, _p, _sz,
                                          _p]
_lib.spardl_distill_workspace_bytes.argtypes = [_i64, _i32]
_lib.spardl_distill_loss.argtypes = [_p, _i64, _p, _p, _i64, _i64, _i32, _i32, _f, _p, _p, _i32, _p, _sz, _p]
_lib.spardl_distill_backward.argtypes = [_p, _i64, _p, _p, _i64, _p, _p, _i64, _i32, _i32, _f, _p, _i64, _i32, _p]
_lib.spardl_distill_loss_backward.argtypes = [_p, _i64, _p, _p, _i64, _p, _i64, _i32, _i32, _f, _p, _p, _p, _i64, _i32,
                                              _p, _sz, _p]
_lib.spardl_gated_ffn_workspace_bytes.argtypes = [_i64, _i32, _i32, _i32, _i32]
_lib.spardl_gated_ffn.argtypes = [_p, _i64] * 5 + [_p, _p, _i64, _i64, _i32, _i32, _i32, _i32, _p, _sz, _p]
_lib.spardl_gated_ffn_backward.argtypes = ([_p, _i64] * 2 + [_p, _p, _i64] + [_p, _i64] * 7
                                           + [_i32, _i32, _i64, _i32, _i32, _i32, _i32, _p, _sz, _p])
for _n in ("rms_norm", "rms_norm_backward", "distill_loss", "distill_backward", "distill_loss_backward", "gated_ffn",
           "gated_ffn_backward"):
    getattr(_lib, "spardl_" + _n).restype = ctypes.c_int
for _n in ("rms_norm", "distill", "gated_ffn"):
    getattr(_lib, f"spardl_{_n}_workspace_bytes").restype = _sz

_TYPES = {torch.bfloat16: BF16, torch.float16: FP16, torch.float32: FP32}


def _check(fn: str, status: int) -> None:
    if status != OK:
        raise SpardlError(fn, status)


def _refuse(fn: str, what: str):
    e = SpardlError(fn, EINVAL)
    e.args = (f"{e.args[0]}: {what}",)
    raise e


def _type(fn: str, t) -> int:
    dt = _TYPES.get(t.dtype)
    if dt is None:
        _refuse(fn, f"no kernel for {t.dtype}")
    return dt


def _lead(fn: str, name: str, t):
    """(its shape, pointer and row distance, type) of the matrix that the other arguments are measured by."""
    try:
        _, cols = shape = t.shape
    except (AttributeError, ValueError):
        _refuse(fn, f"{name} must be a matrix, is {None if t is None else list(t.shape)}")
    return shape, (t.data_ptr(), cols) if t.is_contiguous() else _mat(fn, name, t, shape, t.dtype), t.dtype


def _mat(fn: str, name: str, t, shape, dtype):
    """(pointer, row distance) of a matrix argument; None is passed on."""
    if t is None:
        return None, shape[1]
    if t.shape == shape and t.dtype is dtype:
        if t.is_contiguous():
            return t.data_ptr(), shape[1]
        strides = t.stride()
        if strides[1] == 1 or shape[1] == 1:
            return t.data_ptr(), strides[0] if shape[0] > 1 else shape[1]
    _refuse(fn, f"{name} must be {list(shape)} of {dtype} with contiguous rows, "
                f"is {list(t.shape)} of {t.dtype} with strides {t.stride()}")


def _vec(fn: str, name: str, t, n: int, dtype=torch.float32):
    if t is None:
        return None
    if t.numel() == n and t.dtype is dtype and t.is_contiguous():
        return t.data_ptr()
    _refuse(fn, f"{name} must be {n} contiguous elements of {dtype}, is {list(t.shape)} of {t.dtype}")


def _ws(fn: str, ws):
    if ws is None:
        return None, 0
    if not ws.is_contiguous():
        _refuse(fn, f"the workspace must be contiguous, has strides {ws.stride()}")
    return ws.data_ptr(), ws.nbytes


# the current device and its stream's handle by the shortest way: small calls are bound by what precedes their launch
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)


def _on(fn: str, stream, *tensors) -> int:
    """The stream's handle, after the check that every tensor (or None) is on the device that the launch goes to."""
    at = _current_device() if tensors[0].is_cuda else -1
    for t in tensors:
        if t is not None and t.get_device() != at:
            at = -1
            break
    if at < 0:
        _refuse(fn, "all tensors must be on the current GPU, are on "
                    f"{sorted({str(t.device) for t in tensors if t is not None})}")
    if stream is None and _raw_stream is not None:
        return _raw_stream(at)
    return _stream(stream)


def _new_ws(fn: str, nbytes: int, device):
    if nbytes == 0:
        raise SpardlError(fn, EINVAL)
    return torch.empty(int(nbytes), dtype=torch.uint8, device=device)


# ---------------------------------------------------------------- residual RMS norm

def rms_norm(x, res, weight, sum, y, rstd=None, *, eps: float = 1e-6, stream=None) -> None:
    """sum = x + res, y = sum / rms(sum) * weight; res, sum and rstd may be None."""
    fn = "rms_norm"
    shape, x_at, dt = _lead(fn, "x", x)
    rows, dim = shape
    _check(fn, _lib.spardl_rms_norm(*x_at, *_mat(fn, "res", res, shape, dt),
                                    _vec(fn, "weight", weight, dim, dt), *_mat(fn, "sum", sum, shape, dt),
                                    *_mat(fn, "y", y, shape, dt), _vec(fn, "rstd", rstd, rows), rows, dim, eps,
                                    _type(fn, x), _on(fn, stream, x, res, weight, sum, y, rstd)))


def rms_norm_workspace(rows: int, dim: int, device="cuda"):
    """Scratch for rms_norm_backward over up to `rows` rows."""
    return _new_ws("rms_norm_workspace_bytes", _lib.spardl_rms_norm_workspace_bytes(rows, dim), device)


def rms_norm_backward(dy, sum, weight, rstd, dx, dweight, ws, dsum=None, *, stream=None) -> None:
    """dx (of x and of res alike, dsum included) and dweight (float32)."""
    fn = "rms_norm_backward"
    shape, dy_at, dt = _lead(fn, "dy", dy)
    rows, dim = shape
    _check(fn, _lib.spardl_rms_norm_backward(
        *dy_at, *_mat(fn, "sum", sum, shape, dt), _vec(fn, "weight", weight, dim, dt), _vec(fn, "rstd", rstd, rows),
        *_mat(fn, "dsum", dsum, shape, dt), *_mat(fn, "dx", dx, shape, dt),
        _vec(fn, "dweight", dweight, dim), rows, dim, _type(fn, dy), *_ws(fn, ws),
        _on(fn, stream, dy, sum, weight, rstd, dx, dweight, ws, dsum)))


# ---------------------------------------------------------------- distillation loss

def distill_workspace(rows: int, vocab: int, device="cuda"):
    """Scratch for distill_loss and distill_loss_backward over up to `rows` rows of vocab logits."""
    return _new_ws("distill_workspace_bytes", _lib.spardl_distill_workspace_bytes(rows, vocab), device)


def _lists(fn: str, logits, top_idx, top_val):
    (rows, vocab), (z, ld), _ = _lead(fn, "logits", logits)
    shape, (i, ld_i), dt = _lead(fn, "top_idx", top_idx)
    if shape[0] != rows or dt is not torch.int32:
        _mat(fn, "top_idx", top_idx, (rows, shape[1]), torch.int32)     # refuses
    v, ld_v = _mat(fn, "top_val", top_val, shape, torch.float32)
    if ld_i != ld_v:
        _refuse(fn, "top_idx and top_val must have one row stride")
    return (z, ld, i, v, ld_i), rows, vocab, shape[1]


def distill_loss(logits, top_idx, top_val, loss, stats, ws, *, temperature: float = 1.0, stream=None) -> None:
    """loss [rows] and stats [rows, 2] (float32) of the student's logits against the teacher's lists."""
    fn = "distill_loss"
    lists, rows, vocab, top = _lists(fn, logits, top_idx, top_val)
    _check(fn, _lib.spardl_distill_loss(*lists, rows, vocab, top, temperature, _vec(fn, "loss", loss, rows),
                                        _vec(fn, "stats", stats, 2 * rows), _type(fn, logits), *_ws(fn, ws),
                                        _on(fn, stream, logits, top_idx, top_val, loss, stats, ws)))


def distill_backward(logits, top_idx, top_val, stats, dloss, dlogits, *, temperature: float = 1.0, stream=None) -> None:
    """dlogits from the stats that distill_loss wrote and dloss [rows]; dlogits may be logits."""
    fn = "distill_backward"
    lists, rows, vocab, top = _lists(fn, logits, top_idx, top_val)
    _check(fn, _lib.spardl_distill_backward(*lists, _vec(fn, "stats", stats, 2 * rows),
                                            _vec(fn, "dloss", dloss, rows), rows, vocab, top, temperature,
                                            *_mat(fn, "dlogits", dlogits, logits.shape, logits.dtype),
                                            _type(fn, logits),
                                            _on(fn, stream, logits, top_idx, top_val, stats, dloss, dlogits)))


def distill_loss_backward(logits, top_idx, top_val, dloss, loss, stats, dlogits, ws, *, temperature: float = 1.0,
                          stream=None) -> None:
    """distill_loss and distill_backward in one call, which reads the logits once where it can."""
    fn = "distill_loss_backward"
    lists, rows, vocab, top = _lists(fn, logits, top_idx, top_val)
    _check(fn, _lib.spardl_distill_loss_backward(
        *lists, _vec(fn, "dloss", dloss, rows), rows, vocab, top, temperature,
        _vec(fn, "loss", loss, rows), _vec(fn, "stats", stats, 2 * rows),
        *_mat(fn, "dlogits", dlogits, logits.shape, logits.dtype), _type(fn, logits), *_ws(fn, ws),
        _on(fn, stream, logits, top_idx, top_val, dloss, loss, stats, dlogits, ws)))


# ---------------------------------------------------------------- gated feed-forward block

def gated_ffn_workspace(tokens: int, dim: int, hidden: int, dtype=torch.bfloat16, *, backward: bool = False,
                        unaligned: bool = False, device="cuda"):
    """Scratch for gated_ffn of up to `tokens` tokens, with backward=True for gated_ffn_backward too.
    unaligned: a row of x, dy or a weight may start off a 16-byte boundary
    though its length is a multiple of 8 (a view), or have a stride of 2^21 or more."""
    if dtype not in (torch.bfloat16, torch.float16):
        _refuse("gated_ffn_workspace_bytes", f"no kernel for {dtype}")
    need = [_lib.spardl_gated_ffn_workspace_bytes(tokens, dim, hidden, b, unaligned) for b in range(1 + backward)]
    return _new_ws("gated_ffn_workspace_bytes", max(need), device)


def _act(fn: str, act: str) -> int:
    if act not in ACT:
        _refuse(fn, f"act must be one of {sorted(ACT)}, is {act!r}")
    return ACT[act]


def _gate_up(fn: str, gate, up, rows: int, hidden: int, dt):
    g, ld_g = _mat(fn, "gate", gate, (rows, hidden), dt)
    u, ld_u = _mat(fn, "up", up, (rows, hidden), dt)
    if ld_g != ld_u:
        _refuse(fn, "gate and up must have one row stride")
    return g, u, ld_g


def gated_ffn(x, w_gate, w_up, w_down, y, ws, *, gate=None, up=None, act: str = "silu", stream=None) -> None:
    """y = (act(x w_gate^T) * (x w_up^T)) w_down^T; gate and up receive the two products for the backward pass."""
    fn = "gated_ffn"
    (rows, dim), x_at, dt = _lead(fn, "x", x)
    hidden = _lead(fn, "w_gate", w_gate)[0][0]
    _check(fn, _lib.spardl_gated_ffn(
        *x_at, *_mat(fn, "w_gate", w_gate, (hidden, dim), dt),
        *_mat(fn, "w_up", w_up, (hidden, dim), dt), *_mat(fn, "w_down", w_down, (dim, hidden), dt),
        *_mat(fn, "y", y, (rows, dim), dt), *_gate_up(fn, gate, up, rows, hidden, dt), rows, dim, hidden, _act(fn, act),
        _type(fn, x), *_ws(fn, ws), _on(fn, stream, x, w_gate, w_up, w_down, y, ws, gate, up)))


def gated_ffn_backward(dy, x, gate, up, w_gate, w_up, w_down, dx, dw_gate, dw_up, dw_down, ws, *, act: str = "silu",
                       accumulate: bool = False, stream=None) -> None:
    """dx (may be None) and the weight gradients, in x's type or in float32
    (views of a worker's gradient row, say); accumulate adds to them."""
    fn = "gated_ffn_backward"
    (rows, dim), x_at, dt = _lead(fn, "x", x)
    hidden = _lead(fn, "w_gate", w_gate)[0][0]
    dwt = _lead(fn, "dw_gate", dw_gate)[2]
    _check(fn, _lib.spardl_gated_ffn_backward(
        *_mat(fn, "dy", dy, (rows, dim), dt), *x_at, *_gate_up(fn, gate, up, rows, hidden, dt),
        *_mat(fn, "w_gate", w_gate, (hidden, dim), dt),
        *_mat(fn, "w_up", w_up, (hidden, dim), dt), *_mat(fn, "w_down", w_down, (dim, hidden), dt),
        *_mat(fn, "dx", dx, (rows, dim), dt), *_mat(fn, "dw_gate", dw_gate, (hidden, dim), dwt),
        *_mat(fn, "dw_up", dw_up, (hidden, dim), dwt), *_mat(fn, "dw_down", dw_down, (dim, hidden), dwt),
        _type(fn, dw_gate), accumulate, rows, dim, hidden, _act(fn, act), _type(fn, x), *_ws(fn, ws),
        _on(fn, stream, x, dy, gate, up, w_gate, w_up, w_down, dx, dw_gate, dw_up, dw_down, ws)))
