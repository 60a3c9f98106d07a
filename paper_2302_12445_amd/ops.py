"""Training operators on torch tensors: binding of libdear_ops.so (include/dear_ops.h).

    out, lse = attention(q, k, v, causal=True)                       # [B, S, H, D]
    dq, dk, dv = attention_backward(dout, q, k, v, out, lse, causal=True)
    h, y, kept, rstd = add_rms_norm(x, residual, weight, eps)        # kept: y in 8 bits
    dx, dweight = add_rms_norm_backward(dy, h, weight, rstd, dh=dh)
    kept = checkpoint_encode(x); x = checkpoint_decode(kept, dtype)
    dw = checkpoint_weight_grad(dy, kept)                            # fp32 [outs, ins]

Tensors are on a GPU, bf16 or fp32.  Work is enqueued on the current torch stream of the tensors'
device; outputs and workspaces come from torch's allocator.  Wrong arguments raise ValueError or
DearError before anything is launched.  There is no CPU fallback: if the library is missing,
loading raises.  layers.py has the autograd functions over these calls.
"""
from __future__ import annotations

import ctypes as C
import math
import os
import struct
from typing import NamedTuple, Optional, Tuple

import torch

from .binding import DEAR_BF16, DEAR_F32, DearError

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdear_ops.so")
GROUP = 32  # DEAR_CHECKPOINT_GROUP
NORM_MAX_COLS = 32768

EXPORTS = [
    "dear_attention", "dear_attention_workspace", "dear_attention_backward", "dear_attention_backward_workspace",
    "dear_checkpoint_encode", "dear_checkpoint_decode", "dear_checkpoint_weight_grad", "dear_checkpoint_weight_grad_workspace",
    "dear_add_rms_norm", "dear_add_rms_norm_backward", "dear_add_rms_norm_backward_workspace",
]

_DTYPE = {torch.bfloat16: DEAR_BF16, torch.float32: DEAR_F32}
_lib = None


def load_library() -> C.CDLL:
    """Load libdear_ops.so from the package directory; raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError("libdear_ops.so is not built: run `python -m paper_2302_12445_amd.build` (there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    out64 = C.POINTER(i64)
    # dear_attention_t is passed as the bytes that struct packs
    lib.dear_attention.argtypes = [C.c_char_p, vp]
    lib.dear_attention_backward.argtypes = [C.c_char_p, vp]
    lib.dear_attention_workspace.argtypes = [C.c_char_p, out64]
    lib.dear_attention_backward_workspace.argtypes = [C.c_char_p, out64]
    lib.dear_checkpoint_encode.argtypes = [vp, i32, i64, i64, i64, vp, vp, vp]
    lib.dear_checkpoint_decode.argtypes = [vp, vp, i64, i64, i32, vp, vp]
    lib.dear_checkpoint_weight_grad.argtypes = [vp, i32, i64, vp, vp, i64, i64, i64, vp, vp, i64, vp]
    lib.dear_checkpoint_weight_grad_workspace.argtypes = [i32, i64, i64, i64, out64]
    lib.dear_add_rms_norm.argtypes = [vp, i64, vp, i64, vp, i32, i64, i64, f32, vp, vp, vp, vp, vp, vp]
    lib.dear_add_rms_norm_backward.argtypes = [vp, i64, vp, i64, vp, i64, vp, vp, i32, i64, i64, vp, vp, vp, i64, vp]
    lib.dear_add_rms_norm_backward_workspace.argtypes = [i32, i64, i64, out64]
    for name in EXPORTS:
        getattr(lib, name).restype = C.c_int
    _lib = lib
    return lib


def _check(status: int, where: str) -> None:
    if status:
        raise DearError(status, where)


def _dtype(t: torch.Tensor, what: str) -> int:
    if not t.is_cuda:
        raise ValueError("%s is not on a GPU" % what)
    d = _DTYPE.get(t.dtype)
    if d is None:
        raise ValueError("%s is %s: bfloat16 and float32 are supported" % (what, t.dtype))
    return d


def _like(t: torch.Tensor, ref: torch.Tensor, what: str) -> None:
    if t.dtype != ref.dtype or t.device != ref.device:
        raise ValueError("%s is %s on %s, expected %s on %s" % (what, t.dtype, t.device, ref.dtype, ref.device))


class _on:
    """Makes a tensor's device the current one, where it is not, and gives its current stream."""

    def __init__(self, t: torch.Tensor):
        self.index = t.device.index
        self.guard = None if self.index == torch.cuda.current_device() else torch.cuda.device(self.index)

    def __enter__(self) -> int:
        if self.guard is not None:
            self.guard.__enter__()
        return torch.cuda.current_stream(self.index).cuda_stream

    def __exit__(self, *exc) -> None:
        if self.guard is not None:
            self.guard.__exit__(*exc)


# ------------------------------------------------------------------------------------ attention
# dear_attention_t
_ATTENTION = struct.Struct("@4i2q2ifi2Q" + "Q3q" * 4 + "Q" + "Q3q" * 4 + "Qq")
_NONE = (0, 0, 0, 0)


def _readable(t: torch.Tensor, what: str) -> torch.Tensor:
    """The tensor, or a copy of it that the library can read: head_dim contiguous, pieces of 16 bytes."""
    if t.dim() != 4:
        raise ValueError("%s has shape %s, expected [batch, tokens, heads, head_dim]" % (what, tuple(t.shape)))
    unit = 16 // t.element_size()
    s = t.stride()
    # a stride along an axis of one element says nothing, and may be anything
    fine = (s[3] == 1 or t.shape[3] == 1) and t.data_ptr() % 16 == 0 and all(s[i] % unit == 0 for i in range(3) if t.shape[i] > 1)
    return t if fine else t.contiguous().clone() if t.data_ptr() % 16 else t.contiguous()


def _strided(t: torch.Tensor) -> Tuple[int, int, int, int]:
    """Address and strides; strides along axes of one element as 0."""
    s, n = t.stride(), t.shape
    return t.data_ptr(), s[0] if n[0] > 1 else 0, s[1] if n[1] > 1 else 0, s[2] if n[2] > 1 else 0


def _attention_sizes(q, k, v, scale, q_lens, kv_lens):
    d = _dtype(q, "q")
    _like(k, q, "k")
    _like(v, q, "v")
    q, k, v = _readable(q, "q"), _readable(k, "k"), _readable(v, "v")
    B, Sq, H, D = q.shape
    if k.shape != v.shape or k.shape[0] != B or k.shape[3] != D:
        raise ValueError("shapes do not agree: q %s, k %s, v %s" % (tuple(q.shape), tuple(k.shape), tuple(v.shape)))
    for lens, what in ((q_lens, "q_lens"), (kv_lens, "kv_lens")):
        if lens is not None and (lens.dtype != torch.int32 or lens.device != q.device or lens.shape != (B,) or not lens.is_contiguous()):
            raise ValueError("%s: expected a contiguous int32 tensor of %d on %s" % (what, B, q.device))
    scale = 1.0 / math.sqrt(D) if scale is None else float(scale)
    return q, k, v, (B, H, k.shape[2], D, Sq, k.shape[1], d), scale


def _attention_bytes(sizes, scale, causal, q_lens, kv_lens, q, k, v, out, lse, dout=_NONE, dq=_NONE, dk=_NONE, dv=_NONE,
                     workspace=0, workspace_bytes=0) -> bytes:
    return _ATTENTION.pack(*sizes, 1 if causal else 0, scale, 0, 0 if q_lens is None else q_lens.data_ptr(),
                           0 if kv_lens is None else kv_lens.data_ptr(), *q, *k, *v, *out, lse, *dout, *dq, *dk, *dv,
                           workspace, workspace_bytes)


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = False, scale: Optional[float] = None,
              q_lens: Optional[torch.Tensor] = None, kv_lens: Optional[torch.Tensor] = None
              ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of q [B, Sq, H, D] to k, v [B, Sk, Hkv, D], Hkv dividing H, D a multiple of 8 up to 128.

    Gives (out [B, Sq, H, D], lse [B, H, Sq] fp32).  scale: 1 / sqrt(D) by default.  q_lens, kv_lens: int32 [B], the
    valid tokens of each sequence.  causal: the last valid query sees all valid keys, the one before it one less.
    """
    q, k, v, sizes, scale = _attention_sizes(q, k, v, scale, q_lens, kv_lens)
    B, H, _, D, Sq = sizes[:5]
    lib = load_library()
    with _on(q) as stream:
        out = torch.empty((B, Sq, H, D), dtype=q.dtype, device=q.device)
        lse = torch.empty((B, H, Sq), dtype=torch.float32, device=q.device)
        need = C.c_int64()
        args = (sizes, scale, causal, q_lens, kv_lens, _strided(q), _strided(k), _strided(v), _strided(out), lse.data_ptr())
        packed = _attention_bytes(*args)
        _check(lib.dear_attention_workspace(packed, C.byref(need)), "dear_attention_workspace")
        if need.value:
            space = torch.empty(need.value, dtype=torch.uint8, device=q.device)
            packed = _attention_bytes(*args, workspace=space.data_ptr(), workspace_bytes=need.value)
        _check(lib.dear_attention(packed, stream), "dear_attention")
    return out, lse


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                       lse: torch.Tensor, causal: bool = False, scale: Optional[float] = None,
                       q_lens: Optional[torch.Tensor] = None, kv_lens: Optional[torch.Tensor] = None
                       ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Gradients (dq, dk, dv) from the gradient of out and what attention() gave, with the same arguments."""
    q, k, v, sizes, scale = _attention_sizes(q, k, v, scale, q_lens, kv_lens)
    B, H, Hkv, D, Sq, Sk = sizes[:6]
    _like(out, q, "out")
    _like(dout, q, "dout")
    if out.shape != q.shape or dout.shape != q.shape:
        raise ValueError("out %s and dout %s: expected %s" % (tuple(out.shape), tuple(dout.shape), tuple(q.shape)))
    if lse.dtype != torch.float32 or lse.device != q.device or lse.shape != (B, H, Sq) or not lse.is_contiguous():
        raise ValueError("lse: expected a contiguous float32 tensor of shape %s on %s" % ((B, H, Sq), q.device))
    out, dout = _readable(out, "out"), _readable(dout, "dout")
    lib = load_library()
    with _on(q) as stream:
        dq = torch.empty((B, Sq, H, D), dtype=q.dtype, device=q.device)
        dk = torch.empty((B, Sk, Hkv, D), dtype=q.dtype, device=q.device)
        dv = torch.empty((B, Sk, Hkv, D), dtype=q.dtype, device=q.device)
        need = C.c_int64()
        args = (sizes, scale, causal, q_lens, kv_lens, _strided(q), _strided(k), _strided(v), _strided(out), lse.data_ptr(),
                _strided(dout), _strided(dq), _strided(dk), _strided(dv))
        _check(lib.dear_attention_backward_workspace(_attention_bytes(*args), C.byref(need)), "dear_attention_backward_workspace")
        space = torch.empty(need.value, dtype=torch.uint8, device=q.device)
        packed = _attention_bytes(*args, workspace=space.data_ptr(), workspace_bytes=need.value)
        _check(lib.dear_attention_backward(packed, stream), "dear_attention_backward")
    return dq, dk, dv


# ------------------------------------------------------------------------------------ checkpoints
class Checkpoint(NamedTuple):
    """Rows of `cols` values in 8 bits: codes int8 [rows, cols rounded up to 32], exponents uint8 [rows, cols / 32
    rounded up].  value = code * 2 ** (exponent - 127)."""
    codes: torch.Tensor
    exponents: torch.Tensor
    cols: int


def _as_rows(t: torch.Tensor, what: str) -> torch.Tensor:
    """[..., cols] as [rows, cols] with contiguous columns, copied only if its rows lie at no one distance."""
    if t.dim() < 1 or t.shape[-1] < 1:
        raise ValueError("%s has shape %s, expected [..., cols]" % (what, tuple(t.shape)))
    r = t.reshape(-1, t.shape[-1]) if t.dim() != 2 else t
    return r if (r.stride(1) == 1 or r.shape[1] == 1) and (r.shape[0] <= 1 or r.stride(0) >= r.shape[1]) else r.contiguous()


def _stride(r: torch.Tensor) -> int:
    return r.stride(0) if r.shape[0] > 1 else r.shape[1]


def _empty_checkpoint(rows: int, cols: int, device) -> Checkpoint:
    groups = -(-cols // GROUP)
    return Checkpoint(torch.empty((rows, groups * GROUP), dtype=torch.int8, device=device),
                      torch.empty((rows, groups), dtype=torch.uint8, device=device), cols)


def _checkpoint(kept: Checkpoint) -> int:
    """Checks a checkpoint; gives its rows."""
    codes, exponents, cols = kept
    rows, groups = codes.shape[0] if codes.dim() == 2 else -1, -(-cols // GROUP)
    if (cols < 1 or codes.dtype != torch.int8 or exponents.dtype != torch.uint8 or not codes.is_cuda or codes.device != exponents.device
            or codes.shape != (rows, groups * GROUP) or exponents.shape != (rows, groups)
            or not codes.is_contiguous() or not exponents.is_contiguous()):
        raise ValueError("not a checkpoint of %d columns: codes %s %s, exponents %s %s"
                         % (cols, codes.dtype, tuple(codes.shape), exponents.dtype, tuple(exponents.shape)))
    return rows


def checkpoint_encode(x: torch.Tensor) -> Checkpoint:
    """x [..., cols] in 8 bits: 32 neighbours of a row share the smallest power of two with which they fit 127."""
    d = _dtype(x, "x")
    r = _as_rows(x, "x")
    lib = load_library()
    with _on(x) as stream:
        kept = _empty_checkpoint(r.shape[0], r.shape[1], x.device)
        _check(lib.dear_checkpoint_encode(r.data_ptr(), d, r.shape[0], r.shape[1], _stride(r), kept.codes.data_ptr(),
                                          kept.exponents.data_ptr(), stream), "dear_checkpoint_encode")
    return kept


def checkpoint_decode(kept: Checkpoint, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """What a checkpoint holds, [rows, cols]; exact in either type."""
    rows = _checkpoint(kept)
    if dtype not in _DTYPE:
        raise ValueError("%s: bfloat16 and float32 are supported" % dtype)
    lib = load_library()
    with _on(kept.codes) as stream:
        out = torch.empty((rows, kept.cols), dtype=dtype, device=kept.codes.device)
        _check(lib.dear_checkpoint_decode(kept.codes.data_ptr(), kept.exponents.data_ptr(), rows, kept.cols, _DTYPE[dtype],
                                          out.data_ptr(), stream), "dear_checkpoint_decode")
    return out


def checkpoint_weight_grad(dy: torch.Tensor, kept: Checkpoint) -> torch.Tensor:
    """Gradient [outs, ins] in fp32 of a linear layer's weight, from its output's gradient dy [..., outs] and the
    checkpoint of its input [rows, ins]."""
    rows = _checkpoint(kept)
    d = _dtype(dy, "dy")
    r = _as_rows(dy, "dy")
    if r.shape[0] != rows or dy.device != kept.codes.device:
        raise ValueError("dy has %d rows on %s, the checkpoint %d on %s" % (r.shape[0], dy.device, rows, kept.codes.device))
    outs, ins = r.shape[1], kept.cols
    lib = load_library()
    with _on(dy) as stream:
        dw = torch.empty((outs, ins), dtype=torch.float32, device=dy.device)
        need = C.c_int64()
        _check(lib.dear_checkpoint_weight_grad_workspace(d, rows, outs, ins, C.byref(need)), "dear_checkpoint_weight_grad_workspace")
        space = torch.empty(need.value, dtype=torch.uint8, device=dy.device)
        _check(lib.dear_checkpoint_weight_grad(r.data_ptr(), d, _stride(r), kept.codes.data_ptr(), kept.exponents.data_ptr(), rows,
                                               outs, ins, dw.data_ptr(), space.data_ptr(), need.value, stream),
               "dear_checkpoint_weight_grad")
    return dw


# ------------------------------------------------------------------------------------ norm
def _weight(weight: torch.Tensor, cols: int, device) -> None:
    if weight.dtype != torch.float32 or weight.device != device or weight.shape != (cols,) or not weight.is_contiguous():
        raise ValueError("weight: expected a contiguous float32 tensor of %d on %s" % (cols, device))


def add_rms_norm(x: torch.Tensor, residual: Optional[torch.Tensor], weight: torch.Tensor, eps: float = 1e-5,
                 keep: bool = True) -> Tuple[torch.Tensor, torch.Tensor, Optional[Checkpoint], torch.Tensor]:
    """h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight over the last axis.

    Gives (h, y, kept, rstd): h and y of x's type and shape, kept the checkpoint of y in 8 bits (None without `keep`),
    rstd fp32 [rows].  residual None: h is x itself.  weight: fp32.
    """
    d = _dtype(x, "x")
    r = _as_rows(x, "x")
    rows, cols = r.shape
    _weight(weight, cols, x.device)
    add = None
    if residual is not None:
        _like(residual, x, "residual")
        if residual.shape != x.shape:
            raise ValueError("residual has shape %s, x %s" % (tuple(residual.shape), tuple(x.shape)))
        add = _as_rows(residual, "residual")
    lib = load_library()
    with _on(x) as stream:
        h = x if add is None else torch.empty(x.shape, dtype=x.dtype, device=x.device)
        y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        rstd = torch.empty(rows, dtype=torch.float32, device=x.device)
        kept = _empty_checkpoint(rows, cols, x.device) if keep else None
        _check(lib.dear_add_rms_norm(
            r.data_ptr(), _stride(r), None if add is None else add.data_ptr(), 0 if add is None else _stride(add),
            weight.data_ptr(), d, rows, cols, eps, None if add is None else h.data_ptr(), y.data_ptr(),
            kept.codes.data_ptr() if keep else None, kept.exponents.data_ptr() if keep else None, rstd.data_ptr(), stream),
            "dear_add_rms_norm")
    return h, y, kept, rstd


def add_rms_norm_backward(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor,
                          dh: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Gradients (dx, dweight): dx of x and of residual alike, dweight fp32.  dh: the gradient that reaches h by other
    ways than the norm."""
    d = _dtype(dy, "dy")
    given = [(dy, "dy"), (h, "h")] + ([(dh, "dh")] if dh is not None else [])
    for t, what in given[1:]:
        _like(t, dy, what)
        if t.shape != dy.shape:
            raise ValueError("%s has shape %s, dy %s" % (what, tuple(t.shape), tuple(dy.shape)))
    ry, rh = _as_rows(dy, "dy"), _as_rows(h, "h")
    rd = None if dh is None else _as_rows(dh, "dh")
    rows, cols = ry.shape
    _weight(weight, cols, dy.device)
    if rstd.dtype != torch.float32 or rstd.device != dy.device or rstd.shape != (rows,) or not rstd.is_contiguous():
        raise ValueError("rstd: expected a contiguous float32 tensor of %d on %s" % (rows, dy.device))
    lib = load_library()
    with _on(dy) as stream:
        dx = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
        dweight = torch.empty(cols, dtype=torch.float32, device=dy.device)
        need = C.c_int64()
        _check(lib.dear_add_rms_norm_backward_workspace(d, rows, cols, C.byref(need)), "dear_add_rms_norm_backward_workspace")
        space = torch.empty(need.value, dtype=torch.uint8, device=dy.device)
        _check(lib.dear_add_rms_norm_backward(
            ry.data_ptr(), _stride(ry), rh.data_ptr(), _stride(rh), None if rd is None else rd.data_ptr(),
            0 if rd is None else _stride(rd), weight.data_ptr(), rstd.data_ptr(), d, rows, cols, dx.data_ptr(),
            dweight.data_ptr(), space.data_ptr(), need.value, stream), "dear_add_rms_norm_backward")
    return dx, dweight
