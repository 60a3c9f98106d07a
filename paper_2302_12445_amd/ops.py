"""Training operators on torch tensors: binding of libdear_ops.so (include/dear_ops.h).

    out, lse = attention(q, k, v, causal=True)                       # [B, S, H, D]
    dq, dk, dv = attention_backward(dout, q, k, v, out, lse, causal=True)
    h, y, kept, rstd = add_rms_norm(x, residual, weight, eps)        # kept: y in 8 bits
    dx, dweight = add_rms_norm_backward(dy, h, weight, rstd, dh=dh)
    kept = checkpoint_encode(x); x = checkpoint_decode(kept, dtype)
    dw = checkpoint_weight_grad(dy, kept)                            # fp32 [outs, ins]
    h, last, kept = recurrence(x, gate, state)                       # [B, T, C]; last: fp32 [B, C]
    dx, dgate, dstate = recurrence_backward(dh, x, gate, kept)
    y = expert_linear(x, weight, ends)                               # rows sorted by expert; weight [E, outs, ins]
    dx, dw = expert_input_grad(dy, weight, ends), expert_weight_grad(dy, x, ends)
    norm = clip_grads(grads, max_norm)                               # of all tensors of a list, in place; grad_norm(grads)

Tensors are on a GPU, bf16 or fp32.  Work is enqueued on the current torch stream of the tensors'
device; outputs and workspaces come from torch's allocator.  Wrong arguments raise ValueError or
DearError before anything is launched.  There is no CPU fallback: if the library is missing,
loading raises.  layers.py has the autograd functions over these calls.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import os
import struct
from typing import NamedTuple, Optional, Sequence, Tuple

import torch

from .binding import DEAR_BF16, DEAR_F32, DearError

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdear_ops.so")
GROUP = 32  # DEAR_CHECKPOINT_GROUP
NORM_MAX_COLS = 32768
KEPT = 256  # DEAR_RECURRENCE_KEPT

EXPORTS = [
    "dear_attention", "dear_attention_workspace", "dear_attention_backward", "dear_attention_backward_workspace",
    "dear_checkpoint_encode", "dear_checkpoint_decode", "dear_checkpoint_weight_grad", "dear_checkpoint_weight_grad_workspace",
    "dear_add_rms_norm", "dear_add_rms_norm_backward", "dear_add_rms_norm_backward_workspace",
    "dear_recurrence", "dear_recurrence_backward", "dear_recurrence_workspace",
    "dear_expert_linear", "dear_expert_input_grad", "dear_expert_weight_grad", "dear_expert_linear_workspace",
    "dear_expert_input_grad_workspace", "dear_expert_weight_grad_workspace",
    "dear_grad_norm", "dear_clip_grads", "dear_grad_norm_workspace",
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
    # structures are passed as the bytes that struct packs
    for name in ("dear_attention", "dear_attention_backward", "dear_recurrence", "dear_recurrence_backward", "dear_expert_linear",
                 "dear_expert_input_grad", "dear_expert_weight_grad"):
        getattr(lib, name).argtypes = [C.c_char_p, vp]
    for name in ("dear_attention_workspace", "dear_attention_backward_workspace", "dear_recurrence_workspace",
                 "dear_expert_linear_workspace", "dear_expert_input_grad_workspace", "dear_expert_weight_grad_workspace"):
        getattr(lib, name).argtypes = [C.c_char_p, out64]
    lib.dear_grad_norm.argtypes = [C.c_char_p, i64, vp, vp, i64, vp]
    lib.dear_clip_grads.argtypes = [C.c_char_p, i64, f32, vp, vp, i64, vp]
    lib.dear_grad_norm_workspace.argtypes = [i64, out64]
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


# neither is a name that torch promises to keep
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
_current_device = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device


def _elsewhere(t: torch.Tensor) -> bool:
    """Whether the call has to be made again with the tensor's device as the current one."""
    return t.is_cuda and t.get_device() != _current_device()


@functools.lru_cache(maxsize=1024)
def _attention_workspace(name: str, *head) -> int:
    need = C.c_int64()
    _check(getattr(load_library(), name)(_ATTENTION.pack(*head, *([0] * 37)), C.byref(need)), name)
    return need.value


@functools.lru_cache(maxsize=1024)
def _packed_workspace(name: str, layout: struct.Struct, members: int, *head) -> int:
    """Bytes that a call with a structure of these leading members needs."""
    need = C.c_int64()
    _check(getattr(load_library(), name)(layout.pack(*head, *([0] * (members - len(head)))), C.byref(need)), name)
    return need.value


@functools.lru_cache(maxsize=1024)
def _workspace(name: str, *sizes) -> int:
    """Bytes that a call of these sizes needs."""
    need = C.c_int64()
    _check(getattr(load_library(), name)(*sizes, C.byref(need)), name)
    return need.value


# ------------------------------------------------------------------------------------ attention
# dear_attention_t
_ATTENTION = struct.Struct("@4i2q2ifi2Q" + "Q3q" * 4 + "Q" + "Q3q" * 4 + "Qq")
_NONE = (0, 0, 0, 0)
_F32_MAX = (2 - 2 ** -23) * 2.0 ** 127


def _readable(t: torch.Tensor, what: str):
    """The tensor, or a copy of it that the library can read (head_dim contiguous, pieces of 16 bytes), and its address and
    strides, those along axes of one element, which say nothing, as 0."""
    n = t.shape
    if len(n) != 4:
        raise ValueError("%s has shape %s, expected [batch, tokens, heads, head_dim]" % (what, tuple(n)))
    at, unit = t.data_ptr(), 16 // t.element_size()
    if not t.is_contiguous() or at % 16:
        s = t.stride()
        batch, token, head = s[0] if n[0] > 1 else 0, s[1] if n[1] > 1 else 0, s[2] if n[2] > 1 else 0
        if (s[3] == 1 or n[3] == 1) and at % 16 == 0 and batch % unit == 0 and token % unit == 0 and head % unit == 0:
            return t, (at, batch, token, head)
        t = t.clone(memory_format=torch.contiguous_format)
        at = t.data_ptr()
    return t, (at, n[1] * n[2] * n[3], n[2] * n[3], n[3])


def _empty_as(t: torch.Tensor) -> torch.Tensor:
    """A contiguous output of a tensor's shape and type."""
    return torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=t.dtype, device=t.device)


def _new(like: torch.Tensor, shape):
    """A contiguous output of the shape, and its address and strides."""
    t = _empty_as(like) if like.shape == shape else torch.empty(shape, dtype=like.dtype, device=like.device)
    return t, (t.data_ptr(), shape[1] * shape[2] * shape[3], shape[2] * shape[3], shape[3])


def _attention_sizes(q, k, v, causal, scale, q_lens, kv_lens):
    """(q, k, v) as the library reads them, their places, and the leading members of dear_attention_t."""
    d = _dtype(q, "q")
    _like(k, q, "k")
    _like(v, q, "v")
    (q, pq), (k, pk), (v, pv) = _readable(q, "q"), _readable(k, "k"), _readable(v, "v")
    B, Sq, H, D = q.shape
    Bk, Sk, Hkv, Dk = k.shape
    if k.shape != v.shape or Bk != B or Dk != D:
        raise ValueError("shapes do not agree: q %s, k %s, v %s" % (tuple(q.shape), tuple(k.shape), tuple(v.shape)))
    for lens, what in ((q_lens, "q_lens"), (kv_lens, "kv_lens")):
        if lens is not None and (lens.dtype != torch.int32 or lens.device != q.device or lens.shape != (B,) or not lens.is_contiguous()):
            raise ValueError("%s: expected a contiguous int32 tensor of %d on %s" % (what, B, q.device))
    # (head_dim 0 is refused by the library)
    scale = 1.0 / math.sqrt(D or 1) if scale is None else float(scale)
    if _F32_MAX < abs(scale) < math.inf:  # (others are the library's to refuse)
        raise ValueError("scale %g: fp32 does not hold it" % scale)
    return (q, k, v), (*pq, *pk, *pv), (B, H, Hkv, D, Sq, Sk, d, 1 if causal else 0, scale, 0,
                                        0 if q_lens is None else q_lens.data_ptr(), 0 if kv_lens is None else kv_lens.data_ptr())


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = False, scale: Optional[float] = None,
              q_lens: Optional[torch.Tensor] = None, kv_lens: Optional[torch.Tensor] = None
              ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Attention of q [B, Sq, H, D] to k, v [B, Sk, Hkv, D], Hkv dividing H, D a multiple of 8 up to 128.

    Gives (out [B, Sq, H, D], lse [B, H, Sq] fp32).  scale: 1 / sqrt(D) by default.  q_lens, kv_lens: int32 [B], the
    valid tokens of each sequence.  causal: the last valid query sees all valid keys, the one before it one less.
    """
    if _elsewhere(q):
        with torch.cuda.device(q.device):
            return attention(q, k, v, causal, scale, q_lens, kv_lens)
    kept, places, head = _attention_sizes(q, k, v, causal, scale, q_lens, kv_lens)  # kept: until the work is enqueued
    B, H, _, D, Sq = head[:5]
    lib = load_library()
    out, po = _new(q, (B, Sq, H, D))
    lse = torch.empty((B, H, Sq), dtype=torch.float32, device=q.device)
    need, space = _attention_workspace("dear_attention_workspace", *head[:10]), None
    if need:
        space = torch.empty(need, dtype=torch.uint8, device=q.device)
    _check(lib.dear_attention(_ATTENTION.pack(*head, *places, *po, lse.data_ptr(), *_NONE, *_NONE, *_NONE, *_NONE,
                                              space.data_ptr() if need else 0, need), _raw_stream(q.get_device())), "dear_attention")
    return out, lse


def attention_backward(dout: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                       lse: torch.Tensor, causal: bool = False, scale: Optional[float] = None,
                       q_lens: Optional[torch.Tensor] = None, kv_lens: Optional[torch.Tensor] = None
                       ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Gradients (dq, dk, dv) from the gradient of out and what attention() gave, with the same arguments."""
    if _elsewhere(dout):
        with torch.cuda.device(dout.device):
            return attention_backward(dout, q, k, v, out, lse, causal, scale, q_lens, kv_lens)
    kept, places, head = _attention_sizes(q, k, v, causal, scale, q_lens, kv_lens)
    B, H, Hkv, D, Sq, Sk = head[:6]
    _like(out, q, "out")
    _like(dout, q, "dout")
    if out.shape != q.shape or dout.shape != q.shape:
        raise ValueError("out %s and dout %s: expected %s" % (tuple(out.shape), tuple(dout.shape), tuple(q.shape)))
    if lse.dtype != torch.float32 or lse.device != q.device or lse.shape != (B, H, Sq) or not lse.is_contiguous():
        raise ValueError("lse: expected a contiguous float32 tensor of shape %s on %s" % ((B, H, Sq), q.device))
    (out, po), (dout, pd) = _readable(out, "out"), _readable(dout, "dout")
    lib = load_library()
    (dq, gq), (dk, gk), (dv, gv) = _new(q, (B, Sq, H, D)), _new(k, (B, Sk, Hkv, D)), _new(v, (B, Sk, Hkv, D))
    need = _attention_workspace("dear_attention_backward_workspace", *head[:10])
    space = torch.empty(need, dtype=torch.uint8, device=q.device)
    _check(lib.dear_attention_backward(_ATTENTION.pack(*head, *places, *po, lse.data_ptr(), *pd, *gq, *gk, *gv, space.data_ptr(), need),
                                       _raw_stream(q.get_device())), "dear_attention_backward")
    return dq, dk, dv


# ------------------------------------------------------------------------------------ checkpoints
class Checkpoint(NamedTuple):
    """Rows of `cols` values in 8 bits: codes int8 [rows, cols rounded up to 32], exponents uint8 [rows, cols / 32
    rounded up].  value = code * 2 ** (exponent - 127)."""
    codes: torch.Tensor
    exponents: torch.Tensor
    cols: int


def _as_rows(t: torch.Tensor, what: str) -> Tuple[torch.Tensor, int, int, int]:
    """[..., cols] as rows of contiguous columns, copied only if the rows lie at no one distance: the tensor, rows, cols,
    elements from row to row."""
    n = t.shape
    if not n or n[-1] < 1:
        raise ValueError("%s has shape %s, expected [..., cols]" % (what, tuple(n)))
    cols = n[-1]
    if t.is_contiguous():
        return t, t.numel() // cols, cols, cols
    r = t if len(n) == 2 else t.reshape(-1, cols)
    if (r.stride(1) != 1 and cols > 1) or (r.shape[0] > 1 and r.stride(0) < cols):
        r = r.contiguous()
    return r, r.shape[0], cols, r.stride(0) if r.shape[0] > 1 else cols


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
    if _elsewhere(x):
        with torch.cuda.device(x.device):
            return checkpoint_encode(x)
    d = _dtype(x, "x")
    r, rows, cols, stride = _as_rows(x, "x")
    kept = _empty_checkpoint(rows, cols, x.device)
    _check(load_library().dear_checkpoint_encode(r.data_ptr(), d, rows, cols, stride, kept.codes.data_ptr(), kept.exponents.data_ptr(),
                                                 _raw_stream(x.get_device())), "dear_checkpoint_encode")
    return kept


def checkpoint_decode(kept: Checkpoint, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """What a checkpoint holds, [rows, cols]; exact in either type."""
    if _elsewhere(kept.codes):
        with torch.cuda.device(kept.codes.device):
            return checkpoint_decode(kept, dtype)
    rows = _checkpoint(kept)
    if dtype not in _DTYPE:
        raise ValueError("%s: bfloat16 and float32 are supported" % dtype)
    codes, exponents, cols = kept
    out = torch.empty((rows, cols), dtype=dtype, device=codes.device)
    _check(load_library().dear_checkpoint_decode(codes.data_ptr(), exponents.data_ptr(), rows, cols, _DTYPE[dtype], out.data_ptr(),
                                                 _raw_stream(codes.get_device())), "dear_checkpoint_decode")
    return out


def checkpoint_weight_grad(dy: torch.Tensor, kept: Checkpoint) -> torch.Tensor:
    """Gradient [outs, ins] in fp32 of a linear layer's weight, from its output's gradient dy [..., outs] and the
    checkpoint of its input [rows, ins]."""
    if _elsewhere(dy):
        with torch.cuda.device(dy.device):
            return checkpoint_weight_grad(dy, kept)
    rows = _checkpoint(kept)
    d = _dtype(dy, "dy")
    r, dy_rows, outs, stride = _as_rows(dy, "dy")
    codes, exponents, ins = kept
    if dy_rows != rows or dy.device != codes.device:
        raise ValueError("dy has %d rows on %s, the checkpoint %d on %s" % (dy_rows, dy.device, rows, codes.device))
    lib = load_library()
    dw = torch.empty((outs, ins), dtype=torch.float32, device=dy.device)
    need, space = _workspace("dear_checkpoint_weight_grad_workspace", d, rows, outs, ins), None
    if need:
        space = torch.empty(need, dtype=torch.uint8, device=dy.device)
    _check(lib.dear_checkpoint_weight_grad(r.data_ptr(), d, stride, codes.data_ptr(), exponents.data_ptr(), rows, outs, ins, dw.data_ptr(),
                                           space.data_ptr() if need else None, need, _raw_stream(dy.get_device())),
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
    if _elsewhere(x):
        with torch.cuda.device(x.device):
            return add_rms_norm(x, residual, weight, eps, keep)
    d = _dtype(x, "x")
    r, rows, cols, stride = _as_rows(x, "x")
    device, shape = x.device, x.shape
    _weight(weight, cols, device)
    h, h_at, add, add_at, add_stride = x, None, None, None, 0
    if residual is not None:
        _like(residual, x, "residual")
        if residual.shape != shape:
            raise ValueError("residual has shape %s, x %s" % (tuple(residual.shape), tuple(shape)))
        add, _, _, add_stride = _as_rows(residual, "residual")
        h = _empty_as(x)
        h_at, add_at = h.data_ptr(), add.data_ptr()
    y = _empty_as(x)
    rstd = torch.empty(rows, dtype=torch.float32, device=device)
    kept = _empty_checkpoint(rows, cols, device) if keep else None
    _check(load_library().dear_add_rms_norm(
        r.data_ptr(), stride, add_at, add_stride, weight.data_ptr(), d, rows, cols, eps, h_at, y.data_ptr(),
        kept.codes.data_ptr() if keep else None, kept.exponents.data_ptr() if keep else None, rstd.data_ptr(),
        _raw_stream(x.get_device())), "dear_add_rms_norm")
    return h, y, kept, rstd


def add_rms_norm_backward(dy: torch.Tensor, h: torch.Tensor, weight: torch.Tensor, rstd: torch.Tensor,
                          dh: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Gradients (dx, dweight): dx of x and of residual alike, dweight fp32.  dh: the gradient that reaches h by other
    ways than the norm."""
    if _elsewhere(dy):
        with torch.cuda.device(dy.device):
            return add_rms_norm_backward(dy, h, weight, rstd, dh)
    d = _dtype(dy, "dy")
    device, shape = dy.device, dy.shape
    for t, what in ((h, "h"), (dh, "dh")):
        if t is not None:
            _like(t, dy, what)
            if t.shape != shape:
                raise ValueError("%s has shape %s, dy %s" % (what, tuple(t.shape), tuple(shape)))
    ry, rows, cols, dy_stride = _as_rows(dy, "dy")
    rh, _, _, h_stride = _as_rows(h, "h")
    rd, _, _, dh_stride = (None, 0, 0, 0) if dh is None else _as_rows(dh, "dh")
    _weight(weight, cols, device)
    if rstd.dtype != torch.float32 or rstd.device != device or rstd.shape != (rows,) or not rstd.is_contiguous():
        raise ValueError("rstd: expected a contiguous float32 tensor of %d on %s" % (rows, device))
    lib = load_library()
    dx = _empty_as(dy)
    dweight = torch.empty(cols, dtype=torch.float32, device=device)
    need = _workspace("dear_add_rms_norm_backward_workspace", d, rows, cols)
    space = torch.empty(need, dtype=torch.uint8, device=device)
    _check(lib.dear_add_rms_norm_backward(
        ry.data_ptr(), dy_stride, rh.data_ptr(), h_stride, None if rd is None else rd.data_ptr(), dh_stride, weight.data_ptr(),
        rstd.data_ptr(), d, rows, cols, dx.data_ptr(), dweight.data_ptr(), space.data_ptr(), need, _raw_stream(dy.get_device())),
        "dear_add_rms_norm_backward")
    return dx, dweight


# ------------------------------------------------------------------------------------ recurrence
# dear_recurrence_t
_RECURRENCE = struct.Struct("@2iq2iQ" + "Q2q" * 2 + "2Q" + "Q2q" + "Q" + "Q2q" + "Q" + "Q2q" * 2 + "2Qq")
_RECURRENCE_MEMBERS = 6 + 6 + 2 + 3 + 1 + 3 + 1 + 6 + 3
_MAX_STEP_STRIDE = 1 << 22
_NO_STEPS = (0, 0, 0)


def _steps(t: torch.Tensor, what: str):
    """The tensor, or a copy of it that the library can read (channels contiguous), and its address and strides, those along axes
    of one element, which say nothing, as 0."""
    n = t.shape
    if len(n) != 3 or n[2] < 1:
        raise ValueError("%s has shape %s, expected [batch, steps, channels]" % (what, tuple(n)))
    s = t.stride()
    batch, step = s[0] if n[0] > 1 else 0, s[1] if n[1] > 1 else 0
    if (s[2] != 1 and n[2] > 1) or step >= _MAX_STEP_STRIDE:
        t = t.clone(memory_format=torch.contiguous_format)
        batch, step = n[1] * n[2] if n[0] > 1 else 0, n[2] if n[1] > 1 else 0
    return t, (t.data_ptr(), batch, step)


def _new_steps(like: torch.Tensor):
    t = _empty_as(like)
    n = t.shape
    return t, (t.data_ptr(), n[1] * n[2], n[2])


def _state(t: Optional[torch.Tensor], shape, device, what: str) -> int:
    """The address of fp32 values of the shape, 0 for None."""
    if t is None:
        return 0
    if t.dtype != torch.float32 or t.device != device or t.shape != shape or not t.is_contiguous():
        raise ValueError("%s: expected a contiguous float32 tensor of shape %s on %s" % (what, tuple(shape), device))
    return t.data_ptr()


def _recurrence_sizes(x, gate, lens):
    """(x, gate) as the library reads them, their places, and the leading members of dear_recurrence_t."""
    d = _dtype(x, "x")
    _like(gate, x, "gate")
    if gate.shape != x.shape:
        raise ValueError("gate has shape %s, x %s" % (tuple(gate.shape), tuple(x.shape)))
    (x, px), (gate, pg) = _steps(x, "x"), _steps(gate, "gate")
    B, T, channels = x.shape
    if lens is not None and (lens.dtype != torch.int32 or lens.device != x.device or lens.shape != (B,) or not lens.is_contiguous()):
        raise ValueError("lens: expected a contiguous int32 tensor of %d on %s" % (B, x.device))
    return (x, gate), (*px, *pg), (B, channels, T, d, 0, 0 if lens is None else lens.data_ptr())


def _recurrence_space(head, device):
    need = _packed_workspace("dear_recurrence_workspace", _RECURRENCE, _RECURRENCE_MEMBERS, *head[:5])
    space = torch.empty(need, dtype=torch.uint8, device=device) if need else None
    return space, space.data_ptr() if need else 0, need


def recurrence(x: torch.Tensor, gate: torch.Tensor, state: Optional[torch.Tensor] = None, lens: Optional[torch.Tensor] = None,
               keep: bool = True) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor]]:
    """Gated linear recurrence s[t] = a * s[t-1] + (1 - a) * x[t] with a = sigmoid(gate[t]), channel by channel, of x and gate [B, T, C].

    Gives (h, last, kept): h[t] = s[t], of x's type; last fp32 [B, C], the state behind the last step, which a call on the next steps
    (one token, or many) takes as `state`; kept fp32 [B, ceil(T / 256), C] for recurrence_backward (None without `keep`).
    state: fp32 [B, C] before the first step, zeros by default.  lens: int32 [B], the valid steps of each sequence; behind them h is 0.
    """
    if _elsewhere(x):
        with torch.cuda.device(x.device):
            return recurrence(x, gate, state, lens, keep)
    held, places, head = _recurrence_sizes(x, gate, lens)  # held: until the work is enqueued
    B, channels, T = head[:3]
    at = _state(state, (B, channels), x.device, "state")
    h, ph = _new_steps(x)
    last = torch.empty((B, channels), dtype=torch.float32, device=x.device)
    kept = torch.empty((B, -(-T // KEPT), channels), dtype=torch.float32, device=x.device) if keep else None
    space, space_at, need = _recurrence_space(head, x.device)
    packed = _RECURRENCE.pack(*head, *places, at, kept.data_ptr() if keep else 0, *ph, last.data_ptr(), *_NO_STEPS, 0, *_NO_STEPS, *_NO_STEPS, 0,
                              space_at, need)
    _check(load_library().dear_recurrence(packed, _raw_stream(x.get_device())), "dear_recurrence")
    return h, last, kept


def recurrence_backward(dh: torch.Tensor, x: torch.Tensor, gate: torch.Tensor, kept: torch.Tensor, lens: Optional[torch.Tensor] = None,
                        dlast: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Gradients (dx, dgate, dstate) from the gradient of h, what recurrence() kept, and its arguments; dstate is fp32 [B, C], of the state
    before the first step.  dlast: fp32 [B, C], the gradient of last."""
    if _elsewhere(dh):
        with torch.cuda.device(dh.device):
            return recurrence_backward(dh, x, gate, kept, lens, dlast)
    held, places, head = _recurrence_sizes(x, gate, lens)
    B, channels, T = head[:3]
    _like(dh, x, "dh")
    if dh.shape != x.shape:
        raise ValueError("dh has shape %s, x %s" % (tuple(dh.shape), tuple(x.shape)))
    dh, pd = _steps(dh, "dh")
    kept_at = _state(kept, (B, -(-T // KEPT), channels), x.device, "kept")
    dlast_at = _state(dlast, (B, channels), x.device, "dlast")
    (dx, px), (dgate, pg) = _new_steps(x), _new_steps(gate)
    dstate = torch.empty((B, channels), dtype=torch.float32, device=x.device)
    space, space_at, need = _recurrence_space(head, x.device)
    packed = _RECURRENCE.pack(*head, *places, 0, kept_at, *_NO_STEPS, 0, *pd, dlast_at, *px, *pg, dstate.data_ptr(), space_at, need)
    _check(load_library().dear_recurrence_backward(packed, _raw_stream(x.get_device())), "dear_recurrence_backward")
    return dx, dgate, dstate


# ------------------------------------------------------------------------------------ experts
# dear_experts_t
_EXPERTS = struct.Struct("@q4i2Qq2Qq2Qq")
_EXPERTS_MEMBERS = 14


def _expert_rows(t: torch.Tensor, what: str):
    if t.dim() != 2:
        raise ValueError("%s has shape %s, expected [rows, width]" % (what, tuple(t.shape)))
    return _as_rows(t, what)


def _expert_ends(ends: torch.Tensor, experts: int, device) -> None:
    if ends.dtype != torch.int32 or ends.device != device or ends.shape != (experts,) or not ends.is_contiguous():
        raise ValueError("ends: expected a contiguous int32 tensor of %d on %s" % (experts, device))


def _expert_weight(weight: torch.Tensor, rows: torch.Tensor, axis: int, what: str) -> torch.Tensor:
    """A weight [experts, outs, ins] that rows are multiplied with along one of its axes."""
    _like(weight, rows, "weight")
    if weight.dim() != 3 or weight.shape[axis] != rows.shape[1]:
        raise ValueError("weight has shape %s, %s %s" % (tuple(weight.shape), what, tuple(rows.shape)))
    return weight.contiguous()


def _expert_call(name: str, head, ends, x, x_stride, weight, dy, dy_stride, out) -> None:
    need, space = _packed_workspace(name + "_workspace", _EXPERTS, _EXPERTS_MEMBERS, *head), None
    if need:
        space = torch.empty(need, dtype=torch.uint8, device=out.device)
    packed = _EXPERTS.pack(*head, ends.data_ptr(), x, x_stride, weight, dy, dy_stride, out.data_ptr(), space.data_ptr() if need else 0, need)
    _check(getattr(load_library(), name)(packed, _raw_stream(out.get_device())), name)


def expert_linear(x: torch.Tensor, weight: torch.Tensor, ends: torch.Tensor) -> torch.Tensor:
    """y [rows, outs] of x [rows, ins], sorted by expert, and weight [experts, outs, ins]: expert e has the rows ends[e-1] .. ends[e] - 1.

    ends: int32 [experts], on the GPU; an expert may have no rows, and rows behind the last one's are 0 in y.
    """
    if _elsewhere(x):
        with torch.cuda.device(x.device):
            return expert_linear(x, weight, ends)
    d = _dtype(x, "x")
    r, rows, ins, stride = _expert_rows(x, "x")
    w = _expert_weight(weight, x, 2, "x")
    experts, outs = w.shape[:2]
    _expert_ends(ends, experts, x.device)
    y = torch.empty((rows, outs), dtype=x.dtype, device=x.device)
    _expert_call("dear_expert_linear", (rows, experts, outs, ins, d), ends, r.data_ptr(), stride, w.data_ptr(), 0, 0, y)
    return y


def expert_input_grad(dy: torch.Tensor, weight: torch.Tensor, ends: torch.Tensor) -> torch.Tensor:
    """Gradient [rows, ins] of expert_linear's x from that of its y."""
    if _elsewhere(dy):
        with torch.cuda.device(dy.device):
            return expert_input_grad(dy, weight, ends)
    d = _dtype(dy, "dy")
    r, rows, outs, stride = _expert_rows(dy, "dy")
    w = _expert_weight(weight, dy, 1, "dy")
    experts, _, ins = w.shape
    _expert_ends(ends, experts, dy.device)
    dx = torch.empty((rows, ins), dtype=dy.dtype, device=dy.device)
    _expert_call("dear_expert_input_grad", (rows, experts, outs, ins, d), ends, 0, 0, w.data_ptr(), r.data_ptr(), stride, dx)
    return dx


def expert_weight_grad(dy: torch.Tensor, x: torch.Tensor, ends: torch.Tensor) -> torch.Tensor:
    """Gradient [experts, outs, ins] in fp32 of expert_linear's weight from x and the gradient of y."""
    if _elsewhere(dy):
        with torch.cuda.device(dy.device):
            return expert_weight_grad(dy, x, ends)
    d = _dtype(dy, "dy")
    _like(x, dy, "x")
    ry, rows, outs, dy_stride = _expert_rows(dy, "dy")
    rx, x_rows, ins, x_stride = _expert_rows(x, "x")
    if x_rows != rows:
        raise ValueError("dy has %d rows, x %d" % (rows, x_rows))
    experts = ends.numel()
    _expert_ends(ends, experts, dy.device)
    dw = torch.empty((experts, outs, ins), dtype=torch.float32, device=dy.device)
    _expert_call("dear_expert_weight_grad", (rows, experts, outs, ins, d), ends, rx.data_ptr(), x_stride, 0, ry.data_ptr(), dy_stride, dw)
    return dw


# ------------------------------------------------------------------------------------ gradients
_GRAD_MEMBERS = "2Q2q"  # dear_grad_t, its two types as one number
_dtype_of = torch.Tensor.dtype.__get__


@functools.lru_cache(maxsize=256)
def _grad_layout(count: int) -> struct.Struct:
    return struct.Struct("@" + _GRAD_MEMBERS * count)


def _dense(t: torch.Tensor) -> bool:
    """Whether the elements fill one stretch of memory, in whatever order of axes."""
    if t.is_contiguous():
        return True
    span = 1
    for stride, n in sorted((s, n) for s, n in zip(t.stride(), t.shape) if n != 1):
        if stride != span:
            return False
        span *= n
    return True


def _grad_norm(tensors: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]], max_norm: Optional[float]) -> torch.Tensor:
    tensors = list(tensors)
    if not tensors:
        raise ValueError("no tensors")
    clip = max_norm is not None
    outs = tensors if out is None else list(out)
    if len(outs) != len(tensors):
        raise ValueError("%d tensors and %d outputs" % (len(tensors), len(outs)))
    first = tensors[0]
    if _elsewhere(first):
        with torch.cuda.device(first.device):
            return _grad_norm(tensors, None if out is None else outs, max_norm)
    # a list at a time: a model has some hundred tensors, and each question to one takes the host some 50 ns
    index, count = first.get_device(), len(tensors)
    here, kinds = set(map(torch.Tensor.get_device, tensors)), set(map(_dtype_of, tensors))
    out_kinds = kinds if outs is tensors else set(map(_dtype_of, outs))
    if outs is not tensors:
        here.update(map(torch.Tensor.get_device, outs))
    if len(here) > 1 or index < 0 or not all(k in _DTYPE for k in kinds | out_kinds):
        for t in tensors:
            _dtype(t, "a gradient")
        for t in outs:
            _dtype(t, "an output")
        raise ValueError("tensors are on several devices")
    sizes = list(map(torch.Tensor.numel, tensors))
    if outs is not tensors and sizes != list(map(torch.Tensor.numel, outs)):
        raise ValueError("an output has more or fewer elements than its gradient")
    if not all(map(torch.Tensor.is_contiguous, tensors)) or not (outs is tensors or all(map(torch.Tensor.is_contiguous, outs))):
        if any(o.shape != g.shape for o, g in zip(outs, tensors)):
            raise ValueError("tensors that are not contiguous: an output has another shape than its gradient")
        if clip and not all(_dense(o) for o in outs):
            raise ValueError("an output has gaps between its elements")
        # elements in the outputs' order
        tensors = [g if _dense(g) and (g.stride() == o.stride() or not clip) else
                   torch.empty_strided(o.shape, o.stride(), dtype=g.dtype, device=g.device).copy_(g) if clip else g.contiguous()
                   for g, o in zip(tensors, outs)]
    lib = load_library()
    norm = torch.empty((), dtype=torch.float32, device=first.device)
    need = _workspace("dear_grad_norm_workspace", count)
    space = torch.empty(need, dtype=torch.uint8, device=first.device)
    members = [0] * (4 * count)
    members[::4] = places = list(map(torch.Tensor.data_ptr, tensors))
    members[1::4] = places if outs is tensors else map(torch.Tensor.data_ptr, outs)
    members[2::4] = sizes
    if len(kinds) == 1 and len(out_kinds) == 1:
        members[3::4] = [_DTYPE[first.dtype] | _DTYPE[outs[0].dtype] << 32] * count
    else:
        members[3::4] = [_DTYPE[g.dtype] | _DTYPE[o.dtype] << 32 for g, o in zip(tensors, outs)]
    packed, stream = _grad_layout(count).pack(*members), _raw_stream(index)
    if clip:
        _check(lib.dear_clip_grads(packed, count, max_norm, norm.data_ptr(), space.data_ptr(), need, stream), "dear_clip_grads")
        torch.autograd.graph.increment_version(outs)
    else:
        _check(lib.dear_grad_norm(packed, count, norm.data_ptr(), space.data_ptr(), need, stream), "dear_grad_norm")
    return norm


def grad_norm(tensors: Sequence[torch.Tensor]) -> torch.Tensor:
    """The norm over all elements of the tensors (bf16 or fp32, also both), fp32, on their GPU."""
    return _grad_norm(tensors, None, None)


def clip_grads(tensors: Sequence[torch.Tensor], max_norm: float, out: Optional[Sequence[torch.Tensor]] = None) -> torch.Tensor:
    """Scales the tensors by min(1, max_norm / norm), with norm that over all of them, and gives norm.

    In place, or into `out`: tensors of the same shapes or, contiguous ones, of as many elements (slices of a flat buffer), bf16 or fp32 each,
    so that fp32 gradients can be had of bf16 ones.  Nothing is written that need not change.  The norm stays on the GPU: nothing waits for it.
    """
    max_norm = float(max_norm)
    if not max_norm > 0:
        raise ValueError("max_norm %g: expected a number above 0" % max_norm)
    return _grad_norm(tensors, out, max_norm)
