"""The recurrence, the products grouped by expert and the gradient norm from their definitions, in 64 bits on the CPU, and how far a
result may be from them.

Bounds.  U and R as in ops_reference.py.  Each bound follows an error through the formulas to first order."""
from __future__ import annotations

import torch

from ops_reference import R, U, f64

KEPT = 256


# ------------------------------------------------------------------------------------ recurrence
def gates(gate):
    """a, 1 - a, and their relative errors: the exponential's argument is rounded (|g| U), it, the sum, the reciprocal and the product
    are within a step or two; of the larger of the two only as much of the exponential's error counts as it has a share in it."""
    g = f64(gate)
    a, b = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))
    small = (8 + 2 * torch.where(torch.isfinite(g), g.abs(), 0.0)) * U
    a_off = torch.where(g >= 0, 4 * U + b * small, small)
    b_off = torch.where(g >= 0, small, 4 * U + a * small)
    return a, b, a_off, b_off


def _lens(lens, B, T):
    return [T if lens is None else min(max(int(lens[b]), 0), T) for b in range(B)]


def _valid(lens, B, T):
    return torch.arange(T).view(1, T) < torch.tensor(_lens(lens, B, T)).view(B, 1)


def recurrence(x, gate, state, lens):
    """(h, last, kept) and their bounds.  Of a sum's term the error grows by that of a and by a rounding at each step it passes, and by
    a rounding for each level that joins stretches: within a strip, a wave, a workgroup, and the tiles."""
    dtype, (B, T, C) = x.dtype, x.shape
    valid = _valid(lens, B, T)
    a, b, a_off, b_off = gates(gate)
    x = f64(x)
    s = torch.zeros(B, C, dtype=torch.float64) if state is None else f64(state)
    size, off = s.abs(), torch.zeros_like(s)
    h, h_off = torch.zeros_like(x), torch.zeros_like(x)
    kept, kept_off = [], []
    joins = (32 + -(-T // KEPT)) * U
    for t in range(T):
        if t % KEPT == 0:
            kept.append(s), kept_off.append(off + joins * size + 1e-30)
        v = valid[:, t:t + 1]
        off = torch.where(v, a[:, t] * off + a[:, t] * size * (a_off[:, t] + 2 * U) + (b[:, t] * x[:, t]).abs() * (b_off[:, t] + 2 * U), off)
        size = torch.where(v, a[:, t] * size + (b[:, t] * x[:, t]).abs(), size)
        s = torch.where(v, a[:, t] * s + b[:, t] * x[:, t], s)
        h[:, t] = torch.where(v, s, 0.0)
        h_off[:, t] = off + joins * size + R[dtype] * s.abs() + 1e-30
    none = torch.zeros(B, 0, C, dtype=torch.float64)
    kept, kept_off = (torch.stack(kept, 1), torch.stack(kept_off, 1)) if kept else (none, none)
    return (h, s, kept), (h_off, off + joins * size + 1e-30, kept_off)


def recurrence_backward(dh, x, gate, kept, lens, dlast):
    """(dx, dgate, dstate) from the kept states, and their bounds."""
    dtype, (B, T, C) = x.dtype, x.shape
    valid = _valid(lens, B, T)
    a, b, a_off, b_off = gates(gate)
    dh, x, kept = f64(dh), f64(x), f64(kept)
    before, before_off = torch.zeros_like(x), torch.zeros_like(x)
    for t in range(T):
        if t % KEPT == 0:
            s = kept[:, t // KEPT]
            size, off = s.abs(), torch.zeros_like(s)
        before[:, t], before_off[:, t] = s, off + 32 * U * size
        off = a[:, t] * off + a[:, t] * size * (a_off[:, t] + 2 * U) + (b[:, t] * x[:, t]).abs() * (b_off[:, t] + 2 * U)
        size = a[:, t] * size + (b[:, t] * x[:, t]).abs()
        s = a[:, t] * s + b[:, t] * x[:, t]
    e = torch.zeros(B, C, dtype=torch.float64) if dlast is None else f64(dlast)
    size, off = e.abs(), torch.zeros_like(e)
    out = [torch.zeros_like(x) for _ in range(4)]
    joins = (32 + -(-T // KEPT)) * U
    for t in reversed(range(T)):
        v = valid[:, t:t + 1]
        g, g_size, g_off = dh[:, t] + e, dh[:, t].abs() + size, off + joins * size + 2 * U * (dh[:, t].abs() + size)
        apart, ab = before[:, t] - x[:, t], a[:, t] * b[:, t]
        dx, dg = b[:, t] * g, g * apart * ab
        dx_off = dx.abs() * (b_off[:, t] + 2 * U) + b[:, t] * g_off + R[dtype] * dx.abs()
        apart_off = before_off[:, t] + 2 * U * (before[:, t].abs() + x[:, t].abs())
        dg_off = (g * apart).abs() * ab * (a_off[:, t] + b_off[:, t] + 8 * U) + (g_off * apart.abs() + g.abs() * apart_off) * ab + R[dtype] * dg.abs()
        for o, value in zip(out, (dx, dg, dx_off, dg_off)):
            o[:, t] = torch.where(v, value, 0.0)
        off = torch.where(v, a[:, t] * (off + g_size * (a_off[:, t] + 2 * U)), off)
        size = torch.where(v, a[:, t] * g_size, size)
        e = torch.where(v, a[:, t] * g, e)
    return (out[0], out[1], e), (out[2] + 1e-30, out[3] + 1e-30, off + joins * size + 1e-30)


# ------------------------------------------------------------------------------------ experts
def edges(ends, rows):
    """(first row, behind the last) of each expert: ends ascend and stay within the rows."""
    at, parts = 0, []
    for end in ends.tolist():
        end = max(at, min(max(end, 0), rows))
        parts.append((at, end))
        at = end
    return parts


def expert_linear(x, weight, ends):
    dtype, K = x.dtype, x.shape[1]
    x, w = f64(x), f64(weight)
    y, off = (torch.zeros(x.shape[0], w.shape[1], dtype=torch.float64) for _ in range(2))
    for e, (i, j) in enumerate(edges(ends, x.shape[0])):
        y[i:j] = x[i:j] @ w[e].T
        off[i:j] = (K + 8) * U * (x[i:j].abs() @ w[e].abs().T)
    return y, off + R[dtype] * y.abs() + 1e-30


def expert_input_grad(dy, weight, ends):
    return expert_linear(dy, weight.transpose(1, 2), ends)


def expert_weight_grad(dy, x, ends):
    dy, x, parts = f64(dy), f64(x), edges(ends, x.shape[0])
    dw = torch.stack([dy[i:j].T @ x[i:j] for i, j in parts])
    off = torch.stack([(j - i + 8) * U * (dy[i:j].abs().T @ x[i:j].abs()) for i, j in parts])
    return dw, off + 1e-30


# ------------------------------------------------------------------------------------ gradients
def clip(tensors, max_norm, dtypes):
    """norm, the scaled tensors in `dtypes`, and their bounds: the norm and the factor are rounded once, the product once.  A norm that
    fp32 does not hold is an infinity there; the factor comes from the norm itself."""
    grads = [f64(t) for t in tensors]
    norm = torch.sqrt(sum((g * g).sum() for g in grads))
    by = (max_norm / norm).clamp(max=1.0) if norm > max_norm or torch.isnan(norm) else torch.tensor(1.0, dtype=torch.float64)
    outs = [g * by for g in grads]
    half = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
    said = torch.where(norm > torch.finfo(torch.float32).max, torch.inf, norm)
    return said, outs, 2.0 ** -23 * norm, [o.abs() * (2.0 ** -23 + half[d] + 2.0 ** -30) + 2.0 ** -149 for o, d in zip(outs, dtypes)]
