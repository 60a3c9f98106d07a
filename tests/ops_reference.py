"""The training operators from their definitions, in 64 bits on the CPU, and how far a result may be from them.

Bounds.  U is a unit of fp32 rounding, taken twice as large as 2^-24 because matrix instructions may truncate; a sum of
n products is off by at most (n + 8) U times the sum of their magnitudes, whatever its order.  R[dtype] is the largest
relative error of one rounding to the type.  Each bound below follows an error through the formulas to first order."""
from __future__ import annotations

import math

import torch

U = 2.0 ** -23
R = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -23}
GROUP = 32


def f64(t):
    return t.detach().cpu().double()


def visible(B, Sq, Sk, causal, q_lens, kv_lens):
    """[B, Sq, Sk]"""
    see = torch.zeros(B, Sq, Sk, dtype=torch.bool)
    for b in range(B):
        nq = Sq if q_lens is None else min(max(int(q_lens[b]), 0), Sq)
        nk = Sk if kv_lens is None else min(max(int(kv_lens[b]), 0), Sk)
        for i in range(nq):
            see[b, i, :max(0, min(nk, i + nk - nq + 1) if causal else nk)] = True
    return see


def _scores(q, k, see, scale):
    """Scores [B, H, Sq, Sk] with -inf where nothing is seen, and the bound of their error."""
    G = q.shape[2] // k.shape[2]
    a, c = q.permute(0, 2, 1, 3), k.permute(0, 2, 3, 1).repeat_interleave(G, 1)
    s = scale * a @ c
    off = (q.shape[3] + 16) * U * scale * (a.abs() @ c.abs()) + 4 * U
    return s.masked_fill(~see[:, None], -math.inf), off


def _clean(t, lens):
    """Tokens beyond the lengths as zeros: they are never used."""
    t = f64(t).clone()
    if lens is not None:
        for b in range(t.shape[0]):
            t[b, min(max(int(lens[b]), 0), t.shape[1]):] = 0
    return t


def attention(q, k, v, causal, scale, q_lens, kv_lens):
    """(out, lse), and their bounds."""
    dtype, G = q.dtype, q.shape[2] // k.shape[2]
    q, k, v = _clean(q, q_lens), _clean(k, kv_lens), _clean(v, kv_lens)
    see = visible(q.shape[0], q.shape[1], k.shape[1], causal, q_lens, kv_lens)
    s, off = _scores(q, k, see, scale)
    lse = torch.logsumexp(s, -1) if s.shape[-1] else torch.full(s.shape[:-1], -math.inf, dtype=torch.float64)
    p = torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None])
    vv = v.permute(0, 2, 1, 3).repeat_interleave(G, 1)
    out = p @ vv
    worst = torch.where(see[:, None], off, 0.0).amax(-1, keepdim=True) if off.shape[-1] else torch.zeros_like(lse)[..., None]
    n = k.shape[1]
    out_off = (p @ vv.abs()) * (2 * worst + 2 * (n + 8) * U + (R[dtype] if dtype == torch.bfloat16 else 0)) + R[dtype] * out.abs()
    lse_off = worst[..., 0] + (n + 8) * U + 4 * U * torch.where(lse == -math.inf, 0.0, lse).abs()
    return out.permute(0, 2, 1, 3), lse, out_off.permute(0, 2, 1, 3) + 1e-30, lse_off


def attention_backward(dout, q, k, v, out, lse, causal, scale, q_lens, kv_lens):
    """(dq, dk, dv) by the operator's formulas from the out and lse given, and their bounds."""
    dtype, H, Hkv = q.dtype, q.shape[2], k.shape[2]
    G, D, B, Sq, Sk = H // Hkv, q.shape[3], q.shape[0], q.shape[1], k.shape[1]
    q, k, v = _clean(q, q_lens), _clean(k, kv_lens), _clean(v, kv_lens)
    do, o, z = (x.permute(0, 2, 1, 3) for x in (_clean(dout, q_lens), _clean(out, q_lens), q))
    lse = f64(lse)
    see = visible(B, Sq, Sk, causal, q_lens, kv_lens)
    s, off = _scores(q, k, see, scale)
    p = torch.where(see[:, None], torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None]), 0.0)
    kk, vv = (x.permute(0, 2, 1, 3).repeat_interleave(G, 1) for x in (k, v))
    dp, delta = do @ vv.transpose(-1, -2), (do * o).sum(-1, keepdim=True)
    ds = p * (dp - delta)
    # relative error of p; absolute error of dp - delta; what the rounding of p and ds as operands adds
    p_off = torch.where(see[:, None], off, 0.0) + 4 * U * torch.where(lse == -math.inf, 0.0, lse).abs()[..., None] + 4 * U
    dp_off = (D + 8) * U * (do.abs() @ vv.abs().transpose(-1, -2) + (do * o).abs().sum(-1, keepdim=True))
    half = R[dtype] if dtype == torch.bfloat16 else 0.0
    ds_off = ds.abs() * (p_off + 2 * U + half) + p * dp_off
    n = max(Sq * G, Sk) + 8
    def shared(x):  # gradients of a key head's query heads, added up
        return x.reshape(B, Hkv, G, *x.shape[2:]).sum(2).permute(0, 2, 1, 3)
    dq = scale * ds @ kk
    dq_off = scale * (ds_off + n * U * ds.abs()) @ kk.abs() + R[dtype] * dq.abs()
    dk = shared(scale * ds.transpose(-1, -2) @ z)
    dk_off = shared(scale * (ds_off + n * U * ds.abs()).transpose(-1, -2) @ z.abs()) + R[dtype] * dk.abs()
    dv = shared(p.transpose(-1, -2) @ do)
    dv_off = shared((p * (p_off + half + n * U)).transpose(-1, -2) @ do.abs()) + R[dtype] * dv.abs()
    return (dq.permute(0, 2, 1, 3), dk, dv), (dq_off.permute(0, 2, 1, 3) + 1e-30, dk_off + 1e-30, dv_off + 1e-30)


def encode(x):
    """(codes, exponents) of a 2-D tensor, group by group from the definition."""
    x = f64(x)
    rows, cols = x.shape
    z = torch.zeros(rows, -(-cols // GROUP) * GROUP, dtype=torch.float64)
    z[:, :cols] = x
    z = z.view(rows, z.shape[1] // GROUP, GROUP)
    a = z.abs().amax(-1)
    broken = ~torch.isfinite(z).all(-1)
    a = torch.where(broken, 0.0, a)
    e = torch.full(a.shape, -126, dtype=torch.int64)
    for _ in range(260):  # the smallest e >= -126 with a <= 127 * 2^e
        e = torch.where(a > 127 * torch.pow(2.0, e.double()), e + 1, e)
    codes = torch.round(z * torch.pow(2.0, -e.double()).unsqueeze(-1))
    codes = torch.where(broken.unsqueeze(-1), 0.0, codes)
    return codes.flatten(1).to(torch.int8), torch.where(broken, 255, e + 127).to(torch.uint8)


def decode(codes, exponents, cols):
    step = torch.pow(2.0, exponents.cpu().double() - 127)
    step = torch.where(exponents.cpu() == 255, math.nan, step)
    x = codes.cpu().double().view(*exponents.shape, GROUP) * step.unsqueeze(-1)
    x = torch.where(x.abs() > torch.finfo(torch.float32).max, torch.copysign(torch.tensor(math.inf, dtype=torch.float64), x), x)
    return x.reshape(codes.shape)[:, :cols]


def norm(h, weight, eps):
    """(y, rstd) of the stored h, and their bounds."""
    dtype, h, w = h.dtype, f64(h), f64(weight)
    rstd = 1 / torch.sqrt((h * h).mean(-1) + eps)
    y = h * rstd[:, None] * w
    rel = (h.shape[1] + 16) * U
    return y, rstd, (rel + 2 * R[dtype]) * y.abs() + 1e-30, rel * rstd


def norm_backward(dy, h, weight, rstd, dh):
    dtype, dy, h, w, r = dy.dtype, f64(dy), f64(h), f64(weight), f64(rstd)[:, None]
    rows, cols = dy.shape
    g, n = dy * w, h * r
    mean, size = (g * n).mean(1, keepdim=True), (g * n).abs().mean(1, keepdim=True)
    dx = (g - n * mean) * r + (0 if dh is None else f64(dh))
    whole = ((g.abs() + n.abs() * size) * r).abs() + (0 if dh is None else f64(dh).abs())
    dx_off = 8 * U * whole + (cols + 16) * U * (n.abs() * size * r).abs() + R[dtype] * dx.abs()
    return dx, (dy * n).sum(0), dx_off + 1e-30, (rows + 16) * U * (dy * n).abs().sum(0) + 1e-30


def weight_grad(dy, codes, exponents, cols):
    dy, x = f64(dy), decode(codes, exponents, cols)
    return dy.T @ x, (dy.shape[0] + 8) * U * (dy.abs().T @ x.abs()) + 1e-30


def within(got, want, off, what):
    """Every element of got within its bound of want; infinities and NaNs at the same places."""
    got, bad = f64(got), None
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN elsewhere"
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), what + ": infinities"
    if not got.numel():
        return
    over = torch.where(fine, (got - want).abs() / off.expand_as(want), 0.0)
    bad = over.argmax()
    assert over.max() <= 1, "%s: %g of the bound at %d: %g, expected %g" % (what, over.max(), bad, got.flatten()[bad], want.flatten()[bad])
