"""GPU: the training operators against their definitions in 64 bits, at the sizes, masks, layouts and values where they
can go wrong; bounds as derived in ops_reference.py."""
from __future__ import annotations

import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import ops_reference as ref  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
NAN = math.nan


@pytest.fixture(scope="module")
def ops():
    from paper_2302_12445_amd import ops as m
    m.load_library()
    return m


def normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype).to(DEV)


def lens(values):
    return None if values is None else torch.tensor(values, dtype=torch.int32, device=DEV)


# ------------------------------------------------------------------------------------ attention
def check_attention(ops, q, k, v, causal=False, scale=None, q_lens=None, kv_lens=None, seed=0, label=""):
    """Forward and backward; the backward from the out and lse that the forward gave."""
    q_lens, kv_lens = lens(q_lens), lens(kv_lens)
    s = 1 / math.sqrt(q.shape[3]) if scale is None else scale
    out, lse = ops.attention(q, k, v, causal=causal, scale=scale, q_lens=q_lens, kv_lens=kv_lens)
    want, want_lse, off, lse_off = ref.attention(q, k, v, causal, s, q_lens, kv_lens)
    ref.within(out, want, off, label + " out")
    ref.within(lse, want_lse, lse_off, label + " lse")
    dout = normal(torch.Generator().manual_seed(seed + 1), q.shape, q.dtype)
    if q_lens is not None:  # what stands beyond the lengths is never used
        for b, n in enumerate(q_lens.tolist()):
            dout[b, max(n, 0):] = NAN
    got = ops.attention_backward(dout, q, k, v, out, lse, causal=causal, scale=scale, q_lens=q_lens, kv_lens=kv_lens)
    want, off = ref.attention_backward(dout, q, k, v, out, lse, causal, s, q_lens, kv_lens)
    for g, w, o, name in zip(got, want, off, ("dq", "dk", "dv")):
        ref.within(g, w, o, label + " " + name)
    return out, lse, dout, got


SHAPES = [  # batch, q_len, kv_len, heads, kv_heads, head_dim
    (1, 1, 1, 1, 1, 8), (2, 1, 77, 4, 2, 64), (1, 5, 3, 2, 1, 24), (2, 33, 65, 4, 4, 64), (1, 64, 64, 2, 2, 128),
    (1, 129, 257, 3, 1, 80), (2, 127, 127, 6, 2, 128), (1, 300, 40, 2, 2, 32), (1, 40, 300, 8, 2, 96), (3, 200, 200, 5, 5, 56),
    (1, 513, 513, 4, 1, 64), (1, 1, 1000, 2, 2, 128), (1, 700, 1, 2, 1, 64),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", SHAPES)
def test_attention(ops, shape, causal, dtype):
    B, Sq, Sk, H, Hkv, D = shape
    print("case", shape, causal, dtype, flush=True)
    gen = torch.Generator().manual_seed(sum(shape))
    q, k, v = normal(gen, (B, Sq, H, D), dtype), normal(gen, (B, Sk, Hkv, D), dtype), normal(gen, (B, Sk, Hkv, D), dtype)
    check_attention(ops, q, k, v, causal, seed=7)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dim", [64, 128])
def test_attention_lengths(ops, dim, causal, dtype):
    """Lengths of 0 and 1, whole ones, more than there are and less than none, queries that see no key; NaN and
    infinities in what lies beyond them."""
    print("case lengths", dim, causal, dtype, flush=True)
    nq, nk = [0, 1, 150, 70, 33, 150, 140, -3], [9, 1, 100, 0, 64, 200, 31, 20]
    gen = torch.Generator().manual_seed(5)
    q, k, v = (normal(gen, (8, n, h, dim), dtype) for n, h in ((150, 4), (100, 2), (100, 2)))
    for b in range(8):
        q[b, max(nq[b], 0):] = NAN
        k[b, nk[b]:] = NAN
        v[b, nk[b]:] = math.inf
    out, lse, _, (dq, dk, dv) = check_attention(ops, q, k, v, causal, q_lens=nq, kv_lens=nk)
    assert not out[0].any() and not out[7].any() and not out[3].any() and not dq[3].any() and not dk[0].any() and not dv[7].any()
    assert (lse[3] == -math.inf).all()
    if causal:  # 150 queries on 100 keys: the first 50 see none
        assert not out[2, :50].any() and (lse[2, :, :50] == -math.inf).all() and not dq[2, :50].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(1, 3, 2000, 2, 1, 64), (2, 200, 900, 1, 1, 128), (1, 1500, 130, 2, 2, 40), (2, 640, 640, 4, 1, 64),
                                   (1, 900, 1100, 3, 1, 104)])
def test_attention_few_rows(ops, shape, causal, dtype):
    """Calls of few workgroups, which split the sequences; lengths that leave splits, or all of them, without a token."""
    B, Sq, Sk, H, Hkv, D = shape
    print("case few rows", shape, causal, dtype, flush=True)
    gen = torch.Generator().manual_seed(sum(shape))
    q, k, v = normal(gen, (B, Sq, H, D), dtype), normal(gen, (B, Sk, Hkv, D), dtype), normal(gen, (B, Sk, Hkv, D), dtype)
    check_attention(ops, q, k, v, causal, label="whole")
    check_attention(ops, q, k, v, causal, q_lens=[Sq] + [Sq // 3] * (B - 1), kv_lens=[Sk // 5] + [Sk] * (B - 1), label="short")
    check_attention(ops, q, k, v, causal, q_lens=[Sq] * B, kv_lens=[0] + [1] * (B - 1), label="none")
    k[:, Sk // 2] *= 30  # one split has the maximum of most rows
    check_attention(ops, q, k, v, causal, label="maximum")


def test_attention_of_nothing(ops):
    for B, Sq, Sk in ((0, 4, 4), (2, 0, 4), (2, 4, 0), (2, 0, 0)):
        q, k = torch.zeros(B, Sq, 2, 64, dtype=BF16, device=DEV), torch.zeros(B, Sk, 2, 64, dtype=BF16, device=DEV)
        out, lse = ops.attention(q, k, k)
        assert not out.any() and (lse == -math.inf).all()
        for g in ops.attention_backward(q, q, k, k, out, lse):
            assert not g.any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_layouts(ops, dtype):
    """Packed projections, heads before tokens, keys shared by the whole batch, tensors that start off 16 bytes."""
    gen = torch.Generator().manual_seed(11)
    packed = normal(gen, (2, 70, 3, 4, 64), dtype)
    check_attention(ops, *packed.unbind(2), causal=True, label="packed")
    first = normal(gen, (2, 4, 70, 64), dtype)
    check_attention(ops, first.transpose(1, 2), first.transpose(1, 2), first.transpose(1, 2), label="heads first")
    one = normal(gen, (1, 50, 2, 64), dtype)
    check_attention(ops, packed[:, :, 0], one.expand(2, -1, -1, -1), one.expand(2, -1, -1, -1), label="shared")
    flat = normal(gen, (2 * 70 * 4 * 64 + 3,), dtype)
    odd = flat[3:].view(2, 70, 4, 64)
    check_attention(ops, odd, odd, odd, label="off 16 bytes")
    wide = normal(gen, (2, 70, 4, 67), dtype)[..., :64]
    check_attention(ops, wide, wide, wide, label="odd strides")
    turned = normal(gen, (2, 70, 64, 4), dtype).transpose(2, 3)
    check_attention(ops, turned, turned, turned, label="head_dim not contiguous")


def test_attention_far_offsets(ops):
    """Tokens more than 2^31 elements apart."""
    gen = torch.Generator().manual_seed(3)
    apart = 1 << 26
    base = torch.empty(apart * 69 + 2 * 64, dtype=BF16, device=DEV)
    k = base.as_strided((1, 70, 2, 64), (0, apart, 64, 1))
    k.copy_(normal(gen, (1, 70, 2, 64), BF16))
    q = normal(gen, (1, 70, 2, 64), BF16)
    check_attention(ops, q, k, k, causal=True, label="keys")
    check_attention(ops, k, q, q, causal=True, label="queries")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_attention_large_scores(ops, dtype):
    """Scores of hundreds, whose powers overflow without the running maximum; equal scores; a small scale."""
    gen = torch.Generator().manual_seed(2)
    q, k, v = (normal(gen, (1, 130, 2, 64), dtype, s) for s in (12.0, 12.0, 1.0))
    k[:, 100:] *= 3  # the maximum rises late
    check_attention(ops, q, k, v, label="large")
    check_attention(ops, torch.ones_like(q), torch.ones_like(k), v, causal=True, label="equal")
    check_attention(ops, q, k, v, scale=1e-3, label="scale")


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("shape", [(2, 130, 2, 64), (1, 200, 2, 128), (1, 900, 1, 96)])
def test_attention_scores_far_below_zero(ops, shape, causal, dtype):
    """Scores of minus hundreds alone: powers taken against 0 would all be 0, and those of the first maximum overflow."""
    gen = torch.Generator().manual_seed(5)
    q, k = normal(gen, shape, dtype, 3.0).abs() + 5, -normal(gen, shape, dtype, 3.0).abs() - 5
    v = normal(gen, shape, dtype)
    check_attention(ops, q, k, v, causal, label="low")
    k[:, 100:] /= 4  # the maximum rises late
    check_attention(ops, q, k, v, causal, label="rising")


def test_attention_nan_and_infinity_reach_the_result(ops):
    gen = torch.Generator().manual_seed(2)
    q, k, v = (normal(gen, (2, 40, 2, 64), BF16) for _ in range(3))
    q[0, 7, 1, 3] = NAN
    v[1, 5, 0, 9] = math.inf
    out, lse = ops.attention(q, k, v)
    bad = torch.zeros_like(out, dtype=torch.bool)
    bad[0, 7, 1] = True
    bad[1, :, 0, 9] = True
    assert torch.equal(~torch.isfinite(out), bad)
    assert torch.isnan(lse[0, 1, 7]) and torch.isfinite(lse).sum() == lse.numel() - 1


def test_attention_gradients_against_differences(ops):
    """fp32: the loss sum(out * w) along a random direction, by central differences of the 64-bit definition."""
    gen = torch.Generator().manual_seed(4)
    q, k, v, w = (normal(gen, (1, n, h, 32), F32) for n, h in ((37, 4), (45, 2), (45, 2), (37, 4)))
    out, lse = ops.attention(q, k, v, causal=True)
    grads = ops.attention_backward(w, q, k, v, out, lse, causal=True)
    step = 1e-4
    for n, (t, g) in enumerate(zip((q, k, v), grads)):
        d = normal(gen, t.shape, F32)
        sides = []
        for sign in (1, -1):
            moved = [ref.f64(x) for x in (q, k, v)]
            moved[n] = moved[n] + sign * step * ref.f64(d)
            p, _ = ref._scores(moved[0], moved[1], ref.visible(1, 37, 45, True, None, None), 32 ** -0.5)
            o = torch.softmax(p, -1) @ moved[2].permute(0, 2, 1, 3).repeat_interleave(2, 1)
            sides.append((o.permute(0, 2, 1, 3) * ref.f64(w)).sum())
        slope = (sides[0] - sides[1]) / (2 * step)
        got = (ref.f64(g) * ref.f64(d)).sum()
        # step^2 times the third derivative, and fp32's error of some thousand terms
        assert abs(slope - got) <= 1e-5 * (ref.f64(g) * ref.f64(d)).abs().sum(), n


def test_attention_repeats_bits(ops):
    gen = torch.Generator().manual_seed(8)
    q, k, v = (normal(gen, (2, 333, h, 64), BF16) for h in (8, 2, 2))
    a = ops.attention(q, k, v, causal=True)
    b = ops.attention(q, k, v, causal=True)
    g = ops.attention_backward(q, q, k, v, *a, causal=True)
    f = ops.attention_backward(q, q, k, v, *b, causal=True)
    for x, y in zip(a + g, b + f):
        assert torch.equal(x, y)


# ------------------------------------------------------------------------------------ checkpoints
WIDTHS = [1, 7, 31, 32, 33, 64, 100, 1000, 1024, 4096]


def activations(gen, rows, cols, dtype):
    x = torch.randn(rows, cols, generator=gen) * torch.exp(4 * torch.randn(rows, 1, generator=gen))
    return x.to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", WIDTHS)
@pytest.mark.parametrize("rows", [1, 3, 70])
def test_checkpoint(ops, rows, cols, dtype):
    x = activations(torch.Generator().manual_seed(cols), rows, cols, dtype)
    kept = ops.checkpoint_encode(x)
    codes, exponents = ref.encode(x)
    assert torch.equal(kept.codes.cpu(), codes) and torch.equal(kept.exponents.cpu(), exponents)
    for t in (BF16, F32):
        got = ops.checkpoint_decode(kept, t)
        assert got.dtype == t and torch.equal(ref.f64(got), ref.decode(codes, exponents, cols))
    # half a step of a group whose largest value takes at least 64 steps
    a = torch.nn.functional.pad(ref.f64(x), (0, -cols % 32)).view(rows, -1, 32)
    off = (a.abs().amax(-1, keepdim=True) / 63.5 / 2).expand_as(a).reshape(rows, -1)[:, :cols]
    assert ((ref.f64(got) - ref.f64(x)).abs() <= off).all()


def test_checkpoint_corner_values(ops):
    """Largest values around 127 steps, halves, zeros, the smallest and the largest numbers, NaN and infinities."""
    x = torch.zeros(12, 64)
    x[0, 0], x[0, 1], x[0, 2], x[0, 3] = 127, 0.5, 1.5, -2.5
    x[1, 0] = 127.00001
    x[2, 0], x[2, 33] = 126.9, -128
    x[3, 0] = torch.finfo(F32).max
    x[4, 0], x[4, 1] = 1e-45, -1e-40
    x[5, 0], x[5, 40] = torch.finfo(F32).tiny, 3e-37
    x[6, 5], x[6, 6] = NAN, 3
    x[7, 5], x[7, 40] = math.inf, 2
    x[8, 63], x[8, 0] = -math.inf, -1
    x[9] = -0.0
    x[10] = torch.arange(64) - 31.5
    x[11, 0], x[11, 1] = NAN, math.inf
    for t in (F32, BF16):
        y = x.to(t).to(DEV)
        kept = ops.checkpoint_encode(y)
        codes, exponents = ref.encode(y)
        assert torch.equal(kept.exponents.cpu(), exponents) and torch.equal(kept.codes.cpu(), codes)
        got = ref.f64(ops.checkpoint_decode(kept, F32))
        want = ref.decode(codes, exponents, 64)
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got[~torch.isnan(got)], want[~torch.isnan(want)])


def test_checkpoint_layouts(ops):
    gen = torch.Generator().manual_seed(1)
    big = activations(gen, 20, 200, BF16)
    for x in (big[:, 8:136], big[:, 3:80], big[::2], big.t(), big[3], big.view(4, 5, 200), big[:1].expand(6, -1)):
        kept = ops.checkpoint_encode(x)
        codes, exponents = ref.encode(x.reshape(-1, x.shape[-1]))
        assert torch.equal(kept.codes.cpu(), codes) and torch.equal(kept.exponents.cpu(), exponents)
    empty = ops.checkpoint_encode(big[:0])
    assert empty.codes.shape == (0, 224) and ops.checkpoint_decode(empty).shape == (0, 200)


# ------------------------------------------------------------------------------------ weight gradient
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,outs,ins", [
    (0, 5, 9), (1, 1, 1), (1, 64, 64), (2, 130, 33), (31, 128, 128), (33, 17, 300), (64, 256, 256), (100, 200, 136),
    (257, 129, 127), (1000, 96, 64), (2049, 40, 72), (5000, 8, 32), (700, 520, 264)])
def test_weight_grad(ops, rows, outs, ins, dtype):
    print("case", rows, outs, ins, dtype, flush=True)
    gen = torch.Generator().manual_seed(rows + outs + ins)
    dy = normal(gen, (rows, outs), dtype)
    x = activations(gen, rows, ins, dtype)
    kept = ops.checkpoint_encode(x)
    dw = ops.checkpoint_weight_grad(dy, kept)
    assert dw.dtype == F32
    ref.within(dw, *ref.weight_grad(dy, kept.codes, kept.exponents, ins), "dw")
    assert torch.equal(dw, ops.checkpoint_weight_grad(dy, kept))


def test_weight_grad_layouts(ops):
    gen = torch.Generator().manual_seed(6)
    kept = ops.checkpoint_encode(activations(gen, 90, 70, BF16))
    big = normal(gen, (180, 300), BF16)
    for dy in (big[:90, 8:72], big[:90, 5:70], big[::2, :128], big[:90].t().contiguous().t(), big[:1, :64].expand(90, -1),
               big[:90, :100].reshape(9, 10, 100)):
        ref.within(ops.checkpoint_weight_grad(dy, kept), *ref.weight_grad(dy.reshape(90, -1), kept.codes, kept.exponents, 70), "dw")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_weight_grad_broken_groups(ops, dtype):
    """A group that held a NaN makes its 32 columns NaN, and no others; a NaN of dy its row."""
    gen = torch.Generator().manual_seed(6)
    x, dy = activations(gen, 100, 130, dtype), normal(gen, (100, 50), dtype)
    x[40, 70] = math.inf
    dy[3, 20] = NAN
    dw = ops.checkpoint_weight_grad(dy, ops.checkpoint_encode(x))
    bad = torch.zeros(50, 130, dtype=torch.bool, device=DEV)
    bad[:, 64:96] = True
    bad[20] = True
    assert torch.equal(torch.isnan(dw), bad)


# ------------------------------------------------------------------------------------ norm
NORM_COLS = [1, 5, 8, 64, 100, 504, 520, 768, 1000, 1032, 1600, 2048, 2056, 4096, 5000, 6144, 8192, 8200, 12345, 20480, 32768]


def check_norm(ops, x, residual, weight, eps=1e-5):
    h, y, kept, rstd = ops.add_rms_norm(x, residual, weight, eps)
    want = x if residual is None else (x.float() + residual.float()).to(x.dtype)
    assert torch.equal(h, want)
    rows = h.reshape(-1, h.shape[-1])
    wy, wr, off, roff = ref.norm(rows, weight, eps)
    ref.within(y.reshape(rows.shape), wy, off, "y")
    ref.within(rstd, wr, roff, "rstd")
    codes, exponents = ref.encode(y.reshape(rows.shape))
    assert torch.equal(kept.codes.cpu(), codes) and torch.equal(kept.exponents.cpu(), exponents) and kept.cols == rows.shape[1]
    _, other, none, _ = ops.add_rms_norm(x, residual, weight, eps, keep=False)
    assert none is None and torch.equal(other, y)
    return h, rstd


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("cols", NORM_COLS)
def test_norm(ops, cols, dtype):
    print("case", cols, dtype, flush=True)
    gen = torch.Generator().manual_seed(cols)
    for rows in (1, 6, 67):
        x, residual = activations(gen, rows, cols, dtype), activations(gen, rows, cols, dtype)
        weight = normal(gen, (cols,), F32)
        h, rstd = check_norm(ops, x, residual, weight)
        if rows == 6:
            check_norm(ops, x, None, weight)
        dy, dh = normal(gen, x.shape, dtype), normal(gen, x.shape, dtype)
        for extra in (dh, None):
            dx, dw = ops.add_rms_norm_backward(dy, h, weight, rstd, dh=extra)
            wx, ww, xoff, woff = ref.norm_backward(dy, h, weight, rstd, extra)
            ref.within(dx, wx, xoff, "dx")
            ref.within(dw, ww, woff, "dweight")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_norm_many_rows(ops, dtype):
    gen = torch.Generator().manual_seed(1)
    dy, h = normal(gen, (5000, 72), dtype), normal(gen, (5000, 72), dtype)
    weight = normal(gen, (72,), F32)
    rstd = torch.rsqrt(h.float().square().mean(1) + 1e-5)
    dx, dw = ops.add_rms_norm_backward(dy, h, weight, rstd)
    wx, ww, xoff, woff = ref.norm_backward(dy, h, weight, rstd, None)
    ref.within(dx, wx, xoff, "dx")
    ref.within(dw, ww, woff, "dweight")
    assert torch.equal(dw, ops.add_rms_norm_backward(dy, h, weight, rstd)[1])


def test_norm_layouts(ops):
    gen = torch.Generator().manual_seed(1)
    big = activations(gen, 24, 300, BF16)
    weight = normal(gen, (128,), F32)
    for x in (big[:, 8:136], big[:, 3:131], big[::2, :128], big.view(4, 6, 300)[:, :, 16:144], big[2, :128], big[:0, :128],
              big[:1, :128].expand(5, -1)):
        h, rstd = check_norm(ops, x, x.flip(0) if x.dim() == 2 else x, weight)
        dx, dw = ops.add_rms_norm_backward(x, h, weight, rstd, dh=x)
        flat = [t.reshape(-1, 128) for t in (x, h)]
        wx, ww, xoff, woff = ref.norm_backward(flat[0], flat[1], weight, rstd, flat[0])
        ref.within(dx.reshape(-1, 128), wx, xoff, "dx")
        ref.within(dw, ww, woff, "dweight")
        assert dx.shape == x.shape


def test_norm_corner_values(ops):
    """A row of zeros with no eps gives NaN as 0 times infinity does; infinities and NaN stay in their row."""
    x = torch.ones(4, 64, device=DEV)
    x[0] = 0
    x[1, 3] = NAN
    x[2, 4] = math.inf
    h, y, kept, rstd = ops.add_rms_norm(x, torch.zeros_like(x), torch.ones(64, device=DEV), 0.0)
    assert torch.isinf(rstd[0]) and torch.isnan(y[0]).all() and torch.isnan(y[1]).all()
    assert rstd[2] == 0 and torch.isnan(y[2, 4]) and not y[2, 5:].any()
    assert torch.equal(y[3], torch.ones(64, device=DEV)) and torch.isnan(ops.checkpoint_decode(kept)[1]).all()
    _, y, _, _ = ops.add_rms_norm(x[:1], None, torch.ones(64, device=DEV), 1e-5)
    assert not y.any()


def test_norm_gradient_against_differences(ops):
    gen = torch.Generator().manual_seed(9)
    x, dy, d = (normal(gen, (5, 100), F32) for _ in range(3))
    weight, dw_dir = normal(gen, (100,), F32), normal(gen, (100,), F32)
    _, _, _, rstd = ops.add_rms_norm(x, None, weight, 1e-5)
    dx, dw = ops.add_rms_norm_backward(dy, x, weight, rstd)
    def loss(a, b):
        return (a / torch.sqrt((a * a).mean(1, keepdim=True) + 1e-5) * b * ref.f64(dy)).sum()
    a, b, e = ref.f64(x), ref.f64(weight), 1e-5
    for g, way, sides in ((dx, d, [loss(a + s * e * ref.f64(d), b) for s in (1, -1)]),
                          (dw, dw_dir, [loss(a, b + s * e * ref.f64(dw_dir)) for s in (1, -1)])):
        got = (ref.f64(g) * ref.f64(way)).sum()
        assert abs((sides[0] - sides[1]) / (2 * e) - got) <= 1e-5 * (ref.f64(g) * ref.f64(way)).abs().sum()


# ------------------------------------------------------------------------------------ streams and graphs
def _block(ops, x, res, weight, q_lens):
    h, y, kept, rstd = ops.add_rms_norm(x, res, weight)
    q = y.view(2, 96, 4, 64)
    out, lse = ops.attention(q, q, q, causal=True, q_lens=q_lens, kv_lens=q_lens)
    dq, dk, dv = ops.attention_backward(q, q, q, q, out, lse, causal=True, q_lens=q_lens, kv_lens=q_lens)
    dw = ops.checkpoint_weight_grad(out.view(192, 256), kept)
    dx, dweight = ops.add_rms_norm_backward(dq.view(192, 256), h, weight, rstd, dh=dk.view(192, 256))
    return [h, y, kept.codes, kept.exponents, rstd, out, lse, dq, dk, dv, dw, dx, dweight, ops.checkpoint_decode(ops.checkpoint_encode(dx))]


def test_operators_on_another_stream(ops):
    gen = torch.Generator().manual_seed(9)
    x, res, weight = normal(gen, (192, 256), BF16), normal(gen, (192, 256), BF16), normal(gen, (256,), F32)
    q_lens = lens([96, 50])
    want = _block(ops, x, res, weight, q_lens)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _block(ops, x, res, weight, q_lens)
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_operators_in_a_graph(ops):
    gen = torch.Generator().manual_seed(10)
    x, res, weight = normal(gen, (192, 256), BF16), normal(gen, (192, 256), BF16), normal(gen, (256,), F32)
    q_lens = lens([96, 50])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _block(ops, x, res, weight, q_lens)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _block(ops, x, res, weight, q_lens)
    for n in range(4):
        x.copy_(normal(gen, (192, 256), BF16))
        q_lens.copy_(lens([96 - 10 * n, 7 * n]))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(got, _block(ops, x, res, weight, q_lens)):
            assert torch.equal(a, b), n


# ------------------------------------------------------------------------------------ refusals
def test_refusals(ops):
    from paper_2302_12445_amd import DearError
    q = torch.zeros(2, 8, 4, 64, dtype=BF16, device=DEV)
    out, lse = ops.attention(q, q, q)
    w = torch.ones(64, device=DEV)
    x = torch.zeros(8, 64, dtype=BF16, device=DEV)
    kept = ops.checkpoint_encode(x)
    bad = [
        lambda: ops.attention(q.cpu(), q, q), lambda: ops.attention(q.half(), q.half(), q.half()),
        lambda: ops.attention(q, q.float(), q), lambda: ops.attention(q, q[:1], q), lambda: ops.attention(q, q, q[:, :4]),
        lambda: ops.attention(q, q[..., :32], q[..., :32]), lambda: ops.attention(q[0], q, q),
        lambda: ops.attention(q, q, q, q_lens=torch.zeros(2, device=DEV)), lambda: ops.attention(q, q, q, kv_lens=lens([1, 2, 3])),
        lambda: ops.attention(q, q, q, kv_lens=torch.zeros(2, dtype=torch.int32)),
        lambda: ops.attention_backward(q, q, q, q, out, lse[:, :, :4]), lambda: ops.attention_backward(q[:, :4], q, q, q, out, lse),
        lambda: ops.attention_backward(q.float(), q, q, q, out, lse), lambda: ops.attention_backward(q, q, q, q, out, lse.double()),
        lambda: ops.checkpoint_encode(x.half()), lambda: ops.checkpoint_encode(x[:, :0]), lambda: ops.checkpoint_encode(x.cpu()),
        lambda: ops.checkpoint_decode(kept, torch.float16), lambda: ops.checkpoint_decode(kept._replace(cols=65)),
        lambda: ops.checkpoint_decode(kept._replace(codes=kept.codes[:4])), lambda: ops.checkpoint_weight_grad(x[:4], kept),
        lambda: ops.checkpoint_weight_grad(x.half(), kept), lambda: ops.add_rms_norm(x, x.float(), w),
        lambda: ops.add_rms_norm(x, x[:4], w), lambda: ops.add_rms_norm(x, x, w[:32]), lambda: ops.add_rms_norm(x, x, w.to(BF16)),
        lambda: ops.add_rms_norm_backward(x, x[:4], w, w[:8]), lambda: ops.add_rms_norm_backward(x, x, w, w),
        lambda: ops.add_rms_norm_backward(x, x, w, w[:8], dh=x.float()),
    ]
    for n, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            print("not refused:", n)
    for f in (lambda: ops.attention(q[..., :63].contiguous(), q[..., :63].contiguous(), q[..., :63].contiguous()),
              lambda: ops.attention(q, q[:, :, :3], q[:, :, :3]), lambda: ops.attention(q, q, q, scale=0.0),
              lambda: ops.attention(q, q, q, scale=-1.0), lambda: ops.attention(q, q, q, scale=NAN),
              lambda: ops.attention(torch.cat([q] * 3, -1), torch.cat([q] * 3, -1), torch.cat([q] * 3, -1)),
              lambda: ops.add_rms_norm(x, x, w, -1.0), lambda: ops.add_rms_norm(x, x, w, NAN),
              lambda: ops.add_rms_norm(torch.zeros(1, 32776, device=DEV), None, torch.ones(32776, device=DEV))):
        with pytest.raises(DearError):
            f()
