"""GPU: the gated linear recurrence and its backward pass against their definitions in 64 bits, at the lengths, widths, layouts and
values where they can go wrong; bounds as derived in recurrent_reference.py."""
from __future__ import annotations

import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import ops_reference as ref  # noqa: E402
import recurrent_reference as rec  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
NAN = math.nan


@pytest.fixture(scope="module")
def ops():
    from paper_2302_12445_amd import ops as m
    m.load_library()
    return m


def normal(gen, shape, dtype=F32, scale=1.0):
    return (torch.randn(shape, generator=gen) * scale).to(dtype).to(DEV)


def inputs(shape, dtype, seed, state=True):
    """x, gates of memories from a step to some hundred, and a state."""
    gen = torch.Generator().manual_seed(seed)
    B, T, C = shape
    x = normal(gen, shape, dtype)
    gate = (normal(gen, shape) + 6 * torch.rand(C, generator=gen).to(DEV) - 1).to(dtype)
    return x, gate, normal(gen, (B, C)) if state else None


def check(ops, x, gate, state=None, lens=None, dlast=None, seed=0, label=""):
    """Forward and backward; the backward from the states that the forward kept."""
    lens = None if lens is None else torch.tensor(lens, dtype=torch.int32, device=DEV)
    got = ops.recurrence(x, gate, state, lens)
    clean = (x, gate)
    dh = normal(torch.Generator().manual_seed(seed + 1), x.shape, x.dtype)
    if lens is not None:  # what stands behind the lengths is never used
        behind = ~rec._valid(lens, x.shape[0], x.shape[1]).to(DEV)
        clean = tuple(t.masked_fill(behind.unsqueeze(2), 0.0) for t in (x, gate))
        dh.masked_fill_(behind.unsqueeze(2), NAN)
    want, off = rec.recurrence(*clean, state, lens)
    for g, w, o, name in zip(got, want, off, ("h", "last", "kept")):
        ref.within(g, w, o, label + " " + name)
    assert got[0].dtype == x.dtype and got[1].dtype == got[2].dtype == F32
    grads = ops.recurrence_backward(dh, x, gate, got[2], lens, dlast)
    zeros = dh if lens is None else torch.nan_to_num(dh, 0.0)
    want, off = rec.recurrence_backward(zeros, *clean, got[2], lens, dlast)
    for g, w, o, name in zip(grads, want, off, ("dx", "dgate", "dstate")):
        ref.within(g, w, o, label + " " + name)
    return got, grads


SHAPES = [  # batch, steps, width
    (1, 1, 1), (2, 1, 64), (16, 1, 1024), (3, 5, 3), (1, 8, 4), (1, 31, 7), (2, 32, 65), (1, 33, 64), (2, 96, 128), (2, 97, 130),
    (1, 255, 66), (1, 256, 64), (1, 257, 64), (2, 513, 70), (3, 700, 192), (1, 2049, 32), (2, 1024, 2), (1, 4097, 5),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", SHAPES)
def test_recurrence(ops, shape, dtype):
    print("case", shape, dtype, flush=True)
    x, gate, state = inputs(shape, dtype, sum(shape))
    dlast = normal(torch.Generator().manual_seed(5), state.shape)
    check(ops, x, gate, state, dlast=dlast)
    check(ops, x, gate)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [(513, 300, 6), (65, 600, 520), (600, 40, 64), (530, 80, 33)])
def test_sequences_that_fill_the_chip(ops, shape, dtype):
    """More workgroups than the chip takes at a time, of one tile and of several."""
    print("case", shape, dtype, flush=True)
    x, gate, state = inputs(shape, dtype, sum(shape))
    lens = torch.randint(0, shape[1] + 1, (shape[0],), generator=torch.Generator().manual_seed(1)).tolist()
    check(ops, x, gate, state, lens)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("steps", [1, 40, 300, 1000])
def test_lengths(ops, steps, dtype):
    """Lengths of 0 and 1, at the edges of tiles, more than there are and less than none; NaN and infinities in what lies behind them."""
    print("case lengths", steps, dtype, flush=True)
    lens = [0, 1, steps, steps + 9, -3, steps // 2, min(steps, 255), min(steps, 256), min(steps, 257)]
    x, gate, state = inputs((len(lens), steps, 70), dtype, steps)
    for b, n in enumerate(lens):
        x[b, max(n, 0):] = NAN
        gate[b, max(n, 0):] = math.inf if b % 2 else NAN
    dlast = normal(torch.Generator().manual_seed(6), state.shape)
    got, grads = check(ops, x, gate, state, lens, dlast)
    assert torch.equal(got[1][0], state[0]) and torch.equal(grads[2][0], dlast[0])
    assert not got[0][0].any() and not grads[0][0].any() and not grads[1][0].any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layouts(ops, dtype):
    """Parts of one projection, steps before sequences, broadcast inputs, elements off 16 bytes: all as contiguous copies give."""
    B, T, C = 3, 290, 72
    gen = torch.Generator().manual_seed(3)
    joint = normal(gen, (B, T, 3 * C), dtype)
    turned = normal(gen, (T, B, 2 * C), dtype).transpose(0, 1)
    odd = normal(gen, (B, T, 2 * C + 3), dtype)
    wide = normal(gen, (B, T, C, 2), dtype)
    cases = [(joint[..., :C], joint[..., C:2 * C]), (turned[..., :C], turned[..., C:]), (odd[..., 1:C + 1], odd[..., C + 2:2 * C + 2]),
             (joint[:1, :, :C].expand(B, T, C), joint[:, :1, :C].expand(B, T, C)), (wide[..., 0], wide[..., 1]),
             (joint[..., 1:C], joint[..., C + 1:2 * C]), (joint[..., :2], joint[..., 5:7])]
    dh = normal(gen, (T, B, C), dtype).transpose(0, 1)
    for n, (x, gate) in enumerate(cases):
        print("layout", n, dtype, flush=True)
        d = dh[..., :x.shape[2]]
        h, last, kept = ops.recurrence(x, gate)
        plain = ops.recurrence(x.contiguous(), gate.contiguous())
        # (the channels of a lane may differ, what is computed of a channel does not)
        assert all(torch.equal(a, b) for a, b in zip((h, last, kept), plain))
        got = ops.recurrence_backward(d, x, gate, kept)
        want = ops.recurrence_backward(d.contiguous(), x.contiguous(), gate.contiguous(), kept)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_gates_at_their_ends(ops, dtype):
    """Gates of 0, of large magnitude and of infinity: a and 1 - a are then 1 / 2, tiny, or 0 and 1."""
    values = torch.tensor([0.0, -0.0, 1e-3, 20.0, -20.0, 80.0, -80.0, 1e4, -1e4, math.inf, -math.inf, 5.0], device=DEV)
    gen = torch.Generator().manual_seed(9)
    pick = torch.randint(0, len(values), (2, 600, 40), generator=gen).to(DEV)
    x = normal(gen, pick.shape, dtype)
    check(ops, x, values[pick].to(dtype), normal(gen, (2, 40)))


def test_nan_stays_in_its_channel(ops):
    x, gate, state = inputs((2, 600, 40), BF16, 4)
    x[0, 300, 7] = NAN
    gate[1, 10, 9] = NAN
    h, last, kept = ops.recurrence(x, gate, state)
    bad = torch.isnan(h.float())
    assert bad[0, 300:, 7].all() and bad[1, 10:, 9].all() and bad.sum() == 300 + 590
    dx, dgate, _ = ops.recurrence_backward(torch.ones_like(h), x, gate, kept)
    for t in (dx, dgate):
        bad = torch.isnan(t.float())
        bad[0, :, 7] = bad[1, :, 9] = False
        assert not bad.any()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_continued(ops, dtype):
    """A sequence in pieces, single tokens among them, from the state that each piece leaves: as in one call."""
    x, gate, state = inputs((2, 520, 96), dtype, 11)
    want, off = rec.recurrence(x, gate, state, None)
    s, at, parts = state, 0, []
    for n in (256, 1, 1, 200, 0, 62):
        h, s, kept = ops.recurrence(x[:, at:at + n], gate[:, at:at + n], s, keep=False)
        assert kept is None
        parts.append(h)
        at += n
    ref.within(torch.cat(parts, 1), want[0], off[0], "h")
    ref.within(s, want[1], off[1], "last")


@pytest.mark.parametrize("steps,width", [(1, 5), (40, 3), (300, 2)])
def test_gradients_against_differences(ops, steps, width):
    """Central differences of the definition in 64 bits along random directions."""
    x, gate, state = inputs((2, steps, width), F32, 21)
    gen = torch.Generator().manual_seed(22)
    dh, dlast = normal(gen, x.shape), normal(gen, state.shape)
    lens = torch.tensor([steps, max(1, steps - 3)], dtype=torch.int32, device=DEV)
    _, _, kept = ops.recurrence(x, gate, state, lens)
    grads = ops.recurrence_backward(dh, x, gate, kept, lens, dlast)

    def loss(*t):
        (h, last, _), _ = rec.recurrence(*t, lens)
        return (h * ref.f64(dh)).sum() + (last * ref.f64(dlast)).sum()
    point = [ref.f64(t) for t in (x, gate, state)]
    rec.R[torch.float64] = 0.0
    for n in range(3):
        d = torch.randn(point[n].shape, generator=gen, dtype=torch.float64)
        step = 1e-5
        ends = [loss(*[p + sign * step * d if i == n else p for i, p in enumerate(point)]) for sign in (1, -1)]
        want = (ends[0] - ends[1]) / (2 * step)
        # fp32 sums of some hundred terms; the difference itself is exact to 1e-9
        assert abs((ref.f64(grads[n]) * d).sum() - want) < 2e-5 * (ref.f64(grads[n]).abs() * d.abs()).sum() + 1e-8


def test_same_bits_again_and_on_another_stream(ops):
    x, gate, state = inputs((2, 3000, 256), BF16, 31)
    first = ops.recurrence(x, gate, state)
    grads = ops.recurrence_backward(first[0], x, gate, first[2])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = ops.recurrence(x, gate, state)
        more = ops.recurrence_backward(again[0], x, gate, again[2])
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip((*first, *grads), (*again, *more)))


def test_graph(ops):
    """Captured calls, of long sequences and of a token with its state, replayed on new inputs with eager work in between."""
    x, gate, state = inputs((2, 1500, 128), BF16, 41)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ops.recurrence(x, gate, state)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        h, last, kept = ops.recurrence(x, gate, state)
        grads = ops.recurrence_backward(h, x, gate, kept)
        state.copy_(last)
    for seed in (42, 43, 44):
        fresh = inputs(x.shape, BF16, seed)
        for t, v in zip((x, gate, state), fresh):
            t.copy_(v)
        graph.replay()
        want = ops.recurrence(*fresh)
        more = ops.recurrence_backward(want[0], *fresh[:2], want[2])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((h, last, kept, *grads), (*want, *more))) and torch.equal(state, want[1])


def test_state_in_place(ops):
    """last and dstate may be state and dlast themselves."""
    for shape in ((2, 1, 64), (2, 700, 64), (600, 300, 33)):
        x, gate, state = inputs(shape, F32, 51)
        want = ops.recurrence(x, gate, state)
        s, h = state.clone(), torch.empty_like(x)
        lib, (B, T, C) = ops.load_library(), shape
        held, places, head = ops._recurrence_sizes(x, gate, None)
        space, at, need = ops._recurrence_space(head, x.device)
        none = (0, 0, 0)
        packed = ops._RECURRENCE.pack(*head, *places, s.data_ptr(), 0, h.data_ptr(), T * C, C, s.data_ptr(), *none, 0, *none, *none, 0, at, need)
        assert lib.dear_recurrence(packed, torch.cuda.current_stream().cuda_stream) == 0
        assert torch.equal(h, want[0]) and torch.equal(s, want[1])
        dlast = normal(torch.Generator().manual_seed(52), state.shape)
        grads = ops.recurrence_backward(h, x, gate, want[2], dlast=dlast)
        dx, dg = torch.empty_like(x), torch.empty_like(x)
        packed = ops._RECURRENCE.pack(*head, *places, 0, want[2].data_ptr(), *none, 0, h.data_ptr(), T * C, C, dlast.data_ptr(), dx.data_ptr(),
                                      T * C, C, dg.data_ptr(), T * C, C, dlast.data_ptr(), at, need)
        assert lib.dear_recurrence_backward(packed, torch.cuda.current_stream().cuda_stream) == 0
        assert all(torch.equal(a, b) for a, b in zip((dx, dg, dlast), grads))


@pytest.mark.parametrize("shape", [(4000, 1, 65), (4000, 1, 33), (900, 100, 129), (3, 200, 1001), (1, 20, 1)])
def test_state_in_place_of_odd_widths(ops, shape):
    """The last channels of an odd width are not read by a workgroup that does not write them."""
    x, gate, state = inputs(shape, F32, 51)
    want = ops.recurrence(x, gate, state)
    s, h = state.clone(), torch.empty_like(x)
    lib, (B, T, C) = ops.load_library(), shape
    held, places, head = ops._recurrence_sizes(x, gate, None)
    space, at, need = ops._recurrence_space(head, x.device)
    none = (0, 0, 0)
    packed = ops._RECURRENCE.pack(*head, *places, s.data_ptr(), 0, h.data_ptr(), T * C, C, s.data_ptr(), *none, 0, *none, *none, 0, at, need)
    assert lib.dear_recurrence(packed, torch.cuda.current_stream().cuda_stream) == 0
    assert torch.equal(h, want[0]) and torch.equal(s, want[1])
    dlast = normal(torch.Generator().manual_seed(52), state.shape)
    grads = ops.recurrence_backward(h, x, gate, want[2], dlast=dlast)
    dx, dg = torch.empty_like(x), torch.empty_like(x)
    packed = ops._RECURRENCE.pack(*head, *places, 0, want[2].data_ptr(), *none, 0, h.data_ptr(), T * C, C, dlast.data_ptr(), dx.data_ptr(),
                                  T * C, C, dg.data_ptr(), T * C, C, dlast.data_ptr(), at, need)
    assert lib.dear_recurrence_backward(packed, torch.cuda.current_stream().cuda_stream) == 0
    assert all(torch.equal(a, b) for a, b in zip((dx, dg, dlast), grads))


def test_far_elements(ops):
    """Sequences whose elements lie further apart than 32 bits count."""
    B, T, C = 3, 300, 64
    x, gate, state = inputs((B, T, C), BF16, 61)
    big = torch.empty(2 * (1 << 31) + T * C, dtype=BF16, device=DEV)
    far = big.as_strided((B, T, C), (1 << 31, C, 1))
    far.copy_(x)
    want = ops.recurrence(x, gate, state)
    got = ops.recurrence(far, gate, state)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    wide = big.as_strided((1, T, C), (0, (1 << 22) - 8, 1))  # steps as far apart as a call takes
    wide.copy_(x[:1])
    got = ops.recurrence(wide, gate[:1], state[:1])
    assert all(torch.equal(a, b[:1]) for a, b in zip(got, want))


def test_refusals(ops):
    """Wrong arguments raise before anything is enqueued."""
    from paper_2302_12445_amd import DearError
    x, gate, state = inputs((2, 5, 8), F32, 71)
    _, _, kept = ops.recurrence(x, gate, state)
    lens = torch.tensor([5, 2], dtype=torch.int32, device=DEV)
    for call in (lambda: ops.recurrence(x, gate[:, :4]), lambda: ops.recurrence(x[0], gate[0]), lambda: ops.recurrence(x, gate.cpu()),
                 lambda: ops.recurrence(x, gate, state.cpu()), lambda: ops.recurrence(x, gate, state[:1]), lambda: ops.recurrence(x, gate, state.bfloat16()),
                 lambda: ops.recurrence(x, gate, state, lens.cpu()), lambda: ops.recurrence(x, gate, state, lens.long()),
                 lambda: ops.recurrence(x, gate, state, lens[:1]), lambda: ops.recurrence(x[..., :0], gate[..., :0]),
                 lambda: ops.recurrence_backward(x[:, :4], x, gate, kept), lambda: ops.recurrence_backward(x, x, gate, kept[:, :0]),
                 lambda: ops.recurrence_backward(x, x, gate, kept, dlast=state[:, ::2])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ops.recurrence(x.half(), gate.half()), lambda: ops.recurrence(x, gate.bfloat16()),
                 lambda: ops.recurrence_backward(x.bfloat16(), x, gate, kept)):
        with pytest.raises((TypeError, ValueError)):
            call()
    wide = torch.zeros(1, 1, device=DEV).expand(2, 1 << 22)
    with pytest.raises(DearError):
        ops.recurrence(wide[None], wide[None])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("width", [1, 2, 63, 64, 1001])
def test_one_step(ops, width, dtype):
    """One step, of which some sequences have none, with a state and without, apart and of larger tensors."""
    x, gate, state = inputs((70, 1, width), dtype, 81)
    lens = [int(b % 3 > 0) for b in range(70)]
    check(ops, x, gate, state)
    check(ops, x, gate, state, lens)
    check(ops, x, gate, None, lens)
    wide = torch.empty(70, 3, 2 * width + 1, dtype=dtype, device=DEV).fill_(NAN)
    part = wide[:, 1:2, 1:width + 1]
    part.copy_(x)
    assert all(torch.equal(a, b) for a, b in zip(ops.recurrence(part, gate, state), ops.recurrence(x, gate, state)))


STEADY = [-1.0, 0.0, 2.0, 5.0, 8.0, 9.1, 10.2, 11.5, 12.0, 13.3, 14.1]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("steps", [513, 8192, 32845])
def test_steady_gates_add_nothing_up(ops, steps, dtype):
    """A state of 1, inputs of 1 and gates that stay: all states are 1, and with gradients of 1 - a each step's is 1, however long the
    sequence is.  In half units of fp32: a and b are off by less than 5 from their sum of 1 in each of a strip's sixteen steps, which go by a
    alone; H and 1 - A differ by four at each of the 17 levels that join 129 tiles, by 70 in a strip (of sixteen steps, which a's error and
    a rounding each move) and by 95 in a strip that forgets half (5 over 1 - a of at least 1 / 20), of which as much again is left by the
    maps before; nine levels within a tile go by A alone, two each: 494 in all, below 2^-15.  The gates' own error, below 2^-18 for these,
    moves the gradients with it."""
    print("case steady", steps, dtype, flush=True)
    gate = torch.tensor(STEADY, device=DEV).to(dtype).expand(2, steps, len(STEADY))
    x, state = torch.ones_like(gate), torch.ones(2, len(STEADY), device=DEV)
    h, last, kept = ops.recurrence(x, gate, state)
    for got, r in ((h, ref.R[dtype]), (last, 0.0), (kept, 0.0)):
        off = (got.double() - 1).abs().amax(tuple(range(got.dim() - 1)))
        assert (off <= 2.0 ** -15 + r).all(), off
    b = 1 / (1 + torch.exp(ref.f64(gate[:, 0])))
    dh = b.to(dtype).to(DEV)  # what its rounding makes of the gradients is known
    unit = (ref.f64(dh) / b)[0].to(DEV)
    dlast = (unit * (1 - b[0].to(DEV))).float().expand(2, -1).contiguous()
    dx, _, dstate = ops.recurrence_backward(dh.unsqueeze(1).expand_as(x), x, gate, kept, dlast=dlast)
    for got, want, r in ((dx, unit * b[0].to(DEV), ref.R[dtype]), (dstate, unit * (1 - b[0].to(DEV)), 0.0)):
        off = (got.double() / want - 1).abs().amax(tuple(range(got.dim() - 1)))
        assert (off <= 2.0 ** -15 + 2.0 ** -18 + r).all(), off


@pytest.mark.parametrize("piece", [1, 7, 256])
def test_steady_gates_add_nothing_up_over_calls(ops, piece):
    """The same, token by token and in pieces, each from the state that the one before leaves; a piece is one level or three."""
    gate = torch.tensor(STEADY, device=DEV).expand(2, piece, len(STEADY)).contiguous()
    x, state = torch.ones_like(gate), torch.ones(2, len(STEADY), device=DEV)
    for _ in range(2500):
        h, state, _ = ops.recurrence(x, gate, state, keep=False)
    assert ((h.double() - 1).abs() <= 2.0 ** -15).all() and ((state.double() - 1).abs() <= 2.0 ** -15).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("steps", [2, 16, 40, 257, 700])
def test_what_is_forgotten_stays_so(ops, steps, dtype):
    """Gates whose products pass the smallest number that fp32 holds, and the largest of their inverses, after any number of steps: nothing is left of
    a state, or of a gradient behind, of 10^6."""
    print("case forgotten", steps, dtype, flush=True)
    gate = torch.cat([-torch.logspace(0, 2, 400), torch.linspace(-5.7, -5.3, 101), torch.linspace(-45, -42, 101)]).to(DEV)
    C = gate.numel()
    gen = torch.Generator().manual_seed(111)
    state, dlast = (1e6 * (1 + torch.rand(2, C, generator=gen)).to(DEV) for _ in range(2))
    check(ops, normal(gen, (2, steps, C), dtype), gate.to(dtype).expand(2, steps, C), state, dlast=dlast)
    check(ops, normal(gen, (2, steps, C), dtype), gate.to(dtype).expand(2, steps, C), state, [steps, steps // 2 + 1], dlast)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("gate", [4.0, 12.0])
def test_infinity_stays(ops, gate, dtype):
    """An infinite state of a channel that remembers it stays one, and becomes a NaN only where the other infinity meets it; backward likewise."""
    x = normal(torch.Generator().manual_seed(91), (2, 1300, 6), dtype)
    g = torch.full_like(x, gate)
    state = torch.zeros(2, 6, device=DEV)
    state[0, 1], x[0, 300, 2], x[1, 40, 3], x[0, 20, 4], x[0, 900, 4] = -math.inf, math.inf, -math.inf, math.inf, -math.inf
    want, _, kept = ops.recurrence(x, g, state)
    bad = torch.zeros(2, 1300, 6, device=DEV)
    bad[0, :, 1], bad[0, 300:, 2], bad[1, 40:, 3], bad[0, 20:900, 4] = -math.inf, math.inf, -math.inf, math.inf
    bad[0, 900:, 4] = NAN
    h = want.float()
    assert torch.equal(torch.isnan(h), torch.isnan(bad))
    assert torch.equal(torch.where(torch.isfinite(h), 0.0, h.nan_to_num(7.0, math.inf, -math.inf)), bad.nan_to_num(7.0, math.inf, -math.inf))
    dh = normal(torch.Generator().manual_seed(92), x.shape, dtype)
    dh[1, 700, 0], dh[0, 1299, 5] = math.inf, -math.inf
    dx, _, dstate = ops.recurrence_backward(dh, torch.zeros_like(x), g, torch.zeros_like(kept))
    assert (dx[1, :701, 0] == math.inf).all() and torch.isfinite(dx[1, 701:, 0].float()).all() and (dx[0, :, 5] == -math.inf).all()
    assert dstate[1, 0] == math.inf and dstate[0, 5] == -math.inf and torch.isfinite(dstate).sum() == 10
    token = ops.recurrence(x[:, :1], g[:, :1], state)[1]
    assert token[0, 1] == -math.inf and torch.isfinite(token).sum() == 11


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [(2, 40, 131), (2, 700, 66), (3, 1000, 1003), (1, 5000, 67)])
def test_a_channel_s_place_changes_no_bit(ops, shape, dtype):
    """Of a lane's two channels both are computed alike: shifted by one, and with an odd width, whose last but one is taken twice, a channel has the
    same bits, in each run."""
    x, gate, state = inputs(shape, dtype, 95)
    dh = normal(torch.Generator().manual_seed(96), shape, dtype)
    first = ops.recurrence(x, gate, state)
    grads = ops.recurrence_backward(dh, x, gate, first[2])
    for _ in range(5):
        again = ops.recurrence(x[..., 1:], gate[..., 1:], state[:, 1:].contiguous())
        more = ops.recurrence_backward(dh[..., 1:], x[..., 1:], gate[..., 1:], again[2])
        assert all(torch.equal(a, b[..., 1:]) for a, b in zip((*again, *more), (*first, *grads)))


@pytest.mark.parametrize("steps", [1, 2, 300])
def test_gates_to_all_bits(ops, steps):
    """a and 1 - a of fp32 gates of all sizes, as they come out where the state, the input or the gradient is 1 and the others 0, are each off by
    8 units of 2^-24 and a rounding at most, whatever the gate is; where fp32 does not hold them in full, by exp(-87.3365), 2^-125.99995: 1 / a stops there,
    so that it is in range, and a b below 2^-126 may be 0."""
    least = math.exp(-87.3365) * (1 + 9 * 2.0 ** -24)
    gen = torch.Generator().manual_seed(101)
    gate = torch.cat([torch.linspace(-100, 100, 4001), 20 * torch.randn(4000, generator=gen), torch.randn(4000, generator=gen)]).to(DEV)
    C = gate.numel()
    gates = gate.view(1, 1, C).expand(1, steps, C)
    a, b = 1 / (1 + torch.exp(-ref.f64(gate))), 1 / (1 + torch.exp(ref.f64(gate)))
    x = torch.zeros(1, steps, C, device=DEV)
    x[:, 0] = 1
    none, one = torch.zeros(1, C, device=DEV), torch.ones(1, C, device=DEV)
    got_b = ops.recurrence(x, gates, none)[0][0, 0]
    got_a = ops.recurrence(torch.zeros_like(x), gates, one)[0][0, 0]
    dh = torch.zeros_like(x)
    dh[:, 0] = 1  # (of a step in the middle the sum behind it is 0 likewise)
    dx, _, dstate = ops.recurrence_backward(dh, torch.zeros_like(x), gates, torch.zeros(1, -(-steps // 256), C, device=DEV))
    for got, want, name in ((got_b, b, "b"), (got_a, a, "a"), (dx[0, 0], b, "dx"), (dstate[0], a, "dstate")):
        off = (ref.f64(got) - want).abs()
        worst = ((off - least).clamp(min=0) / want).max().item() * 2 ** 24
        print("steps %d %s: %.2f units" % (steps, name, worst), flush=True)
        assert (off <= 9 * 2.0 ** -24 * want + least).all(), name
