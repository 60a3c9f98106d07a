"""GPU: products grouped by expert and both gradients against their definitions in 64 bits; bounds as derived in
recurrent_reference.py."""
from __future__ import annotations

import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import experts_cases  # noqa: E402
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


def ends_of(counts):
    return torch.tensor(counts).cumsum(0).to(torch.int32).to(DEV)


def check(ops, x, weight, dy, ends):
    """All three products; rows behind the last expert's hold NaN, which reaches nothing."""
    for got, (want, off), name in ((ops.expert_linear(x, weight, ends), rec.expert_linear(x, weight, ends), "y"),
                                   (ops.expert_input_grad(dy, weight, ends), rec.expert_input_grad(dy, weight, ends), "dx"),
                                   (ops.expert_weight_grad(dy, x, ends), rec.expert_weight_grad(dy, x, ends), "dw")):
        assert got.dtype == (F32 if name == "dw" else x.dtype) and got.is_contiguous()
        ref.within(got, want, off, name)


def make(counts, spare, outs, ins, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    M = sum(counts) + spare
    x, dy, w = normal(gen, (M, ins), dtype), normal(gen, (M, outs), dtype), normal(gen, (len(counts), outs, ins), dtype, ins ** -0.5)
    if spare:
        x[-spare:], dy[-spare:] = NAN, NAN
    return x, w, dy, ends_of(counts)


CASES = [  # rows of each expert, rows behind the last, outs, ins
    ([1], 0, 1, 1), ([1], 0, 64, 64), ([0, 1, 0], 0, 24, 40), ([3, 0, 5], 2, 17, 33), ([0, 0], 3, 8, 8), ([128, 128], 0, 128, 128),
    ([127, 129, 0, 1], 0, 136, 72), ([40, 300, 7], 5, 130, 257), ([256, 0, 511, 3, 1], 0, 256, 192), ([33] * 20, 0, 64, 96),
    ([5, 0, 1] * 50, 4, 72, 40), ([700], 100, 320, 136), ([2, 1, 3, 2, 1, 4, 2, 1], 0, 1024, 520), ([17, 16, 33, 15], 9, 520, 1032),
    ([64, 32, 31, 65], 0, 264, 2056), ([1000, 24], 0, 384, 328),
]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_experts(ops, case, dtype):
    counts, spare, outs, ins = CASES[case]
    print("case", len(counts), sum(counts), spare, outs, ins, dtype, flush=True)
    check(ops, *make(counts, spare, outs, ins, dtype, case))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_ends_that_do_not_ascend(ops, dtype):
    """Ends below the one before, below zero and beyond the rows: taken as dear_ops.h says, nothing outside is touched."""
    x, w, dy, _ = make([150, 150], 0, 72, 136, dtype, 3)
    x, dy = x[:290], dy[:290]
    for ends in ([100, 50], [-5, 400], [290, 0], [400, 300], [0, -1], [-2 ** 31, 2 ** 31 - 1]):
        check(ops, x, w, dy, torch.tensor(ends, dtype=torch.int32, device=DEV))


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layouts(ops, dtype):
    """Rows far apart, off 16 bytes, and in columns; a weight whose axes are turned: as contiguous copies give."""
    counts, M, N, K = [30, 0, 171], 201, 72, 136
    gen = torch.Generator().manual_seed(5)
    wide, ends = normal(gen, (M, N + K + 9), dtype), ends_of(counts)
    turned = normal(gen, (3, K, N), dtype).transpose(1, 2)
    for dy, x in ((wide[:, :N], wide[:, N:N + K]), (wide[:, 1:N + 1], wide[:, N + 3:N + K + 3]),
                  (wide[:, :N].t().contiguous().t(), wide[:, N:N + K].t().contiguous().t())):
        check(ops, x, turned, dy, ends)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_not_a_number_stays_with_its_factors(ops, dtype):
    """NaN in one expert's rows and another's weights, and infinities next to the sum's end."""
    x, w, dy, ends = make([100, 40, 60], 0, 136, 200, dtype, 7)
    x[105, 199], dy[99, 135], w[2, 3, 4] = NAN, math.inf, NAN
    y, dx, dw = ops.expert_linear(x, w, ends), ops.expert_input_grad(dy, w, ends), ops.expert_weight_grad(dy, x, ends)
    bad = ~torch.isfinite(y.float())
    assert bad[105].all() and bad[140:, 3].all() and bad.sum() == 136 + 60 - 0
    bad = ~torch.isfinite(dx.float())
    assert bad[99].all() and bad[140:, 4].all() and bad.sum() == 200 + 60
    bad = ~torch.isfinite(dw)
    assert bad[0, 135].all() and bad[1, :, 199].all() and bad.sum() == 200 + 136


def test_nothing(ops):
    x, w, dy, _ = make([4], 0, 24, 40, BF16, 9)
    none = torch.zeros(1, dtype=torch.int32, device=DEV)
    assert ops.expert_linear(x[:0], w, none).shape == (0, 24) and ops.expert_input_grad(dy[:0], w, none).shape == (0, 40)
    dw = ops.expert_weight_grad(dy[:0], x[:0], none)
    assert dw.shape == (1, 24, 40) and not dw.any()


@pytest.mark.parametrize("sizes", [([2048, 700, 0, 1100], 512, 1024), ([900, 20, 5000], 1032, 264)])
def test_long_sums_and_many_tiles(ops, sizes):
    counts, outs, ins = sizes
    check(ops, *make(counts, 0, outs, ins, BF16, 13))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("outs, ins", [(40, 24), (37, 51), (128, 264)])
def test_many_rows_of_few_outputs(ops, outs, ins, dtype):
    """Weight gradients whose rows go to several workgroups; of one expert fewer rows than there are of them."""
    check(ops, *make([3000, 0, 905, 2, 64], 7, outs, ins, dtype, 44))


@pytest.mark.parametrize("counts, outs, ins", [([2500, 0, 2100], 1031, 515), ([600, 900], 37, 2053), ([800, 500], 2053, 130)])
def test_long_sums_of_any_width(ops, counts, outs, ins):
    """Sums beyond 1024 in rows that start anywhere."""
    check(ops, *make(counts, 3, outs, ins, BF16, 46))


@pytest.mark.parametrize("case", range(len(experts_cases.CASES)))
def test_each_way(ops, case):
    """At sizes that take each way that there is (the host's choice is checked on the CPU)."""
    counts, spare, outs, ins, dtype, *ways = experts_cases.CASES[case]
    print("case", len(counts), sum(counts), spare, outs, ins, dtype, ways, flush=True)
    check(ops, *make(counts, spare, outs, ins, {"bf16": BF16, "f32": F32}[dtype], 60 + case))


@pytest.mark.parametrize("outs, ins", [(136, 1000), (1000, 136)])
def test_few_tiles_behind_a_round(ops, outs, ins):
    """66 x 4 tiles of 256: one for each of 256 units, and eight."""
    check(ops, *make([8001, 20, 8200], 5, outs, ins, BF16, 40))


def test_far_weights(ops):
    """Weights of more elements than 31 bits count: the last expert's, and far rows."""
    E, N, K = 9, 16384, 16384
    gen = torch.Generator().manual_seed(15)
    w = torch.empty((E, N, K), dtype=BF16, device=DEV)
    w[E - 1] = normal(gen, (1, K), BF16)  # all rows alike
    w[E - 1, N - 1] = normal(gen, (K,), BF16)
    x, dy = normal(gen, (3, K), BF16), torch.zeros(3, N, dtype=BF16, device=DEV)
    dy[:, N - 1] = 2.0
    ends = torch.tensor([0] * (E - 1) + [3], dtype=torch.int32, device=DEV)
    y = ops.expert_linear(x, w, ends)
    last = w[E - 1][[0, N - 1]].unsqueeze(0)
    want, off = rec.expert_linear(x, last, ends[-1:])
    ref.within(y[:, [0, N - 1]], want, off, "y")
    assert torch.equal(y[:, :1].expand(3, N - 1), y[:, :-1])
    dx = ops.expert_input_grad(dy, w, ends)
    assert torch.equal(dx, (w[E - 1, N - 1].float() * 2).to(BF16).expand(3, K))
    dw = ops.expert_weight_grad(dy, x, torch.tensor([0] * 8 + [3], dtype=torch.int32, device=DEV))
    want, off = rec.expert_weight_grad(dy[:, N - 1:], x, ends[-1:])
    ref.within(dw[E - 1, N - 1:], want[0], off[0], "dw")
    assert not dw[:E - 1].any() and not dw[E - 1, :N - 1].any()


def test_same_bits_again_and_on_another_stream(ops):
    x, w, dy, ends = make([500, 30, 0, 800], 0, 520, 264, BF16, 17)
    first = ops.expert_linear(x, w, ends), ops.expert_input_grad(dy, w, ends), ops.expert_weight_grad(dy, x, ends)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = ops.expert_linear(x, w, ends), ops.expert_input_grad(dy, w, ends), ops.expert_weight_grad(dy, x, ends)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("counts", [[3, 0, 9, 4], [500, 30, 0, 800]])
def test_graph(ops, counts):
    """Captured calls replayed with other rows and other ends, which only the GPU knows."""
    x, w, dy, ends = make(counts, 0, 264, 520, BF16, 19)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ops.expert_linear(x, w, ends)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ops.expert_linear(x, w, ends), ops.expert_input_grad(dy, w, ends), ops.expert_weight_grad(dy, x, ends)
    for n, order in enumerate(([3, 2, 1, 0], [1, 0, 3, 2], [0, 1, 2, 3])):
        fresh = make([counts[i] for i in order], 0, 264, 520, BF16, 20 + n)
        for t, v in zip((x, w, dy, ends), fresh):
            t.copy_(v)
        graph.replay()
        want = ops.expert_linear(*fresh[:2], fresh[3]), ops.expert_input_grad(fresh[2], fresh[1], fresh[3]), ops.expert_weight_grad(fresh[2], fresh[0], fresh[3])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals(ops):
    """Wrong arguments raise before anything is enqueued."""
    from paper_2302_12445_amd import DearError
    x, w, dy, ends = make([3, 4], 1, 16, 24, F32, 81)
    for call in (lambda: ops.expert_linear(x[:, :16], w, ends), lambda: ops.expert_linear(x, w[0], ends), lambda: ops.expert_linear(x, w, ends[:1]),
                 lambda: ops.expert_linear(x, w, ends.long()), lambda: ops.expert_linear(x, w, ends.cpu()), lambda: ops.expert_linear(x, w.cpu(), ends),
                 lambda: ops.expert_linear(x[None], w, ends), lambda: ops.expert_input_grad(dy[:, :8], w, ends),
                 lambda: ops.expert_input_grad(dy, w, ends.view(1, 2)), lambda: ops.expert_weight_grad(dy[:4], x, ends),
                 lambda: ops.expert_weight_grad(dy, x, ends.repeat(2)[::2])):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: ops.expert_linear(x.half(), w.half(), ends), lambda: ops.expert_linear(x, w.bfloat16(), ends),
                 lambda: ops.expert_weight_grad(dy, x.bfloat16(), ends)):
        with pytest.raises((TypeError, ValueError)):
            call()
    with pytest.raises((DearError, ValueError)):
        ops.expert_linear(x, w[:0], ends[:0])
