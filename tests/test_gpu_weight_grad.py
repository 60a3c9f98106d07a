"""GPU: the weight gradient from a checkpoint in the forms that the sizes of test_gpu_ops.py do not reach, against the definition in 64
bits; bounds as derived in ops_reference.py."""
from __future__ import annotations

import ctypes as C
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


@pytest.fixture(scope="module")
def ops():
    from paper_2302_12445_amd import ops as m
    m.load_library()
    return m


def inputs(ops, rows, outs, ins, dtype):
    gen = torch.Generator().manual_seed(rows + outs + ins)
    x = torch.randn(rows, ins, generator=gen) * torch.exp(2 * torch.randn(rows, 1, generator=gen))
    return torch.randn(rows, outs, generator=gen).to(dtype).to(DEV), ops.checkpoint_encode(x.to(dtype).to(DEV))


def check(ops, dy, kept):
    dw = ops.checkpoint_weight_grad(dy, kept)
    ref.within(dw, *ref.weight_grad(dy, kept.codes, kept.exponents, kept.cols), "dw")
    return dw


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("outs,ins", [(64, 130), (50, 96)])
@pytest.mark.parametrize("rows", [1, 3, 31, 33, 100, 127, 129, 260])
def test_infinity_in_the_last_row(ops, rows, outs, ins, dtype):
    """It makes infinities of its output's row (NaN where a code is 0), whatever rows a kernel's last step has to fill up with."""
    dy, kept = inputs(ops, rows, outs, ins, dtype)
    dy[-1, 20] = math.inf
    dy[-1, 37] = -math.inf
    dw = check(ops, dy, kept)
    assert torch.isinf(dw[20]).any() and torch.isinf(dw[37]).any()


def splits(ops, rows, outs, ins):
    """Splits of a bf16 call, from its workspace: the most that one of the kernels that may take it makes."""
    need = C.c_int64()
    assert ops.load_library().dear_checkpoint_weight_grad_workspace(1, rows, outs, ins, C.byref(need)) == 0
    assert need.value % (outs * ins * 4) == 0
    return max(1, need.value // (outs * ins * 4))


# rows in steps of 128: two and three of them, five and six, nine and more, whole ones and not
@pytest.mark.parametrize("rows", [200, 256, 300, 520, 640, 700, 768, 1100, 1280, 1300])
def test_many_steps_in_one_sum(ops, rows):
    """As many tiles as there are CUs, so that rows are not split: bf16, whole vectors, one step after another in two buffers."""
    outs, ins = 2048, 2040
    print("case", rows, flush=True)
    assert splits(ops, rows, outs, ins) == 1
    check(ops, *inputs(ops, rows, outs, ins, BF16))


@pytest.mark.parametrize("rows,outs,ins", [(16384, 512, 2048), (16300, 504, 2040), (9000, 128, 4096), (3001, 1024, 2048)])
def test_many_steps_in_splits(ops, rows, outs, ins):
    n = splits(ops, rows, outs, ins)
    print("case", rows, outs, ins, n, flush=True)
    assert n > 1 and rows > 4 * 128 * n
    check(ops, *inputs(ops, rows, outs, ins, BF16))


@pytest.mark.parametrize("rows,outs,ins", [(128, 2048, 4096), (200, 2056, 4090), (40, 4096, 2048)])
def test_few_rows_of_wide_layers(ops, rows, outs, ins):
    """More tiles than CUs and few steps: bf16, whole vectors, several workgroups a CU."""
    print("case", rows, outs, ins, flush=True)
    assert splits(ops, rows, outs, ins) == 1
    check(ops, *inputs(ops, rows, outs, ins, BF16))


@pytest.mark.parametrize("rows,outs,ins", [(700, 1003, 771), (1300, 2045, 1999)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_many_steps_of_odd_sizes(ops, rows, outs, ins, dtype):
    print("case", rows, outs, ins, dtype, flush=True)
    check(ops, *inputs(ops, rows, outs, ins, dtype))


@pytest.mark.parametrize("apart", [1 << 24, (1 << 24) + 8, (1 << 24) - 8, (1 << 24) + 3])
def test_rows_far_apart(ops, apart):
    """Rows of dy 2^24 elements apart, more than 2^30 in all."""
    dy, kept = inputs(ops, 70, 64, 96, BF16)
    base = torch.empty(69 * apart + 64, dtype=BF16, device=DEV)
    far = base.as_strided((70, 64), (apart, 1))
    far.copy_(dy)
    assert torch.equal(check(ops, far, kept), check(ops, dy, kept)) or apart >= 1 << 24  # (the same kernel: the same bits)
