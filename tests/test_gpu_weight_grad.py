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
