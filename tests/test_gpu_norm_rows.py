"""GPU: the norm and its backward pass where workgroups take several rows of the widest, against the definition in 64 bits; bounds as
derived in ops_reference.py."""
from __future__ import annotations

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


def normal(gen, shape, dtype):
    return torch.randn(shape, generator=gen).to(dtype).to(DEV)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("rows,cols", [(1100, 2056), (1100, 4096), (2100, 3001), (600, 8200), (600, 16384), (600, 20480), (1030, 5000), (520, 32768)])
def test_more_rows_than_workgroups(ops, rows, cols, dtype):
    """A workgroup adds the terms of the weights' gradient of its rows, one after another."""
    print("case", rows, cols, dtype, flush=True)
    gen = torch.Generator().manual_seed(rows + cols)
    x, residual, dy, dh = (normal(gen, (rows, cols), dtype) for _ in range(4))
    weight = normal(gen, (cols,), F32)
    h, y, kept, rstd = ops.add_rms_norm(x, residual, weight)
    assert torch.equal(h, (x.float() + residual.float()).to(dtype))
    wy, wr, off, roff = ref.norm(h, weight, 1e-5)
    ref.within(y, wy, off, "y")
    ref.within(rstd, wr, roff, "rstd")
    other = ops.checkpoint_encode(y)
    assert torch.equal(kept.codes, other.codes) and torch.equal(kept.exponents, other.exponents)
    for extra in (dh, None):
        dx, dw = ops.add_rms_norm_backward(dy, h, weight, rstd, dh=extra)
        wx, ww, xoff, woff = ref.norm_backward(dy, h, weight, rstd, extra)
        ref.within(dx, wx, xoff, "dx")
        ref.within(dw, ww, woff, "dweight")
