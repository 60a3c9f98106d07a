"""GPU: calls of more threads than one launch takes (2^32), on tensors of a few columns; what they give is compared with calls on
parts of them, which test_gpu_ops.py compares with the definitions."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def ops():
    from paper_2302_12445_amd import ops as m
    m.load_library()
    return m


@pytest.fixture(autouse=True)
def memory_given_back():
    yield
    torch.cuda.empty_cache()


def random(rows, cols, dtype, seed):
    return torch.randn(rows, cols, generator=torch.Generator(DEV).manual_seed(seed), device=DEV, dtype=dtype)


def parts(rows, edge):
    """The first rows, those around a multiple of the edge, and the last."""
    return [(0, 1000), (edge - 500, edge + 500), (rows - 1000, rows)]


@pytest.mark.parametrize("residual", [False, True])
def test_norm_of_2_to_the_26_rows(ops, residual):
    """As a norm of the heads of a million tokens."""
    rows, cols = (1 << 26) + 1003, 8
    print("case", rows, cols, residual, flush=True)
    x, r = random(rows, cols, BF16, 1), random(rows, cols, BF16, 2) if residual else None
    weight = random(1, cols, F32, 3)[0]
    h, y, kept, rstd = ops.add_rms_norm(x, r, weight)
    for a, b in parts(rows, 1 << 26):
        want = ops.add_rms_norm(x[a:b], r[a:b] if residual else None, weight)
        got = h[a:b], y[a:b], ops.Checkpoint(kept.codes[a:b], kept.exponents[a:b], cols), rstd[a:b]
        for p, q in zip((*got[:2], *got[2][:2], got[3]), (*want[:2], *want[2][:2], want[3])):
            assert torch.equal(p, q)


@pytest.mark.parametrize("cols", [1, 32])
def test_checkpoint_of_2_to_the_32_pieces(ops, cols):
    """Rows of one value, each filled up to a group, and rows of whole groups: 2^32 pieces of eight codes."""
    rows, edge = (1 << 30) + 1003, 1 << 29
    print("case", rows, cols, flush=True)
    x = random(rows, cols, BF16, 1) if cols == 1 else torch.empty(rows, cols, dtype=BF16, device=DEV)
    near = parts(rows, edge) + parts(rows, 2 * edge)[1:2]
    if cols > 1:  # values where they are looked at
        for n, (a, b) in enumerate(near):
            x[a:b] = random(b - a, cols, BF16, n)
    kept = ops.checkpoint_encode(x)
    for a, b in near:
        want = ops.checkpoint_encode(x[a:b])
        assert torch.equal(kept.codes[a:b], want.codes) and torch.equal(kept.exponents[a:b], want.exponents)
    del x
    got = ops.checkpoint_decode(kept)
    for a, b in near:
        want = ops.checkpoint_decode(ops.Checkpoint(kept.codes[a:b], kept.exponents[a:b], cols))
        assert torch.equal(got[a:b], want)
