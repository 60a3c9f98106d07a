"""GPU: what saved_in_8_bits keeps as checkpoints, and what it leaves as it is."""
from __future__ import annotations

import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
linear, gelu = torch.nn.functional.linear, torch.nn.functional.gelu


@pytest.fixture(scope="module")
def layers():
    from paper_2302_12445_amd import layers as m
    return m


def normal(*shape, seed=0, dtype=F32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).to(DEV)


def gradients(context, loss, *wanted):
    with context:
        out = loss()
    return torch.autograd.grad(out, wanted)


# ------------------------------------------------------------------------------------ weights
WEIGHTS = {
    "whole": lambda w: w, "turned": lambda w: w.t().contiguous().t(), "cast": lambda w: w.to(BF16), "turned and cast": lambda w: w.t().to(BF16).t(),
    "part": lambda w: w[:512], "split": lambda w: w.split([256, 768])[1], "joined": lambda w: torch.cat([w[:300], w[300:]]),
    "joined casts": lambda w: torch.cat([w[:300].to(BF16), w[300:].to(BF16)]), "viewed": lambda w: w.view(2, 512, 256)[1].reshape(-1, 256),
}


@pytest.mark.parametrize("trained", [True, False])
@pytest.mark.parametrize("form", list(WEIGHTS))
def test_weights_are_left_as_they_are(layers, form, trained):
    """A product keeps a view of its weight, or a cast, for its input's gradient, which has to be of the weight itself."""
    weight = torch.nn.Parameter(normal(1024, 256, seed=1), requires_grad=trained)
    used = WEIGHTS[form](weight)
    x = normal(300, 256, dtype=used.dtype).requires_grad_()
    def loss():
        return (linear(x * 1.0, WEIGHTS[form](weight)) * scale).sum()
    scale = normal(300, used.shape[0], seed=2, dtype=used.dtype)
    want, = gradients(torch.autograd.graph.saved_tensors_hooks(lambda t: t.detach(), lambda t: t), loss, x)
    got, = gradients(layers.saved_in_8_bits(), loss, x)
    assert torch.equal(got, want)
    # and the input of the product, an activation, is still kept in 8 bits
    if trained:
        got, = gradients(layers.saved_in_8_bits(), loss, weight)
        want, = gradients(layers.saved_in_8_bits(least=1 << 40), loss, weight)
        assert not torch.equal(got, want) and (got - want).norm() < 0.02 * want.norm()


# ------------------------------------------------------------------------------------ the framework's own functions
@pytest.mark.parametrize("ragged", [False, True])
def test_attend_keeps_what_it_keeps(layers, ragged):
    """Its log-sum-exp in 8 bits would be up to 3 % off in every probability, and NaN beside a padded row's infinity."""
    q, k, v = (normal(16, 512, 16, 64, seed=n, dtype=BF16).requires_grad_() for n in range(3))
    lens = torch.arange(512, 256, -16, dtype=torch.int32, device=DEV) if ragged else None
    scale = normal(16, 512, 16, 64, seed=4, dtype=BF16)
    def loss():
        return (layers.attend(q * 1.0, k * 1.0, v * 1.0, q_lens=lens, kv_lens=lens) * scale).sum()
    want = gradients(layers.saved_in_8_bits(least=1 << 40), loss, q, k, v)
    got = gradients(layers.saved_in_8_bits(), loss, q, k, v)
    for a, b in zip(got, want):
        assert torch.equal(a, b) and torch.isfinite(a).all()


def test_norm_keeps_what_it_keeps(layers):
    norm = layers.AddRMSNorm(64).to(DEV)
    x, residual = (normal(1 << 16, 64, seed=n).requires_grad_() for n in range(2))
    scale = normal(1 << 16, 64, seed=2)
    def loss():
        h, y, _ = norm(x * 1.0, residual * 1.0)
        return (y * scale + h).sum()
    want = gradients(layers.saved_in_8_bits(least=1 << 40), loss, x, residual, norm.weight)
    for a, b in zip(gradients(layers.saved_in_8_bits(), loss, x, residual, norm.weight), want):
        assert torch.equal(a, b)


def test_a_whole_block_in_8_bits(layers):
    """What is not the block's own functions is the GELU, which it keeps in 8 bits itself."""
    torch.manual_seed(3)
    block = layers.TransformerBlock(256, 4, 2).to(DEV)
    x, residual = (normal(8, 100, 256, seed=n, dtype=BF16).requires_grad_() for n in range(2))
    lens = torch.tensor([100, 71, 1, 50, 99, 100, 3, 64], dtype=torch.int32, device=DEV)
    scale = normal(8, 100, 256, seed=2, dtype=BF16)
    def loss():
        out, h = block(x, residual, lens)
        return (out * scale + h).sum()
    wanted = (x, residual, *block.parameters())
    want = gradients(torch.enable_grad(), loss, *wanted)
    for a, b in zip(gradients(layers.saved_in_8_bits(), loss, *wanted), want):
        assert torch.equal(a, b) and torch.isfinite(a).all()


# ------------------------------------------------------------------------------------ what takes no part in the gradient
def test_statistics_are_left_as_they_are(layers):
    """A layer norm of torch's keeps its rows' means and factors, no activations: with as many rows as are worth keeping in 8
    bits, the gradient is that of the input in 8 bits with these."""
    from paper_2302_12445_amd import ops
    rows = 1 << 16
    x = (normal(rows, 96, seed=1) * torch.exp(normal(rows, 1, seed=2))).requires_grad_()
    scale = normal(rows, 96, seed=3)
    def loss():
        return (torch.nn.functional.layer_norm(x * 1.0, (96,)) * scale).sum()
    got, = gradients(layers.saved_in_8_bits(), loss, x)
    # the formula, from the statistics of x and its values in 8 bits
    a = x.detach()
    mean, factor = a.mean(1, keepdim=True), torch.rsqrt(a.var(1, unbiased=False, keepdim=True) + 1e-5)
    n = (ops.checkpoint_decode(ops.checkpoint_encode(a), F32) - mean) * factor
    want = (scale - scale.mean(1, keepdim=True) - n * (scale * n).mean(1, keepdim=True)) * factor
    assert (got - want).norm() <= 1e-5 * want.norm()


# ------------------------------------------------------------------------------------ memory
def requested():
    """Bytes of the tensors that there are, without what the allocator's blocks have beyond them, which depends on the calls before."""
    return torch.cuda.memory_stats()["requested_bytes.all.current"]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("shape", [(512, 1024), (70001, 1), (30000, 33), (200000, 3), (7, 11, 13, 129), (5000, 14)])
def test_what_is_kept_is_never_larger(layers, shape, dtype):
    """33 bytes for every 32 values of a row, the last of which are filled up; where that is no less than the values themselves
    (short rows), these.  The gradient is the GELU's at the values kept."""
    from paper_2302_12445_amd import ops
    n, size = torch.Size(shape).numel(), dtype.itemsize
    codes = n // shape[-1] * -(-shape[-1] // 32) * 33
    u = normal(*shape, dtype=dtype).requires_grad_()
    gelu(u * 1.0).sum().backward()  # (libraries' workspaces)
    u.grad = None
    torch.cuda.synchronize()
    before = requested()
    with layers.saved_in_8_bits(least=1000):
        z = gelu(u * 1.0).sum()
    kept = requested() - before
    assert kept > 0
    assert kept <= min(codes, n * size) + 4096
    z.backward()
    value = u.detach()
    if codes < n * size:
        value = ops.checkpoint_decode(ops.checkpoint_encode(value), dtype).view(shape)
    value = value.requires_grad_()
    gelu(value).sum().backward()
    assert torch.equal(u.grad, value.grad)


def test_a_norm_s_factors_by_hand(layers):
    """A column of factors, one of them huge as a padded row's is: its neighbours' gradients are those of their own factors."""
    x = normal(1 << 16, 64)
    x[100] = 0
    x.requires_grad_()
    scale = normal(1 << 16, 64, seed=1)
    def loss():
        y = x * 1.0
        return (y * torch.rsqrt(y.square().mean(1, keepdim=True) + 1e-12) * scale).sum()
    want, = gradients(layers.saved_in_8_bits(least=1 << 40), loss, x)
    got, = gradients(layers.saved_in_8_bits(), loss, x)
    rest = torch.arange(1 << 16, device=DEV) != 100
    assert (got - want)[rest].norm() < 0.02 * want[rest].norm()


def test_single_values_and_nothing(layers):
    u = normal(3).requires_grad_()
    with layers.saved_in_8_bits(least=0):
        z = gelu(u[0] * 1.0) + gelu(u[1:1] * 1.0).sum() + gelu(u * 1.0).sum()
    z.backward()
    w = u.detach().clone().requires_grad_()
    (gelu(w[0]) + gelu(w).sum()).backward()
    assert (u.grad - w.grad).abs().max() <= 2 * u.abs().max() / 127
