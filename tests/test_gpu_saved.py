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
