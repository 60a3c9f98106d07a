"""CPU checks of the autograd layers: plain torch operations stand in for the calls on the GPU, whose results, as theirs,
carry no graph of their own."""
from __future__ import annotations

import gc
import math
import weakref

import pytest
import torch

from paper_2302_12445_amd import layers, ops


@pytest.fixture
def plain(monkeypatch):
    """The operators in plain torch; gives the names of the calls made."""
    calls = []

    def stand_in(f):
        def call(*args, **kwargs):
            calls.append(f.__name__)
            with torch.no_grad():
                return f(*args, **kwargs)
        monkeypatch.setattr(ops, f.__name__, call)

    def probabilities(q, k):
        return torch.softmax(q.transpose(1, 2) @ k.permute(0, 2, 3, 1) / math.sqrt(q.shape[-1]), -1)

    @stand_in
    def attention(q, k, v, causal=False, scale=None, q_lens=None, kv_lens=None):
        scores = q.transpose(1, 2) @ k.permute(0, 2, 3, 1) / math.sqrt(q.shape[-1])
        return (probabilities(q, k) @ v.transpose(1, 2)).transpose(1, 2).contiguous(), torch.logsumexp(scores, -1)

    @stand_in
    def attention_backward(dout, q, k, v, out, lse, causal=False, scale=None, q_lens=None, kv_lens=None):
        p, g, s = probabilities(q, k), dout.transpose(1, 2), 1 / math.sqrt(q.shape[-1])
        ds = p * (g @ v.permute(0, 2, 3, 1) - (dout * out).sum(-1).transpose(1, 2)[..., None]) * s
        return ((ds @ k.transpose(1, 2)).transpose(1, 2), (ds.transpose(2, 3) @ q.transpose(1, 2)).transpose(1, 2),
                (p.transpose(2, 3) @ g).transpose(1, 2))

    @stand_in
    def add_rms_norm(x, residual, weight, eps=1e-5, keep=True):
        h = x if residual is None else x + residual
        rstd = torch.rsqrt(h.square().mean(-1) + eps)
        y = h * rstd[..., None] * weight
        return h, y, ops.checkpoint_encode(y) if keep else None, rstd.flatten()

    @stand_in
    def add_rms_norm_backward(dy, h, weight, rstd, dh=None):
        r = rstd.view(*h.shape[:-1], 1)
        g, n = dy * weight, h * r
        return (g - n * (g * n).mean(-1, keepdim=True)) * r + (0 if dh is None else dh), (dy * n).flatten(0, -2).sum(0)

    @stand_in
    def checkpoint_encode(x):  # which loses nothing here
        return ops.Checkpoint(x.reshape(-1, x.shape[-1]).clone(), torch.zeros(1, dtype=torch.uint8), x.shape[-1])

    @stand_in
    def checkpoint_weight_grad(dy, kept):
        return dy.reshape(-1, dy.shape[-1]).T @ kept.codes

    return calls


def leaf(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).requires_grad_()


# ------------------------------------------------------------------------------------ second derivatives
# Each loss is taken twice: `near` ends at the layer, whose output's gradient is a constant, `far` goes on behind it.  The penalty has
# a term that does not go through the layer, so that what is missing would not show by itself.
LOSSES = [lambda out: out.sum(), lambda out: out.square().sum()]


@pytest.mark.parametrize("loss", LOSSES)
@pytest.mark.parametrize("which", [0, 1, 2])
def test_attention_refuses_second_derivatives(plain, loss, which):
    t = [leaf(2, 5, 2, 8, seed=n) for n in range(3)]
    first = torch.autograd.grad(loss(layers.attend(*t)), t, create_graph=True)
    with pytest.raises(RuntimeError, match="second"):
        torch.autograd.grad(first[which].square().sum() + t[0].sum() + t[1].sum() + t[2].sum(), t)
    with pytest.raises(RuntimeError, match="second"):
        (first[which].square().sum() + t[0].sum()).backward()


@pytest.mark.parametrize("loss", LOSSES)
@pytest.mark.parametrize("residual", [False, True])
def test_norm_refuses_second_derivatives(plain, loss, residual):
    norm, x, r = layers.AddRMSNorm(8).double(), leaf(6, 8), leaf(6, 8, seed=1) if residual else None
    wanted = [x, norm.weight] + ([r] if residual else [])
    for first in torch.autograd.grad(loss(norm(x, r)[1]), wanted, create_graph=True):
        with pytest.raises(RuntimeError, match="second"):
            torch.autograd.grad(first.square().sum() + x.sum(), x, retain_graph=True)
    # h alone does not need the norm: its gradient is passed on, and that is differentiable
    first, = torch.autograd.grad(norm(x, r)[0].pow(3).sum(), x, create_graph=True)
    h = x if r is None else x + r
    assert torch.allclose(torch.autograd.grad(first.sum(), x)[0], 6 * h)


@pytest.mark.parametrize("loss", LOSSES)
def test_linear_refuses_second_derivatives_of_its_weight_alone(plain, loss):
    linear, x = layers.CheckpointLinear(8, 3).double(), leaf(6, 8)
    dw, = torch.autograd.grad(loss(linear(x)), linear.weight, create_graph=True)
    for t in (x,) if loss is LOSSES[0] else (x, linear.weight, linear.bias):
        with pytest.raises(RuntimeError, match="second"):
            torch.autograd.grad(dw.square().sum() + t.sum(), t, retain_graph=True)
    # the input's gradient is a product with the weight, and the bias's a sum: both can be differentiated
    dx, db = torch.autograd.grad(loss(linear(x)), (x, linear.bias), create_graph=True)
    got = torch.autograd.grad(dx.square().sum() + db.square().sum(), linear.weight)[0]
    w = linear.weight.detach().clone().requires_grad_()
    b = linear.bias.detach().clone().requires_grad_()
    dx, db = torch.autograd.grad(loss(x @ w.t() + b), (x, b), create_graph=True)
    assert torch.allclose(got, torch.autograd.grad(dx.square().sum() + db.square().sum(), w)[0])


def test_first_derivatives_with_a_graph_are_the_same(plain):
    """create_graph alone changes nothing."""
    t = [leaf(2, 5, 2, 8, seed=n) for n in range(3)]
    linear, norm = layers.CheckpointLinear(8, 8).double(), layers.AddRMSNorm(8).double()
    params = t + list(linear.parameters()) + list(norm.parameters())

    def loss():
        h, y, kept = norm(layers.attend(*t))
        return (linear(y, kept) + h).square().sum()
    for a, b in zip(torch.autograd.grad(loss(), params), torch.autograd.grad(loss(), params, create_graph=True)):
        assert torch.equal(a, b) and b.requires_grad and not a.requires_grad


# ------------------------------------------------------------------------------------ work that nobody asks for
def test_linear_makes_no_checkpoint_that_nothing_reads(plain):
    linear, x = layers.CheckpointLinear(8, 3).double(), leaf(6, 8)
    with torch.no_grad():
        want = linear(x)
    assert plain == []
    assert torch.equal(linear(x), want) and plain == ["checkpoint_encode"]
    plain.clear()
    linear.weight.requires_grad_(False)  # a weight that is not trained
    linear(x).sum().backward()
    assert plain == [] and torch.allclose(x.grad, linear.weight.sum(0).expand(6, 8))
    assert linear.bias.grad is not None and linear.weight.grad is None
    with torch.no_grad():
        linear(x, ops.Checkpoint(x, torch.zeros(1, dtype=torch.uint8), 8))
    assert plain == []


def test_norm_without_a_checkpoint(plain, monkeypatch):
    norm, x = layers.AddRMSNorm(8).double(), leaf(6, 8)
    asked = []
    call = ops.add_rms_norm
    monkeypatch.setattr(ops, "add_rms_norm", lambda *args, **kwargs: asked.append(kwargs.get("keep", True)) or call(*args, **kwargs))
    h, y, kept = norm(x, x, keep=False)
    assert kept is None and asked == [False]
    (h + y).sum().backward()
    assert torch.isfinite(x.grad).all() and torch.isfinite(norm.weight.grad).all()
    assert norm(x, x)[2] is not None and norm(x, x, keep=True)[2] is not None and asked == [False, True, True]


def test_block_makes_no_checkpoints_without_gradients(plain, monkeypatch):
    """Nor does the demo's model for its last norm, which no linear layer on a checkpoint follows."""
    from paper_2302_12445_amd.block_demo import TinyTransformer
    asked = []
    call = ops.add_rms_norm
    monkeypatch.setattr(ops, "add_rms_norm", lambda *args, **kwargs: asked.append(kwargs.get("keep", True)) or call(*args, **kwargs))
    torch.manual_seed(0)
    model = TinyTransformer(16, 32, 4, 2, 2, 5, torch.float32)
    tokens, lens = torch.randint(0, 16, (2, 5)), torch.tensor([5, 5], dtype=torch.int32)
    monkeypatch.setattr(layers, "attend", lambda q, k, v, **_: q + k.repeat_interleave(2, 2) + v.repeat_interleave(2, 2))
    with torch.no_grad():
        want = model(tokens, lens)
    assert asked == [False] * 5 and "checkpoint_encode" not in plain
    asked.clear()
    assert torch.equal(model(tokens, lens), want) and asked == [True] * 4 + [False]


# ------------------------------------------------------------------------------------ what saved_in_8_bits leaves as it is
@pytest.mark.parametrize("function", [torch.sigmoid, torch.tanh, torch.exp, lambda x: torch.softmax(x, -1)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.float64])
def test_graphs_of_what_is_left_alone_are_freed(function, dtype):
    """Operations that keep their own output: were that held by the graph itself, a graph that is dropped without a backward
    pass would never be freed."""
    x = torch.randn(8, 8, dtype=dtype, requires_grad=True)
    with layers.saved_in_8_bits():
        source = x * 1.0
        out = function(source)
    alive = [weakref.ref(x), weakref.ref(out)]  # x is held by the graph that leads to it
    del x, source, out
    gc.collect()
    assert [r() for r in alive] == [None, None]


def test_what_is_left_alone_is_the_same_tensor_s_values():
    x = torch.randn(8, 8, dtype=torch.float64, requires_grad=True)

    def gradients():
        first, = torch.autograd.grad((torch.sigmoid(x) * torch.tanh(x * 2)).sum(), x, create_graph=True)
        return first, torch.autograd.grad(first.square().sum(), x)[0]
    want = gradients()
    with layers.saved_in_8_bits():
        got = gradients()
    for a, b in zip(got, want):
        assert torch.equal(a, b)


def test_what_is_left_alone_and_changed_in_place_is_noticed():
    x = torch.randn(8, 8, requires_grad=True)
    with layers.saved_in_8_bits():
        source = x * 1.0
        out = source.square()
    source.add_(1)
    with pytest.raises(RuntimeError, match="in place"):
        out.sum().backward()


def test_whose_values_a_tensor_holds():
    weight, x = torch.nn.Parameter(torch.randn(8, 4)), torch.randn(8, 4, requires_grad=True)
    for f in (lambda t: t.t(), lambda t: t.bfloat16(), lambda t: t.chunk(2)[1], lambda t: torch.stack([t[:4], t[4:]]), lambda t: t.squeeze(0),
              lambda t: t[torch.tensor([1, 3])], lambda t: t.flatten().view(2, 16), lambda t: t.expand(3, 8, 4), lambda t: t.mT.contiguous()):
        assert layers._of_parameters(f(weight).grad_fn) and not layers._of_parameters(f(x * 1).grad_fn)
    for t in (weight * 1, x @ weight.t(), torch.cat([weight, x * 1]), torch.cat([weight * 1, weight])):
        assert not layers._of_parameters(t.grad_fn)
    # long chains, as of what grows piece by piece, and what is joined with itself over and over
    for source in (weight, x * 1):
        chain = doubled = source
        for _ in range(3000):
            chain = chain.view(8, 4)
        for _ in range(64):
            doubled = torch.stack([doubled, doubled])[0]
        assert layers._of_parameters(chain.grad_fn) == layers._of_parameters(doubled.grad_fn) == (source is weight)
