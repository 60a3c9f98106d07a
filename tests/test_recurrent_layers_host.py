"""CPU checks of the recurrence's and the experts' autograd layers: plain torch operations stand in for the calls on the GPU, whose results,
as theirs, carry no graph of their own."""
from __future__ import annotations

import gc
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

    def states(x, gate, state):
        a, s, out = torch.sigmoid(gate), torch.zeros_like(x[:, 0]) if state is None else state, []
        for t in range(x.shape[1]):
            out.append(s)
            s = a[:, t] * s + (1 - a[:, t]) * x[:, t]
        return out, s

    @stand_in
    def recurrence(x, gate, state=None, lens=None, keep=True):
        before, last = states(x, gate, state)
        return torch.stack(before[1:] + [last], 1), last, torch.stack(before[::256], 1) if keep else None

    @stand_in
    def recurrence_backward(dh, x, gate, kept, lens=None, dlast=None):
        before, _ = states(x, gate, kept[:, 0])
        a, e = torch.sigmoid(gate), torch.zeros_like(x[:, 0]) if dlast is None else dlast
        dx, dgate = torch.zeros_like(x), torch.zeros_like(x)
        for t in reversed(range(x.shape[1])):
            g = dh[:, t] + e
            dx[:, t], dgate[:, t] = (1 - a[:, t]) * g, g * (before[t] - x[:, t]) * a[:, t] * (1 - a[:, t])
            e = a[:, t] * g
        return dx, dgate, e

    def parts(ends):
        return list(zip([0] + ends.tolist(), ends.tolist()))

    @stand_in
    def expert_linear(x, weight, ends):
        y = x.new_zeros(x.shape[0], weight.shape[1])
        for e, (i, j) in enumerate(parts(ends)):
            y[i:j] = x[i:j] @ weight[e].T
        return y

    @stand_in
    def expert_input_grad(dy, weight, ends):
        dx = dy.new_zeros(dy.shape[0], weight.shape[2])
        for e, (i, j) in enumerate(parts(ends)):
            dx[i:j] = dy[i:j] @ weight[e]
        return dx

    @stand_in
    def expert_weight_grad(dy, x, ends):
        return torch.stack([dy[i:j].T @ x[i:j] for i, j in parts(ends)])

    return calls


def leaf(*shape, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64).requires_grad_()


def test_gradients_against_differences(plain):
    x, gate, state = leaf(2, 5, 3), leaf(2, 5, 3, seed=1), leaf(2, 3, seed=2)
    assert torch.autograd.gradcheck(lambda *t: layers.recur(*t), (x, gate, state))
    assert torch.autograd.gradcheck(lambda a, b: layers.recur(a, b)[1], (x, gate))
    rows, weight, ends = leaf(7, 4), leaf(3, 5, 4, seed=1), torch.tensor([2, 2, 6])
    assert torch.autograd.gradcheck(lambda a, w: layers._apply(layers._ExpertLinear, a, w, ends), (rows, weight))


def test_experts_layer_against_differences(plain):
    torch.manual_seed(0)
    layer = layers.Experts(4, 6, 5, 2).double()
    y, lens = leaf(2, 6, 4), torch.tensor([6, 3])
    scores = y.reshape(-1, 4).float() @ layer.router.t().float()
    assert scores.topk(3, -1)[0].diff(dim=-1).abs().min() > 1e-4  # no token is near a border, where a difference would cross it
    router = layer.router.data.float()

    def call(y, router, up, down):  # (the router works in fp32, which differences do not see through: its part is left out)
        return torch.func.functional_call(layer, {"router": router, "up.weight": up, "down.weight": down}, (y, lens))
    t = [layer.up.weight.detach().clone().requires_grad_(), layer.down.weight.detach().clone().requires_grad_()]
    assert torch.autograd.gradcheck(lambda u, d: call(y.detach(), router, u, d), t)


LOSSES = [lambda out: out.sum(), lambda out: out.square().sum()]


@pytest.mark.parametrize("loss", LOSSES)
def test_second_derivatives_are_refused(plain, loss):
    x, gate, state = leaf(2, 5, 3), leaf(2, 5, 3, seed=1), leaf(2, 3, seed=2)
    first = torch.autograd.grad(loss(layers.recur(x, gate, state)[0]), (x, gate, state), create_graph=True)
    for g in first:
        with pytest.raises(RuntimeError, match="second derivatives"):
            torch.autograd.grad((g.square().sum() + x.sum() + gate.sum() + state.sum()), (x, gate, state), retain_graph=True)
    rows, weight, ends = leaf(7, 4), leaf(3, 5, 4, seed=1), torch.tensor([2, 2, 6])
    first = torch.autograd.grad(loss(layers._apply(layers._ExpertLinear, rows, weight, ends)), (rows, weight), create_graph=True)
    for g in first:
        with pytest.raises(RuntimeError, match="second derivatives"):
            torch.autograd.grad((g.square().sum() + rows.sum() + weight.sum()), (rows, weight), retain_graph=True)


def test_what_is_not_asked_for_is_not_made(plain):
    x, gate = leaf(2, 5, 3), leaf(2, 5, 3, seed=1)
    with torch.no_grad():
        layers.recur(x, gate)
    assert plain == ["recurrence"]
    rows, weight, ends = leaf(7, 4), leaf(3, 5, 4, seed=1), torch.tensor([2, 2, 6])
    plain.clear()
    layers._apply(layers._ExpertLinear, rows.detach(), weight, ends).sum().backward()
    assert plain == ["expert_linear", "expert_weight_grad"]
    plain.clear()
    layers._apply(layers._ExpertLinear, rows, weight.detach(), ends).sum().backward()
    assert plain == ["expert_linear", "expert_input_grad"]
    h, last = layers.recur(x, gate)
    plain.clear()
    last.sum().backward()  # nobody used h
    assert plain == ["recurrence_backward"]


def test_a_state_carried_in_place(plain):
    """A buffer of states that takes no gradient may be written over before the backward pass, which does not read it, and is not kept alive
    by it; a state that has a gradient has to stay, as an input of it."""
    x, gate, buffer = leaf(2, 5, 3), leaf(2, 5, 3, seed=1), leaf(2, 3, seed=2).detach()
    want = torch.autograd.grad(layers.recur(x, gate, buffer.clone())[0].sum(), (x, gate))
    h, last = layers.recur(x, gate, buffer)
    buffer.copy_(last.detach())
    assert all(torch.equal(p, q) for p, q in zip(torch.autograd.grad(h.sum(), (x, gate)), want))
    state = leaf(2, 3, seed=3).detach()
    h, _ = layers.recur(x, gate, state)
    seen = weakref.ref(state)
    del state
    gc.collect()
    assert seen() is None
    start = leaf(2, 3, seed=4)
    h, _ = layers.recur(x, gate, start)
    assert torch.autograd.grad(h.sum(), start)[0].shape == start.shape


def test_graphs_are_freed(plain):
    x, gate = leaf(2, 5, 3), leaf(2, 5, 3, seed=1)
    h, last = layers.recur(x * 1, gate * 1)
    seen = weakref.ref(h.grad_fn)
    del h, last
    gc.collect()
    assert seen() is None


def test_experts_refuse_more_than_there_are():
    for top in (0, 3):
        with pytest.raises(ValueError, match="top"):
            layers.Experts(4, 4, 2, top)


@pytest.mark.parametrize("fill", [float("nan"), float("inf")])
def test_gradients_behind_the_lengths_reach_nothing(plain, fill):
    """What the incoming gradient holds behind the lengths changes no gradient, the router's among them."""
    torch.manual_seed(1)
    layer = layers.Experts(4, 6, 5, 2)
    y, dout, lens = torch.randn(3, 6, 4), torch.randn(3, 6, 4), torch.tensor([6, 0, 3])
    results = []
    for behind in (0.0, fill):
        a, d = y.clone().requires_grad_(), dout.clone()
        d[1], d[2, 3:] = behind, behind
        layer.zero_grad()
        layer(a, lens).backward(d)
        results.append([a.grad] + [p.grad.clone() for p in layer.parameters()])
    assert all(torch.equal(p, q) for p, q in zip(*results)) and results[1][1].any()
