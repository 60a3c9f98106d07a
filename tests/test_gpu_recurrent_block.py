"""GPU: recurrent blocks with expert layers against plain torch in 64 bits, their training under DistOptim with clipped gradients, and
DistOptim's clipping by itself."""
from __future__ import annotations

import copy
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import recurrent_reference as rec  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class PlainBlock:
    """RecurrentBlock's mathematics in plain torch operations, on 64-bit copies of its parameters."""

    def __init__(self, block):
        self.block = block
        self.p = {n: t.detach().cpu().double().requires_grad_() for n, t in block.named_parameters()}

    def norm(self, name, h):
        return h / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-5) * self.p[name + ".weight"]

    def linear(self, name, x):
        return x @ self.p[name + ".weight"].T + self.p[name + ".bias"]

    def feed_forward(self, y, valid):
        b = self.block
        if b.experts is None:
            return self.linear("down", torch.nn.functional.gelu(self.linear("up", y)))
        scores, chosen = (y @ self.p["experts.router"].T).topk(b.experts.top, -1)
        share = torch.softmax(scores, -1)
        out = torch.zeros_like(y)
        for e in range(b.experts.experts):
            z = torch.nn.functional.gelu(y @ self.p["experts.up.weight"][e].T) @ self.p["experts.down.weight"][e].T
            out = out + z * (share * (chosen == e)).sum(-1, keepdim=True)
        return out * valid

    def __call__(self, x, residual, lens, state=None):
        B, T, C = x.shape
        valid = rec._valid(lens, B, T).unsqueeze(2)
        h = x + residual
        v, gate, open_ = self.linear("into", self.norm("norm1", h)).split(C, 2)
        a = torch.sigmoid(gate)
        s = torch.zeros(B, C, dtype=torch.float64) if state is None else state
        steps = []
        for t in range(T):
            s = torch.where(valid[:, t], a[:, t] * s + (1 - a[:, t]) * v[:, t], s)
            steps.append(torch.where(valid[:, t], s, torch.zeros_like(s)))
        h = h + self.linear("proj", torch.stack(steps, 1) * torch.nn.functional.silu(open_))
        return self.feed_forward(self.norm("norm2", h), valid), h, s


def share(got, want):
    return ((got.detach().cpu().double() - want.detach()).norm() / want.detach().norm()).item()


@pytest.mark.parametrize("experts", [0, 5])
def test_block_against_plain_torch(experts):
    """Outputs and input gradients in fp32 through some ten operations of a few hundred terms each; weight gradients from inputs kept in 8
    bits, and a GELU's derivative taken at one, within what that rounding does (a value off by 1/127 of its group's largest at most).
    Without experts, whose inputs are kept as they are, the recurrence's own gradients are no further off than those behind it."""
    from paper_2302_12445_amd.layers import RecurrentBlock
    torch.manual_seed(3)
    block = RecurrentBlock(64, 96, experts).to(DEV)
    for n, t in block.named_parameters():
        if "norm" in n:
            t.data += 0.1 * torch.randn_like(t)
    plain = PlainBlock(block)
    x, residual = (torch.randn(3, 40, 64, device=DEV) for _ in range(2))
    state = torch.randn(3, 64, device=DEV)
    lens = torch.tensor([40, 17, 1], dtype=torch.int32, device=DEV)
    a, r, s = (t.clone().requires_grad_() for t in (x, residual, state))
    out, h, last = block(a, r, lens, s)
    grads = [torch.randn_like(t) for t in (out, h, last)]
    torch.autograd.backward([out, h, last], grads)
    pa, pr, ps = (t.detach().cpu().double().requires_grad_() for t in (x, residual, state))
    want = plain(pa, pr, lens.cpu(), ps)
    torch.autograd.backward(list(want), [g.cpu().double() for g in grads])
    assert share(out, want[0]) < 1e-5 and share(h, want[1]) < 1e-5 and share(last, want[2]) < 1e-5
    for got, w in ((a.grad, pa.grad), (r.grad, pr.grad), (s.grad, ps.grad)):
        assert share(got, w) < 1e-2
    for n, t in block.named_parameters():
        assert t.grad.dtype == torch.float32 and share(t.grad, plain.p[n].grad) < 2e-2, n


def test_tokens_one_by_one():
    """A block fed a token at a time with its state gives what it gives for the sequence."""
    from paper_2302_12445_amd.layers import RecurrentBlock
    torch.manual_seed(4)
    block = RecurrentBlock(64, experts=4).to(DEV)
    x = torch.randn(2, 30, 64, device=DEV)
    with torch.no_grad():
        want, _ = block(x)
        state, parts = torch.zeros(2, 64, device=DEV), []
        for t in range(30):
            out, _, state = block(x[:, t:t + 1], state=state)
            parts.append(out)
    # fp32 sums of a few hundred terms, in other orders
    assert share(torch.cat(parts, 1), want.double().cpu()) < 1e-5


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_experts_take_nothing_from_behind_the_sequences(dtype):
    """What stands behind the lengths, NaN here, reaches neither results nor gradients."""
    from paper_2302_12445_amd.layers import Experts
    torch.manual_seed(6)
    layer = Experts(32, 48, 5, 2).to(DEV)
    y = torch.randn(3, 7, 32, device=DEV).to(dtype)
    lens = torch.tensor([7, 0, 3], dtype=torch.int32, device=DEV)
    results = []
    for fill in (0.0, math.nan):
        a = y.clone()
        a[1], a[2, 3:] = fill, fill
        a.requires_grad_()
        layer.zero_grad()
        out = layer(a, lens)
        out.float().square().sum().backward()
        results.append([out, a.grad] + [p.grad.clone() for p in layer.parameters()])
    assert all(torch.equal(a, b) for a, b in zip(*results))
    assert not results[1][0][1].any() and not results[1][1][2, 3:].any()


@pytest.mark.parametrize("fill", [math.nan, math.inf])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_behind_the_sequences_reach_nothing(dtype, fill):
    """What the incoming gradient holds behind the lengths changes no gradient."""
    from paper_2302_12445_amd.layers import Experts
    torch.manual_seed(8)
    layer = Experts(32, 48, 5, 2).to(DEV)
    y, dout = (torch.randn(3, 7, 32, device=DEV).to(dtype) for _ in range(2))
    lens = torch.tensor([7, 0, 3], dtype=torch.int32, device=DEV)
    results = []
    for behind in (0.0, fill):
        a, d = y.clone().requires_grad_(), dout.clone()
        d[1], d[2, 3:] = behind, behind
        layer.zero_grad()
        layer(a, lens).backward(d)
        results.append([a.grad] + [p.grad.clone() for p in layer.parameters()])
    assert all(torch.equal(p, q) for p, q in zip(*results)) and results[1][1].any()


def test_experts_spread_and_gather():
    """Each token goes to its experts and back, none to others; gradients of tokens that go to several are added."""
    from paper_2302_12445_amd.layers import Experts
    torch.manual_seed(5)
    layer = Experts(32, 48, 6, 3).to(DEV)
    y = torch.randn(4, 9, 32, device=DEV)
    lens = torch.tensor([9, 0, 4, 1], dtype=torch.int32, device=DEV)
    a = y.clone().requires_grad_()
    out = layer(a, lens)
    out.square().sum().backward()
    block = type("", (), {"experts": layer})()
    plain = PlainBlock.__new__(PlainBlock)
    plain.block, plain.p = block, {"experts." + n: t.detach().cpu().double().requires_grad_() for n, t in layer.named_parameters()}
    b = y.cpu().double().requires_grad_()
    want = plain.feed_forward(b, rec._valid(lens.cpu(), 4, 9).unsqueeze(2))
    want.square().sum().backward()
    assert share(out, want) < 1e-5 and not out[1].any() and not out[2, 4:].any()
    assert share(a.grad, b.grad) < 1e-2 and not a.grad[1].any()
    for n, t in layer.named_parameters():
        assert share(t.grad, plain.p["experts." + n].grad) < 2e-2, n


def plain_training(replicas, width, heads, kv_heads, layers, tokens, batch, steps, lr, experts, max_grad_norm, seed=0):
    """block_demo.train in plain 64-bit torch on the CPU: one model, SGD with momentum on the clipped mean of the replicas' gradients."""
    from paper_2302_12445_amd.block_demo import TinyTransformer, batch_of
    torch.manual_seed(seed)
    model = TinyTransformer(64, width, heads, kv_heads, layers, tokens, torch.float32, "recurrence", experts, 2)
    blocks = [PlainBlock(b) for b in model.blocks]
    outer = {n: t.detach().double().requires_grad_() for n, t in model.named_parameters() if not n.startswith("blocks.")}
    params = list(outer.values()) + [t for b in blocks for t in b.p.values()]
    moms = [torch.zeros_like(t) for t in params]
    gen = torch.Generator().manual_seed(seed + 1)
    losses = []
    for _ in range(steps):
        total = 0.0
        for _ in range(replicas):
            x, lens, y = batch_of(64, batch, tokens, gen, "cpu")
            a = outer["embed.weight"][x] + outer["position.weight"]
            residual = torch.zeros_like(a)
            for block in blocks:
                a, residual, _ = block(a, residual, lens)
            h = a + residual
            h = h / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-5) * outer["norm.weight"]
            logits = h @ outer["head.weight"].T + outer["head.bias"]
            loss = torch.nn.functional.cross_entropy(logits.flatten(0, 1), y.flatten(), ignore_index=-100)
            (loss / replicas).backward()
            total += loss.item() / replicas
        norm = torch.sqrt(sum((t.grad ** 2).sum() for t in params))
        by = min(1.0, max_grad_norm / norm.item())
        for t, m in zip(params, moms):
            m.mul_(0.9).add_(by * t.grad)
            t.data.sub_(lr * m)
            t.grad = None
        losses.append(total)
    return losses


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_blocks_train_under_dist_optim(dtype):
    """Replicas stay the same bit for bit.  In fp32 the losses are those of the same training in 64 bits: off by what weight gradients
    that are off by 2 % at most (the test above) make of a step, 2 % of what the steps have changed, and rounding.  In bf16 tokens near a
    border between experts go another way."""
    from paper_2302_12445_amd.block_demo import train
    print("case: recurrent blocks under DistOptim", dtype, flush=True)
    setup = dict(replicas=2, width=64, heads=4, kv_heads=2, layers=2, tokens=24, batch=8, steps=15, lr=0.1)
    losses, _, models = train(dtype=dtype, mixer="recurrence", experts=4, max_grad_norm=0.5, **setup)
    for a, b in zip(models[0].parameters(), models[1].parameters()):
        assert torch.equal(a, b) and torch.isfinite(a).all()
    if dtype == torch.float32:
        want = plain_training(experts=4, max_grad_norm=0.5, **setup)
        for got, w in zip(losses, want):
            assert abs(got - w) <= 1e-3 + 0.05 * abs(want[0] - w)


@pytest.mark.parametrize("max_norm", [0.05, 1e6])
@pytest.mark.parametrize("threshold", [0, 1 << 12, 25 << 20])
def test_dist_optim_clips_the_mean_gradient(threshold, max_norm):
    """Against the mean of the replicas' gradients, clipped and applied in 64 bits: parameters within 2e-4 of their changes, the norm
    within fp32's rounding of sums of some thousand terms; where nothing is clipped, the same bits as without."""
    from paper_2302_12445_amd.dist_optim import DistOptim
    print("case: clipping", threshold, max_norm, flush=True)
    P, lr, mu = 3, 0.1, 0.9
    torch.manual_seed(7)
    model = torch.nn.Sequential(torch.nn.Linear(33, 50), torch.nn.Tanh(), torch.nn.Linear(50, 7)).to(DEV)
    data = [[torch.randn(16, 33, device=DEV) for _ in range(P)] for _ in range(3)]

    def run(**options):
        models = [copy.deepcopy(model) for _ in range(P)]
        optim, norms = DistOptim(models, lr, mu, fusion_threshold_bytes=threshold, **options), []
        for batch in data:
            for m, x in zip(models, batch):
                m(x).square().mean().backward()
            optim.step()
            norms.append(optim.grad_norm)
        optim.synchronize()
        torch.cuda.synchronize()
        optim.close()
        for m in models[1:]:
            for a, b in zip(m.parameters(), models[0].parameters()):
                assert torch.equal(a, b)
        return models[0], norms
    got, norms = run(max_grad_norm=max_norm)
    want = copy.deepcopy(model).double()
    moms = [torch.zeros_like(p) for p in want.parameters()]
    for n, batch in enumerate(data):
        want.zero_grad()
        for x in batch:
            (want(x.double()).square().mean() / P).backward()
        norm = torch.sqrt(sum((p.grad ** 2).sum() for p in want.parameters()))
        assert abs(norms[n].item() - norm.item()) <= 1e-5 * norm.item()
        by = min(1.0, max_norm / norm.item())
        for p, m in zip(want.parameters(), moms):
            m.mul_(mu).add_(by * p.grad)
            p.data.sub_(lr * m)
    for a, w, first in zip(got.parameters(), want.parameters(), model.parameters()):
        assert (a.double() - w).norm() <= 2e-4 * (w - first.double()).norm() + 1e-7 * w.norm()
    if max_norm == 1e6:
        plain, none = run(fused_update=False)
        assert none[0] is None
        for a, b in zip(got.parameters(), plain.parameters()):
            assert torch.equal(a, b)


def test_dist_optim_refuses_a_norm_that_is_none():
    from paper_2302_12445_amd.dist_optim import DistOptim
    for bad in (0.0, -1.0, math.nan):
        with pytest.raises(ValueError, match="max_grad_norm"):
            DistOptim([torch.nn.Linear(2, 2).to(DEV)], 0.1, 0.9, max_grad_norm=bad)


def test_a_step_s_gradients_repeat_bits():
    """The same block on the same inputs gives the same bits."""
    from paper_2302_12445_amd.layers import RecurrentBlock
    torch.manual_seed(6)
    block = RecurrentBlock(128, 256, 4).to(DEV)
    x, residual, dout = (torch.randn(4, 300, 128, device=DEV).bfloat16() for _ in range(3))
    lens = torch.tensor([300, 20, 257, 30], dtype=torch.int32, device=DEV)
    runs = []
    for _ in range(2):
        block.zero_grad()
        a = x.clone().requires_grad_()
        out, h = block(a, residual, lens)
        out.backward(dout)
        runs.append([out.detach(), h.detach(), a.grad] + [t.grad.clone() for n, t in block.named_parameters() if not n.endswith("bias")])
    for p, q in zip(*runs):
        assert torch.equal(p, q)


def test_demo_refuses_experts_behind_attention():
    from paper_2302_12445_amd.block_demo import TinyTransformer
    with pytest.raises(ValueError, match="experts"):
        TinyTransformer(64, 32, 2, 2, 1, 8, torch.float32, "attention", 4)
