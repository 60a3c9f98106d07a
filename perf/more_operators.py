"""Performance cases of the operators of a recurrent block with expert layers: a gated linear recurrence with its
backward pass, products grouped by expert with both gradients, and the global gradient norm with clipping.

listed() and draw() give cases (dicts of plain values); prepare() makes the tensors that a training program has
in hand before the call; run() is one pass, in plain 32-bit torch operations or, where `own` is true, through the
framework; work() is the traffic and arithmetic that a pass cannot do without; exact() is the result in 64 bits.

Paths (case["path"]):
  recurrence           s[t] = a[t] s[t-1] + (1 - a[t]) x[t] with a = sigmoid(gate), along the steps of each sequence
  recurrence_backward  gradients of x, of the gates and of the state before the first step
  experts              rows, sorted by expert, times the weights of their expert
  experts_input_grad   gradient of the rows
  experts_weight_grad  gradient of each expert's weights, in fp32
  clip                 norm over the gradients of a model's tensors, and the gradients scaled down to a largest norm, in fp32
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
KEPT = 256  # steps from one kept state to the next
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------------------------ the cases
def _recurrence(path, dtype, batch, steps, width, ragged=False, state=False):
    return {"path": path, "dtype": dtype, "batch": batch, "steps": steps, "width": width, "ragged": ragged, "state": state}


def _experts(path, dtype, rows, experts, outs, ins, skew, spare=0):
    return {"path": path, "dtype": dtype, "rows": rows, "experts": experts, "outs": outs, "ins": ins, "skew": skew, "spare": spare}


def _clip(dtype, width, layers, vocab, sigma):
    return {"path": "clip", "dtype": dtype, "width": width, "layers": layers, "vocab": vocab, "sigma": sigma}


def listed():
    return [
        # one more token of sixteen sequences that are being answered: latency counts
        dict(_recurrence("recurrence", "bf16", 16, 1, 1024, state=True), name="recurrence_token"),
        # a BERT-Large batch of padded sequences of 512
        dict(_recurrence("recurrence", "bf16", 16, 512, 1024, ragged=True), name="recurrence_padded"),
        # two long sequences, forward and backward: few channels for the chip, many steps
        dict(_recurrence("recurrence", "bf16", 2, 8192, 1024), name="recurrence_long"),
        dict(_recurrence("recurrence_backward", "bf16", 2, 8192, 1024), name="recurrence_backward_long"),
        # a program that trains in fp32, with odd lengths and widths
        dict(_recurrence("recurrence_backward", "f32", 3, 1111, 771, ragged=True), name="recurrence_backward_odd_f32"),
        # sixteen tokens, each to two of eight experts, some of which get none: reading weights counts
        dict(_experts("experts", "bf16", 32, 8, 4096, 1024, 1.5), name="experts_tokens"),
        # a BERT-Large batch, 8192 tokens to two experts each: the feed-forward layer's first product and its gradients
        dict(_experts("experts", "bf16", 16384, 8, 4096, 1024, 0.5), name="experts_batch"),
        dict(_experts("experts_input_grad", "bf16", 16384, 8, 4096, 1024, 0.5), name="experts_input_grad_batch"),
        dict(_experts("experts_weight_grad", "bf16", 16384, 8, 4096, 1024, 0.5), name="experts_weight_grad_batch"),
        # narrow experts of odd sizes in fp32
        dict(_experts("experts", "f32", 1111, 6, 771, 1003, 1.0, spare=13), name="experts_odd_f32"),
        # a small model's gradients, and BERT-Large's
        dict(_clip("f32", 64, 2, 512, 0.05), name="clip_small"),
        dict(_clip("f32", 1024, 24, 30522, 0.001), name="clip_model"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the ranges above: sequences from one step to 32768, batches to 32, widths to 4096; rows from one to
    32768 over up to 64 experts, even or skewed, with rows behind the last expert's or none; models of one to 24 layers,
    clipped or not."""
    path = rng.choice(["recurrence", "recurrence", "recurrence_backward", "recurrence_backward", "experts", "experts",
                       "experts_input_grad", "experts_input_grad", "experts_weight_grad", "clip"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if path in ("recurrence", "recurrence_backward"):
        width = _log_uniform(rng, 16, 4096)
        if rng.random() < 0.6:  # widths are mostly multiples of 64
            width = max(64, width // 64 * 64)
        steps = _log_uniform(rng, 1, 32768)
        batch = rng.randint(1, 32)
        most = 1 << 24  # elements of the long listed cases
        while batch > 1 and batch * steps * width > most:
            batch -= 1
        while steps * width > most:
            steps = steps * 3 // 4
        return _recurrence(path, dtype, batch, steps, width, rng.random() < 0.4, rng.random() < 0.5)
    if path == "clip":
        return _clip(dtype, _log_uniform(rng, 16, 1024), rng.randint(1, 24), _log_uniform(rng, 64, 30522),
                     rng.choice([1e-6, 1e-3, 0.05, 2.0]))
    rows, experts = _log_uniform(rng, 1, 32768), _log_uniform(rng, 1, 64)
    outs, ins = _log_uniform(rng, 16, 8192), _log_uniform(rng, 16, 8192)
    if rng.random() < 0.6:
        outs, ins = max(64, outs // 64 * 64), max(64, ins // 64 * 64)
    most = 16384 * 4096 * 1024 // (1 if dtype == "bf16" else 16)
    while rows * outs * ins > most:
        rows = rows * 3 // 4
    while experts * outs * ins > 1 << 28:
        experts = experts * 3 // 4
    while outs * ins > 1 << 25:
        outs, ins = outs * 3 // 4, ins * 3 // 4
    return _experts(path, dtype, max(1, rows), max(1, experts), outs, ins, rng.choice([0.0, 0.5, 1.0, 2.0]),
                    rng.choice([0, 0, 0, rows // 16]))


# ------------------------------------------------------------------------------------ inputs
def _normal(shape, gen, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * scale).to(TYPES[dtype])


def _lengths(case):
    """Steps of each sequence: in a ragged batch they fall from the whole length to about half."""
    B, T = case["batch"], case["steps"]
    return [max(1, T - (b * T) // (2 * B)) if case["ragged"] else T for b in range(B)]


def _counts(case):
    """Rows of each expert, from the busiest on: shares fall as 1 / place ** skew."""
    share = [1.0 / (i + 1) ** case["skew"] for i in range(case["experts"])]
    edge, at, all_ = [0], 0.0, sum(share)
    for s in share:
        at += s
        edge.append(min(case["rows"], int(case["rows"] * at / all_ + 0.5)))
    edge[-1] = case["rows"]
    return [b - a for a, b in zip(edge, edge[1:])]


def _sizes(case):
    """Elements of the tensors of a transformer of this width: embeddings, and for each layer four square projections, two
    of four times the width, and two norms, with their biases."""
    w = case["width"]
    layer = 4 * [w * w, w] + [4 * w * w, 4 * w, 4 * w * w, w] + 4 * [w]
    return [case["vocab"] * w, 512 * w, w, w] + case["layers"] * layer


def _places(sizes):
    """Where tensors start in a buffer that has each on a multiple of 64 elements, and the buffer's elements."""
    at, starts = 0, []
    for n in sizes:
        starts.append(at)
        at += -(-n // 64) * 64
    return starts, at


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    path, t = case["path"], case["dtype"]
    s = {"case": case}
    if path in ("recurrence", "recurrence_backward"):
        B, T, C = case["batch"], case["steps"], case["width"]
        # x and the gates are parts of one projection; gates hold on to a state for one step to some hundred
        both = torch.randn(B, T, 2 * C, generator=gen, device=DEV)
        both[..., C:] += 6 * torch.rand(C, generator=gen, device=DEV) - 0.5
        s["x"], s["gate"] = both.to(TYPES[t]).split(C, 2)
        s["state"] = torch.randn(B, C, generator=gen, device=DEV) if case["state"] else None
        s["lens"] = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV) if case["ragged"] else None
        if path == "recurrence_backward":
            s["dh"] = _normal((B, T, C), gen, t, 0.01)
            s["kept"] = _plain_recurrence(s)["kept"]
    elif path == "clip":
        sizes = _sizes(case)
        starts, n = _places(sizes)
        flat = _normal(n, gen, t, case["sigma"])
        s["grads"] = [flat[at:at + size] for at, size in zip(starts, sizes)]
        s["flat"] = torch.zeros(n, device=DEV)  # the fp32 gradients that the optimizer reads
        s["out"] = [s["flat"][at:at + size] for at, size in zip(starts, sizes)]
    else:
        E, N, K, M = case["experts"], case["outs"], case["ins"], case["rows"] + case["spare"]
        # which expert is busy changes with the seed
        order = torch.randperm(E, generator=gen, device=DEV).tolist()
        by_place = _counts(case)
        counts = [by_place[p] for p in order]
        s["counts"] = counts
        s["ends"] = torch.tensor(counts, device=DEV).cumsum(0).to(torch.int32)
        if path != "experts":
            s["dy"] = _normal((M, N), gen, t, 0.01)
        if path != "experts_input_grad":
            x = torch.randn(M, K, generator=gen, device=DEV)
            loud = torch.rand(K, generator=gen, device=DEV) < 0.01  # a few channels of activations are much larger
            s["x"] = (x * torch.where(loud, 12.0, 1.0)).to(TYPES[t])
        if path != "experts_weight_grad":
            s["weight"] = _normal((E, N, K), gen, t, 1 / math.sqrt(K))
    return s


# ------------------------------------------------------------------------------------ the plain forms
def _scan(a, b):
    """s[t] = a[t] s[t-1] + b[t] along axis 1, with s[-1] = 0: each round joins maps of d steps to maps of 2 d."""
    d = 1
    while d < a.shape[1]:
        b = torch.cat([b[:, :d], b[:, d:] + a[:, d:] * b[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return b


def _plain_gates(s):
    """a, 1 - a and x in 32 bits; steps beyond the length keep the state as it is (a = 1)."""
    a, b, x = torch.sigmoid(s["gate"].float()), torch.sigmoid(-s["gate"].float()), s["x"].float()
    if s["lens"] is None:
        return a, b, x, None
    valid = (torch.arange(x.shape[1], device=DEV) < s["lens"].view(-1, 1)).unsqueeze(2)
    return a.masked_fill(~valid, 1.0), b.masked_fill(~valid, 0.0), x.masked_fill(~valid, 0.0), valid


def _plain_states(s, a, b, x):
    """[B, T + 1, C]: the state before each step, and behind the last."""
    first = torch.zeros_like(x[:, 0]) if s["state"] is None else s["state"]
    b = b * x
    b = torch.cat([b[:, :1] + (a[:, 0] * first).unsqueeze(1), b[:, 1:]], 1)
    return torch.cat([first.unsqueeze(1), _scan(a, b)], 1)


def _plain_recurrence(s):
    a, b, x, valid = _plain_gates(s)
    states = _plain_states(s, a, b, x)
    h = states[:, 1:]
    if valid is not None:
        h = h.masked_fill(~valid, 0.0)
    out = {"h": h.to(s["x"].dtype), "last": states[:, -1].contiguous()}
    if s["case"]["path"] == "recurrence_backward" or not s["case"]["state"]:
        out["kept"] = states[:, :-1:KEPT].contiguous()
    return out


def _plain_recurrence_backward(s):
    a, b, x, valid = _plain_gates(s)
    before = _plain_states(s, a, b, x)[:, :-1]
    dh = s["dh"].float()
    if valid is not None:
        dh = dh.masked_fill(~valid, 0.0)
    after = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1)
    g = _scan(after.flip(1), dh.flip(1)).flip(1)
    t = s["x"].dtype
    dx, dgate = b * g, g * (before - x) * a * b
    if valid is not None:
        dgate = dgate.masked_fill(~valid, 0.0)
    return {"dx": dx.to(t), "dgate": dgate.to(t), "dstate": a[:, 0] * g[:, 0]}


def _plain_parts(s, x):
    """The rows of each expert, and those behind the last, in 32 bits."""
    return x.float().split(s["counts"] + [s["case"]["spare"]])


def _plain_rows(s, parts, width):
    return torch.cat([*parts, torch.zeros(s["case"]["spare"], width, device=DEV)])


def _plain_clip(s):
    flat = torch.cat([g.float() for g in s["grads"]])
    norm = flat.double().square().sum().sqrt().float()
    flat = flat * torch.clamp(1.0 / norm, max=1.0)
    torch._foreach_copy_(s["out"], list(flat.split([g.numel() for g in s["grads"]])))
    return {"norm": norm, "grads": s["flat"]}


# ------------------------------------------------------------------------------------ one pass
def run(state):
    s, case = state, state["case"]
    path = case["path"]
    if own:
        return _run_own(s, case, path)
    if path == "recurrence":
        return _plain_recurrence(s)
    if path == "recurrence_backward":
        return _plain_recurrence_backward(s)
    if path == "clip":
        return _plain_clip(s)
    if path == "experts":
        parts = [x @ w.t() for x, w in zip(_plain_parts(s, s["x"]), s["weight"].float())]
        return _plain_rows(s, parts, case["outs"]).to(s["x"].dtype)
    if path == "experts_input_grad":
        parts = [dy @ w for dy, w in zip(_plain_parts(s, s["dy"]), s["weight"].float())]
        return _plain_rows(s, parts, case["ins"]).to(s["dy"].dtype)
    pairs = zip(_plain_parts(s, s["dy"])[:-1], _plain_parts(s, s["x"]))
    return torch.stack([dy.t() @ x for dy, x in pairs])


def _run_own(s, case, path):
    from paper_2302_12445_amd import ops
    if path == "recurrence":
        keep = not case["state"]
        h, last, kept = ops.recurrence(s["x"], s["gate"], state=s["state"], lens=s["lens"], keep=keep)
        return {"h": h, "last": last, "kept": kept} if keep else {"h": h, "last": last}
    if path == "recurrence_backward":
        dx, dgate, dstate = ops.recurrence_backward(s["dh"], s["x"], s["gate"], s["kept"], lens=s["lens"])
        return {"dx": dx, "dgate": dgate, "dstate": dstate}
    if path == "clip":
        return {"norm": ops.clip_grads(s["grads"], 1.0, out=s["out"]), "grads": s["flat"]}
    if path == "experts":
        return ops.expert_linear(s["x"], s["weight"], s["ends"])
    if path == "experts_input_grad":
        return ops.expert_input_grad(s["dy"], s["weight"], s["ends"])
    return ops.expert_weight_grad(s["dy"], s["x"], s["ends"])


# ------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    path, g = case["path"], SIZE[case["dtype"]]
    if path in ("recurrence", "recurrence_backward"):
        B, T, C = case["batch"], case["steps"], case["width"]
        read, whole, states = sum(_lengths(case)) * C, B * T * C, 4 * B * C
        kept = -(-T // KEPT) * states
        if path == "recurrence":
            return {"bytes": 2 * read * g + whole * g + states + (states if case["state"] else kept), "flops": 10 * read}
        return {"bytes": 3 * read * g + 2 * whole * g + kept + states, "flops": 25 * read}
    if path == "clip":
        n = sum(_sizes(case))
        return {"bytes": n * (g + 4) + 4, "flops": 3 * n}
    m, n, k = case["rows"], case["outs"], case["ins"]
    all_ = m + case["spare"]
    used = sum(c > 0 for c in _counts(case))
    if path == "experts":
        moved = m * k * g + used * n * k * g + all_ * n * g
    elif path == "experts_input_grad":
        moved = m * n * g + used * n * k * g + all_ * k * g
    else:
        moved = m * (n + k) * g + case["experts"] * n * k * 4
    return {"bytes": moved, "flops": 2 * m * n * k}


# ------------------------------------------------------------------------------------ in 64 bits
def _exact_recurrence(case, s):
    """By the definition, one step after another, in place of the last state where a sequence has ended."""
    x, gate = s["x"].double(), s["gate"].double()
    B, T, C = x.shape
    lens = torch.tensor(_lengths(case), device=DEV).view(B, 1)
    state = torch.zeros(B, C, dtype=torch.float64, device=DEV) if s["state"] is None else s["state"].double()
    a = 1 / (1 + torch.exp(-gate))
    b = 1 / (1 + torch.exp(gate))
    h, before = torch.zeros_like(x), torch.zeros_like(x)
    for t in range(T):
        before[:, t] = state
        state = torch.where(t < lens, a[:, t] * state + b[:, t] * x[:, t], state)
        h[:, t] = state
    steps = torch.arange(T, device=DEV).view(1, T, 1)
    if case["path"] == "recurrence":
        out = {"h": torch.where(steps < lens.view(B, 1, 1), h, 0.0), "last": state}
        if not case["state"]:
            out["kept"] = before[:, ::KEPT]
        return out
    dh, g = s["dh"].double(), torch.zeros(B, C, dtype=torch.float64, device=DEV)
    dx, dgate = torch.zeros_like(x), torch.zeros_like(x)
    for t in reversed(range(T)):
        g = torch.where(t < lens, g + dh[:, t], g)
        dx[:, t] = b[:, t] * g
        dgate[:, t] = g * (before[:, t] - x[:, t]) * a[:, t] * b[:, t]
        g = torch.where(t < lens, a[:, t] * g, g)
    return {"dx": torch.where(steps < lens.view(B, 1, 1), dx, 0.0), "dgate": torch.where(steps < lens.view(B, 1, 1), dgate, 0.0), "dstate": g}


def exact(case, seed):
    s, path = prepare(case, seed), case["path"]
    if path in ("recurrence", "recurrence_backward"):
        return _exact_recurrence(case, s)
    if path == "clip":
        grads = [g.double() for g in s["grads"]]
        norm = math.sqrt(math.fsum(float(g.pow(2).sum()) for g in grads))
        flat = torch.zeros(s["flat"].shape, dtype=torch.float64, device=DEV)
        for at, g in zip(_places(_sizes(case))[0], grads):
            flat[at:at + g.numel()] = g / norm if norm > 1 else g
        return {"norm": torch.tensor(norm, dtype=torch.float64), "grads": flat}
    edges = [0] + s["ends"].tolist()
    E, N, K, M = case["experts"], case["outs"], case["ins"], case["rows"] + case["spare"]
    shape = {"experts": (M, N), "experts_input_grad": (M, K), "experts_weight_grad": (E, N, K)}[path]
    out = torch.zeros(shape, dtype=torch.float64, device=DEV)
    for e, (i, j) in enumerate(zip(edges, edges[1:])):
        if path == "experts":
            out[i:j] = s["x"][i:j].double() @ s["weight"][e].double().T
        elif path == "experts_input_grad":
            out[i:j] = s["dy"][i:j].double() @ s["weight"][e].double()
        else:
            out[e] = s["dy"][i:j].double().T @ s["x"][i:j].double()
    return out
