"""Training demo of the operators under the paper's optimizer: P replicas of a small pre-norm transformer on one GPU, batches
of padded sequences, attention / norm / checkpoints in 8 bits from ops.py, gradients aggregated and parameters updated by
DistOptim inside the backward passes.  The task: predict the token before (a causal model reaches a loss near zero).
Prints one JSON line: losses and step time.

    python -m paper_2302_12445_amd.block_demo --replicas 4 --width 256 --layers 2 --steps 150
"""
from __future__ import annotations

import argparse
import copy
import json
import sys
import time

import torch

from .layers import AddRMSNorm, TransformerBlock


class TinyTransformer(torch.nn.Module):
    """Embedding, blocks, norm and a projection to the vocabulary; activations in `dtype`, parameters fp32."""

    def __init__(self, vocab: int, width: int, heads: int, kv_heads: int, layers: int, tokens: int, dtype: torch.dtype):
        super().__init__()
        self.embed = torch.nn.Embedding(vocab, width)
        self.position = torch.nn.Embedding(tokens, width)
        self.blocks = torch.nn.ModuleList(TransformerBlock(width, heads, kv_heads) for _ in range(layers))
        self.norm = AddRMSNorm(width)
        self.head = torch.nn.Linear(width, vocab)
        self.dtype = dtype

    def forward(self, tokens: torch.Tensor, lens: torch.Tensor) -> torch.Tensor:
        at = torch.arange(tokens.shape[1], device=tokens.device)
        x, residual = (self.embed(tokens) + self.position(at)).to(self.dtype), None
        for block in self.blocks:
            x, residual = block(x, residual, lens)
        _, y, _ = self.norm(x, residual, keep=False)
        return self.head(y.float())


def batch_of(vocab: int, batch: int, tokens: int, gen: torch.Generator, device: str):
    """Random sequences, padded: (tokens, lengths, targets: the token before, -100 where there is none)."""
    x = torch.randint(0, vocab, (batch, tokens), generator=gen)
    lens = torch.randint(tokens // 2, tokens + 1, (batch,), generator=gen)
    y = torch.cat([torch.full((batch, 1), -100), x[:, :-1]], 1)
    y[torch.arange(tokens).expand(batch, -1) >= lens[:, None]] = -100
    return x.to(device), lens.to(device, torch.int32), y.to(device)


def train(replicas: int, width: int, heads: int, kv_heads: int, layers: int, tokens: int, batch: int, steps: int, lr: float,
          dtype: torch.dtype, seed: int = 0, device: str = "cuda:0"):
    """Losses of the steps, seconds a step behind the first five, and the replicas."""
    from .dist_optim import DistOptim
    vocab = 64
    torch.manual_seed(seed)
    model = TinyTransformer(vocab, width, heads, kv_heads, layers, tokens, dtype).to(device)
    models = [copy.deepcopy(model) for _ in range(replicas)]
    optim = DistOptim(models, lr=lr, momentum=0.9, fusion_threshold_bytes=4 << 20)
    gen = torch.Generator().manual_seed(seed + 1)
    losses, began = [], 0.0
    for step in range(steps):
        if step == min(5, steps - 1):
            torch.cuda.synchronize()
            began = time.perf_counter()
        total = 0.0
        for m in models:
            x, lens, y = batch_of(vocab, batch, tokens, gen, device)
            loss = torch.nn.functional.cross_entropy(m(x, lens).flatten(0, 1), y.flatten(), ignore_index=-100)
            loss.backward()
            total = total + loss.detach()
        optim.step()
        losses.append(total / replicas)
    optim.synchronize()
    torch.cuda.synchronize()
    seconds = (time.perf_counter() - began) / max(1, steps - min(5, steps - 1))
    optim.close()
    return [float(v) for v in losses], seconds, models


def main() -> None:
    ap = argparse.ArgumentParser()
    ap.add_argument("--replicas", type=int, default=4)
    ap.add_argument("--width", type=int, default=256)
    ap.add_argument("--heads", type=int, default=4)
    ap.add_argument("--kv-heads", type=int, default=2)
    ap.add_argument("--layers", type=int, default=2)
    ap.add_argument("--tokens", type=int, default=64)
    ap.add_argument("--batch", type=int, default=16, help="sequences per replica")
    ap.add_argument("--steps", type=int, default=150)
    ap.add_argument("--lr", type=float, default=0.2)
    ap.add_argument("--dtype", default="bf16", choices=["bf16", "f32"], help="type of the activations")
    args = ap.parse_args()
    if not torch.cuda.is_available():
        print("block_demo needs a GPU", file=sys.stderr)
        sys.exit(2)
    dtype = torch.bfloat16 if args.dtype == "bf16" else torch.float32
    losses, seconds, _ = train(args.replicas, args.width, args.heads, args.kv_heads, args.layers, args.tokens, args.batch, args.steps,
                               args.lr, dtype)
    print(json.dumps({"demo": "transformer blocks under DistOptim", "replicas": args.replicas, "width": args.width,
                      "layers": args.layers, "tokens": args.tokens, "batch": args.batch, "dtype": args.dtype,
                      "first_loss": losses[0], "last_loss": losses[-1], "ms_per_step": seconds * 1e3}))


if __name__ == "__main__":
    main()
