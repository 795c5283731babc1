"""A small pre-norm attention model trained with the framework's operators, on one GPU:

    norm (with the residual addition) -> fused Q|K|V projection with PAMM -> rotary positions in place
    -> attention over the fused row -> output projection (torch) -> dropout, and the gradients clipped by their global norm.

The task: tokens of a random alphabet, where every second half of a sequence repeats the first; the model
has to find out.  Run: ``python examples/train_qkv_block.py [--steps N] [--dropout P]``.
"""
from __future__ import annotations

import argparse
import sys
from pathlib import Path

import torch
import torch.nn.functional as F

ROOT = Path(__file__).resolve().parent.parent
if str(ROOT) not in sys.path:
    sys.path.insert(0, str(ROOT))

from paper_2506_02939_b200 import pamm  # noqa: E402
from paper_2506_02939_b200.autograd import Dropout, Norm, PammLinear, attention, clip_grad_norm_, rotary  # noqa: E402


class Block(torch.nn.Module):
    """One attention block with ``heads`` query heads that share ``kv_heads`` key and value heads."""

    def __init__(self, n: int, heads: int, kv_heads: int, head_dim: int, r: float, dtype=torch.bfloat16, dropout: float = 0.0, seed: int = 0):
        super().__init__()
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.norm = Norm(n, rms=True, dtype=dtype)
        self.qkv = PammLinear(n, (heads + 2 * kv_heads) * head_dim, r=r, dtype=dtype)
        self.out = torch.nn.Linear(heads * head_dim, n, bias=False, dtype=dtype, device="cuda")
        self.dropout = Dropout(dropout, seed=seed)

    def forward(self, x, stream, table):
        """``x``: the last block's output; ``stream``: the residual stream before it.  Returns the same pair."""
        y, stream = self.norm(x, stream)
        batch, seq, _ = y.shape
        total = self.heads + 2 * self.kv_heads
        z = self.qkv(y).view(batch, seq, total, self.head_dim)
        z = rotary(z, table, rotated=self.heads + self.kv_heads, inplace=True)        # V is not touched
        a = attention(z, self.kv_heads, causal=True)
        return self.dropout(self.out(a.flatten(2))), stream


class Model(torch.nn.Module):
    def __init__(self, alphabet=64, n=256, blocks=2, heads=4, kv_heads=2, head_dim=64, length=128, r=1.0 / 16, dtype=torch.bfloat16, dropout=0.0):
        super().__init__()
        self.embed = torch.nn.Embedding(alphabet, n, dtype=dtype, device="cuda")
        self.blocks = torch.nn.ModuleList(Block(n, heads, kv_heads, head_dim, r, dtype, dropout, seed=i) for i in range(blocks))
        self.norm = Norm(n, rms=True, dtype=dtype)
        self.head = torch.nn.Linear(n, alphabet, bias=False, dtype=dtype, device="cuda")
        self.register_buffer("table", pamm.rotary_table(length, *pamm.rotary_frequencies(head_dim)), persistent=False)

    def forward(self, tokens):
        x = self.embed(tokens)
        stream = torch.zeros_like(x)
        for block in self.blocks:
            x, stream = block(x, stream, self.table)
        y, _ = self.norm(x, stream)
        return self.head(y)


def train(steps: int = 200, batch: int = 32, length: int = 128, alphabet: int = 64, limit: float = 1.0, seed: int = 0, report=print,
          dropout: float = 0.0):
    torch.manual_seed(seed)
    model = Model(alphabet, length=length, dropout=dropout)
    optimizer = torch.optim.AdamW(model.parameters(), lr=2e-3, weight_decay=0.0)
    losses = []
    for step in range(steps):
        half = torch.randint(0, alphabet, (batch, length // 2), device="cuda")
        tokens = torch.cat((half, half), 1)
        logits = model(tokens[:, :-1])
        # the second half alone can be known
        loss = F.cross_entropy(logits[:, length // 2 - 1:].float().flatten(0, 1), tokens[:, length // 2:].flatten())
        optimizer.zero_grad()
        loss.backward()
        norm = clip_grad_norm_(model.parameters(), limit)
        optimizer.step()
        losses.append(loss.detach())
        if report is not None and (step % 20 == 0 or step == steps - 1):
            report(f"step {step:4d}  loss {float(loss.detach()):.4f}  gradient norm {float(norm):.3f}")
    return torch.stack(losses).float().cpu()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--dropout", type=float, default=0.0)
    args = ap.parse_args()
    train(args.steps, dropout=args.dropout)
