"""A small decoder-only language model trained on packed sequences, with the
library on its whole hot path between the projections and behind them:

* attention over the pack: ``layers.PackedAttention`` (forward and backward); with
  ``--window``, every other layer sees a window and the sequence's first tokens;
* with ``--rotary``, norms of queries and keys and the rotation of their positions
  in place of learned places: ``layers.QKNormRotary``;
* every linear layer keeps its input in 8 bits and takes its weight gradient
  from there: ``layers.linear``;
* the gated MLP keeps gate and up in 8 bits: ``layers.swiglu``;
* with ``--clip``, the gradients are clipped by their global norm:
  ``optim.clip_grad_norm_``;
* the hidden matrices are updated by ``NormPreOptimizer``, embeddings and norms
  by AdamW, as in the paper's setup.

The data are synthetic (no corpus is needed): each sequence repeats a random
phrase, so that a model that attends to the phrase's last occurrence predicts
all but its first tokens.  Lengths differ from sequence to sequence and every
step packs other ones into a buffer of fixed size.

    python -m examples.train_packed_lm --steps 60
    python -m examples.train_packed_lm --steps 60 --window 32 --sinks 4 --rotary --clip 1.0
"""
from __future__ import annotations

import argparse
import time

import torch
import torch.nn.functional as F

from paper_2609_36692_gb300 import layers
from paper_2609_36692_gb300.optim import NormPreOptimizer, clip_grad_norm_


class Block(torch.nn.Module):
    """Pre-norm attention and gated MLP; bf16 activations, fp32 matrices."""

    def __init__(self, width: int, heads: int, kv_heads: int, mlp: int, rotary: bool = False):
        super().__init__()
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, width // heads
        self.norm1, self.norm2 = (torch.nn.Parameter(torch.ones(width)) for _ in range(2))
        w = lambda rows, cols: torch.nn.Parameter(torch.randn(rows, cols) * cols ** -0.5)  # noqa: E731
        self.qkv = w((heads + 2 * kv_heads) * self.head_dim, width)
        self.out, self.gate, self.up, self.down = w(width, width), w(mlp, width), w(mlp, width), w(width, mlp)
        if rotary:
            self.q_norm, self.k_norm = (torch.nn.Parameter(torch.ones(self.head_dim)) for _ in range(2))

    def matrices(self):
        return [self.qkv, self.out, self.gate, self.up, self.down]

    def forward(self, x: torch.Tensor, attention: layers.PackedAttention, rotary=None, places=None) -> torch.Tensor:
        h, hk, d = self.heads, self.kv_heads, self.head_dim
        y = layers.linear(F.rms_norm(x, x.shape[-1:], self.norm1.to(x.dtype)), self.qkv).view(-1, h + 2 * hk, d)
        q, k = y[:, :h], y[:, h:h + hk]
        if rotary is not None:
            q, k = rotary(q, k, places, self.q_norm, self.k_norm, used=sum(attention.lengths))
        y = attention(q, k, y[:, h + hk:])
        x = x + layers.linear(y.reshape(x.shape), self.out)
        y = F.rms_norm(x, x.shape[-1:], self.norm2.to(x.dtype))
        return x + layers.linear(layers.swiglu(layers.linear(y, self.gate), layers.linear(y, self.up)), self.down)


class Model(torch.nn.Module):
    def __init__(self, vocab: int, width: int, heads: int, kv_heads: int, mlp: int, depth: int, max_len: int,
                 rotary: bool = False):
        super().__init__()
        self.tokens = torch.nn.Parameter(torch.randn(vocab, width) * 0.02)
        self.places = None if rotary else torch.nn.Parameter(torch.randn(max_len, width) * 0.02)
        self.rotary = layers.QKNormRotary(heads, kv_heads, width // heads) if rotary else None
        self.blocks = torch.nn.ModuleList(Block(width, heads, kv_heads, mlp, rotary) for _ in range(depth))
        self.norm = torch.nn.Parameter(torch.ones(width))

    def forward(self, ids, places, *attention):
        """attention: a plan, or several that the layers take in turn."""
        x = (self.tokens[ids] if self.rotary else self.tokens[ids] + self.places[places]).to(torch.bfloat16)
        for i, block in enumerate(self.blocks):
            x = block(x, attention[i % len(attention)], self.rotary, places)
        return F.rms_norm(x, x.shape[-1:], self.norm.to(x.dtype)).float() @ self.tokens.t()


def batch(rng: torch.Generator, tokens: int, vocab: int, max_len: int):
    """Lengths, and for each row of the pack its token, its place and the token
    to predict (-100: none); rows past the last sequence are padding."""
    lengths, ids, places, targets = [], [], [], []
    while sum(lengths) < tokens - 16:
        n = min(int(torch.randint(16, max_len + 1, (1,), generator=rng)), tokens - sum(lengths))
        period = int(torch.randint(4, 12, (1,), generator=rng))
        phrase = torch.randint(0, vocab, (period,), generator=rng)
        seq = phrase[torch.arange(n + 1) % period]
        lengths.append(n)
        ids.append(seq[:-1])
        targets.append(torch.where(torch.arange(1, n + 1) >= period, seq[1:], -100))
        places.append(torch.arange(n))
    pad = tokens - sum(lengths)
    cat = lambda xs, fill: torch.cat(xs + [torch.full((pad,), fill)]).cuda()  # noqa: E731
    return lengths, cat(ids, 0), cat(places, 0), cat(targets, -100)


def train(steps: int = 60, tokens: int = 2048, vocab: int = 256, width: int = 256, heads: int = 4, kv_heads: int = 2,
          mlp: int = 704, depth: int = 2, max_len: int = 256, lr: float = 0.02, variant: str = "G", seed: int = 0,
          log=None, window: int = 0, sinks: int = 0, rotary: bool = False, clip: float = 0.0):
    """Trains for `steps` steps; returns the losses.  window: the layers with even
    numbers see that many rows up to their own, and the first `sinks`.  clip: the
    gradients' norm is held to it (0: not)."""
    torch.manual_seed(seed)
    rng = torch.Generator().manual_seed(seed + 1)
    model = Model(vocab, width, heads, kv_heads, mlp, depth, max_len, rotary).cuda()
    matrices = [w for block in model.blocks for w in block.matrices()]
    ids_of = {id(w) for w in matrices}
    others = [p for p in model.parameters() if id(p) not in ids_of]
    opts = [NormPreOptimizer(matrices, lr=lr, variant=variant), torch.optim.AdamW(others, lr=3e-3, weight_decay=0.0)]
    plan = lambda **kw: layers.PackedAttention(heads, kv_heads, width // heads, max_tokens=tokens, max_seqs=tokens // 16, **kw)  # noqa: E731
    attention = ([plan(window=window, sinks=sinks)] if window else []) + [plan()]
    losses = []
    for step in range(steps):
        lengths, ids, places, targets = batch(rng, tokens, vocab, max_len)
        for a in attention:
            a.set_lengths(lengths)                # once per batch, for every layer and both directions
        for opt in opts:
            opt.zero_grad(set_to_none=True)
        start = time.perf_counter()
        loss = F.cross_entropy(model(ids, places, *attention), targets, ignore_index=-100)
        loss.backward()
        if clip:
            clip_grad_norm_(model.parameters(), clip)
        for opt in opts:
            opt.step()
        losses.append(float(loss.detach()))
        if log and (step % 10 == 0 or step + 1 == steps):
            log("step %3d  %2d sequences  loss %.3f  %.1f ms" % (step, len(lengths), losses[-1],
                                                                (time.perf_counter() - start) * 1e3))
    for a in attention:
        a.status()
    layers.ckpt_status()
    return losses


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=60)
    ap.add_argument("--tokens", type=int, default=2048)
    ap.add_argument("--variant", default="G", choices=["G", "L", "muon"])
    ap.add_argument("--window", type=int, default=0)
    ap.add_argument("--sinks", type=int, default=0)
    ap.add_argument("--rotary", action="store_true")
    ap.add_argument("--clip", type=float, default=0.0)
    a = ap.parse_args()
    train(steps=a.steps, tokens=a.tokens, variant=a.variant, log=print, window=a.window, sinks=a.sinks, rotary=a.rotary,
          clip=a.clip)


if __name__ == "__main__":
    main()
