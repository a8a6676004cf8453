"""A pipeline stage with attention between two boundaries, trained on packed sequences, then served from a cache of pages.

The hidden states of sequences of different lengths arrive packed behind each other through a compressed boundary, pass the
block's first half (layer norm, queries, keys and values by a product in 8-bit blocks, rotation, attention, a product) and its second one, and
the loss is the distance from a target that a random stage of the same form makes.  Then a prompt and token after token go through the trained stage with
a cache.  Run it on a GPU:

    python examples/attention_stage.py [--tokens 1024] [--hidden 768] [--heads 12] [--inner 2048] [--steps 30]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2311_05827_amd as A


class Block(torch.nn.Module):
    """Attention and a two-layer product, each with its residual."""

    def __init__(self, hidden, heads, kv_heads, inner):
        super().__init__()
        self.attention = A.stage.SelfAttention(hidden, heads, kv_heads)
        self.entry, self.out = A.stage.NormLinear(hidden, inner), A.stage.BlockLinear(inner, hidden)

    def forward(self, x, offsets=None, cache=None):
        x = x + self.attention(x, offsets, cache)
        return x + self.out(torch.relu(self.entry(x)))


def lengths_of(tokens, sequences):
    """Some short, some long."""
    weights = [1 + 3 * (s % 3) for s in range(sequences)]
    lengths = [tokens * w // sum(weights) for w in weights]
    lengths[-1] += tokens - sum(lengths)
    return lengths


def train(tokens, hidden, heads, kv_heads, inner, steps, sequences=5, seed=0, say=print):
    """Losses of the steps, the gradient that goes back in the last one, and the trained block."""
    torch.manual_seed(seed)
    block, teacher = Block(hidden, heads, kv_heads, inner), Block(hidden, heads, kv_heads, inner)
    forward = A.boundary.ForwardCompressor(tokens, hidden, in_dtype=A.BF16, out_dtype=A.BF16)
    backward = A.boundary.BackwardCompressor(tokens, hidden, in_dtype=A.BF16, out_dtype=A.BF16)
    for _ in range(2):
        forward.controller.on_lr_change()   # 4 bits
    offsets = torch.tensor([0] + lengths_of(tokens, sequences), device="cuda").cumsum(0).int()
    optimizer = torch.optim.AdamW(block.parameters(), lr=1e-3, weight_decay=0.0)
    losses, sent = [], None
    for step in range(steps):
        x = torch.randn(tokens, hidden, device="cuda", dtype=torch.bfloat16)
        with torch.no_grad():
            target = teacher(x, offsets)
        sent = x.clone().requires_grad_(True)                 # the previous stage's output
        y = block(A.boundary.boundary(sent, forward, backward), offsets)
        loss = (y.float() - target.float()).square().mean()
        optimizer.zero_grad()
        loss.backward()                                        # sent.grad: what the previous stage receives
        optimizer.step()
        losses.append(loss.detach())
    losses = torch.stack(losses).tolist()
    for step in range(0, steps, max(1, steps // 6)):
        say("step %3d  loss %.4f" % (step, losses[step]))
    return losses, sent.grad, block


@torch.no_grad()
def serve(block, tokens, prompt):
    """The first `prompt` tokens at once, then one after the other."""
    block.eval()
    cache = block.attention.cache(1, len(tokens), page_size=16)
    parts = [tokens[:prompt]] + list(tokens[prompt:].split(1))
    return torch.cat([block(part, cache=cache) for part in parts])


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 1024), ("hidden", 768), ("heads", 12), ("kv_heads", 4), ("inner", 2048), ("steps", 30)):
        ap.add_argument("--" + name.replace("_", "-"), type=int, default=value)
    a = ap.parse_args()
    losses, _, block = train(a.tokens, a.hidden, a.heads, a.kv_heads, a.inner, a.steps)
    x = torch.randn(40, a.hidden, device="cuda", dtype=torch.bfloat16)
    y = serve(block, x, 30)
    print("loss %.4f -> %.4f; served %d tokens, mean square %.4f" % (losses[0], losses[-1], len(y), float(y.float().square().mean())))


if __name__ == "__main__":
    main()
