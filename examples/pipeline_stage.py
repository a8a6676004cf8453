"""A pipeline stage of a transformer between two boundaries, trained for a few steps, then served token by token.

The hidden states arrive through a compressed boundary (4 sign bits a value forward, 8-bit codes for the gradient that goes
back), pass the stage's entry (layer norm, then a product in 8-bit blocks) and leave through a second product; the loss
is the distance from a target that a random stage of the same form makes.  Run it on a GPU:

    python examples/pipeline_stage.py [--tokens 1024] [--hidden 768] [--inner 2048] [--steps 30]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2311_05827_amd as A


def train(tokens, hidden, inner, steps, dtype=torch.bfloat16, seed=0, say=print):
    """Losses of the steps, and the trained stage."""
    torch.manual_seed(seed)
    code = A.F32 if dtype == torch.float32 else A.BF16
    entry, out = A.stage.NormLinear(hidden, inner), A.stage.BlockLinear(inner, hidden)
    teacher_entry, teacher_out = A.stage.NormLinear(hidden, inner), A.stage.BlockLinear(inner, hidden)
    forward = A.boundary.ForwardCompressor(tokens, hidden, in_dtype=code, out_dtype=code)
    backward = A.boundary.BackwardCompressor(tokens, hidden, in_dtype=code, out_dtype=code)
    for _ in range(2):
        forward.controller.on_lr_change()   # 4 bits
    optimizer = torch.optim.AdamW([*entry.parameters(), *out.parameters()], lr=3e-3, weight_decay=0.0)
    losses = []
    for step in range(steps):
        x = torch.randn(tokens, hidden, device="cuda", dtype=dtype)
        with torch.no_grad():
            target = teacher_out(torch.relu(teacher_entry(x)))
        sent = x.clone().requires_grad_(True)                 # the previous stage's output
        received = A.boundary.boundary(sent, forward, backward)
        y = out(torch.relu(entry(received)))
        loss = (y.float() - target.float()).square().mean()
        optimizer.zero_grad()
        loss.backward()                                        # sent.grad: what the previous stage receives
        optimizer.step()
        losses.append(loss.detach())
    losses = torch.stack(losses).tolist()
    for step in range(0, steps, max(1, steps // 6)):
        say("step %3d  loss %.4f" % (step, losses[step]))
    return losses, entry, out


@torch.no_grad()
def serve(entry, out, tokens, dtype=torch.bfloat16):
    """One token after the other through the stage, its weights laid out once."""
    entry.eval().linear.freeze()
    out.eval().freeze()
    return torch.cat([out(torch.relu(entry(t[None]))) for t in tokens.to(dtype)])


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 1024), ("hidden", 768), ("inner", 2048), ("steps", 30)):
        ap.add_argument("--" + name, type=int, default=value)
    a = ap.parse_args()
    losses, entry, out = train(a.tokens, a.hidden, a.inner, a.steps)
    y = serve(entry, out, torch.randn(4, a.hidden, device="cuda"))
    print("loss %.4f -> %.4f; served %d tokens, mean square %.4f" % (losses[0], losses[-1], len(y), float(y.float().square().mean())))


if __name__ == "__main__":
    main()
