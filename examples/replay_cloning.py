"""A token model clones replayed behaviour, every operator on the GPU.

    python examples/replay_cloning.py [--steps 20] [--windows 64] [--length 32] [--bits 8]

A replay table holds trajectories of tokens (discretised observations and
actions), some of them padding.  Each step selects windows by priority,
collects them, runs norm, gated recurrence and norm over each window, takes the
cross entropy of the next tokens weighted by the importance-sampling weights
(the padding takes no part), clips the gradients and steps all parameters at
once, their averages in 8 bits, and writes the windows' mean losses back as
priorities.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2310_05205_amd import gear, learn  # noqa: E402

TOKENS, WIDTH = 500, 128


class Cloner(torch.nn.Module):
    """Tokens -> embedding -> norm -> recurrence -> residual sum and norm -> token head."""

    def __init__(self, dtype=torch.float32):
        super().__init__()
        self.embed = torch.nn.Parameter(torch.randn(TOKENS, WIDTH, dtype=dtype))
        self.project = torch.nn.Linear(WIDTH, 2 * WIDTH, dtype=dtype)
        self.head = torch.nn.Parameter(torch.randn(TOKENS, WIDTH, dtype=dtype) / WIDTH ** 0.5)
        self.norm = torch.nn.Parameter(torch.stack([torch.ones(2, WIDTH), torch.zeros(2, WIDTH)], 1))  # weight, bias of both

    def forward(self, tokens):
        """Normed states before the head."""
        x = self.embed[tokens]
        p = self.project(learn.layer_norm(x, self.norm[0, 0], self.norm[0, 1]))
        h, _ = learn.recurrence(p[..., :WIDTH], p[..., WIDTH:], form=gear.GEAR_GATE_SIGMOID)
        return learn.layer_norm(h, self.norm[1, 0], self.norm[1, 1], residual=x)[0]

    def loss(self, tokens, mask, weight=None):
        """Weighted mean loss of the next tokens, and their log-probabilities."""
        y = self.forward(tokens[:, :-1].long())
        return learn.token_loss(y, self.head, tokens[:, 1:].contiguous(), weight=weight, mask=mask[:, 1:].contiguous())[:2]


def fill(table, n, T, seed):
    """Trajectories that walk the tokens by a fixed step, now and then a random one; the last part is padding."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    first = torch.randint(0, TOKENS, (n, 1), generator=g, device="cuda")
    stray = torch.randint(0, TOKENS, (n, T), generator=g, device="cuda") * (torch.rand(n, T, generator=g, device="cuda") < 0.05)
    tokens = (first + 7 * torch.arange(T, device="cuda") + stray.cumsum(1)) % TOKENS
    length = T - torch.randint(0, T // 4 + 1, (n, 1), generator=g, device="cuda")
    mask = torch.arange(T, device="cuda") < length
    table.insert({"token": tokens.int(), "mask": mask.to(torch.uint8)}, np.full(n, 1000, np.uint32))


def train(steps=20, windows=64, length=32, bits=8, seed=0, dtype=torch.bfloat16, log=print):
    """Runs the loop; returns the losses and the gradients' norms."""
    torch.manual_seed(seed)
    table = gear.Table([("token", torch.int32, ()), ("mask", torch.uint8, ())], capacity=8 * windows, T=2 * length)
    try:
        fill(table, 8 * windows, 2 * length, seed)
        model = Cloner(dtype).cuda()
        opt = learn.AdamW(model.parameters(), lr=3e-3, betas=(0.9, 0.98), bits=bits, max_norm=1.0)
        seen = []
        for step in range(steps):
            idx, start, weight = table.select(gear.GEAR_PRIORITIZED, windows, length, seed=seed + step, beta=0.4, weights=True)
            batch = table.collect_fields(idx, start, length)
            loss, logp = model.loss(batch["token"], batch["mask"], weight)
            opt.zero_grad()
            loss.backward()
            norm = opt.step()
            per_window = -logp.sum(1) / batch["mask"][:, 1:].sum(1).clamp(min=1)
            table.update_priorities(idx, (1 + 1000 * per_window).to(torch.int32))
            seen.append((loss.detach(), norm))
        assert table.sync() == 0
        seen = [(float(l), float(n)) for l, n in seen]
        for step, (l, n) in enumerate(seen):
            if step % max(1, steps // 5) == 0 or step == steps - 1:
                log("step %3d  loss %.4f  gradients' norm %.3f" % (step, l, n))
        return seen
    finally:
        table.close()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--windows", type=int, default=64)
    ap.add_argument("--length", type=int, default=32)
    ap.add_argument("--bits", type=int, default=8, choices=(8, 32))
    a = ap.parse_args()
    train(a.steps, a.windows, a.length, a.bits)
