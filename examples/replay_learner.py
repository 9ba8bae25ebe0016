"""A recurrent agent learns from prioritized replay, every operator on the GPU.

    python examples/replay_learner.py [--steps 20] [--windows 256] [--length 32]

A replay table holds trajectories of 8 agents' observations with actions,
rewards, done flags and the log-probabilities their actions had.  Each step
selects windows by priority, collects them, runs a gated recurrence over each
window (its state cleared where an episode began), estimates advantages, takes
the clipped policy loss weighted by the importance-sampling weights, steps the
parameters, and writes the windows' mean absolute advantages back as
priorities.  At the end the agent acts: one recurrence step per environment
step, its states updated in place.

The data stays that of random agents, so the clipped ratio lets the probability
of a rewarded action rise by about a fifth; how far it got is printed.
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2310_05205_amd import gear, learn  # noqa: E402

AGENTS, OBS, ACTIONS, WIDTH = 8, 8, 16, 256
# An action is rewarded at once.  A longer horizon would add the rewards of later actions, of all agents, as noise: with
# 0.99 and 0.95 nothing is learned from this much data.
GAMMA, LAMBDA = 0.5, 0.5


class Agent(torch.nn.Module):
    """Observations -> gate and input of a recurrence -> logits per agent and a value."""

    def __init__(self):
        super().__init__()
        self.project = torch.nn.Linear(AGENTS * OBS, 2 * WIDTH)
        self.policy = torch.nn.Linear(WIDTH, AGENTS * ACTIONS)
        self.value = torch.nn.Linear(WIDTH, 1)

    def forward(self, obs, reset):
        p = self.project(obs)
        h, _ = learn.recurrence(p[..., :WIDTH], p[..., WIDTH:], form=gear.GEAR_GATE_SIGMOID, reset=reset)
        logits = self.policy(h).view(*h.shape[:2], AGENTS, ACTIONS)
        return logits, self.value(h).squeeze(-1)

    def act(self, obs, state, reset):
        p = self.project(obs)
        h, _ = gear.recurrence_step(p[:, :WIDTH], p[:, WIDTH:], state, form=gear.GEAR_GATE_SIGMOID, reset=reset, out=state)
        return self.policy(h).view(-1, AGENTS, ACTIONS).argmax(-1)


def observe(n, T, generator):
    """Observations, and for each the action that is rewarded: the one that the signs of the first four name."""
    obs = torch.randn(n, T, AGENTS, OBS, generator=generator, device="cuda").to(torch.bfloat16)
    bits = (obs[..., :4] > 0).int()
    return obs, (bits * torch.tensor([1, 2, 4, 8], device="cuda", dtype=torch.int32)).sum(-1)


def rewarded(agent, seed=1 << 20):
    """Mean probability that the agent gives the rewarded action on new observations; 1/16 for one that knows nothing."""
    obs, right = observe(64, 64, torch.Generator(device="cuda").manual_seed(seed))
    with torch.no_grad():
        logits, _ = agent(obs.float().flatten(2), None)
    return float(torch.softmax(logits, -1).gather(-1, right.long()[..., None]).mean())


def fill(table, n, T, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    obs, right = observe(n, T, g)
    action = torch.randint(0, ACTIONS, (n, T, AGENTS), generator=g, device="cuda", dtype=torch.int32)
    reward = (action == right).float().mean(-1)
    done = (torch.rand(n, T, generator=g, device="cuda") < 0.02).to(torch.uint8)
    logp = torch.full((n, T, AGENTS), -float(np.log(ACTIONS)), device="cuda")
    table.insert({"obs": obs, "action": action, "reward": reward, "done": done, "logp": logp},
                 np.full(n, 1000, np.uint32))


def train(steps=20, windows=256, length=32, seed=0, log=print, agent=None):
    """Runs the loop, for a new agent or a given one; returns the losses and the last actions."""
    torch.manual_seed(seed)
    table = gear.Table([("obs", torch.bfloat16, (AGENTS, OBS)), ("action", torch.int32, (AGENTS,)),
                        ("reward", torch.float32, ()), ("done", torch.uint8, ()), ("logp", torch.float32, (AGENTS,))],
                       capacity=4 * windows, T=2 * length)
    try:
        fill(table, 4 * windows, 2 * length, seed)
        agent = Agent().cuda() if agent is None else agent
        before = rewarded(agent)
        opt = torch.optim.Adam(agent.parameters(), lr=3e-3)
        losses = []
        for step in range(steps):
            idx, start, weight = table.select(gear.GEAR_PRIORITIZED, windows, length, seed=seed + step, beta=0.4, weights=True)
            batch = table.collect_fields(idx, start, length)
            # The state is cleared before the step that follows an episode's end.
            reset = torch.nn.functional.pad(batch["done"][:, :-1], (1, 0))
            logits, value = agent(batch["obs"].float().flatten(2), reset)
            # The value after the window's last step is not in it; its own stands in.
            values = torch.cat([value, value[:, -1:]], dim=1).detach()
            adv, ret = gear.advantages(batch["reward"], values, GAMMA, LAMBDA, done=batch["done"])
            loss, logp, entropy, stats = learn.policy_loss(logits, batch["action"], batch["logp"], adv, weight=weight,
                                                           entropy=0.001)
            critic = (weight[:, None] * (value - ret).square()).mean()
            opt.zero_grad()
            (loss + 0.5 * critic).backward()
            opt.step()
            table.update_priorities(idx, (1 + 1000 * adv.abs().mean(1)).to(torch.int32))
            losses.append((loss.detach(), critic.detach(), stats))
        assert table.sync() == 0
        losses = [(float(l), float(c), s.tolist()) for l, c, s in losses]
        for step, (l, c, s) in enumerate(losses):
            if step % max(1, steps // 5) == 0 or step == steps - 1:
                log("step %3d  policy loss %+.4f  critic %.4f  entropy %.3f  clipped %.3f" % (step, l, c, s[2], s[3]))
        log("probability of the rewarded action: %.4f -> %.4f" % (before, rewarded(agent)))
        # Acting: 64 environments, states in place.
        state = torch.zeros(64, WIDTH, device="cuda")
        with torch.no_grad():
            for _ in range(8):
                action = agent.act(torch.randn(64, AGENTS * OBS, device="cuda"), state, None)
        return losses, action
    finally:
        table.close()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=20)
    ap.add_argument("--windows", type=int, default=256)
    ap.add_argument("--length", type=int, default=32)
    a = ap.parse_args()
    train(a.steps, a.windows, a.length)
