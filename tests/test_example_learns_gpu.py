"""The example's agent learns what its rewards say (GPU)."""
import pytest
import torch

from tests.helpers import say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", [0, 1])
def test_the_rewarded_action_becomes_likelier(seed):
    """On observations it has not seen.  The clip lets a probability rise from 1/16 by a fifth before it takes the
    gradient away; a twentieth is asked for.  Untrained agents are within a hundredth of 1/16: whatever their logits,
    the rewarded action depends on signs that these treat alike."""
    from examples import replay_learner as example
    torch.manual_seed(seed)
    agent = example.Agent().cuda()
    say("examples/replay_learner.py, 60 steps, seed %d" % seed)
    before = example.rewarded(agent)
    assert abs(before - 1 / 16) < 0.01 / 16
    losses, _ = example.train(steps=60, seed=seed, log=say, agent=agent)
    assert len(losses) == 60 and example.rewarded(agent) > 1.05 / 16
