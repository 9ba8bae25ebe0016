"""The differentiable forms against the calls they make, gradients against
torch's own through plain operations, and the example that runs the operators
together (GPU)."""
import numpy as np
import pytest
import torch

from paper_2310_05205_amd import gear, learn
from tests.helpers import cuda, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sigmoid", [False, True])
def test_recurrence_gradients_reach_every_input(sigmoid):
    """fp32 gradients through the halves of one projection, against the same steps in float64 autograd."""
    form = gear.GEAR_GATE_SIGMOID if sigmoid else gear.GEAR_GATE_VALUE
    g = torch.Generator().manual_seed(1)
    p0 = torch.rand(3, 40, 14, generator=g, dtype=torch.float64)
    s0 = torch.randn(3, 7, generator=g, dtype=torch.float64)
    r = torch.rand(3, 40, generator=g) < 0.05
    p, s = (t.clone().requires_grad_() for t in (p0, s0))
    h, ys = s, []
    for t in range(40):
        gate, x = p[:, t, :7], p[:, t, 7:]
        kept = torch.where(r[:, t, None], torch.zeros_like(h), h)
        f = torch.sigmoid(gate) if sigmoid else gate
        h = f * kept + ((1 - f) * x if sigmoid else x)
        ys.append(h)
    y64 = torch.stack(ys, 1)
    (y64.square().sum() + h.sum()).backward()
    q, u = (t.float().to(cuda()).requires_grad_() for t in (p0, s0))
    say("learn.recurrence sigmoid=%s" % sigmoid)
    y, final = learn.recurrence(q[..., :7], q[..., 7:], u, form=form, reset=r.to(cuda()))
    (y.square().sum() + final.sum()).backward()
    # Values and gradients stay below 1e3 here; 40 steps of correctly rounded fp32 operations, a few units each.
    for got, want in ((y, y64), (q.grad, p.grad), (u.grad, s.grad)):
        scale = want.detach().abs().max().item()
        assert (got.detach().cpu().double() - want.detach()).abs().max().item() < 40 * 16 * 2.0 ** -24 * scale


def test_recurrence_output_gradients_of_any_kind():
    """None, broadcast and transposed gradients of the outputs."""
    gate = torch.rand(2, 20, 6, device=cuda(), requires_grad=True)
    x = torch.randn(2, 20, 6, device=cuda(), requires_grad=True)
    y, final = learn.recurrence(gate, x)
    final.sum().backward()
    only_final = x.grad.clone()
    x.grad = gate.grad = None
    y, final = learn.recurrence(gate, x)
    y.sum().backward()  # a gradient expanded from one value
    only_y = x.grad.clone()
    x.grad = gate.grad = None
    y, final = learn.recurrence(gate, x)
    (y.transpose(1, 2).contiguous().sum() + final.sum()).backward()
    torch.testing.assert_close(x.grad, only_y + only_final, rtol=1e-5, atol=1e-5)


def test_policy_loss_gradient_scales_and_repeats():
    g = torch.Generator().manual_seed(2)
    z = torch.randn(6, 5, 9, generator=g).to(cuda()).requires_grad_()
    act = torch.randint(0, 9, (6, 5), generator=g).to(cuda())
    old, adv = torch.full((6, 5), -2.0, device=cuda()), torch.randn(6, 5, generator=g).to(cuda())
    want = gear.policy_loss(z.detach(), act, old, adv, entropy=0.1)
    loss, logp, ent, stats = learn.policy_loss(z, act, old, adv, entropy=0.1)
    assert torch.equal(loss.detach(), want[0]) and torch.equal(logp, want[1]) and not logp.requires_grad
    (4 * loss).backward(retain_graph=True)
    assert torch.equal(z.grad, 4 * want[4])
    z.grad = None
    loss.backward()
    assert torch.equal(z.grad, want[4])


def test_example_runs():
    """Every operator in one loop: finite losses and a policy that moves."""
    from examples import replay_learner
    say("examples/replay_learner.py")
    losses, action = replay_learner.train(steps=12, windows=128, length=16, log=say)
    assert len(losses) == 12 and np.isfinite([l[:2] for l in losses]).all()
    entropy, clipped = [s[2] for _, _, s in losses], [s[3] for _, _, s in losses]
    assert all(0 < e < np.log(16) + 1e-5 for e in entropy) and len(set(entropy)) == 12 and 0 < clipped[-1] < 1
    assert action.shape == (64, 8) and int(action.min()) >= 0 and int(action.max()) < 16
