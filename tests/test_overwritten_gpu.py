"""Calls that write over a tensor of the caller's (GPU): autograd hears of it, and
memory that the call reads elsewhere is refused."""
import pytest
import torch

from paper_2310_05205_amd import gear, learn
from tests.helpers import cuda, say

pytestmark = pytest.mark.gpu


def rows(n=6, V=9):
    act = torch.arange(n, device=cuda()) % V
    old, adv = torch.full((n,), -2.0, device=cuda()), torch.linspace(-1, 1, n, device=cuda())
    return act, old, adv


def test_logits_saved_by_autograd():
    """tanh keeps its result for its gradient; a product with a constant keeps nothing."""
    act, old, adv = rows()
    a = torch.randn(6, 9, device=cuda(), requires_grad=True)
    z = torch.tanh(a)
    say("policy loss over logits that autograd has saved")
    grad = gear.policy_loss(z, act, old, adv, in_place=True)[4]
    assert grad.data_ptr() == z.data_ptr()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        z.backward(grad.detach().clone())
    z = 3.0 * a
    want = gear.policy_loss(z.detach().clone(), act, old, adv)[4]
    grad = gear.policy_loss(z, act, old, adv, in_place=True)[4].detach().clone()
    z.backward(grad)
    assert torch.equal(a.grad, 3.0 * want)


def test_versions_of_logits():
    act, old, adv = rows()
    z = torch.randn(6, 9, device=cuda())
    before = z._version
    gear.policy_loss(z, act, old, adv)
    gear.policy_loss(z, act, old, adv, grad=False, in_place=True)
    assert z._version == before  # not written
    gear.policy_loss(z.view(2, 3, 9), act.view(2, 3), old.view(2, 3), adv.view(2, 3), in_place=True)
    assert z._version == before + 1


def test_states_saved_by_autograd():
    """An actor steps a state in place that a recorded window started from."""
    gate, x = (torch.rand(2, 5, 6, device=cuda(), requires_grad=True) for _ in range(2))
    state = torch.randn(2, 6, device=cuda())
    say("recurrence step over a state that autograd has saved")
    y, _ = learn.recurrence(gate, x, state)
    before = state._version
    gear.recurrence_step(gate[:, 0].detach(), x[:, 0].detach(), state, out=state)
    assert state._version == before + 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    y, _ = learn.recurrence(gate, x, state)
    other = torch.empty_like(state)
    gear.recurrence_step(gate[:, 0].detach(), x[:, 0].detach(), state, out=other)
    assert state._version == before + 1 and other._version == 1
    y.sum().backward()


def test_inference_tensors():
    """An actor's states and logits made without autograd, written over inside its scope and out of it."""
    act, old, adv = rows()
    with torch.inference_mode():
        gate, x = torch.rand(2, 6, device=cuda()), torch.rand(2, 6, device=cuda())
        state, z = torch.ones(2, 6, device=cuda()), torch.randn(6, 9, device=cuda())
        want = gate * (gate * state + x) + x
        gear.recurrence_step(gate, x, state, out=state)
    say("recurrence step over an inference tensor")
    gear.recurrence_step(gate, x, state, out=state)
    torch.testing.assert_close(state, want, rtol=1e-6, atol=1e-6)
    assert gear.policy_loss(z, act, old, adv, in_place=True)[4].data_ptr() == z.data_ptr()
