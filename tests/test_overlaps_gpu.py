"""Outputs in memory that the same call reads elsewhere are refused (GPU)."""
import pytest
import torch

from paper_2310_05205_amd import gear
from tests.helpers import cuda, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D", [1, 4, 5, 64])
def test_a_step_over_its_inputs(D):
    """Lanes share channels of some widths: one would read what another has written."""
    B = 3
    buf = torch.rand(4 * B * D + 16, device=cuda())
    x, gate, state = (buf[k * B * D:(k + 1) * B * D].view(B, D) for k in range(3))
    free = buf[3 * B * D:4 * B * D].view(B, D)
    reset = buf[:B * D].view(torch.uint8)[:B]
    kept = buf.clone()
    for kw in ({"out": x}, {"out": gate}, {"out": buf[1:B * D + 1].view(B, D)},
               {"state": x, "out": x}, {"state": free, "reset": reset, "out": x, "x": gate}):
        xx = kw.pop("x", x)
        say("recurrence step over its inputs D=%d" % D)
        with pytest.raises(ValueError, match="overlap"):
            gear.recurrence_step(gate, xx, kw.pop("state", state), **kw)
    torch.cuda.synchronize()
    assert torch.equal(buf, kept)
    y, s = gear.recurrence_step(gate, x, state, out=free)  # neighbours are no overlap
    want_y, want_s = gear.recurrence_step(gate, x, state)
    assert torch.equal(s, want_s) and torch.equal(y, want_y) and s.data_ptr() == free.data_ptr()


def test_a_step_between_the_rows_of_its_inputs():
    """Inputs at a stride leave room for a state of one window among their rows."""
    buf = torch.rand(4, 24, device=cuda())
    x, gate = buf[::2, :6], buf[::2, 6:12]
    state = torch.rand(2, 6, device=cuda())
    want = gear.recurrence_step(gate, x, state)[1]
    out = buf[1, 0:12].view(2, 6)
    assert torch.equal(gear.recurrence_step(gate, x, state, out=out)[1], want)
    with pytest.raises(ValueError, match="overlap"):
        gear.recurrence_step(gate, x, state, out=buf.view(-1)[37:49].view(2, 6))  # one element into the third row


@pytest.mark.parametrize("which", ["action", "old_logp", "ref_logp", "adv", "weight", "mask", "grad_loss"])
def test_a_gradient_over_the_rows_inputs(which):
    """The gradient takes the logits' memory; what the rows' terms come from must not lie in it."""
    n, V = 8, 6
    z = torch.randn(n, V, device=cuda())
    row = z.view(-1)[10:10 + n]
    kw = {"action": torch.zeros(n, dtype=torch.int32, device=cuda()), "old_logp": torch.full((n,), -2.0, device=cuda()),
          "adv": torch.ones(n, device=cuda())}
    kw[which] = {"action": row.view(torch.int32), "mask": row.view(torch.uint8)[:n], "grad_loss": row[:1]}.get(which, row)
    kept = z.clone()
    args = [kw.pop(k) for k in ("action", "old_logp", "adv")]
    say("policy gradient over its %s" % which)
    with pytest.raises(ValueError, match="%s must not overlap" % which):
        gear.policy_loss(z, *args, in_place=True, **kw)
    torch.cuda.synchronize()
    assert torch.equal(z, kept)
    gear.policy_loss(z, *args, **kw)  # reads them, and writes elsewhere
    gear.policy_loss(z, *args, grad=False, in_place=True, **kw)
    assert torch.equal(z, kept)
