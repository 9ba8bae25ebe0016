"""Rows of the policy calls whose logits are NaN throughout, or beside -inf (GPU)."""
import numpy as np
import pytest
import torch

from paper_2310_05205_amd import gear
from tests.helpers import cuda, say
from tests.test_policy_gpu import DTYPES, make

pytestmark = pytest.mark.gpu

# Rows of less than a piece, of one lane, of several lanes, of a wave, of a workgroup, and longer than registers hold
# (the last in 32 bits alone for the shorter of the two).
WIDTHS = [2, 3, 16, 100, 1000, 5000, 9000, 40000, 70000, 140000]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("V", WIDTHS)
@pytest.mark.parametrize("n", [4, 3000])
def test_nan_throughout_a_row_shows(V, n, dtype):
    """Rows of NaN, or of NaN beside -inf, are no rows without a distribution."""
    if n * V > 1 << 22:
        n = 40
    z, act, old, refl, _, adv = make((n,), V, dtype, 3)
    z[1] = float("nan")
    z[2] = float("-inf")
    z[2, V - 1] = float("nan")
    z[n - 1] = float("-inf")  # as a whole: no distribution
    act[2] = 0
    m = torch.ones(n, dtype=torch.bool, device=cuda())
    say("policy with rows of NaN n=%d V=%d %s" % (n, V, dtype))
    logp, ent = gear.action_logp(z, act)
    assert bool(torch.isnan(logp[1:3]).all()) and bool(torch.isnan(ent[1:3]).all())
    assert float(logp[n - 1]) == float("-inf") and float(ent[n - 1]) == 0
    loss, logp2, ent2, stats, grad = gear.policy_loss(z, act, old, adv, ref_logp=refl, mask=m, kl=0.1, entropy=0.1)
    assert bool(torch.isnan(logp2[1:3]).all()) and bool(torch.isnan(ent2[1:3]).all())
    assert np.isnan(float(loss)) and bool(torch.isnan(stats[:3]).all())
    assert bool(torch.isnan(grad[1]).all()) and bool(torch.isnan(grad[2]).all())
    rest = [0] + list(range(3, n))
    assert bool(torch.isfinite(grad[rest]).all()) and not bool(grad[n - 1].any())
    # Where the mask or the action leaves those rows out, nothing of them shows.
    m[1], act[2] = False, -1
    loss, logp2, ent2, stats, grad = gear.policy_loss(z, act, old, adv, ref_logp=refl, mask=m, kl=0.1, entropy=0.1)
    assert np.isfinite(float(loss)) and bool(torch.isfinite(stats).all()) and not bool(grad[1:3].any())
    assert not bool(logp2[1:3].any()) and not bool(ent2[1:3].any())
