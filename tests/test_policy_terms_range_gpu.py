"""Rows of the policy loss with ratios and terms beyond fp32, where a 0 multiplies them (GPU)."""
import numpy as np
import pytest
import torch

from paper_2310_05205_amd import gear
from tests.helpers import cuda, say
from tests.test_policy_gpu import check, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [3, 18, 700, 5000, 40000])
def test_a_ratio_beyond_range_times_no_advantage(V):
    """exp(lp - old) passes fp32 where the acting policy held the action for all but impossible; an advantage of 0
    leaves nothing of it."""
    z, act, old, refl, _, adv = make((12,), V, "float32", V)
    old[3], old[4], old[7] = -120.0, -1e4, -3e38
    adv[3] = adv[4] = adv[5] = 0.0
    adv[7] = 1.0  # clipped
    say("policy with ratios beyond range V=%d" % V)
    out = gear.policy_loss(z, act, old, adv, ref_logp=refl, kl=0.1, entropy=0.02)
    assert np.isfinite(float(out[0])) and bool(torch.isfinite(out[3]).all()) and bool(torch.isfinite(out[4]).all())
    check(z, act, old.clamp(min=-600), refl, None, adv)  # exp of more overflows 64 bits, too


@pytest.mark.parametrize("V", [3, 18, 700, 5000, 40000])
def test_a_weight_of_zero_leaves_nothing(V):
    """Of a row whose terms pass fp32, either."""
    z, act, old, refl, _, adv = make((12,), V, "float32", V + 1)
    weight = torch.rand(12, device=cuda())
    weight[2] = weight[5] = weight[6] = 0.0
    old[2], adv[2], refl[5], refl[6] = -120.0, -1.0, 110.0, 95.0
    say("policy with weights of 0 V=%d" % V)
    loss, logp, ent, stats, grad = gear.policy_loss(z, act, old, adv, ref_logp=refl, weight=weight, kl=0.1, entropy=0.02)
    some = torch.ones(12, dtype=torch.bool, device=cuda())
    some[[2, 5, 6]] = False
    want = gear.policy_loss(z, act, old, adv, ref_logp=refl, weight=weight, mask=some, kl=0.1, entropy=0.02, denom=12.0)
    np.testing.assert_allclose(float(loss), float(want[0]), rtol=1e-6, atol=1e-7)
    assert torch.equal(grad[some], want[4][some]) and not bool(grad[~some].any())
