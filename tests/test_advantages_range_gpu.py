"""Advantages of windows that are split into segments, where the discounts' product
passes what 32 bits hold (GPU)."""
import numpy as np
import pytest
import torch

from paper_2310_05205_amd import gear
from tests.helpers import cuda, say
from tests.test_advantages_gpu import check, make, wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("L", [6, 500, 3000, 30000])
@pytest.mark.parametrize("gamma,lam", [(0.99, 0.95), (0.5, 0.5), (1.0, 1.0), (1e-3, 1e-3)])
def test_an_infinite_reward_stays(L, gamma, lam):
    """It reaches every step before it in its episode, as the steps' sums give it, and no other."""
    r, v, d, _ = make(4, L, "float32", "float32", L, 0, False)
    r[0, L - 1], r[1, L // 2], r[2, L - 1] = float("inf"), float("-inf"), float("-inf")
    d = torch.zeros(4, L, dtype=torch.bool, device=cuda())
    d[2, L // 3] = True
    say("advantages with infinite rewards L=%d gamma=%s lambda=%s" % (L, gamma, lam))
    adv, ret = gear.advantages(r, v, gamma, lam, done=d)
    for t in (adv, ret):
        assert bool((t[0] == float("inf")).all()) and bool((t[1, :L // 2 + 1] == float("-inf")).all())
        assert bool((t[2, L // 3 + 1:] == float("-inf")).all())
        assert bool(torch.isfinite(t[1, L // 2 + 1:]).all() & torch.isfinite(t[2, :L // 3 + 1]).all())
        assert bool(torch.isfinite(t[3]).all())


@pytest.mark.parametrize("gamma,lam", [(0.9, 0.5), (0.5, 0.25), (1e-4, 1e-4), (0.0, 0.5)])
def test_discounts_that_vanish(gamma, lam):
    r, v, d, n = make(3, 9000, "float32", "bfloat16", 5, 0.001, True)
    r[:, -1] = 1e30
    say("advantages gamma=%s lambda=%s" % (gamma, lam))
    check(r, v, gamma, lam, d, n)
    assert np.isfinite(wide(gear.advantages(r, v, gamma, lam, done=d, lengths=n)[0])).all()
