"""The learner's formulas against differences, in 64 bits (CPU)."""
import numpy as np
import pytest

from tests import learner_reference as ref


def _slope(f, x, d, step=1e-6):
    return (f(x + step * d) - f(x - step * d)) / (2 * step)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("T", [1, 7])
def test_recurrence_gradients_are_slopes(sigmoid, T):
    rng = np.random.default_rng(T)
    B, D = 3, 4
    gate, x, dy = rng.normal(size=(3, B, T, D))
    state, dfinal = rng.normal(size=(2, B, D))
    reset = rng.random((B, T)) < 0.3
    lengths = np.array([0, T, (T + 1) // 2])

    def loss(g, x_, s):
        (y, _), (h, _), _, _ = ref.recurrence(g, x_, s, sigmoid, reset, lengths)
        return (y * dy).sum() + (h * dfinal).sum()
    (dg, _), (dx, _), (ds, _) = ref.recurrence_backward(gate, x, state, dy, dfinal, sigmoid, reset, lengths)
    for grad, at in ((dg, 0), (dx, 1), (ds, 2)):
        args = [gate, x, state]
        d = rng.normal(size=args[at].shape)

        def f(v):
            return loss(*[v if i == at else a for i, a in enumerate(args)])
        # Central differences: rounding 1e-16 / 1e-6 and a third-order term of 1e-12, on values of order 10.
        assert abs(_slope(f, args[at], d) - (grad * d).sum()) < 1e-7


def test_policy_gradient_is_a_slope():
    rng = np.random.default_rng(5)
    n, V = 40, 9
    z = 2 * rng.normal(size=(n, V))
    action = rng.integers(0, V, n)
    action[3] = -1
    mask = rng.random(n) < 0.8
    kw = dict(mask=mask, adv=rng.normal(size=n), weight=rng.random(n), clip=(0.1, 0.3), kl=0.2, entropy=0.05, denom=None)
    lp = ref.policy(z, action)["logp"][0]
    kw["old"], kw["ref"] = lp - 0.3 * rng.normal(size=n), lp - 0.3 * rng.normal(size=n)
    out = ref.policy(z, action, **kw)
    assert 0 < out["stats"][0][3] < 1  # some rows clipped, some not
    d = rng.normal(size=z.shape)
    slope = _slope(lambda v: ref.policy(v, action, **kw)["loss"][0], z, d)
    assert abs(slope - (out["grad"][0] * d).sum()) < 1e-7
    assert not out["grad"][0][~mask].any() and not out["grad"][0][3].any()


def test_advantages_sum_the_discounted_errors():
    rng = np.random.default_rng(6)
    r, v = rng.normal(size=(2, 9)), rng.normal(size=(2, 10))
    done = np.zeros((2, 9), bool)
    done[0, 4] = True
    (adv, _), (ret, _) = ref.advantages(r, v, 0.5, 0.25, done)
    for b in range(2):
        for t in range(9):
            total, k = 0.0, 1.0
            for u in range(t, 9):
                live = not done[b, u]
                total += k * (r[b, u] + 0.5 * live * v[b, u + 1] - v[b, u])
                k *= 0.125
                if not live:
                    break
            assert abs(adv[b, t] - total) < 1e-12
    np.testing.assert_allclose(ret, adv + v[:, :-1], atol=1e-12)
