"""The clipped policy loss and its gradient, and the actions' log-probabilities,
against their definition in 64 bits: action counts from one to past what
registers hold, types, masks, shared advantages and weights, logits of the
lowest value and of -inf (GPU)."""
import numpy as np
import pytest
import torch

from paper_2310_05205_amd import gear
from tests import learner_reference as ref
from tests.helpers import cuda, host, say

pytestmark = pytest.mark.gpu

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
ACTIONS = {"int32": torch.int32, "int64": torch.int64, "uint8": torch.uint8}


def wide(t):
    return None if t is None else host(t.double() if t.is_floating_point() else t)


def edges(lr, clip):
    """Log ratios moved half a percent off the clip's edges, where one rounding decides the gradient."""
    for edge in (np.log(1 - clip[0]) if clip[0] < 1 else -1e9, np.log(1 + clip[1])):
        d = lr - edge
        lr = torch.where(d.abs() < 5e-3, edge + torch.where(d < 0, -5e-3, 5e-3), lr)
    return lr


def make(lead, V, dtype, seed, mask=False, scale=2.0, clip=(0.2, 0.3), action="int32"):
    g = torch.Generator().manual_seed(seed)
    z = (scale * torch.randn(*lead, V, generator=g)).to(DTYPES[dtype])
    act = torch.randint(0, V, lead, generator=g)
    lp = torch.log_softmax(z.double(), -1).gather(-1, act[..., None])[..., 0]
    old = (lp - edges(0.3 * torch.randn(lead, generator=g, dtype=torch.float64), clip)).float()
    refl = (lp - 0.3 * torch.randn(lead, generator=g, dtype=torch.float64)).float()
    m = (torch.rand(lead, generator=g) < 0.8).to(cuda()) if mask else None
    adv = torch.randn(lead, generator=g)
    return z.to(cuda()), act.to(ACTIONS[action]).to(cuda()), old.to(cuda()), refl.to(cuda()), m, adv.to(cuda())


def rows_of(t, lead):
    """A per-row array from one whose shape is the first of the leading sizes."""
    if t is None:
        return None
    a = wide(t)
    return np.broadcast_to(a.reshape(a.shape + (1,) * (len(lead) - a.ndim)), lead).reshape(-1)


def check(z, act, old, refl, m, adv, weight=None, clip=(0.2, 0.3), kl=0.1, entropy=0.02, denom=None, scale=1.0):
    lead, V = tuple(z.shape[:-1]), z.shape[-1]
    dtype = str(z.dtype).replace("torch.", "")
    loss, logp, ent, stats, grad = gear.policy_loss(z, act, old, adv, ref_logp=refl, weight=weight, mask=m, clip=clip,
                                                    kl=kl, entropy=entropy, denom=denom, grad_scale=scale)
    assert grad.dtype == z.dtype and grad.shape == z.shape and loss.dim() == 0 and logp.shape == lead
    w = ref.policy(wide(z).reshape(-1, V), wide(act).reshape(-1), mask=rows_of(m, lead), old=wide(old).reshape(-1),
                   adv=rows_of(adv, lead), ref=None if refl is None else wide(refl).reshape(-1),
                   weight=rows_of(weight, lead), clip=clip, kl=kl, entropy=entropy, denom=denom, scale=scale)
    ref.within(wide(logp).reshape(-1), *w["logp"])
    ref.within(wide(ent).reshape(-1), *w["entropy"])
    ref.within(wide(grad).reshape(-1, V), *w["grad"], dtype)
    ref.within(wide(loss), *w["loss"])
    ref.within(wide(stats), *w["stats"])
    l2, e2 = gear.action_logp(z, act, mask=m)
    assert torch.equal(l2, logp) and torch.equal(e2, ent)
    l3, _, _, s3, none = gear.policy_loss(z, act, old, adv, ref_logp=refl, weight=weight, mask=m, clip=clip, kl=kl,
                                          entropy=entropy, denom=denom, grad=False)
    assert none is None and torch.equal(l3, loss) and torch.equal(s3, stats)
    again = gear.policy_loss(z.clone(), act, old, adv, ref_logp=refl, weight=weight, mask=m, clip=clip, kl=kl,
                             entropy=entropy, denom=denom, grad_scale=scale, in_place=z.is_contiguous())
    assert torch.equal(again[4], grad) and torch.equal(again[0], loss)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("lead,V,mask", [
    ((1,), 1, False), ((5,), 2, True), ((64,), 3, False), ((3, 7), 5, True), ((130,), 7, False), ((33,), 8, True),
    ((257,), 9, False), ((1000,), 16, True), ((77,), 18, False), ((40,), 31, True), ((9, 5), 33, False), ((21,), 64, True),
    ((19,), 65, False), ((13,), 127, True), ((17,), 200, False), ((11,), 257, True), ((9,), 511, False), ((7,), 513, True),
    ((6,), 1023, False), ((5,), 1025, True), ((6,), 2047, False), ((4,), 4096, False), ((3,), 4099, True),
    ((3,), 8192, False), ((3,), 10007, True), ((3,), 16385, False), ((2,), 32768, False), ((2,), 50001, True),
    ((2,), 65537, False), ((2,), 131072, False), ((2,), 150001, True)])
def test_against_definition(lead, V, mask, dtype):
    say("policy rows=%s V=%d %s mask=%s" % (lead, V, dtype, mask))
    check(*make(lead, V, dtype, V, mask), scale=64.0)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("V", [2500, 3071, 3073, 5000, 6143, 6144, 6145])
def test_longest_rows_of_a_wave(V, dtype):
    say("policy V=%d %s" % (V, dtype))
    check(*make((2100 if V == 5000 else 6,), V, dtype, V, True), scale=64.0)


@pytest.mark.parametrize("action", list(ACTIONS))
@pytest.mark.parametrize("case", ["plain", "no-kl", "no-ref", "no-entropy", "denom", "wide-clip", "negative"])
def test_terms(case, action):
    kw = {"plain": {}, "no-kl": {"kl": 0.0}, "no-ref": {}, "no-entropy": {"entropy": 0.0}, "denom": {"denom": 17.5},
          "wide-clip": {"clip": (1.0, 3.0)}, "negative": {"kl": -0.1, "entropy": -0.3}}[case]
    z, act, old, refl, m, adv = make((60,), 21, "float32", 4, True, clip=kw.get("clip", (0.2, 0.3)), action=action)
    say("policy terms %s %s" % (case, action))
    check(z, act, old, None if case == "no-ref" else refl, m, adv, **kw)


@pytest.mark.parametrize("depth", [1, 2, 3])
def test_shared_advantages_weights_and_masks(depth):
    """Values of a window or a step serve every row below it."""
    lead = (6, 5, 3)
    z, act, old, refl, _, _ = make(lead, 12, "bfloat16", 8)
    adv, weight = torch.randn(lead[:depth], device=cuda()), torch.rand(lead[:4 - depth], device=cuda())
    m = torch.rand(lead[:depth], device=cuda()) < 0.7
    say("policy with shared values, depth %d" % depth)
    check(z, act, old, refl, m, adv, weight)


def test_rows_at_a_stride():
    z, act, old, refl, m, adv = make((4, 6), 50, "float16", 9, True)
    big = torch.full((4, 6, 77), 3.0, dtype=torch.float16, device=cuda())
    big[..., 5:55] = z
    say("policy with strided rows")
    check(big[..., 5:55], act, old, refl, m, adv)
    a = gear.policy_loss(big[..., 5:55], act, old, adv, mask=m)
    b = gear.policy_loss(z, act, old, adv, mask=m)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("V", [3, 16, 300, 9000])
def test_lowest_values_and_infinities(V, dtype):
    """Unavailable actions at the type's lowest value or at -inf have probability 0, also the first and the last."""
    n = 12
    z, act, old, refl, _, adv = make((n,), V, dtype, V)
    low = torch.finfo(DTYPES[dtype]).min
    act[:] = V // 2
    for r, v in enumerate([low, float("-inf")] * (n // 2)):
        z[r, :V // 2] = v
        z[r, -1] = v
    z[4] = low                     # all at the lowest value: uniform
    z[5, torch.arange(V, device=cuda()) != V // 2] = float("-inf")  # one action left
    lp, ent = gear.action_logp(z, act)
    old = lp - 0.1
    say("policy with lowest values V=%d %s" % (V, dtype))
    check(z, act, old, lp + 0.05, None, adv)
    check(z, act, old, lp + 0.05, None, adv, entropy=5.0, scale=1024.0)
    assert abs(float(lp[4]) + np.log(V)) < 1e-5 * np.log(V) + 1e-6 and float(lp[5]) == 0 and float(ent[5]) == 0


@pytest.mark.parametrize("V", [4, 18, 700, 40000])
def test_rows_without_part_or_distribution(V):
    """Masked rows and actions out of range leave zeros whatever their logits hold; rows of -inf add nothing."""
    n = 10
    z, act, old, refl, _, adv = make((n,), V, "float32", 3)
    m = torch.ones(n, dtype=torch.uint8, device=cuda())
    m[2] = m[3] = 0
    z[2], z[3] = float("nan"), float("inf")
    old[2] = adv[3] = float("nan")
    act[4], act[5] = -100, V
    z[4], z[5] = float("nan"), float("nan")
    z[6] = float("-inf")
    say("policy with rows without part V=%d" % V)
    loss, logp, ent, stats, grad = gear.policy_loss(z, act, old, adv, ref_logp=refl, mask=m, kl=0.1, entropy=0.1)
    assert not bool(grad[2:7].any()) and not bool(logp[2:6].any()) and not bool(ent[2:7].any())
    assert float(logp[6]) == float("-inf") and np.isfinite(float(loss)) and bool(torch.isfinite(stats).all())
    keep = [0, 1, 7, 8, 9]
    few = gear.policy_loss(z[keep], act[keep], old[keep], adv[keep], ref_logp=refl[keep], kl=0.1, entropy=0.1, denom=6.0)
    assert torch.equal(few[4], grad[keep]) and torch.equal(few[1], logp[keep])
    np.testing.assert_allclose(float(few[0]), float(loss), rtol=1e-6)
    # Nothing takes part at all.
    out = gear.policy_loss(z, act, old, adv, mask=torch.zeros_like(m))
    assert float(out[0]) == 0 and not bool(out[3].any()) and not bool(out[4].any())


def test_an_action_that_cannot_be_taken():
    """Its log-probability is -inf, its ratio 0: no policy gradient, and no NaN."""
    z, act, old, _, _, adv = make((8,), 9, "float32", 3)
    z[torch.arange(8), act.long()] = float("-inf")
    loss, logp, ent, stats, grad = gear.policy_loss(z, act, old, adv)
    assert bool((logp == float("-inf")).all()) and np.isfinite(float(loss)) and not bool(grad.any())
    want = torch.where(adv < 0, -0.8 * adv, torch.zeros_like(adv)).double().mean()
    np.testing.assert_allclose(float(loss), float(want), rtol=1e-6)


def test_nan_and_infinity_show():
    """A NaN or +inf in a row that takes part is not hidden, and stays in its row's gradient."""
    for V in (6, 100, 5000):
        z, act, old, _, _, adv = make((4,), V, "float32", 3)
        act[:] = 1
        z[1, V - 1], z[2, 0] = float("nan"), float("inf")
        loss, logp, _, _, grad = gear.policy_loss(z, act, old, adv, denom=4.0)
        assert np.isnan(float(loss)) and bool(torch.isnan(grad[1]).all()) and not bool(torch.isfinite(logp[1:3]).all())
        assert bool(torch.isfinite(grad[[0, 3]]).all())


def test_no_rows():
    z = torch.zeros(0, 5, device=cuda())
    e = torch.zeros(0, device=cuda())
    loss, logp, ent, stats, grad = gear.policy_loss(z, e.int(), e, e)
    assert float(loss) == 0 and not bool(stats.any()) and grad.shape == (0, 5) and logp.shape == (0,)
    assert gear.action_logp(z, e.int())[0].shape == (0,)


def test_gradient_factors():
    z, act, old, refl, m, adv = make((30,), 40, "float32", 6, True)
    g1 = gear.policy_loss(z, act, old, adv, mask=m)[4]
    g2 = gear.policy_loss(z, act, old, adv, mask=m, grad_scale=8.0, grad_loss=torch.tensor(0.25, device=cuda()))[4]
    assert torch.equal(g2, 2 * g1)


def test_gradient_is_a_slope():
    """Central differences of the loss itself, along the gradient."""
    z, act, old, refl, m, adv = make((50,), 33, "float32", 12, True)
    kw = dict(ref_logp=refl, mask=m, kl=0.1, entropy=0.05, clip=(0.2, 0.3))
    g = gear.policy_loss(z, act, old, adv, **kw)[4].double()
    d = g / g.norm()
    # Rows are half a percent off the clip's edges and a step moves log ratios by less than 2e-3.  The loss is of
    # order 1 and correct to 1e-6, so its rounding leaves 1e-3 of the slope's unit at this step; the slope's own
    # third-order term is below 1e-6.
    step = 1e-3
    up = gear.policy_loss((z.double() + step * d).float(), act, old, adv, grad=False, **kw)[0].double()
    down = gear.policy_loss((z.double() - step * d).float(), act, old, adv, grad=False, **kw)[0].double()
    assert abs(float((up - down) / (2 * step)) - float(g.norm())) < 1e-3


def test_offsets_past_32_bits():
    big = torch.empty((1 << 32) + 64, dtype=torch.bfloat16, device=cuda())
    z = big.as_strided((3, 20), (1 << 31, 1))
    v, act, old, _, _, adv = make((3,), 20, "bfloat16", 2)
    z.copy_(v)
    say("policy rows 2^31 elements apart")
    a = gear.policy_loss(z, act, old, adv)
    b = gear.policy_loss(v, act, old, adv)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("lead,V", [((700, 3), 16), ((40,), 9001)])
def test_streams_and_graphs(lead, V):
    z, act, old, refl, m, adv = make(lead, V, "bfloat16", 2, True)

    def call(**kw):
        return gear.policy_loss(z, act, old, adv, ref_logp=refl, mask=m, kl=0.1, entropy=0.01, **kw)
    want = call()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = call(stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for _ in range(3):
        z.copy_(torch.randn(z.shape, device=cuda()))
        m.logical_not_()
        graph.replay()
        torch.cuda.synchronize()
        want = call()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals():
    z, act, old, refl, m, adv = make((4, 3), 5, "float32", 1, True)
    for args, kw, words in [
            ((z, act[:3], old, adv), {}, "action must have shape"), ((z, act.float(), old, adv), {}, "action must be"),
            ((z, act.t().contiguous().t(), old, adv), {}, "action must be contiguous"),
            ((z.double(), act, old, adv), {}, "float32"), ((z, act, old.half(), adv), {}, "old_logp must be float32"),
            ((z, act, None, adv), {}, "old_logp is missing"), ((z, act, old, None), {}, "adv is missing"),
            ((z, act, old, adv[:, :2].contiguous()), {}, "adv must have the first sizes"),
            ((z, act, old, adv, ), {"ref_logp": refl[0]}, "ref_logp must have shape"),
            ((z, act, old, adv), {"mask": m.int()}, "mask must be uint8"),
            ((z, act, old, adv), {"mask": m.cpu()}, "mask must be on"),
            ((z, act, old, adv), {"denom": 0.0}, "denom"),
            ((z, act, old, adv), {"grad_loss": torch.ones(2, device=cuda())}, "grad_loss"),
            ((torch.randn(4, 5, 3, device=cuda()).transpose(1, 2), act, old, adv), {}, "contiguous along"),
            ((torch.randn(3, 4, 5, device=cuda()).transpose(0, 1), act, old, adv), {}, "one stride"),
            ((torch.randn(4, 1, 5, device=cuda()).expand(4, 3, 5), act, old, adv), {}, "one stride"),
            ((torch.randn(1, 1, 5, device=cuda()).expand(4, 3, 5), act, old, adv), {}, "overlap")]:
        with pytest.raises(ValueError, match=words):
            gear.policy_loss(*args, **kw)
    for kw, words in [({"clip": (-0.1, 0.2)}, "clip"), ({"kl": float("nan")}, "coefficient"),
                      ({"grad_scale": float("inf")}, "coefficient"), ({"denom": float("inf")}, "denom")]:
        with pytest.raises(gear.GearError) as e:
            gear.policy_loss(z, act, old, adv, **kw)
        assert e.value.code == gear.GEAR_E_INVAL and words in str(e.value)
