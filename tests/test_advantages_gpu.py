"""Advantages and returns against their definition in 64 bits: lengths from
none to several segments, types, strides, ended episodes and ragged windows (GPU)."""
import pytest
import torch

from paper_2310_05205_amd import gear
from tests import learner_reference as ref
from tests.helpers import cuda, host, say

pytestmark = pytest.mark.gpu

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def wide(t):
    return None if t is None else host(t.double() if t.is_floating_point() else t)


def make(B, L, rt, vt, seed, done, ragged):
    g = torch.Generator().manual_seed(seed)
    r = torch.randn(B, L, generator=g).to(DTYPES[rt]).to(cuda())
    v = (3 * torch.randn(B, L + 1, generator=g)).to(DTYPES[vt]).to(cuda())
    d = (torch.rand(B, L, generator=g) < done).to(cuda()) if done else None
    n = torch.randint(-1, L + 2, (B,), generator=g, dtype=torch.int32).to(cuda()) if ragged else None
    return r, v, d, n


def check(r, v, gamma, lam, d, n):
    adv, ret = gear.advantages(r, v, gamma, lam, done=d, lengths=n)
    assert adv.dtype == ret.dtype == torch.float32 and adv.shape == r.shape
    (wa, ea), (wr, er) = ref.advantages(wide(r), wide(v), gamma, lam, wide(d), wide(n))
    ref.within(wide(adv), wa, ea)
    ref.within(wide(ret), wr, er)


@pytest.mark.parametrize("rt,vt", [("float32", "float32"), ("float32", "bfloat16"), ("float16", "float32"),
                                   ("bfloat16", "float16")])
@pytest.mark.parametrize("B,L,done,ragged", [
    (1, 1, 0, False), (3, 0, 0, False), (0, 5, 0, False), (2, 3, 0.5, False), (5, 4, 0, True), (70, 5, 0.2, True),
    (9, 8, 0, False), (33, 9, 0.1, True), (100, 17, 0.1, False), (7, 63, 0.05, True), (3, 128, 0, False),
    (4, 255, 0.02, True), (2, 256, 0.01, False), (2, 257, 0.01, True), (300, 32, 0.03, False), (1, 5000, 0.001, False),
    (3, 20011, 0.0005, True), (2, 70001, 0, False)])
def test_against_definition(B, L, done, ragged, rt, vt):
    say("advantages B=%d L=%d %s %s done=%s ragged=%s" % (B, L, rt, vt, done, ragged))
    check(*make(B, L, rt, vt, B + L, done, ragged)[:2], 0.99, 0.95, *make(B, L, rt, vt, B + L, done, ragged)[2:])


@pytest.mark.parametrize("B,L", [(2, 513), (2, 2560), (2, 2561), (1023, 2600), (1024, 2600), (1030, 600)])
def test_around_the_split(B, L):
    """Windows just too short and just long enough for segments, and calls of nearly too many and too many windows."""
    r, v, d, n = make(B, L, "bfloat16", "float32", B + L, 0.01, True)
    say("advantages around the split B=%d L=%d" % (B, L))
    check(r, v, 0.99, 0.95, d, n)


@pytest.mark.parametrize("gamma,lam", [(0.0, 0.95), (1.0, 0.0), (1.0, 1.0), (0.5, 1.0)])
def test_limits_of_the_discounts(gamma, lam):
    r, v, d, n = make(4, 900, "float32", "float32", 1, 0.01, True)
    say("advantages gamma=%s lambda=%s" % (gamma, lam))
    check(r, v, gamma, lam, d, n)


@pytest.mark.parametrize("L", [7, 300, 30000])
def test_ended_episodes_and_padding_pass_nothing_on(L):
    """NaN after a step that ended its episode, and past a window's length, stays there."""
    r, v, _, _ = make(3, L, "float32", "float32", 2, 0, False)
    d = torch.zeros(3, L, dtype=torch.uint8, device=cuda())
    n = torch.tensor([L, L, L // 2], dtype=torch.int32, device=cuda())
    d[0, L // 2] = 7
    r[0, L // 2 + 1:] = float("nan")
    v[0, L // 2 + 1:] = float("inf")
    r[2, L // 2:] = float("nan")
    v[2, L // 2 + 1:] = float("nan")
    say("advantages with NaN after the end, L=%d" % L)
    adv, ret = gear.advantages(r, v, 0.99, 0.95, done=d, lengths=n)
    assert bool(torch.isfinite(adv[0, :L // 2 + 1]).all()) and bool(torch.isnan(adv[0, L // 2 + 1:]).all())
    assert bool(torch.isfinite(adv[1:]).all()) and bool(torch.isfinite(ret[1:]).all())
    assert not bool(adv[2, L // 2:].any()) and not bool(ret[2, L // 2:].any())
    r2, v2 = torch.nan_to_num(r, 0, 0, 0), torch.nan_to_num(v, 0, 0, 0)
    again, _ = gear.advantages(r2, v2, 0.99, 0.95, done=d, lengths=n)
    assert torch.equal(again[0, :L // 2 + 1], adv[0, :L // 2 + 1]) and torch.equal(again[1:], adv[1:])


def test_strides():
    big = torch.randn(5, 200, device=cuda())
    value = torch.randn(5, 150, device=cuda()).bfloat16()
    done = torch.rand(5, 99, device=cuda()) < 0.05
    check(big[:, 3:80], value[:, 1:79], 0.97, 0.9, done[:, 7:84], None)
    check(big[0, :77].expand(5, 77), value[0, :78].expand(5, 78), 0.97, 0.9, done[:, :77], None)


def test_on_another_stream_and_captured():
    r, v, d, _ = make(3, 50000, "float32", "float32", 2, 0.001, False)
    want = gear.advantages(r, v, 0.99, 0.95, done=d)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = gear.advantages(r, v, 0.99, 0.95, done=d, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = gear.advantages(r, v, 0.99, 0.95, done=d)
    for k in range(3):
        r.copy_(torch.randn(r.shape, device=cuda()))
        graph.replay()
        torch.cuda.synchronize()
        want = gear.advantages(r, v, 0.99, 0.95, done=d)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals():
    r, v = torch.randn(2, 5, device=cuda()), torch.randn(2, 6, device=cuda())
    for args, kw, words in [
            ((r, r), {}, "value must have shape"), ((r.double(), v), {}, "float32"), ((r.t(), v), {}, "value must"),
            ((r, v.cpu()), {}, "must be on"), ((r[0], v), {}, "reward must have shape"),
            ((torch.randn(5, 2, device=cuda()).t(), v), {}, "contiguous along"),
            ((r, v), {"done": torch.zeros(2, 5, dtype=torch.int32, device=cuda())}, "done must be uint8"),
            ((r, v), {"done": torch.zeros(2, 6, dtype=torch.bool, device=cuda())}, "done must have shape"),
            ((r, v), {"lengths": torch.zeros(5, dtype=torch.int32, device=cuda())}, "lengths must have shape")]:
        with pytest.raises(ValueError, match=words):
            gear.advantages(*args, 0.99, 0.95, **kw)
    for gamma, lam in ((1.5, 0.9), (0.9, -0.1), (float("nan"), 0.9)):
        with pytest.raises(gear.GearError) as e:
            gear.advantages(r, v, gamma, lam)
        assert e.value.code == gear.GEAR_E_INVAL and "[0, 1]" in str(e.value)
