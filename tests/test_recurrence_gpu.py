"""The gated recurrence against its definition in 64 bits: lengths from none to
many tiles and segments, odd widths, strides, resets, ragged windows, states
that are not finite, streams and graphs (GPU)."""
import numpy as np
import pytest
import torch

from paper_2310_05205_amd import gear
from tests import learner_reference as ref
from tests.helpers import cuda, host, say

pytestmark = pytest.mark.gpu

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}


def wide(t):
    return None if t is None else host(t.double() if t.is_floating_point() else t)


def make(B, T, D, dtype, seed, sigmoid, packed=False, reset=0.0, ragged=False):
    g = torch.Generator().manual_seed(seed)
    gate = 2 + 1.5 * torch.randn(B, T, D, generator=g)
    if not sigmoid:
        gate = torch.sigmoid(gate) * torch.where(torch.rand(B, T, D, generator=g) < 0.2, -1.0, 1.0)
    x, dy = torch.randn(2, B, T, D, generator=g)
    state, dfinal = torch.randn(2, B, D, generator=g).to(cuda())
    dt = DTYPES[dtype]
    if packed:
        p = torch.cat([gate, x], dim=2).to(dt).to(cuda())
        gate, x = p[..., :D], p[..., D:]
    else:
        gate, x = gate.to(dt).to(cuda()), x.to(dt).to(cuda())
    r = (torch.rand(B, T, generator=g) < reset).to(torch.uint8).to(cuda()) if reset else None
    n = torch.randint(-1, T + 2, (B,), generator=g, dtype=torch.int32).to(cuda()) if ragged else None
    return gate, x, dy.to(dt).to(cuda()), state, dfinal, r, n


def check(gate, x, dy, state, dfinal, r, n, dtype, sigmoid):
    form = gear.GEAR_GATE_SIGMOID if sigmoid else gear.GEAR_GATE_VALUE
    B, T, D = x.shape
    y, final, saved = gear.recurrence(gate, x, state, form=form, reset=r, lengths=n, save=True)
    assert y.dtype == x.dtype and final.dtype == torch.float32 and y.is_contiguous()
    dgate, dx, dstate = gear.recurrence_backward(gate, x, saved, dy, dfinal, state, form=form, reset=r, lengths=n)
    args = [wide(gate), wide(x), wide(state)]
    kw = dict(sigmoid=sigmoid, reset=wide(r), lengths=wide(n))
    (wy, ey), (wf, ef), _, _ = ref.recurrence(*args, **kw)
    ref.within(wide(y), wy, ey, dtype)
    ref.within(wide(final), wf, ef)
    (wg, eg), (wx, ex), (ws, es) = ref.recurrence_backward(*args, wide(dy), wide(dfinal), **kw)
    ref.within(wide(dx), wx, ex, dtype)
    ref.within(wide(dgate), wg, eg, dtype)
    ref.within(wide(dstate), ws, es)
    y2, final2, none = gear.recurrence(gate, x, state, form=form, reset=r, lengths=n)
    assert none is None and torch.equal(y2, y) and torch.equal(final2, final)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("B,T,D,packed,reset,ragged", [
    (1, 1, 1, False, 0, False), (3, 0, 5, False, 0, False), (0, 4, 5, False, 0, False), (2, 5, 0, False, 0, False),
    (2, 15, 3, False, 0.3, False), (2, 16, 2, False, 0, True), (2, 17, 4, True, 0.1, False),
    (5, 33, 7, True, 0.1, True), (3, 48, 64, False, 0.05, True), (1, 100, 257, False, 0, False),
    (700, 20, 130, False, 0.05, False), (1, 3001, 6, False, 0.01, False), (2, 1111, 65, True, 0, True),
    (1, 777, 1, False, 0.02, False)])
def test_against_definition(B, T, D, packed, reset, ragged, dtype, sigmoid):
    say("recurrence B=%d T=%d D=%d %s sigmoid=%s packed=%s reset=%s ragged=%s" % (B, T, D, dtype, sigmoid, packed, reset,
                                                                                  ragged))
    check(*make(B, T, D, dtype, 7 * B + T + D, sigmoid, packed, reset, ragged), dtype, sigmoid)


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("B,T,D", [(2, 80, 9), (2, 81, 9), (3, 96, 66), (3, 97, 66), (270, 97, 256), (505, 83, 260)])
def test_around_the_split(B, T, D, dtype):
    """Windows just too short and just long enough for segments, and calls of nearly too many and too many channels."""
    say("recurrence around the split B=%d T=%d D=%d %s" % (B, T, D, dtype))
    check(*make(B, T, D, dtype, B + T, True, True, 0.05, True), dtype, True)


@pytest.mark.parametrize("T", [5, 40, 2000])
def test_without_states_and_gradients(T):
    gate, x, dy, _, _, r, n = make(2, T, 9, "float32", 3, True, reset=0.1)
    say("recurrence without states T=%d" % T)
    check(gate, x, dy, None, None, r, n, "float32", True)
    _, _, saved = gear.recurrence(gate, x, form=gear.GEAR_GATE_SIGMOID, reset=r, save=True)
    dgate, dx, dstate = gear.recurrence_backward(gate, x, saved, None, form=gear.GEAR_GATE_SIGMOID, reset=r)
    assert not bool(dgate.any()) and not bool(dx.any()) and not bool(dstate.any())


@pytest.mark.parametrize("T", [3, 40, 3000])
def test_resets_cut_infinities_and_nan(T):
    """A state or gradient that is not finite ends at a reset, whole tiles and segments away included."""
    gate, x, dy, state, dfinal, _, _ = make(3, T, 5, "float32", 11, False)
    r = torch.zeros(3, T, dtype=torch.bool, device=cuda())
    r[0, 0] = r[1, T // 2] = True
    state[0, 0], state[1, 1], state[2, 2] = float("inf"), float("nan"), float("-inf")
    dfinal[1, 1], dfinal[0, 0] = float("nan"), float("inf")
    say("recurrence with infinities T=%d" % T)
    y, final, saved = gear.recurrence(gate, x, state, reset=r, save=True)
    assert bool(torch.isfinite(y[0]).all()) and bool(torch.isfinite(final[:2]).all())
    assert bool(torch.isfinite(y[1, T // 2:]).all()) and bool(torch.isnan(y[1, :T // 2, 1]).all())
    assert not bool(torch.isfinite(y[2, :, 2]).any()) and bool(torch.isfinite(y[2, :, [0, 1, 3, 4]]).all())
    dgate, dx, dstate = gear.recurrence_backward(gate, x, saved, dy, dfinal, state, reset=r)
    assert bool((dstate[0] == 0).all()) and bool(torch.isfinite(dstate[1]).all())
    assert bool(torch.isfinite(dx[1, :T // 2]).all()) and bool(torch.isnan(dx[1, T // 2:, 1]).all())


def test_extreme_gates():
    g = torch.tensor([-1e30, -200.0, -90.0, -30.0, 0.0, 30.0, 90.0, 200.0, 1e30, float("inf"), float("-inf")])
    gate = g.view(1, 1, -1).expand(2, 3, -1).contiguous().to(cuda())
    x = torch.full((2, 3, 11), 3.0, device=cuda())
    state = torch.full((2, 11), 5.0, device=cuda())
    y, final, saved = gear.recurrence(gate, x, state, form=gear.GEAR_GATE_SIGMOID, save=True)
    f = 1 / (1 + np.exp(-np.clip(g.numpy().astype(np.float64), -700, 700)))
    np.testing.assert_allclose(host(y)[0, 0], f * 5 + (1 - f) * 3, rtol=1e-6)
    dgate, dx, dstate = gear.recurrence_backward(gate, x, saved, torch.ones_like(x), None, state,
                                                 form=gear.GEAR_GATE_SIGMOID)
    assert bool(torch.isfinite(dgate).all()) and bool(torch.isfinite(dx).all()) and bool(torch.isfinite(dstate).all())
    assert bool((dgate[:, :, [0, 8, 9, 10]] == 0).all())


def test_padding_is_not_read():
    """Steps past a window's length hold NaN and resets; nothing of them comes through."""
    gate, x, dy, state, dfinal, _, _ = make(4, 37, 6, "bfloat16", 5, True)
    n = torch.tensor([0, 5, 32, 37], dtype=torch.int32, device=cuda())
    r = torch.zeros(4, 37, dtype=torch.uint8, device=cuda())
    for b, k in enumerate(n.tolist()):
        for t in (gate, x, dy):
            t[b, k:] = float("nan")
        r[b, k:] = 255
    say("recurrence with NaN past the lengths")
    check_args = [wide(torch.nan_to_num(t)) for t in (gate, x)]
    y, final, saved = gear.recurrence(gate, x, state, form=gear.GEAR_GATE_SIGMOID, reset=r, lengths=n, save=True)
    (wy, ey), (wf, ef), _, _ = ref.recurrence(*check_args, wide(state), True, None, wide(n))
    ref.within(wide(y), wy, ey, "bfloat16")
    ref.within(wide(final), wf, ef)
    assert torch.equal(final[0], state[0])
    grads = gear.recurrence_backward(gate, x, saved, dy, dfinal, state, form=gear.GEAR_GATE_SIGMOID, reset=r, lengths=n)
    want = ref.recurrence_backward(*check_args, wide(state), wide(torch.nan_to_num(dy)), wide(dfinal), True, None, wide(n))
    for got, (w, e), dt in zip(grads, want, ("bfloat16", "bfloat16", "float32")):
        ref.within(wide(got), w, e, dt)


def test_strides():
    """Transposed time and batch, windows that share one gate, every second step, views at odd offsets."""
    base = torch.randn(12, 4, 30, device=cuda())
    x = base.transpose(0, 1)[:, ::2, 3:24]                       # [4, 6, 21]
    gate = torch.rand(1, 6, 21, device=cuda()).expand(4, 6, 21)  # stride 0
    dy = torch.randn(4 * 6 * 21 + 1, device=cuda())[1:].view(4, 6, 21)
    r = (torch.rand(4, 40, device=cuda()) < 0.3)[:, 5:11]
    state, dfinal = torch.randn(2, 4, 21, device=cuda())
    check(gate, x, dy, state, dfinal, r, None, "float32", False)
    check(gate.half(), x.half().as_strided((4, 6, 21), (126, 21, 1)), dy.half(), state, dfinal, r, None, "float16", True)


@pytest.mark.parametrize("sigmoid", [False, True])
@pytest.mark.parametrize("B,D", [(1, 1), (5, 3), (7, 64), (300, 129), (2, 1024)])
@pytest.mark.parametrize("dtype", list(DTYPES))
def test_steps_equal_the_window(B, D, dtype, sigmoid):
    """An actor's steps, states in place or not, are the window's, bit for bit."""
    form = gear.GEAR_GATE_SIGMOID if sigmoid else gear.GEAR_GATE_VALUE
    gate, x, _, state, _, r, _ = make(B, 6, D, dtype, B + D, sigmoid, reset=0.2)
    say("recurrence steps B=%d D=%d %s" % (B, D, dtype))
    y, final, _ = gear.recurrence(gate, x, state, form=form, reset=r)
    kept, inplace = state, state.clone()
    for t in range(6):
        yt, kept = gear.recurrence_step(gate[:, t], x[:, t], kept, form=form, reset=r[:, t])
        y2, back = gear.recurrence_step(gate[:, t], x[:, t], inplace, form=form, reset=r[:, t], out=inplace)
        assert back.data_ptr() == inplace.data_ptr()
        assert torch.equal(yt, y[:, t]) and torch.equal(y2, yt) and torch.equal(inplace, kept)
    assert torch.equal(kept, final)


def test_offsets_past_32_bits():
    """A window whose strides pass 2^31 elements, read in place."""
    big = torch.empty((1 << 31) + 100, dtype=torch.bfloat16, device=cuda())
    x = big.as_strided((2, 2, 40), (1 << 30, 1 << 30, 1))
    v = torch.randn(2, 40, device=cuda()).bfloat16()
    x[0, 0], x[1, 1] = v[0], v[1]
    x[0, 1] = v[0]  # the same memory as x[1, 0]
    say("recurrence with strides of 2^30 elements")
    gate = torch.full((2, 2, 40), 0.5, device=cuda()).bfloat16()
    y, final, saved = gear.recurrence(gate, x, save=True)
    assert torch.equal(final[1], 0.5 * v[0].float() + v[1].float())
    dgate, dx, _ = gear.recurrence_backward(gate, x, saved, torch.ones_like(gate))
    assert bool((dx[:, 0] == 1.5).all()) and torch.equal(dgate[1, 1], v[0])


def test_on_another_stream():
    gate, x, dy, state, dfinal, r, _ = make(3, 2000, 33, "float32", 2, True, reset=0.01)
    want = gear.recurrence(gate, x, state, form=gear.GEAR_GATE_SIGMOID, reset=r, save=True)
    wb = gear.recurrence_backward(gate, x, want[2], dy, dfinal, state, form=gear.GEAR_GATE_SIGMOID, reset=r)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for _ in range(3):
        got = gear.recurrence(gate, x, state, form=gear.GEAR_GATE_SIGMOID, reset=r, save=True, stream=s)
        gb = gear.recurrence_backward(gate, x, got[2], dy, dfinal, state, form=gear.GEAR_GATE_SIGMOID, reset=r, stream=s)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got + gb, want + wb))


def test_captured_calls_replay():
    gate, x, dy, state, dfinal, r, _ = make(3, 1500, 33, "bfloat16", 2, True, reset=0.01)
    form = gear.GEAR_GATE_SIGMOID

    def both():
        y, f, s = gear.recurrence(gate, x, state, form=form, reset=r, save=True)
        return (y, f) + gear.recurrence_backward(gate, x, s, dy, dfinal, state, form=form, reset=r)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        both()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    for k in range(3):
        x.copy_(torch.randn(x.shape, device=cuda()))
        state.fill_(float(k))
        graph.replay()
        torch.cuda.synchronize()
        want = both()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_refusals():
    x = torch.randn(2, 3, 4, device=cuda())
    for args, kw, words in [
            ((x[:, :2], x), {}, "shape"), ((x.half(), x), {}, "dtype"), ((x.double(), x.double()), {}, "float32"),
            ((x.cpu(), x), {}, "must be on"), ((x, x.transpose(1, 2)), {}, "shape"),
            ((x.transpose(0, 2).contiguous().transpose(0, 2),) * 2, {}, "contiguous along"),
            ((x, x, x[0]), {}, "state"), ((x, x, x[:, 0].half()), {}, "state must be float32"),
            ((x, x), {"reset": torch.zeros(2, 3, device=cuda())}, "reset must be uint8"),
            ((x, x), {"reset": torch.zeros(2, 4, dtype=torch.bool, device=cuda())}, "reset must have shape"),
            ((x, x), {"lengths": torch.zeros(2, dtype=torch.int64, device=cuda())}, "lengths must be int32"),
            ((x, x), {"lengths": torch.zeros(3, dtype=torch.int32, device=cuda())}, "lengths must have shape")]:
        with pytest.raises(ValueError, match=words):
            gear.recurrence(*args, **kw)
    with pytest.raises(gear.GearError) as e:
        gear.recurrence(x, x, form=2)
    assert e.value.code == gear.GEAR_E_INVAL and "form" in str(e.value)
    with pytest.raises(ValueError, match="GPU"):
        gear.recurrence(x.cpu(), x.cpu())
    with pytest.raises(ValueError, match="saved"):
        gear.recurrence_backward(x, x, None, x)
    with pytest.raises(ValueError, match="saved must have shape"):
        gear.recurrence_backward(x, x, torch.zeros(5, device=cuda()), x)
    state = torch.zeros(9, device=cuda())
    with pytest.raises(ValueError, match="overlap"):
        gear.recurrence_step(x[:, 0], x[:, 0], state[:8].view(2, 4), out=state[1:].view(2, 4))
