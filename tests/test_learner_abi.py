"""Argument checks of the learner's entry points, without a device."""
import ctypes

import pytest

from paper_2310_05205_amd import gear

FAKE = 4096  # never dereferenced: every call here is refused or has nothing to do


def _rec(**kw):
    d = dict(dtype=gear.GEAR_DTYPE_BF16, form=gear.GEAR_GATE_VALUE, B=2, T=100, D=8)
    d.update(kw)
    return gear.gear_recurrence_desc(**d)


def _adv(**kw):
    lam = kw.pop("lam", 0.9)
    d = gear.gear_advantages_desc(**dict(dict(reward_dtype=gear.GEAR_DTYPE_F32, value_dtype=gear.GEAR_DTYPE_F32, B=2, L=9,
                                              gamma=0.9), **kw))
    setattr(d, "lambda", lam)
    return d


def _pol(**kw):
    return gear.gear_policy_desc(**dict(dict(dtype=gear.GEAR_DTYPE_F32, action_dtype=gear.GEAR_DTYPE_I32, n=4, V=3,
                                             row_stride=3, d_action=FAKE, mask_group=1, adv_group=1, weight_group=1,
                                             grad_scale=1.0), **kw))


def _sizes(f, d, k):
    out = [ctypes.c_int64(-1) for _ in range(k)]
    rc = f(ctypes.byref(d) if d is not None else None, *[ctypes.byref(o) for o in out])
    return rc, [o.value for o in out]


@pytest.mark.parametrize("d,words", [
    (None, "NULL"), (_rec(dtype=gear.GEAR_DTYPE_I32), "dtype"), (_rec(form=7), "form"), (_rec(B=-1), "negative"),
    (_rec(B=1 << 30, T=1 << 30, D=1), "range"), (_rec(B=1 << 41, T=0), "range"), (_rec(B=1 << 30, T=0, D=1 << 30), "range")])
def test_recurrence_descriptors(d, words):
    lib = gear.lib()
    p = ctypes.byref(d) if d is not None else None
    for rc in (_sizes(lib.gear_recurrence_sizes, d, 2)[0],
               lib.gear_recurrence(p, FAKE, FAKE, None, FAKE, None, None, FAKE, 1 << 30, None),
               lib.gear_recurrence_backward(p, FAKE, FAKE, None, FAKE, FAKE, None, FAKE, FAKE, None, FAKE, 1 << 30, None)):
        assert rc == gear.GEAR_E_INVAL and words in gear.gear_last_error()


def test_recurrence_arguments():
    lib = gear.lib()
    d = _rec()
    rc, (saved, work) = _sizes(lib.gear_recurrence_sizes, d, 2)
    assert rc == gear.GEAR_OK and saved == 6 * 2 * 8 * 4 and work > 0
    assert lib.gear_recurrence_sizes(ctypes.byref(d), None, None) == gear.GEAR_OK
    call = lib.gear_recurrence
    assert call(ctypes.byref(d), None, FAKE, None, FAKE, None, None, FAKE, work, None) == gear.GEAR_E_INVAL
    assert call(ctypes.byref(d), FAKE, FAKE, None, FAKE, None, None, FAKE, work - 1, None) == gear.GEAR_E_INVAL
    assert "workspace" in gear.gear_last_error()
    assert call(ctypes.byref(d), FAKE, FAKE, FAKE, FAKE, FAKE, None, FAKE, work, None) == gear.GEAR_E_INVAL
    assert "one step" in gear.gear_last_error()
    back = lib.gear_recurrence_backward
    assert back(ctypes.byref(d), FAKE, FAKE, None, None, FAKE, None, FAKE, FAKE, None, FAKE, work, None) == gear.GEAR_E_INVAL
    assert "saved" in gear.gear_last_error()
    assert back(ctypes.byref(d), FAKE, FAKE, None, FAKE, FAKE, None, FAKE, None, None, FAKE, work, None) == gear.GEAR_E_INVAL
    # One tile saves and needs nothing, and nothing is enqueued for no channels.
    assert _sizes(lib.gear_recurrence_sizes, _rec(T=16), 2) == (gear.GEAR_OK, [0, 0])
    assert call(ctypes.byref(_rec(D=0)), None, None, None, None, None, None, None, 0, None) == gear.GEAR_OK


@pytest.mark.parametrize("d,words", [
    (None, "NULL"), (_adv(reward_dtype=gear.GEAR_DTYPE_F64), "dtype"), (_adv(value_dtype=99), "dtype"), (_adv(L=-1), "range"),
    (_adv(B=1 << 30, L=1 << 30), "range"), (_adv(gamma=1.01), "[0, 1]"), (_adv(gamma=float("nan")), "[0, 1]"),
    (_adv(lam=-0.5), "[0, 1]")])
def test_advantage_descriptors(d, words):
    lib = gear.lib()
    p = ctypes.byref(d) if d is not None else None
    assert _sizes(lib.gear_advantages_sizes, d, 1)[0] == gear.GEAR_E_INVAL and words in gear.gear_last_error()
    assert lib.gear_advantages(p, FAKE, FAKE, FAKE, FAKE, FAKE, 1 << 30, None) == gear.GEAR_E_INVAL
    assert words in gear.gear_last_error()


def test_advantage_arguments():
    lib = gear.lib()
    d = _adv()
    assert lib.gear_advantages(ctypes.byref(d), None, FAKE, FAKE, FAKE, None, 0, None) == gear.GEAR_E_INVAL
    assert lib.gear_advantages(ctypes.byref(d), FAKE, FAKE, None, FAKE, None, 0, None) == gear.GEAR_E_INVAL
    long = _adv(L=1 << 20)
    rc, (work,) = _sizes(lib.gear_advantages_sizes, long, 1)
    assert rc == gear.GEAR_OK and work > 0
    assert lib.gear_advantages(ctypes.byref(long), FAKE, FAKE, FAKE, FAKE, FAKE, work - 1, None) == gear.GEAR_E_INVAL
    assert "workspace" in gear.gear_last_error()
    assert lib.gear_advantages(ctypes.byref(_adv(B=0)), None, None, None, None, None, 0, None) == gear.GEAR_OK


@pytest.mark.parametrize("d,words", [
    (None, "NULL"), (_pol(dtype=gear.GEAR_DTYPE_U8), "dtype"), (_pol(action_dtype=gear.GEAR_DTYPE_F32), "action"),
    (_pol(V=0), "range"), (_pol(V=1 << 31, row_stride=1 << 31), "range"), (_pol(n=-1), "range"), (_pol(n=1 << 40), "range"),
    (_pol(row_stride=2), "row_stride"), (_pol(mask_group=0), "group"), (_pol(adv_group=0), "group"),
    (_pol(weight_group=-3), "group")])
def test_policy_descriptors(d, words):
    lib = gear.lib()
    p = ctypes.byref(d) if d is not None else None
    assert _sizes(lib.gear_policy_sizes, d, 1)[0] == gear.GEAR_E_INVAL and words in gear.gear_last_error()
    assert lib.gear_action_logp(p, FAKE, FAKE, FAKE, None) == gear.GEAR_E_INVAL and words in gear.gear_last_error()
    assert lib.gear_policy_loss(p, FAKE, FAKE, None, FAKE, None, None, FAKE, None, None, None, None, FAKE, 1 << 30,
                                None) == gear.GEAR_E_INVAL
    assert words in gear.gear_last_error()


def test_policy_arguments():
    lib = gear.lib()
    d = _pol()
    rc, (work,) = _sizes(lib.gear_policy_sizes, d, 1)
    assert rc == gear.GEAR_OK and work > 0

    def call(d, logits=FAKE, old=FAKE, adv=FAKE, loss=FAKE, grad=None, w=FAKE, bytes=work):
        return lib.gear_policy_loss(ctypes.byref(d), logits, old, None, adv, None, None, loss, None, None, None, grad, w,
                                    bytes, None)
    for kw in ({"logits": None}, {"old": None}, {"adv": None}, {"loss": None}, {"w": None}, {"bytes": work - 1}):
        assert call(d, **kw) == gear.GEAR_E_INVAL, kw
    assert call(_pol(d_action=None)) == gear.GEAR_E_INVAL
    assert call(_pol(row_stride=4), grad=FAKE) == gear.GEAR_E_INVAL and "logits' place" in gear.gear_last_error()
    for kw in ({"clip_low": -0.1}, {"clip_high": float("nan")}, {"denom": -1.0}, {"denom": float("inf")},
               {"kl": float("inf")}, {"entropy": float("nan")}, {"grad_scale": float("inf")}):
        assert call(_pol(**kw)) == gear.GEAR_E_INVAL, kw
    assert lib.gear_action_logp(ctypes.byref(_pol(d_action=None)), FAKE, FAKE, FAKE, None) == gear.GEAR_E_INVAL
    assert lib.gear_action_logp(ctypes.byref(_pol(n=0)), None, None, None, None) == gear.GEAR_OK
