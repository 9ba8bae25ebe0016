"""Argument checks of layer norm, the token head's loss and the optimizer's step, without a device."""
import ctypes

import pytest
import torch

from paper_2310_05205_amd import gear, learn

FAKE = 4096  # never dereferenced: every call here is refused or has nothing to do


def _norm(**kw):
    return gear.gear_norm_desc(**dict(dict(dtype=gear.GEAR_DTYPE_BF16, param_dtype=gear.GEAR_DTYPE_F32, n=3, D=8, x_row=8,
                                           residual_row=8, dy_row=8, dtotal_row=8, eps=1e-5), **kw))


def _token(**kw):
    return gear.gear_token_desc(**dict(dict(dtype=gear.GEAR_DTYPE_BF16, target_dtype=gear.GEAR_DTYPE_I32, n=4, D=8, V=9,
                                            hidden_row=8, head_row=8, d_target=FAKE, mask_group=1, weight_group=1,
                                            grad_scale=1.0), **kw))


def _tensor(**kw):
    return gear.gear_step_tensor(**dict(dict(dtype=gear.GEAR_DTYPE_BF16, n=5, d_grad=FAKE, d_param=FAKE, d_exp_avg=FAKE,
                                             d_exp_avg_sq=FAKE), **kw))


def _adamw(**kw):
    return gear.gear_adamw_desc(**dict(dict(state_bits=32, lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1), **kw))


def _ref(d):
    return ctypes.byref(d) if d is not None else None


def _sizes(f, d, k):
    out = [ctypes.c_int64(-1) for _ in range(k)]
    return f(_ref(d), *[ctypes.byref(o) for o in out]), [o.value for o in out]


@pytest.mark.parametrize("d,words", [
    (None, "NULL"), (_norm(dtype=gear.GEAR_DTYPE_I32), "dtype"), (_norm(param_dtype=gear.GEAR_DTYPE_F16), "param_dtype"),
    (_norm(n=-1), "range"), (_norm(D=0), "range"), (_norm(D=(1 << 20) + 1), "range"), (_norm(n=1 << 40), "range"),
    (_norm(x_row=-1), "stride"), (_norm(residual_row=-1), "stride"), (_norm(dy_row=-8), "stride"), (_norm(dtotal_row=-8), "stride"),
    (_norm(eps=-1e-9), "eps"), (_norm(eps=float("nan")), "eps"), (_norm(eps=float("inf")), "eps")])
def test_norm_descriptors(d, words):
    lib = gear.lib()
    for rc in (_sizes(lib.gear_layer_norm_sizes, d, 1)[0],
               lib.gear_layer_norm(_ref(d), FAKE, None, FAKE, FAKE, FAKE, None, None, None),
               lib.gear_layer_norm_backward(_ref(d), FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE, FAKE, 1 << 40, None)):
        assert rc == gear.GEAR_E_INVAL and words in gear.gear_last_error()


def test_norm_arguments():
    lib = gear.lib()
    d = _norm()
    rc, (work,) = _sizes(lib.gear_layer_norm_sizes, d, 1)
    assert rc == gear.GEAR_OK and work > 0
    assert lib.gear_layer_norm_sizes(ctypes.byref(d), None) == gear.GEAR_OK
    for args in ((None, None, FAKE, None), (FAKE, None, None, None), (FAKE, None, FAKE, FAKE)):
        x, res, y, total = args
        assert lib.gear_layer_norm(ctypes.byref(d), x, res, None, None, y, total, None, None) == gear.GEAR_E_INVAL
    back = lib.gear_layer_norm_backward
    for t, saved, dy in ((None, FAKE, FAKE), (FAKE, None, FAKE), (FAKE, FAKE, None)):
        assert back(ctypes.byref(d), t, saved, None, dy, None, FAKE, FAKE, FAKE, FAKE, work, None) == gear.GEAR_E_INVAL
    for w, n in ((None, work), (FAKE, work - 1)):
        assert back(ctypes.byref(d), FAKE, FAKE, None, FAKE, None, FAKE, FAKE, None, w, n, None) == gear.GEAR_E_INVAL
        assert "workspace" in gear.gear_last_error()
    none = _norm(n=0)
    assert lib.gear_layer_norm(ctypes.byref(none), None, None, None, None, None, None, None, None) == gear.GEAR_OK
    assert back(ctypes.byref(none), None, None, None, None, None, None, None, None, None, 0, None) == gear.GEAR_OK


@pytest.mark.parametrize("d,words", [
    (None, "NULL"), (_token(dtype=gear.GEAR_DTYPE_F64), "dtype"), (_token(target_dtype=gear.GEAR_DTYPE_F32), "target"),
    (_token(n=-1), "range"), (_token(n=gear.GEAR_TOKEN_MAX + 1), "range"), (_token(V=0), "range"),
    (_token(V=gear.GEAR_TOKEN_MAX + 1), "range"), (_token(n=1 << 24, V=1 << 13), "range"), (_token(D=0), "range"),
    (_token(D=65537, hidden_row=65537, head_row=65537), "range"), (_token(hidden_row=7), "stride"), (_token(head_row=7), "stride"),
    (_token(mask_group=0), "group"), (_token(weight_group=-1), "group"), (_token(denom=-1.0), "denom"),
    (_token(denom=float("inf")), "denom"), (_token(denom=float("nan")), "denom"), (_token(grad_scale=float("inf")), "grad_scale")])
def test_token_descriptors(d, words):
    lib = gear.lib()
    for rc in (_sizes(lib.gear_token_loss_sizes, d, 2)[0],
               lib.gear_token_loss(_ref(d), FAKE, FAKE, FAKE, None, None, FAKE, 1 << 50, None),
               lib.gear_token_loss_backward(_ref(d), FAKE, FAKE, FAKE, None, FAKE, FAKE, FAKE, 1 << 50, None)):
        assert rc == gear.GEAR_E_INVAL and words in gear.gear_last_error()


def test_token_arguments():
    lib = gear.lib()
    d = _token()
    rc, (loss, back) = _sizes(lib.gear_token_loss_sizes, d, 2)
    assert rc == gear.GEAR_OK and loss > 0 and back > 0
    assert lib.gear_token_loss_sizes(ctypes.byref(d), None, None) == gear.GEAR_OK
    for h, W, out, w, n in ((None, FAKE, FAKE, FAKE, loss), (FAKE, None, FAKE, FAKE, loss), (FAKE, FAKE, None, FAKE, loss),
                            (FAKE, FAKE, FAKE, None, loss), (FAKE, FAKE, FAKE, FAKE, loss - 1), (FAKE, FAKE, FAKE, FAKE + 8, loss)):
        assert lib.gear_token_loss(ctypes.byref(d), h, W, out, None, None, w, n, None) == gear.GEAR_E_INVAL
    for h, W, lse, w, n in ((None, FAKE, FAKE, FAKE, back), (FAKE, None, FAKE, FAKE, back), (FAKE, FAKE, None, FAKE, back),
                            (FAKE, FAKE, FAKE, None, back), (FAKE, FAKE, FAKE, FAKE, back - 1), (FAKE, FAKE, FAKE, FAKE + 4, back)):
        assert lib.gear_token_loss_backward(ctypes.byref(d), h, W, lse, None, FAKE, FAKE, w, n, None) == gear.GEAR_E_INVAL
    bare = _token(d_target=None)
    assert lib.gear_token_loss(ctypes.byref(bare), FAKE, FAKE, FAKE, None, None, FAKE, loss, None) == gear.GEAR_E_INVAL
    # Nothing to compute: nothing is enqueued.
    assert lib.gear_token_loss_backward(ctypes.byref(d), FAKE, FAKE, FAKE, None, None, None, FAKE, back, None) == gear.GEAR_OK


@pytest.mark.parametrize("n,D,V", [(1, 1, 1), (1 << 24, 64, 4096), (8192, 4096, 131072), (1, 65536, 1 << 24), (0, 5, 7)])
def test_token_workspaces_of_every_size(n, D, V):
    """Sizes at the ends of the range have workspaces that a GPU holds."""
    for dtype in (gear.GEAR_DTYPE_F32, gear.GEAR_DTYPE_BF16):
        rc, (loss, back) = _sizes(gear.lib().gear_token_loss_sizes, _token(dtype=dtype, n=n, D=D, V=V, hidden_row=D, head_row=D), 2)
        assert rc == gear.GEAR_OK and 0 < loss < 250 << 30 and 0 < back < 250 << 30


def test_step_arguments():
    lib = gear.lib()
    norm, adam = ctypes.c_int64(), ctypes.c_int64()
    assert lib.gear_step_sizes(ctypes.byref(norm), ctypes.byref(adam)) == gear.GEAR_OK and lib.gear_step_sizes(None, None) == gear.GEAR_OK

    def grad_norm(t=_tensor(), count=1, scale=1.0, limit=1.0, out=FAKE, factor=FAKE, work=FAKE, n=norm.value):
        return lib.gear_grad_norm(_ref(t), count, scale, limit, out, factor, work, n, None)
    for kw in ({"t": None}, {"count": -1}, {"t": _tensor(dtype=gear.GEAR_DTYPE_F64)}, {"t": _tensor(n=-1)}, {"t": _tensor(n=(1 << 40) + 1)},
               {"t": _tensor(d_grad=None)}, {"scale": 0.0}, {"scale": float("nan")}, {"scale": float("inf")}, {"limit": 0.0},
               {"limit": float("nan")}, {"out": None}, {"factor": None}, {"work": None}, {"n": norm.value - 1}):
        assert grad_norm(**kw) == gear.GEAR_E_INVAL, kw

    def adamw(d=_adamw(), t=_tensor(), count=1, step=FAKE, work=FAKE, n=adam.value):
        return lib.gear_adamw(_ref(d), _ref(t), count, step, work, n, None)
    for kw in ({"d": None}, {"t": None}, {"count": -2}, {"step": None}, {"work": None}, {"n": adam.value - 1},
               {"t": _tensor(dtype=gear.GEAR_DTYPE_I32)}, {"t": _tensor(d_param=None)}, {"t": _tensor(d_grad=None)},
               {"t": _tensor(d_exp_avg=None)}, {"t": _tensor(d_exp_avg_sq=None)}, {"d": _adamw(state_bits=8)}, {"d": _adamw(state_bits=16)},
               {"t": _tensor(dtype=gear.GEAR_DTYPE_F32, d_master=FAKE)}, {"d": _adamw(lr=-0.1)}, {"d": _adamw(lr=float("nan"))},
               {"d": _adamw(beta1=1.0)}, {"d": _adamw(beta2=-0.5)}, {"d": _adamw(beta2=float("nan"))}, {"d": _adamw(eps=0.0)},
               {"d": _adamw(eps=1e-60)}, {"d": _adamw(weight_decay=float("inf"))}):
        assert adamw(**kw) == gear.GEAR_E_INVAL, kw


def test_tensors_have_to_be_on_the_gpu():
    x, t = torch.ones(2, 3), torch.zeros(2, dtype=torch.int64)
    for call in (lambda: gear.layer_norm(x), lambda: gear.layer_norm_backward(x, x, torch.ones(2, 2)), lambda: gear.token_loss(x, x, t),
                 lambda: gear.token_loss_backward(x, x, t, torch.ones(2)), lambda: gear.grad_norm([x]), lambda: gear.grad_norm([]),
                 lambda: gear.adamw([x], [x], [x], [x], torch.zeros(1, dtype=torch.int64), lr=0.1)):
        with pytest.raises(ValueError):
            call()


def test_optimizers_take_lists():
    """A tensor alone would be taken for its rows, which never have a gradient."""
    with pytest.raises(TypeError):
        learn.AdamW(torch.nn.Parameter(torch.ones(3, 4)))
