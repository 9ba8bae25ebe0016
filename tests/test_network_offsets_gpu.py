"""The network's operators on tensors whose offsets pass 32 bits: what lies at both ends (GPU)."""
import pytest
import torch

from paper_2310_05205_amd import gear
from tests.helpers import cuda, say
from tests.network_reference import Norm, STEP, Token, U, U32, d64, near

pytestmark = pytest.mark.gpu
D = 1024
ROWS = (1 << 22) + 5  # of D values: 2^32 and more
ENDS = 100


@pytest.fixture(autouse=True)
def give_back():
    """Tens of GB, for the tests that allocate by themselves."""
    yield
    torch.cuda.empty_cache()


def ends(t):
    return torch.cat([t[:ENDS], t[-ENDS:]])


def with_ends(seed, dtype=torch.bfloat16):
    """Zeros but for the first and the last rows, and those."""
    t = torch.zeros(ROWS, D, dtype=dtype, device=cuda())
    part = torch.randn(2 * ENDS, D, generator=torch.Generator().manual_seed(seed)).to(dtype)
    t[:ENDS], t[-ENDS:] = part[:ENDS].to(cuda()), part[ENDS:].to(cuda())
    return t, part


@pytest.mark.parametrize("part", [0, 7])
def test_layer_norm(part):
    """Rows of D - part values at a stride of D: whole lines, and not."""
    say("layer_norm of %d rows of %d" % (ROWS, D - part))
    (x, a), (dy, b) = with_ends(1), with_ends(2)
    x, a, dy, b = (t[:, :D - part] for t in (x, a, dy, b))
    dy = dy.contiguous()
    weight, bias = (1 + 0.1 * torch.randn(D - part, generator=torch.Generator().manual_seed(s)) for s in (3, 4))
    y, _, saved = gear.layer_norm(x, weight.to(cuda()), bias.to(cuda()), save=True)
    want = Norm(a, weight, bias, 1e-5, None)
    near(ends(y), want.y, want.y_bound, "y")
    dx, dw, db = gear.layer_norm_backward(dy, x, saved, weight.to(cuda()))
    want.backward(b, None, torch.float32)
    near(ends(dx), want.dx, want.dx_bound, "dx")
    # The other rows add exact zeros.
    near(dw, want.dw, want.dw_bound, "dweight")
    near(db, want.db, want.db_bound, "dbias")
    assert not dx[ENDS:-ENDS].any()


def test_token_loss_of_many_rows():
    say("token_loss of %d rows" % ROWS)
    h, part = with_ends(1)
    W = (torch.randn(5, D, generator=torch.Generator().manual_seed(2)) / 16).to(torch.bfloat16)
    on = torch.zeros(ROWS, dtype=torch.bool, device=cuda())
    on[:ENDS] = on[-ENDS:] = True
    t = (torch.arange(ROWS, device=cuda()) % 5).int()
    want = Token(part, W, ends(t).cpu())
    loss, logp, lse = gear.token_loss(h, W.to(cuda()), t, mask=on)
    near(ends(logp), want.logp, want.logp_off, "logp")
    near(loss, want.loss, want.loss_off, "loss")
    want.gradients(100.0)
    dh, dW = gear.token_loss_backward(h, W.to(cuda()), t, lse, mask=on, grad_scale=100.0)
    near(ends(dh), want.dh, want.dh_bound, "dhidden")
    near(dW, want.dW, want.dW_bound, "dhead")
    assert not dh[ENDS:-ENDS].any() and not logp[ENDS:-ENDS].any()


def test_token_loss_of_many_tokens():
    """A head with zeros between its ends: those tokens' logits are 0."""
    say("token_loss of %d tokens" % ROWS)
    W, part = with_ends(1)
    W, part = W.div_(16), part / 16
    h = torch.randn(7, D, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16)
    t = torch.tensor([0, 1, ENDS - 1, ROWS - 1, ROWS - ENDS, ROWS - 2, 5])
    at = torch.where(t < ENDS, t, t - ROWS + 2 * ENDS)
    z = d64(h) @ d64(part).t()
    lse = torch.logsumexp(torch.cat([z, torch.full((7, 1), float(ROWS - 2 * ENDS)).double().log()], 1), 1)
    logp = z.gather(1, at[:, None])[:, 0] - lse
    # Exact products added 32 at a time; exponentials of up to |z|, their sums, a logarithm below 2^5.
    z_off = (U32 * (8 + D / 16) * (d64(h).abs() @ d64(part).abs().t())).amax(1)
    lse_off = 2 * z_off + U32 * (16 + 2 * z.abs().amax(1)) + U32 * lse.abs()
    args = [x.to(cuda()) for x in (h, )] + [W, t.to(cuda())]
    loss, got, got_lse = gear.token_loss(*args)
    near(got_lse, lse, lse_off, "lse")
    near(got, logp, z_off + lse_off + 2 * U32 * logp.abs(), "logp")
    dh, dW = gear.token_loss_backward(*args, got_lse, grad_scale=7.0)
    e = torch.exp(z - lse[:, None])
    e_off = e * (z_off + lse_off + 8 * U32)[:, None]
    e[torch.arange(7), at] -= 1.0
    e_off = e_off + (U[torch.bfloat16] * 1.01 + 8 * U32) * e.abs() + 2.0 ** -38
    # The tokens between add exact zeros to dh.
    off = e_off @ d64(part).abs() + U32 * (64 + 2 * ENDS / 16) * (e.abs() @ d64(part).abs())
    want = e @ d64(part)
    near(dh, want, U[torch.bfloat16] * want.abs() + 1.01 * off + STEP[torch.bfloat16], "dhidden")
    want = e.t() @ d64(h)
    off = (e_off + 2.0 ** -38).t() @ d64(h).abs() + U32 * 65 * (e.abs().t() @ d64(h).abs())
    near(ends(dW), want, U[torch.bfloat16] * want.abs() + 1.01 * off + STEP[torch.bfloat16], "dhead")


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(bits):
    n, tail = (1 << 32) + 1003, (1 << 32) - 4096
    say("adamw of %d values, %d bits" % (n, bits))
    kind = torch.float32 if bits == 32 else torch.uint8
    p, g = (torch.ones(n, dtype=torch.bfloat16, device=cuda()) for _ in range(2))
    m, v = (torch.zeros(n, dtype=kind, device=cuda()) for _ in range(2))
    s = [torch.zeros((n + 255) // 256, device=cuda()) for _ in range(2)] if bits == 8 else []
    g[tail:] = torch.randn(n - tail, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).to(cuda())
    apart = [x[tail:].clone() for x in (p, g, m, v)] + [x[tail // 256:].clone() for x in s]
    form = lambda x: x.view(torch.float8_e4m3fn) if x.dtype == torch.uint8 else x  # noqa: E731
    call = lambda p, g, m, v, *s: gear.adamw([p], [g], [form(m)], [form(v)], torch.zeros(1, dtype=torch.int64, device=cuda()),  # noqa: E731
                                             lr=0.125, weight_decay=0.0, scales=([s[0]], [s[1]]) if s else None)
    norm, _ = gear.grad_norm([g])
    want = float(tail + d64(g[tail:]).square().sum()) ** 0.5
    assert abs(float(norm) - want) <= 2 * U32 * want
    call(p, g, m, v, *s)
    call(*apart)
    for x, y in zip([x[tail:] for x in (p, g, m, v)] + [x[tail // 256:] for x in s], apart):
        assert torch.equal(x.view(torch.uint8), y.view(torch.uint8))
    assert (p[:tail] == 0.875).all()
