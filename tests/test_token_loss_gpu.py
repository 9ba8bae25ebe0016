"""The loss of a token head and its gradients against their formulas in 64 bits (GPU)."""
import pytest
import torch

from paper_2310_05205_amd import gear, learn
from tests.helpers import cuda, say
from tests.network_reference import Token, near

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def inputs(n, D, V, dtype, seed=1):
    g = torch.Generator().manual_seed(seed)
    head = torch.randn(V, D, generator=g) * 2 / D ** 0.5
    t = torch.randint(0, V, (n,), generator=g)
    h = torch.randn(n, D, generator=g) + torch.rand(n, 1, generator=g) * head[t]
    return h.to(dtype), head.to(dtype), t, 0.2 + torch.rand(n, generator=g)


def check(hidden, head, target, on=None, weight=None, denom=None, scale=1.0, what=""):
    """Inputs on the GPU, of any layout; on and weight a value per row."""
    say("token_loss %s" % what)
    n, D = target.numel(), hidden.shape[-1]
    cpu = lambda t: None if t is None else t.detach().cpu()  # noqa: E731
    want = Token(cpu(hidden).reshape(n, D), cpu(head), cpu(target).reshape(n), cpu(on), cpu(weight), denom)
    mask = None if on is None else on.reshape(target.shape)
    w = None if weight is None else weight.reshape(target.shape)
    loss, logp, lse = gear.token_loss(hidden, head, target, weight=w, mask=mask, denom=denom)
    assert logp.shape == lse.shape == target.shape
    near(logp.reshape(n), want.logp, want.logp_off, "logp")
    near(lse.reshape(n), torch.where(want.on, want.lse, 0.0), want.lse_off, "lse")
    near(loss, want.loss, want.loss_off, "loss")
    want.gradients(scale)
    dh, dW = gear.token_loss_backward(hidden, head, target, lse, weight=w, mask=mask, denom=denom, grad_scale=scale)
    assert dh.shape == hidden.shape and dW.shape == head.shape and dh.dtype == dW.dtype == hidden.dtype
    near(dh.reshape(n, D), want.dh, want.dh_bound, "dhidden")
    near(dW, want.dW, want.dW_bound, "dhead")
    one, none = gear.token_loss_backward(hidden, head, target, lse, weight=w, mask=mask, denom=denom, grad_scale=scale, dhead=False)
    assert none is None and torch.equal(one, dh)
    none, one = gear.token_loss_backward(hidden, head, target, lse, weight=w, mask=mask, denom=denom, grad_scale=scale, dhidden=False)
    assert none is None and torch.equal(one, dW)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,V", [(1, 1, 1), (1, 1, 2), (2, 3, 5), (320, 64, 18), (17, 64, 128), (16, 128, 129),
                                   (129, 65, 127), (128, 63, 256), (5, 200, 1000), (300, 192, 300), (257, 320, 513),
                                   (1, 512, 4097), (64, 100, 777), (33, 1003, 2001), (700, 8, 4)])
def test_sizes(dtype, n, D, V):
    h, W, t, w = (x.to(cuda()) for x in inputs(n, D, V, dtype))
    g = torch.Generator().manual_seed(7)
    on = (torch.rand(n, generator=g) < 0.8).to(cuda())
    # 1/64 of a step of fp16 and more stays representable with this scale.
    check(h, W, t, on, w, scale=1024.0, what="%d x %d x %d %s, masked" % (n, D, V, dtype))
    check(h, W, t.int(), scale=64.0 * n, what="%d x %d x %d %s" % (n, D, V, dtype))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,V", [(300, 72, 11000), (520, 520, 30001), (5000, 70, 40), (9000, 200, 3), (3000, 300, 700)])
def test_sizes_of_other_tiles(dtype, n, D, V):
    """Middle and big tiles in each product, rows split for small heads."""
    h, W, t, w = (x.to(cuda()) for x in inputs(n, D, V, dtype))
    on = (torch.rand(n, generator=torch.Generator().manual_seed(7)) < 0.8).to(cuda())
    check(h, W, t, on, w, scale=16.0 * n, what="%d x %d x %d %s" % (n, D, V, dtype))


@pytest.mark.parametrize("dtype", TYPES)
def test_several_pieces_of_the_vocabulary(dtype):
    """Tokens beyond one piece, forward and backward."""
    h, W, t, w = (x.to(cuda()) for x in inputs(40, 24, 140001, dtype))
    check(h, W, t, None, w, scale=512.0, what="140001 tokens %s" % dtype)


def test_pieces_of_many_rows():
    h, W, t, w = (x.to(cuda()) for x in inputs(40000, 8, 4000, torch.bfloat16))
    check(h, W, t, None, w, what="40000 rows of 4000 tokens")


@pytest.mark.parametrize("dtype", TYPES)
def test_layouts(dtype):
    """Rows that begin anywhere and lie apart, leading dimensions, targets of every type."""
    h, W, t, w = (x.to(cuda()) for x in inputs(24, 64, 100, dtype))
    wide = torch.zeros(24, 131, dtype=dtype, device=cuda())
    tall = torch.zeros(100, 90, dtype=dtype, device=cuda())
    wide[:, 1:65], tall[:, 3:67] = h, W
    check(wide[:, 1:65], tall[:, 3:67], t, None, w, scale=64.0, what="slices %s" % dtype)
    wide = torch.zeros(24, 128, dtype=dtype, device=cuda())
    wide[:, 64:] = h
    check(wide[:, 64:], W, t.to(torch.uint8), None, w, scale=64.0, what="a half %s" % dtype)
    check(h.reshape(2, 3, 4, 64), W, t.reshape(2, 3, 4), (w < 1).flatten(), w, scale=64.0, what="leading dimensions %s" % dtype)
    check(h[0], W, t[0], scale=64.0, what="one row of one dimension %s" % dtype)


def test_shared_weights_and_masks():
    """Values of the first dimensions serve every row below them."""
    h, W, t, _ = (x.to(cuda()) for x in inputs(24, 64, 100, torch.float32))
    h, t = h.reshape(4, 6, 64), t.reshape(4, 6)
    w, on = torch.rand(4, device=cuda()) + 0.5, torch.tensor([True, False, True, True], device=cuda())
    say("token_loss shared")
    a = gear.token_loss(h, W, t, weight=w, mask=on)
    b = gear.token_loss(h, W, t, weight=w[:, None].expand(4, 6).contiguous(), mask=on[:, None].expand(4, 6).contiguous())
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    da = gear.token_loss_backward(h, W, t, a[2], weight=w, mask=on)
    db = gear.token_loss_backward(h, W, t, a[2], weight=w[:, None].expand(4, 6).contiguous(),
                                  mask=on[:, None].expand(4, 6).contiguous())
    assert all(torch.equal(x, y) for x, y in zip(da, db))


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_that_take_no_part(dtype):
    """NaN and infinities in them reach nothing; targets out of range; no row at all."""
    h, W, t, w = inputs(200, 96, 300, dtype)
    on = torch.rand(200, generator=torch.Generator().manual_seed(2)) < 0.7
    h[~on] = float("nan")
    h[(~on).nonzero()[:5, 0]] = float("inf")
    w[~on] = float("nan")
    t[~on] = -100
    check(h.to(cuda()), W.to(cuda()), t.to(cuda()), None, w.to(cuda()), scale=64.0, what="targets out of range %s" % dtype)
    t[~on] = 5
    check(h.to(cuda()), W.to(cuda()), t.to(cuda()), on.to(cuda()), w.to(cuda()), denom=77.0, scale=64.0, what="masked %s" % dtype)
    none = torch.zeros(200, dtype=torch.bool, device=cuda())
    say("token_loss no row takes part %s" % dtype)
    loss, logp, lse = gear.token_loss(h.to(cuda()), W.to(cuda()), t.to(cuda()), mask=none)
    dh, dW = gear.token_loss_backward(h.to(cuda()), W.to(cuda()), t.to(cuda()), lse, mask=none)
    assert float(loss) == 0 and not logp.any() and not lse.any() and not dh.any() and not dW.any()


@pytest.mark.parametrize("dtype", TYPES)
def test_no_rows(dtype):
    h, W = torch.empty(0, 8, dtype=dtype, device=cuda()), torch.ones(5, 8, dtype=dtype, device=cuda())
    t = torch.empty(0, dtype=torch.int64, device=cuda())
    loss, logp, lse = gear.token_loss(h, W, t)
    dh, dW = gear.token_loss_backward(h, W, t, lse)
    assert float(loss) == 0 and logp.shape == (0,) and dh.shape == (0, 8) and not dW.any()


@pytest.mark.parametrize("dtype", TYPES)
def test_weights_of_every_kind(dtype):
    """Zero, negative, and of sizes far apart: small ones count where they are alone."""
    h, W, t, w = inputs(150, 64, 90, dtype)
    w[:50] = 0.0
    w[50:100] *= -1
    w[100:] *= 1e-3
    check(h.to(cuda()), W.to(cuda()), t.to(cuda()), None, w.to(cuda()), denom=1.0, scale=16.0, what="weights %s" % dtype)
    check(h.to(cuda()), W.to(cuda()), t.to(cuda()), None, (w * 1e-20).to(cuda()), denom=1e-20, scale=16.0, what="tiny weights %s" % dtype)


def test_large_logits():
    """Distances beyond fp32's exponential; a certain row's log-probability is 0."""
    h, W, t, w = inputs(60, 64, 200, torch.float32)
    check((100 * h).to(cuda()), W.to(cuda()), t.to(cuda()), None, w.to(cuda()), what="logits of hundreds")
    big = 1e30 * torch.eye(8, 16)
    say("token_loss certain rows")
    loss, logp, lse = gear.token_loss(big.to(cuda()), torch.eye(20, 16).to(cuda()), torch.arange(8).to(cuda()))
    assert float(loss) == 0 and not logp.any()


@pytest.mark.parametrize("dtype", TYPES)
def test_logits_far_from_zero(dtype):
    """All logits of a row are 2^21 + a small integer, exact in 32 bits: log-probabilities depend on the small part alone."""
    n, V = 70, 300
    g = torch.Generator().manual_seed(3)
    h = torch.tensor([2048.0, 1.0]).expand(n, 2).contiguous()
    W = torch.stack([torch.full((V,), 1024.0), torch.randint(-9, 10, (V,), generator=g).float()], 1)
    t = torch.randint(0, V, (n,), generator=g)
    say("token_loss logits of 2^21 %s" % dtype)
    loss, logp, lse = gear.token_loss(h.to(dtype).to(cuda()), W.to(dtype).to(cuda()), t.to(cuda()))
    want = W.double()[t, 1] - torch.logsumexp(W.double()[:, 1], 0)
    # Distances are whole numbers up to 18.  An exponential takes one rounding of distance times log2 e, at most 26 * 2^-24 / 2
    # in the power and ln 2 of that in the value, and two units of its own: 11 * 2^-24.  A sum of 300 positive terms in tiles adds at
    # most 16 roundings in a row per level and three levels: 48 * 2^-24.  A logarithm below 8 adds 2 units of 2^-21 at most,
    # 16 * 2^-24; the difference below 32 one of 2^-20, 16 * 2^-24.
    near(logp, want, torch.full_like(want, 91 * 2.0 ** -24), "logp")
    # lse's last digit is 2^-2.
    near(lse, 2.0 ** 21 + torch.logsumexp(W.double()[:, 1], 0).expand(n), torch.full((n,), 2.0 ** -2, dtype=torch.float64), "lse")


@pytest.mark.parametrize("dtype", TYPES)
def test_certain_rows_of_every_type(dtype):
    """The largest logits of the type, up to 1.5 * 2^127, are certain: 0, and no other value."""
    far = 2.0 ** 15 if dtype == torch.float16 else 2.0 ** 63
    h, W = torch.zeros(40, 8), torch.zeros(90, 8)
    h[:, 0] = 2.0 ** torch.linspace(0, 15 if dtype == torch.float16 else 64, 40).round()
    W[33, 0] = 1.5 * far
    say("token_loss certain rows %s" % dtype)
    t = torch.full((40,), 33)
    args = [x.to(cuda()) for x in (h.to(dtype), W.to(dtype), t)]
    loss, logp, lse = gear.token_loss(*args)
    assert float(loss) == 0 and not logp.any()
    assert torch.equal(lse.cpu(), h[:, 0] * 1.5 * far)
    dh, dW = gear.token_loss_backward(*args, lse)
    assert not dh.any() and not dW.any()


@pytest.mark.parametrize("hidden,head", [(1e30, 1e-30), (1e-30, 1e30), (1e-36, 1e34), (3e38, 1e-38), (0.0, 1.0), (1.0, 0.0), (1e-42, 1.0)])
def test_32_bit_values_of_any_size(hidden, head):
    """Ends of the range, zeros, subnormal values; rows that take no part are far larger."""
    h, W, t, w = inputs(150, 64, 200, torch.float32)
    h, W = h / h.abs().max() * hidden, W / W.abs().max() * head
    on = torch.rand(150, generator=torch.Generator().manual_seed(2)) < 0.7
    h[~on] = 1e38 if hidden < 1e37 else float("inf")
    check(h.to(cuda()), W.to(cuda()), t.to(cuda()), on.to(cuda()), w.to(cuda()), what="values of %g and %g" % (hidden, head))


def test_32_bit_rows_stand_for_themselves():
    """A row far larger than the others, or of infinities, changes none of them."""
    h, W, t, w = inputs(150, 100, 200, torch.float32)
    args = [x.to(cuda()) for x in (W, t)]
    say("token_loss rows of their own")
    _, logp, lse = gear.token_loss(h.to(cuda()), *args)
    for odd in (1e30, float("inf"), float("nan")):
        h[7] = odd
        _, other, other_lse = gear.token_loss(h.to(cuda()), *args)
        keep = torch.arange(150) != 7
        assert torch.equal(other.cpu()[keep], logp.cpu()[keep]) and torch.equal(other_lse.cpu()[keep], lse.cpu()[keep])


def test_32_bit_rows_of_different_sizes():
    """Rows and columns that differ by a thousand, the head's the other way round: every logit counts."""
    h, W, t, w = inputs(150, 64, 200, torch.float32)
    by = 10.0 ** torch.linspace(-3, 3, 64)
    check((h * by).to(cuda()), (W / by).to(cuda()), t.to(cuda()), None, w.to(cuda()), what="columns of different sizes")
    check((h * 10.0 ** torch.linspace(-6, 0, 150)[:, None]).to(cuda()), W.to(cuda()), t.to(cuda()), None, w.to(cuda()), what="rows of different sizes")


@pytest.mark.parametrize("dtype", TYPES)
def test_nan_and_infinity_show(dtype):
    h, W, t, w = inputs(40, 64, 130, dtype)
    h[3, 7] = float("nan")
    say("token_loss NaN %s" % dtype)
    loss, logp, lse = gear.token_loss(h.to(cuda()), W.to(cuda()), t.to(cuda()))
    bad = torch.isnan(logp.cpu())
    assert torch.isnan(loss) and bad[3] and int(bad.sum()) == 1 and torch.isnan(lse[3])
    dh, dW = gear.token_loss_backward(h.to(cuda()), W.to(cuda()), t.to(cuda()), lse)
    assert torch.isnan(dh[3]).all() and torch.isfinite(dh[:3]).all() and torch.isnan(dW).all()
    h[3, 7] = float("inf")
    loss, logp, lse = gear.token_loss(h.to(cuda()), W.to(cuda()), t.to(cuda()))
    assert not torch.isfinite(logp[3]) and torch.isfinite(logp[:3]).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [20, 320, 2000, 20000])
def test_nan_weights_show(dtype, n):
    """One NaN weight on a row that takes part, among zeros and among others, and NaN weights alone: the formula's NaN in
    the loss, in the row's dhidden and in all of dhead.  On a row that takes no part it reaches nothing."""
    h, W, t, w = (x.to(cuda()) for x in inputs(n, 24, 30, dtype))
    nan = float("nan")
    for at in (0, n // 2, n - 1):
        for rest in (0.0, -2.0, nan):
            weight = torch.full((n,), rest, device=cuda())
            weight[at] = nan
            say("token_loss NaN weight at %d of %d beside %s, %s" % (at, n, rest, dtype))
            loss, logp, lse = gear.token_loss(h, W, t, weight=weight)
            dh, dW = gear.token_loss_backward(h, W, t, lse, weight=weight)
            assert torch.isnan(loss) and torch.isfinite(logp).all()
            assert torch.equal(torch.isnan(dh).all(1), torch.isnan(weight)) and torch.equal(torch.isnan(dh).any(1), torch.isnan(weight))
            assert torch.isnan(dW).all()
    on = torch.ones(n, dtype=torch.bool, device=cuda())
    on[n // 2] = False
    w[n // 2] = nan
    loss, logp, lse = gear.token_loss(h, W, t, weight=w, mask=on)
    dh, dW = gear.token_loss_backward(h, W, t, lse, weight=w, mask=on)
    assert torch.isfinite(loss) and torch.isfinite(dh).all() and torch.isfinite(dW).all() and not dh[n // 2].any()


def test_gradient_scales_and_repeats():
    h, W, t, w = (x.to(cuda()) for x in inputs(300, 100, 500, torch.bfloat16))
    say("token_loss repeats")
    loss, logp, lse = gear.token_loss(h, W, t, weight=w)
    first = gear.token_loss_backward(h, W, t, lse, weight=w, grad_scale=4.0)
    for _ in range(3):
        assert torch.equal(loss, gear.token_loss(h, W, t, weight=w)[0])
        assert all(torch.equal(a, b) for a, b in zip(first, gear.token_loss_backward(h, W, t, lse, weight=w, grad_scale=4.0)))
    by = torch.tensor(2.0, device=cuda())
    assert all(torch.equal(a, b) for a, b in zip(first, gear.token_loss_backward(h, W, t, lse, weight=w, grad_scale=2.0, grad_loss=by)))


def test_gradients_by_differences():
    """learn.token_loss against differences of the 64-bit definition along random directions."""
    h, W, t, w = inputs(20, 33, 70, torch.float32)
    hg, Wg = h.to(cuda()).requires_grad_(), W.to(cuda()).requires_grad_()
    say("learn.token_loss")
    loss, logp, lse = learn.token_loss(hg, Wg, t.to(cuda()), weight=w.to(cuda()))
    assert not logp.requires_grad and not lse.requires_grad
    (3 * loss).backward()
    f = lambda a, b: 3 * Token(a, b, t, None, w.double()).loss  # noqa: E731
    g = torch.Generator().manual_seed(4)
    for k, (x, grad) in enumerate(((h, hg.grad), (W, Wg.grad))):
        way = torch.randn(x.shape, generator=g, dtype=torch.float64)
        ends = [(x.double() + s * way, W.double()) if k == 0 else (h.double(), x.double() + s * way) for s in (1e-5, -1e-5)]
        # Token's bounds need a type; its values are those of the doubles.
        slope = (f(*(e.double() for e in ends[0])) - f(*(e.double() for e in ends[1]))) / 2e-5
        got = (grad.cpu().double() * way).sum()
        size = float((grad.cpu().double().abs() * way.abs()).sum())
        assert abs(float(slope - got)) < 1e-4 * abs(float(slope)) + 1e-5 * size


def test_only_what_needs_a_gradient():
    h, W, t, _ = (x.to(cuda()) for x in inputs(20, 64, 70, torch.float32))
    W.requires_grad_()
    learn.token_loss(h, W, t)[0].backward()
    assert W.grad is not None and h.grad is None


def test_captured_calls_replay():
    h, W, t, w = (x.to(cuda()) for x in inputs(150, 72, 700, torch.bfloat16))

    def run():
        loss, logp, lse = gear.token_loss(h, W, t, weight=w)
        return (loss, logp, lse) + gear.token_loss_backward(h, W, t, lse, weight=w)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = run()
    for seed in (11, 12, 13):
        h2, W2, t2, w2 = inputs(150, 72, 700, torch.bfloat16, seed)
        h.copy_(h2), W.copy_(W2), t.copy_(t2), w.copy_(w2)
        want = run()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), seed


def test_two_streams_at_once():
    """Calls in flight together have workspaces of their own."""
    sets = [tuple(x.to(cuda()) for x in inputs(500, 128, 3000, torch.bfloat16, s)) for s in (1, 2)]
    want = [gear.token_loss(h, W, t, weight=w) for h, W, t, w in sets]
    want = [o + gear.token_loss_backward(h, W, t, o[2], weight=w) for o, (h, W, t, w) in zip(want, sets)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    say("token_loss on two streams")
    for _ in range(3):
        got = []
        for s, (h, W, t, w) in zip(streams, sets):
            o = gear.token_loss(h, W, t, weight=w, stream=s)
            got.append(o + gear.token_loss_backward(h, W, t, o[2], weight=w, stream=s))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_refusals():
    h, W, t, w = (x.to(cuda()) for x in inputs(6, 8, 10, torch.float32))
    bad = [((h, W.half(), t), {}), ((h, W[:, :7], t), {}), ((h, W.t(), t), {}), ((h.t(), W, t), {}), ((h, W, t[:5]), {}),
           ((h, W, t.float()), {}), ((h, W, t), {"weight": w[:3]}), ((h, W, t), {"weight": w.half()}),
           ((h, W, t), {"mask": w}), ((h, W, t), {"denom": 0.0}), ((h[:1].expand(6, 8), W, t), {}),
           ((h, W[:0], t), {}), ((h.cpu(), W, t), {}), ((h, W.cpu(), t), {}), ((h.double(), W.double(), t), {})]
    for args, kw in bad:
        with pytest.raises((ValueError, TypeError)):
            gear.token_loss(*args, **kw)
    lse = gear.token_loss(h, W, t)[2]
    for args, kw in [((h, W, t, None), {}), ((h, W, t, lse[:3]), {}), ((h, W, t, lse.double()), {}),
                     ((h, W, t, lse), {"grad_loss": w})]:
        with pytest.raises((ValueError, TypeError)):
            gear.token_loss_backward(*args, **kw)
    with pytest.raises(gear.GearError):
        gear.token_loss_backward(h, W, t, lse, grad_scale=float("nan"))
