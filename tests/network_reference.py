"""Layer norm, a token head's loss and AdamW from their definitions in float64 on
the CPU, and the error bounds that their tests hold the kernels to.

U is half a step of a type, relative to a value: a rounding is off by that much at
most.  Kernels compute in 32 bits, so a bound is the rounding of the output and a
number of 32-bit roundings of the terms that enter it."""
import torch

U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
U32 = 2.0 ** -24
# The least step of a type: what is below its normal range is rounded to multiples of it.
STEP = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def d64(t):
    return None if t is None else t.detach().cpu().double()


def near(got, want, bound, what):
    """Every element within its bound; equal where both are infinite or NaN."""
    got = d64(got)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), what + ": NaN"
    assert torch.equal(got[odd & ~torch.isnan(want)], want[odd & ~torch.isnan(want)]), what + ": infinities"
    off = (got - want).abs()[~odd]
    lim = bound.expand_as(want)[~odd] if torch.is_tensor(bound) else torch.full_like(off, bound)
    bad = off > lim
    assert not bad.any(), "%s: off by %g where %g is allowed" % (what, off[bad][0], lim[bad][0])


# --- layer norm -----------------------------------------------------------------

class Norm:
    """One call and its bounds.  x, residual, dy, dtotal [n, D] on the CPU in their own types."""

    def __init__(self, x, weight, bias, eps, residual=None):
        self.x_dtype = x.dtype
        t = d64(x)
        if residual is not None:
            t = d64((x.float() + residual.float()).to(x.dtype))
        n, D = t.shape
        self.t = t
        self.w = torch.ones(D, dtype=torch.float64) if weight is None else d64(weight)
        b = torch.zeros(D, dtype=torch.float64) if bias is None else d64(bias)
        self.mean = t.mean(1, keepdim=True)
        c = t - self.mean
        self.rstd = 1 / torch.sqrt(c.square().mean(1, keepdim=True) + eps)
        self.u = c * self.rstd
        self.y = self.u * self.w + b
        # A 32-bit sum of D values is off by its depth in roundings of the mean magnitude: lanes add up to D / 256
        # values in turn, then 8 levels; the sums around the mean correct that again, which leaves the subtraction's
        # own rounding, of the values' size, and a few of u's.
        self.units = 16 + D / 64
        self.u_off = U32 * (8 * t.abs().amax(1, keepdim=True) * self.rstd + self.units * self.u.abs())
        self.y_bound = U[x.dtype] * self.y.abs() + 2 * (self.u_off * self.w.abs() + 4 * U32 * b.abs()) + STEP[x.dtype]

    def backward(self, dy, dtotal, w_dtype):
        dy = d64(dy)
        n, D = dy.shape
        g = dy * self.w
        a, k = g.mean(1, keepdim=True), (g * self.u).mean(1, keepdim=True)
        self.dx = (g - a - self.u * k) * self.rstd
        size = (g.abs() + g.abs().mean(1, keepdim=True) + self.u.abs() * (g * self.u).abs().mean(1, keepdim=True)) * self.rstd
        off = U32 * self.units * size + self.rstd * (self.u_off * k.abs() + self.u.abs() * (g.abs() * self.u_off).mean(1, keepdim=True))
        if dtotal is not None:
            self.dx = self.dx + d64(dtotal)
            off = off + 2 * U32 * d64(dtotal).abs()
        self.dx_bound = U[self.x_dtype] * self.dx.abs() + 2 * off + STEP[self.x_dtype]
        self.dw, self.db = (dy * self.u).sum(0), dy.sum(0)
        # Sums over rows: in turn over a slice of them, then over slices.
        units = 32 + n / 256
        dw_off = U32 * units * (dy * self.u).abs().sum(0) + (dy.abs() * self.u_off).sum(0)
        self.dw_bound = U[w_dtype] * self.dw.abs() + 2 * dw_off + STEP[w_dtype]
        self.db_bound = U[w_dtype] * self.db.abs() + U32 * units * dy.abs().sum(0) + STEP[w_dtype]


# --- the loss of a token head ---------------------------------------------------

class Token:
    """One call and its bounds: hidden [n, D], head [V, D], target [n], on [n] bool, weight [n] or None."""

    def __init__(self, hidden, head, target, on=None, weight=None, denom=None):
        self.dtype = hidden.dtype
        n, V = hidden.shape[0], head.shape[0]
        t = target.long()
        on = torch.ones(n, dtype=torch.bool) if on is None else on.bool()
        self.on = on & (t >= 0) & (t < V)
        # Rows that take no part hold anything.
        self.h = torch.where(self.on[:, None], d64(hidden), 0.0)
        self.W = d64(head)
        self.t = torch.where(self.on, t, 0)
        w = torch.ones(n, dtype=torch.float64) if weight is None else d64(weight)
        self.w = torch.where(self.on, w, 0.0)
        self.denom = float(denom) if denom is not None else max(1.0, float(self.on.sum()))
        z = self.h @ self.W.t()
        self.lse = torch.logsumexp(z, 1)
        lp = z.gather(1, self.t[:, None])[:, 0] - self.lse
        D = self.h.shape[1]
        # A logit: products added 32 at a time in 32 bits.  Those of 16-bit values are exact.  32-bit values enter as two
        # fp16 parts: the first is off by 2^-11 of the value at most, the second by 2^-11 of that, 2^-22 in all, or by
        # 2^-25 of the unit that the row's largest value has 2^14 of, 2^-39 of that value; the product of the second
        # parts, left out, is 2^-22 at most.  Three times 2^-22 are 12 units of 2^-24.
        size = self.h.abs() @ self.W.abs().t()
        self.z_off = (U32 * (8 + D / 16) * size).amax(1)
        self.parts_off = 0.0
        if self.dtype == torch.float32 and n:
            self.parts_off = 12 * U32
            h, W = self.h.abs(), self.W.abs()
            low = 2.0 ** -39 * (h.amax(1)[:, None] * W.sum(1) + W.amax(1) * h.sum(1)[:, None])
            self.z_off = self.z_off + (12 * U32 * size + low).amax(1)
        # Exponentials of rounded products of up to |z|, a logarithm, and sums over the vocabulary, all positive.
        self.lse_off = 2 * self.z_off + U32 * (16 + 2 * z.abs().amax(1)) + U32 * self.lse.abs()
        self.logp = torch.where(self.on, lp, 0.0)
        self.logp_off = self.z_off + self.lse_off + 2 * U32 * lp.abs()
        self.loss = -(self.w * self.logp).sum() / self.denom
        self.loss_off = (self.w.abs() * (self.logp_off + 2 * U32 * self.logp.abs())).sum() / self.denom + 4 * U32 * self.loss.abs()
        self.p = torch.exp(z - self.lse[:, None])

    def gradients(self, scale):
        dt = self.dtype
        e = self.p.clone()
        e[torch.arange(len(e)), self.t] -= 1.0
        c = (self.w * scale / self.denom)[:, None]
        held = U[dt] if dt != torch.float32 else U32
        # e: the exponential's own error, the subtraction's, the rounding to the products' type (its floor: 2^-39), and
        # the rounding of e times the weight.
        e_off = self.p * (self.z_off + self.lse_off + 8 * U32)[:, None] + (held * 1.01 + 8 * U32) * e.abs() + 2.0 ** -38
        # The products of parts once more, and hidden values and head where they are far below the tensor's largest.
        e_off = e_off + self.parts_off * e.abs()
        low = 2.0 ** -39 if dt == torch.float32 else 0.0
        low_W, low_h = (low * t.abs().max() if t.numel() else 0.0 for t in (self.W, self.h))
        n, V = e.shape
        self.dh = c * (e @ self.W)
        off = c.abs() * (e_off @ self.W.abs() + U32 * (64 + V / 16) * (e.abs() @ self.W.abs()) + low_W * e.abs().sum(1, keepdim=True))
        self.dh_bound = U[dt] * self.dh.abs() + 1.01 * off + STEP[dt]
        ce = c * e
        self.dW = ce.t() @ self.h
        # The floor is one of the largest weight.
        floor = 2.0 ** -38 * c.abs().max() if n else 0.0
        off = (c.abs() * e_off + floor).t() @ self.h.abs() + U32 * (64 + n / 16) * (ce.abs().t() @ self.h.abs())
        off = off + low_h * ce.abs().sum(0)[:, None]
        self.dW_bound = U[dt] * self.dW.abs() + 1.01 * off + STEP[dt]


# --- AdamW ----------------------------------------------------------------------

BLOCK, TOP, LEAST = 256, 448.0, 2.0 ** -9


def decoded(q, scale):
    """Values of an 8-bit average."""
    n = q.numel()
    s = scale.cpu().double().repeat_interleave(BLOCK)[:n]
    return q.cpu().float().double().reshape(-1) * s


def adamw(p, g, m, v, t, lr, betas, eps, wd):
    """(p, m, v, the update's size) after step t, all float64."""
    m = betas[0] * m + (1 - betas[0]) * g
    v = betas[1] * v + (1 - betas[1]) * g * g
    up = lr * (m / (1 - betas[0] ** t)) / (torch.sqrt(v / (1 - betas[1] ** t)) + eps)
    return p * (1 - lr * wd) - up, m, v, up.abs()
