"""The learner's operators in 64 bits, step by step in numpy, with bounds on
what 32-bit arithmetic may make of them.

Each function returns its results and, for every value, the error that
correctly rounded fp32 operations and the stated errors of exp (|x| + 2 units in
the last place), log, reciprocal and their like can add up to: the recursions
below run the same steps over the errors.  ``within`` compares with twice that,
plus the rounding to the output's type."""
import numpy as np

EPS = 2.0 ** -24  # half a unit in the last place, relative
ROUND = {"float32": (2.0 ** -24, 2.0 ** -149), "bfloat16": (2.0 ** -8, 2.0 ** -133), "float16": (2.0 ** -11, 2.0 ** -24)}


def within(got, want, err, dtype="float32"):
    """Every value near enough; equal where the expected one is not finite."""
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    assert got.shape == want.shape, (got.shape, want.shape)
    fin = np.isfinite(want)
    np.testing.assert_array_equal(got[~fin], want[~fin])
    rel, tiny = ROUND[dtype]
    tol = 2.0 * np.asarray(err, np.float64) + rel * np.abs(want) + tiny
    bad = fin & ~(np.abs(got - want) <= tol)
    assert not bad.any(), "%d of %d off, worst %g of its tolerance at %s: %g for %g" % (
        bad.sum(), bad.size, np.nanmax(np.where(bad, np.abs(got - want) / tol, 0)),
        np.unravel_index(np.argmax(np.where(bad, np.abs(got - want) / tol, 0)), bad.shape),
        got[bad][0], want[bad][0])


def _sigmoid(g):
    t = np.exp(-np.abs(g))
    return np.where(g >= 0, 1 / (1 + t), t / (1 + t)), np.where(g >= 0, t / (1 + t), 1 / (1 + t))


def _gates(gate, sigmoid):
    """Decay, input weight and the relative error of either in units of EPS."""
    if sigmoid:
        f, w = _sigmoid(gate)
        return f, w, np.abs(gate) + 8
    return gate, np.ones_like(gate), np.zeros_like(gate)


def recurrence(gate, x, state, sigmoid=False, reset=None, lengths=None):
    """((y, err), (final, err), states before every step, their errors)."""
    gate, x = np.asarray(gate, np.float64), np.asarray(x, np.float64)
    B, T, D = x.shape
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    z = np.zeros((B, T), bool) if reset is None else np.asarray(reset) != 0
    f, w, ge = _gates(gate, sigmoid)
    h = np.zeros((B, D)) if state is None else np.array(state, np.float64)
    e = np.zeros((B, D))
    y, ye, before, be = (np.zeros((B, T, D)) for _ in range(4))
    for t in range(T):
        on, cut = (t < n)[:, None], z[:, t][:, None]
        hp, ep = np.where(cut, 0.0, h), np.where(cut, 0.0, e)
        before[:, t], be[:, t] = hp, ep
        with np.errstate(invalid="ignore"):
            kept = np.where(cut, 0.0, f[:, t] * hp)
            new = kept + w[:, t] * x[:, t]
            ne = np.abs(f[:, t]) * ep + EPS * ((ge[:, t] + 1) * (np.abs(kept) + np.abs(w[:, t] * x[:, t])) + 2 * np.abs(new))
        h, e = np.where(on, new, h), np.where(on, ne, e)
        y[:, t], ye[:, t] = np.where(on, h, 0.0), np.where(on, e, 0.0)
    return (y, ye), (h, e), before, be


def recurrence_backward(gate, x, state, dy, dfinal, sigmoid=False, reset=None, lengths=None):
    """((dgate, err), (dx, err), (dstate, err))."""
    gate, x = np.asarray(gate, np.float64), np.asarray(x, np.float64)
    B, T, D = x.shape
    n = np.full(B, T) if lengths is None else np.clip(lengths, 0, T)
    z = np.zeros((B, T), bool) if reset is None else np.asarray(reset) != 0
    f, w, ge = _gates(gate, sigmoid)
    _, _, before, be = recurrence(gate, x, state, sigmoid, reset, lengths)
    dy = np.zeros((B, T, D)) if dy is None else np.asarray(dy, np.float64)
    G = np.zeros((B, D)) if dfinal is None else np.array(dfinal, np.float64)
    e = np.zeros((B, D))
    dgate, dge, dx, dxe = (np.zeros((B, T, D)) for _ in range(4))
    for t in range(T - 1, -1, -1):
        on, cut = (t < n)[:, None], z[:, t][:, None]
        t_ = G + dy[:, t]
        te = e + EPS * np.abs(t_)
        if sigmoid:
            diff = before[:, t] - x[:, t]
            de = be[:, t] + EPS * np.abs(diff)
            slope = f[:, t] * w[:, t]
            dg = t_ * diff * slope
            ee = te * np.abs(diff) * slope + np.abs(t_) * de * slope + EPS * (2 * ge[:, t] + 4) * np.abs(dg)
            ox, oe = t_ * w[:, t], te * w[:, t] + EPS * (ge[:, t] + 1) * np.abs(t_ * w[:, t])
        else:
            dg = t_ * before[:, t]
            ee = te * np.abs(before[:, t]) + np.abs(t_) * be[:, t] + EPS * np.abs(dg)
            ox, oe = t_, te
        dgate[:, t], dge[:, t] = np.where(on, dg, 0.0), np.where(on, ee, 0.0)
        dx[:, t], dxe[:, t] = np.where(on, ox, 0.0), np.where(on, oe, 0.0)
        new = np.where(cut, 0.0, f[:, t] * t_)
        ne = np.where(cut, 0.0, np.abs(f[:, t]) * te + EPS * (ge[:, t] + 2) * np.abs(new))
        G, e = np.where(on, new, G), np.where(on, ne, e)
    return (dgate, dge), (dx, dxe), (G, e)


def advantages(reward, value, gamma, lam, done=None, lengths=None):
    """((adv, err), (ret, err))."""
    r, v = np.asarray(reward, np.float64), np.asarray(value, np.float64)
    B, L = r.shape
    gamma, decay = float(np.float32(gamma)), float(np.float32(np.float32(gamma) * np.float32(lam)))
    n = np.full(B, L) if lengths is None else np.clip(lengths, 0, L)
    end = np.zeros((B, L), bool) if done is None else np.asarray(done) != 0
    a, e = np.zeros(B), np.zeros(B)
    adv, ae, ret, re = (np.zeros((B, L)) for _ in range(4))
    for t in range(L - 1, -1, -1):
        on, cut = t < n, end[:, t]
        nxt = np.where(cut, 0.0, gamma * np.where(cut, 0.0, v[:, t + 1]))
        delta = r[:, t] + nxt - v[:, t]
        de = EPS * (3 * np.abs(nxt) + 2 * np.abs(r[:, t] + nxt) + np.abs(delta))
        more, me = np.where(cut, 0.0, decay * np.where(cut, 0.0, a)), np.where(cut, 0.0, decay * e)
        new = delta + more
        a = np.where(on, new, a)
        # Maps composed in another order round their products as well: two more units each.
        e = np.where(on, de + me + EPS * (3 * np.abs(more) + 2 * np.abs(new) + np.abs(delta)), e)
        adv[:, t], ae[:, t] = np.where(on, a, 0.0), np.where(on, e, 0.0)
        ret[:, t] = np.where(on, a + v[:, t], 0.0)
        re[:, t] = np.where(on, e + EPS * np.abs(a + v[:, t]), 0.0)
    return (adv, ae), (ret, re)


def policy(logits, action, mask=None, old=None, adv=None, ref=None, weight=None, clip=(0.2, 0.2), kl=0.0, entropy=0.0,
           denom=None, scale=1.0, need=True):
    """A dict of (value, err) for rows [n, V]; every per-row input of shape [n]."""
    with np.errstate(all="ignore"):
        return _policy(np.asarray(logits, np.float64), np.asarray(action, np.int64), mask, old, adv, ref, weight, clip, kl,
                       entropy, denom, scale)


def _policy(z, action, mask, old, adv, ref, weight, clip, kl, entropy, denom, scale):
    n, V = z.shape
    on = (action >= 0) & (action < V)
    if mask is not None:
        on &= np.asarray(mask) != 0
    act = np.where(on, action, 0)
    zz = np.where(on[:, None], z, 0.0)
    m = zz.max(1)
    empty = np.isneginf(m)
    d = zz - np.where(empty, 0.0, m)[:, None]
    E = np.exp(d)
    S = E.sum(1)
    ln = np.log(S)
    p = E / np.where(empty, 1.0, S)[:, None]
    dd = np.where(p > 0, d, 0.0)
    pd = (p * np.abs(dd)).sum(1)
    lp = np.where(empty, -np.inf, d[np.arange(n), act] - ln)
    H = np.where(empty, 0.0, ln - (p * dd).sum(1))
    # Sums: every lane adds V / 256 values one after the other at most, then the lanes in pairs.
    units = 16 + V / 256
    lpe = EPS * (2 * np.abs(np.where(np.isfinite(lp), lp, 0)) + 2 * np.abs(ln) + pd + units)
    He = EPS * ((p * np.abs(dd) * (np.abs(dd) + units)).sum(1) + (pd + np.abs(ln)) * units + units)
    out = {"logp": (np.where(on, lp, 0.0), np.where(on, lpe, 0.0)), "entropy": (np.where(on, H, 0.0), np.where(on, He, 0.0))}
    if old is None:
        return out
    live = on & ~empty
    A, w = np.asarray(adv, np.float64), np.ones(n) if weight is None else np.asarray(weight, np.float64)
    count = float(max(on.sum(), 1)) if denom is None else float(np.float32(denom))
    lo, hi = float(np.float32(1) - np.float32(clip[0])), float(np.float32(1) + np.float32(clip[1]))
    kl, entropy = float(np.float32(kl)), float(np.float32(entropy))
    x = lp - np.asarray(old, np.float64)
    r = np.exp(x)
    re = np.where(np.isfinite(r), r, 0) * (lpe + EPS * (np.abs(np.where(np.isfinite(x), x, 0)) + 3))
    free, held = r * A, np.clip(r, lo, hi) * A
    clipped = held < free
    pg = -np.minimum(free, held)
    pge = np.where(clipped, 0.0, re * np.abs(A)) + EPS * np.abs(pg)
    c, ce = np.where(clipped, 0.0, -free), np.where(clipped, 0.0, re * np.abs(A) + EPS * np.abs(free))
    k, ke = np.zeros(n), np.zeros(n)
    row, rowe = pg, pge
    if ref is not None:
        q = np.asarray(ref, np.float64) - lp
        em = np.expm1(q)
        qe = lpe + EPS * np.abs(q)
        k = em - q
        ke = qe * np.abs(em) + EPS * (3 * np.abs(em) + np.abs(q) + np.abs(k))
        if kl != 0:
            row, rowe = row + kl * k, rowe + abs(kl) * ke + EPS * 2 * np.abs(kl * k)
            c, ce = c - kl * em, ce + abs(kl) * (qe * (np.abs(em) + 1) + 3 * EPS * np.abs(em))
    if entropy != 0:
        row, rowe = row - entropy * H, rowe + abs(entropy) * (He + EPS * np.abs(H))
    rowe = np.abs(w) * (rowe + 2 * EPS * np.abs(row))
    row = w * row
    s = np.where(live, w * scale / count, 0.0)
    logp = np.where(p > 0, dd - ln[:, None], 0.0)
    inner = entropy * (logp + H[:, None]) - c[:, None]
    pe = p * EPS * (np.abs(dd) + pd[:, None] + units + 4)
    ie = abs(entropy) * ((lpe + He)[:, None] + EPS * (np.abs(dd) + 3 * np.abs(logp))) + ce[:, None] + EPS * 2 * np.abs(inner)
    g, ge = p * inner, pe * np.abs(inner) + p * ie
    rows = np.arange(n)
    g[rows, act] += np.where(live, c, 0.0)
    ge[rows, act] += np.where(live, ce + EPS * 2 * np.abs(c), 0.0)
    s1 = s[:, None]
    out["grad"] = np.where(live[:, None], g * s1, 0.0), np.where(live[:, None], np.abs(s1) * (ge + EPS * 6 * np.abs(g)), 0.0)

    def mean(v, e):
        v, e = np.where(live, v, 0.0), np.where(live, e, 0.0)
        return v.sum() / count, (e.sum() + EPS * 16 * np.abs(v).sum()) / abs(count)
    out["loss"] = mean(row, rowe)
    parts = [mean(pg, pge), mean(k, ke), mean(H, He), mean(clipped.astype(float), np.zeros(n))]
    out["stats"] = np.array([v for v, _ in parts]), np.array([e for _, e in parts])
    return out
