"""Cases of the learner's operators on replayed windows: the gated linear
recurrence over a window (forward, backward and one step), the advantages of
its rewards, and the clipped policy loss with its gradient.

``listed()`` names them, ``draw(rng)`` gives more of the same ranges,
``prepare`` makes a case's inputs on the GPU, ``run`` is one pass, in plain
torch operations or, with ``own``, through ``paper_2310_05205_amd.gear``;
``work`` is what a pass cannot do without and ``exact`` its outputs in 64 bits.

Kinds of pass:

  train    recurrence over windows, forward and backward
  forward  recurrence over windows, forward alone
  step     recurrence of one step, as an actor calls it
  policy   clipped policy loss with KL and entropy terms, and its gradient
  logp     log-probabilities of the actions and entropies alone
  adv      advantages and returns of windows
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
CLIP = (0.2, 0.28)
KL, ENTROPY = 0.05, 0.01
GAMMA, LAM = 0.99, 0.95


def listed():
    return [
        # An actor's step: 64 environments, one recurrent layer.
        {"name": "step", "kind": "step", "form": "sigmoid", "dtype": "bf16", "B": 64, "D": 1024, "reset": True},
        # Training on windows of the agents table: 8192 windows of 32 steps, 8 agents' 64 values, gate and
        # input the two halves of one projection.
        {"name": "train-windows", "kind": "train", "form": "sigmoid", "dtype": "bf16", "B": 8192, "T": 32, "D": 512,
         "reset": True, "ragged": False, "packed": True},
        # Few long trajectories, the split over time: gates as given, kept in 32 bits.
        {"name": "train-long", "kind": "train", "form": "value", "dtype": "f32", "B": 4, "T": 16384, "D": 512,
         "reset": True, "ragged": False, "packed": False},
        # Odd and ragged: whole 1000-step trajectories that ended early, a width that is no multiple of anything.
        {"name": "train-ragged", "kind": "train", "form": "sigmoid", "dtype": "f16", "B": 37, "T": 1000, "D": 1003,
         "reset": False, "ragged": True, "packed": False},
        # One long context read before acting from it.
        {"name": "forward-context", "kind": "forward", "form": "sigmoid", "dtype": "bf16", "B": 1, "T": 131072,
         "D": 512, "reset": False, "ragged": False, "packed": True},
        # A small discrete policy on 16 windows of 20 steps: latency.
        {"name": "policy-small", "kind": "policy", "dtype": "f32", "W": 16, "L": 20, "agents": 1, "V": 18,
         "mask": True, "unavailable": False},
        # The agents table's batch: 2.1 M rows of 16 logits, some actions unavailable, shared advantages.
        {"name": "policy-agents", "kind": "policy", "dtype": "bf16", "W": 8192, "L": 32, "agents": 8, "V": 16,
         "mask": True, "unavailable": True},
        # A token policy over a large vocabulary.
        {"name": "policy-tokens", "kind": "policy", "dtype": "bf16", "W": 32, "L": 128, "agents": 1, "V": 32768,
         "mask": False, "unavailable": False},
        # An odd vocabulary (rows aligned to nothing) and an odd number of rows.
        {"name": "policy-odd", "kind": "policy", "dtype": "f16", "W": 31, "L": 49, "agents": 1, "V": 50001,
         "mask": True, "unavailable": False},
        # Log-probabilities under the reference policy over the largest vocabulary.
        {"name": "logp-tokens", "kind": "logp", "dtype": "bf16", "W": 8, "L": 256, "agents": 1, "V": 131072,
         "mask": False, "unavailable": False},
        # Advantages of a training batch of 32-step windows.
        {"name": "adv-windows", "kind": "adv", "dtype": "f32", "B": 8192, "L": 32, "done": True, "ragged": False},
        # Few long streams of odd length, ended early.
        {"name": "adv-long", "kind": "adv", "dtype": "bf16", "B": 19, "L": 262147, "done": True, "ragged": True},
    ]


def _log(rng, lo, hi):
    """A size spread over its logarithm; large ones are odd or an odd multiple of 64, half of each."""
    n = max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))
    if n < 256:
        return n
    n = n | 1 if rng.random() < 0.5 else (n // 64 | 1) * 64
    return n if n <= hi else n - 64


def draw(rng):
    kind = rng.choice(["step", "train", "train", "forward", "policy", "policy", "logp", "adv"])
    c = {"kind": kind, "dtype": rng.choice(["f32", "bf16", "f16"])}
    if kind == "adv":
        c["L"] = _log(rng, 1, 300000)
        c["B"] = _log(rng, 1, min(20000, 5000000 // c["L"]))
        c["done"], c["ragged"] = rng.random() < 0.7, rng.random() < 0.5
    elif kind in ("policy", "logp"):
        c["V"] = _log(rng, 2, 131072)
        c["agents"] = rng.choice([1, 1, 3, 8])
        c["L"] = _log(rng, 1, 128)
        rows = min(1 << 20, (1 << 26) // c["V"])
        c["W"] = _log(rng, 1, max(1, rows // (c["L"] * c["agents"])))
        c["mask"], c["unavailable"] = rng.random() < 0.5, rng.random() < 0.5
    else:
        c["form"] = rng.choice(["value", "sigmoid"])
        c["D"] = _log(rng, 1, 4096)
        c["reset"] = rng.random() < 0.5
        if kind == "step":
            c["B"] = _log(rng, 1, 2048)
        else:
            c["T"] = _log(rng, 1, 65536)
            c["D"] = min(c["D"], max(1, (1 << 25) // c["T"]))
            c["B"] = _log(rng, 1, max(1, min(8192, (1 << 25) // (c["T"] * c["D"]))))
            c["ragged"], c["packed"] = rng.random() < 0.4, rng.random() < 0.5
    return c


class _Random:
    """Seeded inputs on the GPU."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(shape, generator=self.g, device="cuda")

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda")

    def below(self, n, *shape):
        return torch.randint(0, n, shape, generator=self.g, device="cuda")


def prepare(case, seed):
    r = _Random(seed)
    dt = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["kind"] == "adv":
        B, L = case["B"], case["L"]
        # Sparse-ish rewards and a critic that is roughly right.
        s["reward"] = r.normal(B, L).to(dt)
        s["value"] = (3.0 * r.normal(B, L + 1)).to(dt)
        s["done"] = (r.uniform(B, L) < 0.01).to(torch.uint8) if case["done"] else None
        s["lengths"] = r.below(L + 1, B).to(torch.int32) if case["ragged"] else None
    elif case["kind"] in ("policy", "logp"):
        W, L, K, V = case["W"], case["L"], case["agents"], case["V"]
        z = (2.0 * r.normal(W, L, K, V)).to(dt)
        s["action"] = r.below(V, W, L, K).to(torch.int32)
        if case["unavailable"]:
            # Unavailable actions hold the type's lowest value, never the one taken.
            off = r.uniform(W, L, K, V) < 0.25
            off.scatter_(3, s["action"].long()[..., None], False)
            z.masked_fill_(off, torch.finfo(dt).min)
        s["logits"] = z
        s["mask"] = (r.uniform(W, L, K) < 0.9).to(torch.uint8) if case["mask"] else None
        if case["kind"] == "policy":
            s["adv"] = r.normal(W, L)
            s["weight"] = 0.2 + 0.8 * r.uniform(W)
            # The behaviour policy is a few updates old.  At the clip's very edges the gradient jumps, and one
            # rounding decides its side; ratios there are moved off them by half a percent.
            lp = _log_softmax(z.float()).gather(3, s["action"].long()[..., None])[..., 0]
            lr = 0.15 * r.normal(W, L, K)
            for edge in (math.log(1 - CLIP[0]), math.log(1 + CLIP[1])):
                d = lr - edge
                lr = torch.where(d.abs() < 5e-3, edge + torch.where(d < 0, -5e-3, 5e-3), lr)
            s["old_logp"] = lp - lr
            s["ref_logp"] = lp - 0.3 * r.normal(W, L, K)
            # A loss scale where gradients would underflow 16 bits.
            rows = W * L * K
            s["grad_scale"] = float(2 ** int(math.log2(rows))) if case["dtype"] == "f16" else 1.0
    else:
        B, T, D = case["B"], case.get("T", 1), case["D"]
        if case.get("packed"):
            # Gate and input as one projection leaves them: [B, T, 2 D].
            p = torch.empty(B, T, 2 * D, dtype=dt, device="cuda")
            gate, x = p[..., :D], p[..., D:]
        else:
            gate, x = torch.empty(B, T, D, dtype=dt, device="cuda"), torch.empty(B, T, D, dtype=dt, device="cuda")
        g = 3.0 + 1.5 * r.normal(B, T, D)
        gate.copy_(g if case["form"] == "sigmoid" else torch.sigmoid(g))
        x.copy_(r.normal(B, T, D))
        s["gate"], s["x"] = gate, x
        s["state"] = r.normal(B, D)
        s["reset"] = (r.uniform(B, T) < 0.01).to(torch.uint8) if case["reset"] else None
        s["lengths"] = r.below(T + 1, B).to(torch.int32) if case.get("ragged") else None
        if case["kind"] == "train":
            s["dy"] = r.normal(B, T, D).to(dt)
            s["dfinal"] = r.normal(B, D)
        if case["kind"] == "step":
            s["gate"], s["x"] = gate[:, 0], x[:, 0]
            s["reset"] = s["reset"][:, 0].contiguous() if case["reset"] else None
    return s


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _OWN[kind](s)
    return _PLAIN[kind](s)


# --- the framework's operators ---------------------------------------------

def _form(s):
    from paper_2310_05205_amd import gear
    return gear.GEAR_GATE_SIGMOID if s["case"]["form"] == "sigmoid" else gear.GEAR_GATE_VALUE


def _own_train(s):
    from paper_2310_05205_amd import gear
    form = _form(s)
    y, final, saved = gear.recurrence(s["gate"], s["x"], s["state"], form=form, reset=s["reset"],
                                      lengths=s["lengths"], save=True)
    dgate, dx, dstate = gear.recurrence_backward(s["gate"], s["x"], saved, s["dy"], s["dfinal"], s["state"], form=form,
                                                 reset=s["reset"], lengths=s["lengths"])
    return {"y": y, "final": final, "dgate": dgate, "dx": dx, "dstate": dstate}


def _own_forward(s):
    from paper_2310_05205_amd import gear
    y, final, _ = gear.recurrence(s["gate"], s["x"], s["state"], form=_form(s), reset=s["reset"],
                                  lengths=s["lengths"])
    return {"y": y, "final": final}


def _own_step(s):
    from paper_2310_05205_amd import gear
    y, state = gear.recurrence_step(s["gate"], s["x"], s["state"], form=_form(s), reset=s["reset"])
    return {"y": y, "state": state}


def _own_policy(s):
    from paper_2310_05205_amd import gear
    loss, logp, entropy, stats, grad = gear.policy_loss(
        s["logits"], s["action"], s["old_logp"], s["adv"], ref_logp=s["ref_logp"], weight=s["weight"], mask=s["mask"],
        clip=CLIP, kl=KL, entropy=ENTROPY, grad=True, grad_scale=s["grad_scale"])
    return {"loss": loss, "logp": logp, "entropy": entropy, "stats": stats, "grad": grad}


def _own_logp(s):
    from paper_2310_05205_amd import gear
    logp, entropy = gear.action_logp(s["logits"], s["action"], mask=s["mask"])
    return {"logp": logp, "entropy": entropy}


def _own_adv(s):
    from paper_2310_05205_amd import gear
    adv, ret = gear.advantages(s["reward"], s["value"], GAMMA, LAM, done=s["done"], lengths=s["lengths"])
    return {"adv": adv, "ret": ret}


_OWN = {"train": _own_train, "forward": _own_forward, "step": _own_step, "policy": _own_policy, "logp": _own_logp,
        "adv": _own_adv}


# --- plain torch operations in 32 bits --------------------------------------

def _scan(a, u):
    """h_t = a_t h_{t-1} + u_t along dimension 1, by doubling spans."""
    T, k = a.shape[1], 1
    while k < T:
        h = u.clone()
        h[:, k:] += a[:, k:] * u[:, :-k]
        u = h
        if 2 * k < T:
            p = a.clone()
            p[:, k:] *= a[:, :-k]
            a = p
        k *= 2
    return u


def _valid(lengths, B, T):
    if lengths is None:
        return torch.ones(B, T, dtype=torch.bool, device="cuda")
    return torch.arange(T, device="cuda")[None] < lengths[:, None]


def _plain_parts(s):
    """Decays (0 after a reset, 1 past the end), the inputs' weights, inputs and masks of a recurrence."""
    gate, x = s["gate"].float(), s["x"].float()
    B, T, _ = gate.shape
    valid = _valid(s["lengths"], B, T)[..., None]
    if s["case"]["form"] == "sigmoid":
        f = 1.0 / (1.0 + torch.exp(-gate))
        w = 1.0 / (1.0 + torch.exp(gate))
    else:
        f, w = gate, torch.ones_like(gate)
    a = f if s["reset"] is None else torch.where(s["reset"][..., None] != 0, 0.0, f)
    a = torch.where(valid, a, 1.0)
    u = torch.where(valid, w * x, 0.0)
    return a, w, x, f, u, valid


def _plain_states(a, u, state):
    u = u.clone()
    u[:, 0] += a[:, 0] * state
    return _scan(a, u)


def _plain_forward(s):
    a, _, x, _, u, valid = _plain_parts(s)
    h = _plain_states(a, u, s["state"])
    return {"y": torch.where(valid, h, 0.0).to(s["x"].dtype), "final": h[:, -1].clone()}


def _plain_train(s):
    dt = s["x"].dtype
    a, w, x, f, u, valid = _plain_parts(s)
    h = _plain_states(a, u, s["state"])
    before = torch.cat([s["state"][:, None], h[:, :-1]], dim=1)
    if s["reset"] is not None:
        before = torch.where(s["reset"][..., None] != 0, 0.0, before)
    d = torch.where(valid, s["dy"].float(), 0.0)
    d[:, -1] += s["dfinal"]
    after = torch.cat([a[:, 1:], torch.zeros_like(a[:, :1])], dim=1)
    G = _scan(after.flip(1), d.flip(1)).flip(1)
    if s["case"]["form"] == "sigmoid":
        dgate = G * (before - x) * f * w
    else:
        dgate = G * before
    return {"y": torch.where(valid, h, 0.0).to(dt), "final": h[:, -1].clone(),
            "dgate": torch.where(valid, dgate, 0.0).to(dt), "dx": torch.where(valid, G * w, 0.0).to(dt),
            "dstate": a[:, 0] * G[:, 0]}


def _plain_step(s):
    one = dict(s, gate=s["gate"][:, None], x=s["x"][:, None], lengths=None,
               reset=None if s["reset"] is None else s["reset"][:, None])
    r = _plain_forward(one)
    return {"y": r["y"][:, 0], "state": r["final"]}


def _log_softmax(z):
    m = z.amax(-1, keepdim=True)
    return z - m - torch.log(torch.exp(z - m).sum(-1, keepdim=True))


def _plain_rows(s):
    lsm = _log_softmax(s["logits"].float())
    p = torch.exp(lsm)
    plogp = torch.where(p > 0, p * lsm, 0.0)
    lp = lsm.gather(-1, s["action"].long()[..., None])[..., 0]
    H = -plogp.sum(-1)
    on = torch.ones_like(lp, dtype=torch.bool) if s["mask"] is None else s["mask"] != 0
    return p, plogp, torch.where(on, lp, 0.0), torch.where(on, H, 0.0), on


def _plain_logp(s):
    _, _, lp, H, _ = _plain_rows(s)
    return {"logp": lp, "entropy": H}


def _plain_policy(s):
    p, plogp, lp, H, on = _plain_rows(s)
    A, w = s["adv"][..., None].expand_as(lp), s["weight"][:, None, None].expand_as(lp)
    count = on.sum().clamp(min=1).float()
    ratio = torch.exp(lp - s["old_logp"])
    free, clipped = ratio * A, ratio.clamp(1 - CLIP[0], 1 + CLIP[1]) * A
    pg = -torch.minimum(free, clipped)
    q = s["ref_logp"] - lp
    kl = torch.exp(q) - q - 1
    is_clipped = clipped < free

    def mean(v):
        return torch.where(on, v, 0.0).sum() / count
    loss = mean(w * (pg + KL * kl - ENTROPY * H))
    stats = torch.stack([mean(pg), mean(kl), mean(H), mean(is_clipped.float())])
    c = torch.where(is_clipped, 0.0, -free) + KL * (1 - torch.exp(q))
    scale = torch.where(on, w, 0.0) * (s["grad_scale"] / count)
    g = ENTROPY * (plogp + p * H[..., None]) - c[..., None] * p
    g.scatter_add_(-1, s["action"].long()[..., None], c[..., None])
    g *= scale[..., None]
    return {"loss": loss, "logp": lp, "entropy": H, "stats": stats, "grad": g.to(s["logits"].dtype)}


def _plain_adv(s):
    r, v = s["reward"].float(), s["value"].float()
    B, L = r.shape
    valid = _valid(s["lengths"], B, L)
    live = valid if s["done"] is None else valid & (s["done"] == 0)
    d = torch.where(valid, r + torch.where(live, GAMMA * v[:, 1:], 0.0) - v[:, :-1], 0.0)
    c = torch.where(live, GAMMA * LAM, 0.0)
    A = _scan(c.flip(1)[..., None], d.flip(1)[..., None])[..., 0].flip(1)
    A = torch.where(valid, A, 0.0)
    return {"adv": A, "ret": torch.where(valid, A + v[:, :-1], 0.0)}


_PLAIN = {"train": _plain_train, "forward": _plain_forward, "step": _plain_step, "policy": _plain_policy,
          "logp": _plain_logp, "adv": _plain_adv}


# --- what a pass cannot do without ------------------------------------------

def work(case):
    size = DTYPES[case["dtype"]].itemsize
    if case["kind"] == "adv":
        n = case["B"] * case["L"]
        b = size * (n + n + case["B"]) + (n if case["done"] else 0) + 8 * n + (4 * case["B"] if case["ragged"] else 0)
        return {"bytes": b, "flops": 7 * n}
    if case["kind"] in ("policy", "logp"):
        W, L = case["W"], case["L"]
        rows = W * L * case["agents"]
        n = rows * case["V"]
        b = size * n + 4 * rows + (rows if case["mask"] else 0) + 8 * rows
        if case["kind"] == "logp":
            return {"bytes": b, "flops": 6 * n}
        return {"bytes": b + size * n + 8 * rows + 4 * W * L + 4 * W + 20, "flops": 12 * n}
    B, T, D = case["B"], case.get("T", 1), case["D"]
    n = B * T * D
    extra = (B * T if case["reset"] else 0) + (4 * B if case.get("ragged") else 0)
    sig = case["form"] == "sigmoid"
    fwd = size * 3 * n + 8 * B * D + extra
    if case["kind"] != "train":
        return {"bytes": fwd, "flops": (8 if sig else 2) * n}
    # The rest of the model and its loss lie between the two calls, so the backward call reads gate and input again.
    return {"bytes": fwd + size * 5 * n + 12 * B * D + extra, "flops": (24 if sig else 6) * n}


# --- the definitions in 64 bits, one step or row after the other ------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "adv":
        return _exact_adv(s)
    if case["kind"] in ("policy", "logp"):
        return _exact_policy(s)
    return _exact_recurrence(s)


def _exact_recurrence(s):
    case = s["case"]
    gate, x = s["gate"].double(), s["x"].double()
    if case["kind"] == "step":
        gate, x = gate[:, None], x[:, None]
    B, T, D = x.shape
    f = torch.sigmoid(gate) if case["form"] == "sigmoid" else gate
    w = 1.0 - f if case["form"] == "sigmoid" else torch.ones_like(f)
    keep = torch.ones(B, T, 1, dtype=torch.float64, device="cuda")
    if s["reset"] is not None:
        keep -= (s["reset"].reshape(B, T, 1) != 0).double()
    inside = torch.ones(B, T, 1, dtype=torch.float64, device="cuda")
    if s["lengths"] is not None:
        inside = (torch.arange(T, device="cuda")[None, :, None] < s["lengths"][:, None, None]).double()
    decay = inside * keep * f + (1 - inside)
    added = inside * w * x
    h = s["state"].double()
    prev = torch.empty(B, T, D, dtype=torch.float64, device="cuda")
    y = torch.empty_like(prev)
    for t in range(T):
        prev[:, t] = h
        h = torch.addcmul(added[:, t], decay[:, t], h)
        y[:, t] = h
    y *= inside
    if case["kind"] == "step":
        return {"y": y[:, 0], "state": h}
    if case["kind"] == "forward":
        return {"y": y, "final": h}
    dy = s["dy"].double() * inside
    G = s["dfinal"].double()
    back = torch.empty_like(prev)
    for t in range(T - 1, -1, -1):
        G = G + dy[:, t]
        back[:, t] = G
        G = decay[:, t] * G
    back *= inside
    dgate = back * (keep * prev - x) * f * w if case["form"] == "sigmoid" else back * keep * prev
    return {"y": y, "final": h, "dgate": dgate, "dx": back * w, "dstate": G}


def _exact_policy(s):
    V = s["case"]["V"]
    z = s["logits"].double().reshape(-1, V)
    n = z.shape[0]
    a = s["action"].long().reshape(-1)
    rows = torch.arange(n, device="cuda")
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    lp = z[rows, a] - lse
    H = lse - (p * z.clamp(min=-1e30)).sum(1)
    on = torch.ones(n, dtype=torch.float64, device="cuda") if s["mask"] is None else s["mask"].reshape(-1).double()
    shape = s["action"].shape
    out = {}
    if s["case"]["kind"] == "policy":
        W, L, K = shape
        A = s["adv"].double().repeat_interleave(K, 1).reshape(-1)
        w = s["weight"].double().repeat_interleave(L * K)
        count = on.sum().clamp(min=1)
        r = torch.exp(lp - s["old_logp"].double().reshape(-1))
        lo, hi = 1 - CLIP[0], 1 + CLIP[1]
        # With A >= 0 the ratio counts up to hi, with A < 0 from lo on.
        limit = torch.where(A >= 0, r.clamp(max=hi), r.clamp(min=lo))
        flat = (limit != r).double() * (A != 0)
        pg = -limit * A
        d = s["ref_logp"].double().reshape(-1) - lp
        kl = torch.expm1(d) - d
        out["loss"] = (on * w * (pg + KL * kl - ENTROPY * H)).sum() / count
        c = (flat - 1) * A * r - KL * torch.expm1(d)
        out["logp"], out["entropy"] = (on * lp).reshape(shape), (on * H).reshape(shape)
        out["stats"] = torch.stack([(on * t).sum() / count for t in (pg, kl, H, flat)])
        g = p * (ENTROPY * ((z - lse[:, None]).clamp(min=-1e30) + H[:, None]) - c[:, None])
        g[rows, a] += c
        out["grad"] = (g * (on * w * s["grad_scale"] / count)[:, None]).reshape(s["logits"].shape)
        return out
    return {"logp": (on * lp).reshape(shape), "entropy": (on * H).reshape(shape)}


def _exact_adv(s):
    r, v = s["reward"].double().cpu().numpy(), s["value"].double().cpu().numpy()
    B, L = r.shape
    go = 1.0 - (s["done"].cpu().numpy() != 0) if s["done"] is not None else r * 0 + 1.0
    n = s["lengths"].cpu().numpy() if s["lengths"] is not None else [L] * B
    adv, ret = r * 0, r * 0
    for b in range(B) if B < L else ():
        a, m = 0.0, int(n[b])
        rb, vb, gb, col = r[b].tolist(), v[b].tolist(), go[b].tolist(), [0.0] * L
        for t in range(m - 1, -1, -1):
            a = rb[t] + GAMMA * gb[t] * vb[t + 1] - vb[t] + GAMMA * LAM * gb[t] * a
            col[t] = a
        adv[b] = col
        ret[b, :m] = adv[b, :m] + v[b, :m]
    if B >= L:
        a = r[:, 0] * 0
        for t in range(L - 1, -1, -1):
            a = r[:, t] + GAMMA * go[:, t] * v[:, t + 1] - v[:, t] + GAMMA * LAM * go[:, t] * a
            a = a * (t < torch.as_tensor(n).numpy())
            adv[:, t] = a
            ret[:, t] = (a + v[:, t]) * (t < torch.as_tensor(n).numpy())
    return {"adv": torch.from_numpy(adv), "ret": torch.from_numpy(ret)}
