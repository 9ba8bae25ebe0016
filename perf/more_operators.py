"""Cases of what a learner's network needs around its recurrence and losses:
layer norm with the residual sum before it, the loss of a token head over a
vocabulary without its logits, and the AdamW step of all parameters at once.

``listed()`` names them, ``draw(rng)`` gives more of the same ranges,
``prepare`` makes a case's inputs on the GPU, ``run`` is one pass, in plain
torch operations or, with ``own``, through ``paper_2310_05205_amd.gear``;
``work`` is what a pass cannot do without and ``exact`` its outputs in 64 bits.

Kinds of pass:

  norm        layer norm, forward alone
  norm-train  layer norm of a residual sum, forward and backward
  token       loss and log-probabilities of targets under a token head
  token-train the same, and the gradients of hidden states and head
  adamw       norm of all gradients, then one clipped AdamW step of all tensors
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5                # of layer norm
BETAS, ADAM_EPS, DECAY, LR, MAX_NORM = (0.9, 0.98), 1e-8, 0.05, 1e-3, 1.0
BLOCK = 256               # elements of an 8-bit state that share a scale
TOP, LEAST = 448.0, 2.0 ** -9  # e4m3: its largest value and its smallest above 0


def listed():
    return [
        # Before an actor's step: 64 environments.
        {"name": "norm-step", "kind": "norm", "dtype": "bf16", "wide": True, "rows": 64, "D": 1024},
        # Training on the agents table's windows: 8192 x 32 steps of 512 channels, the block's residual stream.
        {"name": "norm-windows", "kind": "norm-train", "dtype": "bf16", "wide": True, "rows": 262144, "D": 512,
         "residual": True},
        # Whole 1000-step trajectories of a width that is no multiple of anything, parameters in 16 bits.
        {"name": "norm-odd", "kind": "norm-train", "dtype": "f16", "wide": False, "rows": 37000, "D": 1003,
         "residual": False},
        # Few, very long rows in 32 bits.
        {"name": "norm-long", "kind": "norm-train", "dtype": "f32", "wide": True, "rows": 1024, "D": 20000,
         "residual": True},
        # A small discrete head on 16 windows of 20 steps: latency.
        {"name": "token-small", "kind": "token-train", "dtype": "f32", "rows": 320, "D": 64, "V": 18, "mask": True},
        # Log-probabilities of 16 sequences' next tokens: the head is read once.
        {"name": "token-step", "kind": "token", "dtype": "bf16", "rows": 16, "D": 2048, "V": 32768, "mask": False},
        # A token policy cloned from replayed windows, 32 of 128 tokens.
        {"name": "token-windows", "kind": "token-train", "dtype": "bf16", "rows": 4096, "D": 1024, "V": 32768,
         "mask": False},
        # An odd vocabulary, an odd width, an odd number of rows, padding among them.
        {"name": "token-odd", "kind": "token-train", "dtype": "f16", "rows": 1519, "D": 1003, "V": 50001, "mask": True},
        # A head kept in 32 bits.
        {"name": "token-f32", "kind": "token-train", "dtype": "f32", "rows": 1000, "D": 512, "V": 8192, "mask": True},
        # A small agent's parameters: latency.
        {"name": "adamw-small", "kind": "adamw", "dtype": "f32", "bits": 32, "master": False, "layers": 2, "D": 64,
         "V": 18},
        # 218 M parameters in 16 bits over a 32-bit copy, states in 32 bits.
        {"name": "adamw-wide", "kind": "adamw", "dtype": "bf16", "bits": 32, "master": True, "layers": 12, "D": 2048,
         "V": 32768},
        # 123 tensors of odd sizes, states in 8 bits.
        {"name": "adamw-odd", "kind": "adamw", "dtype": "bf16", "bits": 8, "master": True, "layers": 24, "D": 1003,
         "V": 50001},
    ]


def _log(rng, lo, hi):
    """A size spread over its logarithm; large ones are odd or an odd multiple of 64, half of each."""
    n = max(lo, min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))
    if n < 256:
        return n
    n = n | 1 if rng.random() < 0.5 else (n // 64 | 1) * 64
    return n if n <= hi else n - 64


def draw(rng):
    kind = rng.choice(["norm", "norm-train", "norm-train", "token", "token-train", "token-train", "adamw", "adamw"])
    c = {"kind": kind, "dtype": rng.choice(["f32", "bf16", "f16"])}
    if kind in ("norm", "norm-train"):
        c["wide"] = c["dtype"] == "f32" or rng.random() < 0.5
        # Of rows of one or two values the normalisation keeps no more than signs, and gradients of rounding alone.
        c["D"] = _log(rng, 8, 32768)
        c["rows"] = _log(rng, 1, min(300000, (1 << 26) // c["D"]))
        if kind == "norm-train":
            c["residual"] = rng.random() < 0.5
    elif kind in ("token", "token-train"):
        c["V"] = _log(rng, 8, 131072)
        c["D"] = _log(rng, 1, min(4096, (1 << 27) // c["V"]))
        most = min((1 << 27) // c["V"], (1 << (35 if c["dtype"] == "f32" else 37)) // (c["V"] * c["D"]))
        # A batch to learn from has some rows that are still uncertain; one row alone may have a gradient of rounding.
        c["rows"] = _log(rng, 1 if kind == "token" else 16, max(16, min(8192, most)))
        c["mask"] = rng.random() < 0.5
    else:
        c["bits"] = rng.choice([8, 32])
        c["master"] = c["dtype"] != "f32" and rng.random() < 0.5
        c["layers"] = rng.randint(1, 24)
        c["D"] = _log(rng, 4, 2048)
        while c["layers"] * c["D"] ** 2 > 1 << 25:
            c["layers"] -= 1
        c["V"] = _log(rng, 2, min(50001, (1 << 26) // c["D"]))
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


def _shapes(case):
    """A network's tensors: per layer a projection to gate and input, one back, their biases and a norm; then the head."""
    D = case["D"]
    return [(2 * D, D), (2 * D,), (D, D), (D,), (D,)] * case["layers"] + [(case["V"], D), (case["V"],), (D,)]


def prepare(case, seed):
    r = _Random(seed)
    dt = DTYPES[case["dtype"]]
    s = {"case": case}
    if case["kind"] in ("norm", "norm-train"):
        n, D = case["rows"], case["D"]
        wt = torch.float32 if case["wide"] else dt
        # A residual stream: rows of their own size and offset, channels of their own size.
        size = 1.0 + 2.0 * r.uniform(D).square()
        s["x"] = (r.normal(n, D) * size * (0.5 + r.uniform(n, 1)) + 0.5 * r.normal(n, 1)).to(dt)
        s["residual"] = r.normal(n, D).to(dt) if case.get("residual") else None
        s["weight"] = (1.0 + 0.2 * r.normal(D)).to(wt)
        s["bias"] = (0.2 * r.normal(D)).to(wt)
        if case["kind"] == "norm-train":
            s["dy"] = (r.normal(n, D) * (0.5 + r.uniform(D))).to(dt)
            s["dtotal"] = r.normal(n, D).to(dt) if case["residual"] else None
    elif case["kind"] in ("token", "token-train"):
        n, D, V = case["rows"], case["D"], case["V"]
        head = r.normal(V, D) * (2.0 / math.sqrt(D))
        y = r.below(V, n)
        # A network that has learned part of the data: most rows lean towards their target.
        lean = 2.0 * (r.uniform(n) < 0.8).float() * r.uniform(n)
        h = r.normal(n, D) + lean[:, None] * head[y] / head[y].norm(dim=1, keepdim=True).clamp(min=0.1)
        s["hidden"], s["head"], s["target"] = h.to(dt), head.to(dt), y.to(torch.int32)
        s["mask"] = (r.uniform(n) < 0.8).to(torch.uint8) if case["mask"] else None
        s["weight"] = 0.2 + 0.8 * r.uniform(n)
        # A loss scale where gradients would underflow 16 bits.
        s["grad_scale"] = float(2 ** int(math.log2(n) + 4)) if case["dtype"] == "f16" else 1.0
    else:
        shapes = _shapes(case)
        sizes = [math.prod(x) for x in shapes]
        at, total = [], 0
        for k in sizes:
            at.append(total)
            total += (k + BLOCK - 1) // BLOCK * BLOCK
        # One buffer holds all parameters, another all gradients, and so on; what lies between tensors stays 0.
        inside = torch.zeros(total, dtype=torch.bool, device="cuda")
        for a, k in zip(at, sizes):
            inside[a:a + k] = True
        # Tensors' gradients differ in size by orders of magnitude, and so do a tensor's.
        order = torch.empty(total, device="cuda")
        for a, k, u in zip(at, sizes, r.uniform(len(at)).tolist()):
            order[a:a + k] = 10.0 ** (-4.0 * u)
        order = torch.where(inside, order * (0.1 + r.uniform(total)), 0.0)
        flat = {"grad": (r.normal(total) * order).to(dt), "param": torch.where(inside, 0.05 * r.normal(total), 0.0)}
        m, root = 0.3 * r.normal(total) * order, (0.5 + r.uniform(total)) * order
        if case["master"]:
            flat["master"] = flat["param"].clone()
        flat["param"] = flat["param"].to(dt)
        if case["bits"] == 32:
            flat["exp_avg"], flat["exp_avg_sq"] = m, root.square()
        else:
            flat["exp_avg"], flat["exp_avg_scale"] = _in_8_bits(m)
            flat["exp_avg_sq"], flat["exp_avg_sq_scale"] = _in_8_bits(root)
        s["flat"] = flat
        # The tensors themselves, parts of the buffers, as a program holds them in lists.
        s["lists"] = {}
        for name, f in flat.items():
            if name.endswith("_scale"):
                s["lists"][name] = [f[a // BLOCK:a // BLOCK + (k + BLOCK - 1) // BLOCK] for a, k in zip(at, sizes)]
            else:
                s["lists"][name] = [f[a:a + k].view(x) for a, k, x in zip(at, sizes, shapes)]
        s["step"] = torch.tensor([100], device="cuda")
    return s


def run(s):
    kind = s["case"]["kind"]
    if own:
        return _OWN[kind](s)
    return _PLAIN[kind](s)


# --- the framework's operators ---------------------------------------------

def _own_norm(s):
    from paper_2310_05205_amd import gear
    y, _, _ = gear.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS)
    return {"y": y}


def _own_norm_train(s):
    from paper_2310_05205_amd import gear
    y, total, saved = gear.layer_norm(s["x"], s["weight"], s["bias"], eps=EPS, residual=s["residual"], save=True)
    dx, dw, db = gear.layer_norm_backward(s["dy"], s["x"] if total is None else total, saved, s["weight"],
                                          dtotal=s["dtotal"])
    return {"y": y, "total": total, "dx": dx, "dweight": dw, "dbias": db}


def _own_token(s):
    from paper_2310_05205_amd import gear
    loss, logp, lse = gear.token_loss(s["hidden"], s["head"], s["target"], weight=s["weight"], mask=s["mask"])
    return {"loss": loss, "logp": logp, "lse": lse}


def _own_token_train(s):
    from paper_2310_05205_amd import gear
    loss, logp, lse = gear.token_loss(s["hidden"], s["head"], s["target"], weight=s["weight"], mask=s["mask"])
    dhidden, dhead = gear.token_loss_backward(s["hidden"], s["head"], s["target"], lse, weight=s["weight"],
                                              mask=s["mask"], grad_scale=s["grad_scale"])
    return {"loss": loss, "logp": logp, "lse": lse, "dhidden": dhidden, "dhead": dhead}


def _own_adamw(s):
    from paper_2310_05205_amd import gear
    t = s["lists"]
    norm, factor = gear.grad_norm(t["grad"], max_norm=MAX_NORM)
    scales = None
    if s["case"]["bits"] == 8:
        scales = (t["exp_avg_scale"], t["exp_avg_sq_scale"])
    gear.adamw(t["param"], t["grad"], t["exp_avg"], t["exp_avg_sq"], s["step"], scales=scales, master=t.get("master"),
               lr=LR, betas=BETAS, eps=ADAM_EPS, weight_decay=DECAY, factor=factor)
    return dict({k: v for k, v in s["flat"].items() if k != "grad"}, step=s["step"], norm=norm, factor=factor)


_OWN = {"norm": _own_norm, "norm-train": _own_norm_train, "token": _own_token, "token-train": _own_token_train,
        "adamw": _own_adamw}


# --- plain torch operations in 32 bits --------------------------------------

def _plain_stats(total):
    t = total.float()
    mean = t.mean(-1, keepdim=True)
    d = t - mean
    rstd = 1.0 / torch.sqrt(d.square().mean(-1, keepdim=True) + EPS)
    return d * rstd, rstd


def _plain_norm(s):
    xhat, _ = _plain_stats(s["x"])
    return {"y": (xhat * s["weight"].float() + s["bias"].float()).to(s["x"].dtype)}


def _plain_norm_train(s):
    dt, wt = s["x"].dtype, s["weight"].dtype
    total = None if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(dt)
    w = s["weight"].float()
    xhat, rstd = _plain_stats(s["x"] if total is None else total)
    y = (xhat * w + s["bias"].float()).to(dt)
    dy = s["dy"].float()
    g = dy * w
    dx = (g - g.mean(-1, keepdim=True) - xhat * (g * xhat).mean(-1, keepdim=True)) * rstd
    if s["dtotal"] is not None:
        dx = dx + s["dtotal"].float()
    return {"y": y, "total": total, "dx": dx.to(dt), "dweight": (dy * xhat).sum(0).to(wt), "dbias": dy.sum(0).to(wt)}


def _plain_rows(s):
    z = s["hidden"].float() @ s["head"].float().t()
    top = z.amax(-1, keepdim=True)
    lse = (top + torch.log(torch.exp(z - top).sum(-1, keepdim=True)))[:, 0]
    logp = z.gather(1, s["target"].long()[:, None])[:, 0] - lse
    on = torch.ones_like(lse, dtype=torch.bool) if s["mask"] is None else s["mask"] != 0
    share = torch.where(on, s["weight"], 0.0) / on.sum().clamp(min=1).float()
    out = {"loss": -(share * logp).sum(), "logp": torch.where(on, logp, 0.0), "lse": torch.where(on, lse, 0.0)}
    return out, z, lse, share


def _plain_token(s):
    return _plain_rows(s)[0]


def _plain_token_train(s):
    out, z, lse, share = _plain_rows(s)
    g = torch.exp(z - lse[:, None])
    g.scatter_add_(1, s["target"].long()[:, None], torch.full_like(lse, -1.0)[:, None])
    g *= (share * s["grad_scale"])[:, None]
    dt = s["hidden"].dtype
    out["dhidden"] = (g @ s["head"].float()).to(dt)
    out["dhead"] = (g.t() @ s["hidden"].float()).to(dt)
    return out


def _in_8_bits(x):
    """Blocks of values as e4m3 under the block's own scale; what is not 0 stays not 0."""
    x = x.view(-1, BLOCK)
    scale = x.abs().amax(1) / TOP
    q = x / torch.where(scale > 0, scale, 1.0)[:, None]
    q = torch.where(x != 0, torch.copysign(q.abs().clamp(LEAST, TOP), q), 0.0)
    return q.to(torch.float8_e4m3fn).view(-1), scale


def _from_8_bits(q, scale):
    return (q.to(scale.dtype).view(-1, BLOCK) * scale[:, None]).view(-1)


def _plain_adamw(s):
    f, case = s["flat"], s["case"]
    g = f["grad"].float()
    norm = torch.sqrt(g.double().square().sum()).float()
    factor = torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)
    g = g * factor
    s["step"] += 1
    t = s["step"].double()
    c1, c2 = (1.0 - BETAS[0] ** t).float(), (1.0 - BETAS[1] ** t).float()
    if case["bits"] == 32:
        m, v = f["exp_avg"], f["exp_avg_sq"]
    else:
        m = _from_8_bits(f["exp_avg"], f["exp_avg_scale"])
        v = _from_8_bits(f["exp_avg_sq"], f["exp_avg_sq_scale"]).square()
    m = BETAS[0] * m + (1.0 - BETAS[0]) * g
    v = BETAS[1] * v + (1.0 - BETAS[1]) * g.square()
    p = f["master"] if case["master"] else f["param"].float()
    p = p * (1.0 - LR * DECAY) - LR * (m / c1) / (torch.sqrt(v / c2) + ADAM_EPS)
    if case["master"]:
        f["master"].copy_(p)
    f["param"].copy_(p)
    if case["bits"] == 32:
        f["exp_avg"].copy_(m)
        f["exp_avg_sq"].copy_(v)
    else:
        parts = _in_8_bits(m) + _in_8_bits(torch.sqrt(v))
        f["exp_avg"].copy_(parts[0])
        f["exp_avg_scale"].copy_(parts[1])
        f["exp_avg_sq"].copy_(parts[2])
        f["exp_avg_sq_scale"].copy_(parts[3])
    return dict({k: x for k, x in f.items() if k != "grad"}, step=s["step"], norm=norm, factor=factor)


_PLAIN = {"norm": _plain_norm, "norm-train": _plain_norm_train, "token": _plain_token, "token-train": _plain_token_train,
          "adamw": _plain_adamw}


# --- what a pass cannot do without ------------------------------------------

def work(case):
    size = DTYPES[case["dtype"]].itemsize
    if case["kind"] in ("norm", "norm-train"):
        n = case["rows"] * case["D"]
        par = (4 if case["wide"] else size) * case["D"]
        if case["kind"] == "norm":
            return {"bytes": 2 * size * n + 2 * par, "flops": 8 * n}
        # The rest of the model and its loss lie between the two calls, so the backward call reads the rows again.
        return {"bytes": size * n * (8 if case["residual"] else 5) + 5 * par + 16 * case["rows"], "flops": 24 * n}
    if case["kind"] in ("token", "token-train"):
        n, D, V = case["rows"], case["D"], case["V"]
        rows = n * (4 + 4 + 8 + (1 if case["mask"] else 0))
        if case["kind"] == "token":
            return {"bytes": size * (n + V) * D + rows, "flops": 2.0 * n * V * D}
        # Three products; the logits once more, which backward cannot have from forward, are not counted.
        return {"bytes": 3 * size * (n + V) * D + 2 * rows, "flops": 6.0 * n * V * D}
    n = sum(math.prod(x) for x in _shapes(case))
    state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (3 * size + (8 if case["master"] else 0) + state), "flops": 20 * n}


# --- the definitions in 64 bits ---------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("norm", "norm-train"):
        return _exact_norm(s)
    if case["kind"] in ("token", "token-train"):
        return _exact_token(s)
    return _exact_adamw(s)


def _exact_norm(s):
    x = s["x"].double()
    total = None
    if s["residual"] is not None:
        # The sum is rounded to the rows' type, and what is normalised is what was written.
        total = (x + s["residual"].double()).to(s["x"].dtype).double()
        x = total
    n, D = x.shape
    w = s["weight"].double()
    var, mean = torch.var_mean(x, dim=1, correction=0)
    sd = torch.sqrt(var + EPS)
    u = (x - mean[:, None]) / sd[:, None]
    out = {"y": torch.addcmul(s["bias"].double(), u, w)}
    if s["case"]["kind"] == "norm":
        return out
    dy = s["dy"].double()
    # Of the Jacobian (I - 1 1' / D - u u' / D) / sd of the normalisation.
    dw = dy * w
    along = (dw * u).sum(1) / D
    dx = (dw - dw.sum(1, keepdim=True) / D - along[:, None] * u) / sd[:, None]
    out["total"] = total
    out["dx"] = dx if s["dtotal"] is None else dx + s["dtotal"].double()
    out["dweight"], out["dbias"] = torch.einsum("nd,nd->d", dy, u), dy.sum(0)
    return out


def _exact_token(s):
    h, W, y = s["hidden"].double(), s["head"].double(), s["target"].long()
    n, V = h.shape[0], W.shape[0]
    keep = torch.ones(n, dtype=torch.float64, device="cuda") if s["mask"] is None else s["mask"].double()
    count = max(1.0, float(keep.sum()))
    z = torch.mm(h, W.t())
    lse = torch.logsumexp(z, 1)
    row = torch.arange(n, device="cuda")
    logp = z[row, y] - lse
    w = s["weight"].double() * keep / count
    out = {"loss": -(w * logp).sum(), "logp": keep * logp, "lse": keep * lse}
    if s["case"]["kind"] == "token-train":
        p = z.sub_(lse[:, None]).exp_()
        p[row, y] -= 1.0
        p *= (w * s["grad_scale"])[:, None]
        out["dhidden"], out["dhead"] = torch.mm(p, W), torch.mm(p.t(), h)
    return out


def _exact_adamw(s):
    f, case = s["flat"], s["case"]
    g = f["grad"].double()
    norm = torch.linalg.vector_norm(g)
    factor = 1.0 if float(norm) <= MAX_NORM else MAX_NORM / float(norm)
    t = int(s["step"]) + 1
    b1, b2 = BETAS
    if case["bits"] == 32:
        m, v = f["exp_avg"].double(), f["exp_avg_sq"].double()
    else:
        m = _from_8_bits(f["exp_avg"], f["exp_avg_scale"].double())
        v = _from_8_bits(f["exp_avg_sq"], f["exp_avg_sq_scale"].double()) ** 2
    g *= factor
    m.mul_(b1).add_(g, alpha=1 - b1)
    v.mul_(b2).addcmul_(g, g, value=1 - b2)
    p = (f["master"] if case["master"] else f["param"]).double() * (1 - LR * DECAY)
    p -= LR / (1 - b1 ** t) * m / (torch.sqrt(v) / math.sqrt(1 - b2 ** t) + ADAM_EPS)
    out = {"param": p, "norm": norm, "factor": torch.tensor(factor, dtype=torch.float64), "step": torch.tensor([t])}
    if case["master"]:
        out["master"] = p
    if case["bits"] == 32:
        out["exp_avg"], out["exp_avg_sq"] = m, v
    else:
        for name, x in (("exp_avg", m), ("exp_avg_sq", torch.sqrt(v))):
            x = x.view(-1, BLOCK)
            largest = x.abs().max(1).values
            a = x * TOP / largest.where(largest != 0, torch.ones_like(largest))[:, None]
            # e4m3 holds multiples of an eighth of the power of two below, of 2^-9 at least.
            ulp = torch.exp2(torch.floor(torch.log2(a.abs().clamp(min=2.0 ** -6))) - 3)
            q = torch.round(a / ulp) * ulp
            q[(q == 0) & (a > 0)], q[(q == 0) & (a < 0)] = LEAST, -LEAST
            out[name], out[name + "_scale"] = q.view(-1), largest / TOP
    return out
