"""The learner's operators as differentiable torch functions, and its optimizer.

``recurrence``, ``policy_loss``, ``layer_norm`` and ``token_loss`` here take
what their namesakes in ``gear`` take and record a gradient; every step, forward
and backward, runs in the HIP library.  ``advantages`` and ``action_logp`` need
no gradient: see ``gear``.  ``AdamW`` steps a model's parameters by ``gear.adamw``.

A backward pass that is captured into a HIP graph must not meet leaves that an eager
autograd graph still holds (torch's rule: it ends the process); the calls in ``gear``
are captured without one.
"""
import torch

from . import gear


class _Recurrence(torch.autograd.Function):
    @staticmethod
    def forward(ctx, gate, x, state, form, reset, lengths):
        y, final, saved = gear.recurrence(gate, x, state, form=form, reset=reset, lengths=lengths, save=True)
        ctx.save_for_backward(gate, x, state, reset, lengths, saved)
        ctx.form = form
        ctx.set_materialize_grads(False)
        return y, final

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dfinal):
        gate, x, state, reset, lengths, saved = ctx.saved_tensors
        if dy is not None and dy.dim() and dy.stride(-1) != 1:
            dy = dy.contiguous()  # a gradient broadcast from a sum, say
        if dfinal is not None:
            dfinal = dfinal.contiguous()
        dgate, dx, dstate = gear.recurrence_backward(gate, x, saved, dy, dfinal, state, form=ctx.form, reset=reset,
                                                     lengths=lengths)
        return (dgate if ctx.needs_input_grad[0] else None, dx if ctx.needs_input_grad[1] else None,
                dstate if ctx.needs_input_grad[2] else None, None, None, None)


def recurrence(gate, x, state=None, *, form=gear.GEAR_GATE_VALUE, reset=None, lengths=None):
    """(y, final state) of gear.recurrence, differentiable in gate, x and state."""
    return _Recurrence.apply(gate, x, state, form, reset, lengths)


class _PolicyLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, action, old_logp, adv, ref_logp, weight, mask, clip, kl, entropy, denom):
        loss, logp, ent, stats, _ = gear.policy_loss(logits, action, old_logp, adv, ref_logp=ref_logp, weight=weight,
                                                     mask=mask, clip=clip, kl=kl, entropy=entropy, denom=denom, grad=False)
        ctx.save_for_backward(logits, action, old_logp, adv, ref_logp, weight, mask)
        ctx.terms = clip, kl, entropy, denom
        ctx.mark_non_differentiable(logp, ent, stats)
        return loss, logp, ent, stats

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss, *_):
        logits, action, old_logp, adv, ref_logp, weight, mask = ctx.saved_tensors
        clip, kl, entropy, denom = ctx.terms
        grad = gear.policy_loss(logits, action, old_logp, adv, ref_logp=ref_logp, weight=weight, mask=mask, clip=clip, kl=kl,
                                entropy=entropy, denom=denom, grad_loss=dloss)[4]
        return (grad,) + (None,) * 10


def policy_loss(logits, action, old_logp, adv, *, ref_logp=None, weight=None, mask=None, clip=(0.2, 0.2), kl=0.0,
                entropy=0.0, denom=None):
    """(loss, logp, entropy, stats) of gear.policy_loss, the loss differentiable
    in the logits.  The backward call reads the logits again and multiplies by the
    loss's own gradient before it rounds, so a loss scale serves 16-bit logits.  A
    program whose loss is this alone saves that reading: gear.policy_loss gives
    loss and gradient at once, for ``logits.backward(grad)``.
    """
    return _PolicyLoss.apply(logits, action, old_logp, adv, ref_logp, weight, mask, clip, kl, entropy, denom)


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, residual):
        y, total, saved = gear.layer_norm(x, weight, bias, eps=eps, residual=residual, save=True)
        ctx.save_for_backward(x if total is None else total, weight, saved)
        ctx.set_materialize_grads(False)
        return y if total is None else (y, total)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy, dtotal=None):
        t, weight, saved = ctx.saved_tensors
        need = ctx.needs_input_grad
        if dy is None:
            return dtotal, None, None, None, dtotal if need[4] else None
        # Gradients broadcast from a sum, say, or turned.
        dy, dtotal = dy.contiguous(), None if dtotal is None else dtotal.contiguous()
        dx, dweight, dbias = gear.layer_norm_backward(dy, t, saved, weight, dtotal=dtotal)
        return (dx if need[0] else None, dweight if need[1] else None, dbias if need[2] else None, None,
                dx if need[4] else None)


def layer_norm(x, weight=None, bias=None, *, eps=1e-5, residual=None):
    """y of gear.layer_norm, or (y, total) with a residual, differentiable in x,
    weight, bias and residual."""
    return _LayerNorm.apply(x, weight, bias, eps, residual)


class _TokenLoss(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, head, target, weight, mask, denom):
        loss, logp, lse = gear.token_loss(hidden, head, target, weight=weight, mask=mask, denom=denom)
        ctx.save_for_backward(hidden, head, target, weight, mask, lse)
        ctx.denom = denom
        ctx.mark_non_differentiable(logp, lse)
        return loss, logp, lse

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dloss, *_):
        hidden, head, target, weight, mask, lse = ctx.saved_tensors
        dhidden, dhead = gear.token_loss_backward(hidden, head, target, lse, weight=weight, mask=mask, denom=ctx.denom,
                                                  grad_loss=dloss, dhidden=ctx.needs_input_grad[0],
                                                  dhead=ctx.needs_input_grad[1])
        return dhidden, dhead, None, None, None, None


def token_loss(hidden, head, target, *, weight=None, mask=None, denom=None):
    """(loss, logp, lse) of gear.token_loss, the loss differentiable in hidden and
    head.  The loss's own gradient multiplies theirs before they are rounded, so a loss
    scale serves 16-bit types."""
    return _TokenLoss.apply(hidden, head, target, weight, mask, denom)


def _versions(params):
    """What a write to a parameter counts up; tensors of inference mode have none."""
    try:
        return [p._version for p in params]
    except RuntimeError:
        return [None if p.is_inference() else p._version for p in params]


class AdamW:
    """AdamW over a model's parameters, each step one call for all of them.

    params: tensors on one GPU, contiguous.  With bits=8 the averages are held in
    8 bits (gear.adamw).  A value whose gradient is 0 from some step on comes to rest;
    where it only turns small, the first average is rounded to nearest and may stay: at up to
    2^-15 of its block's largest with betas[0] of 0.9, at any size from 0.95 on.
    16-bit parameters step as float32 masters, which `master`
    turns off.  max_norm clips the gradients' common norm.  lr is a number or a
    float32 tensor of one value on the GPU, and may be set between steps.  Parameters
    without a gradient stay as they are; the count of steps is one for all.  A step
    whose gradients are not finite is left out, on the device, where norm or scale
    are asked for.

    A parameter that the program writes between steps (a model's state that is
    loaded, a reset) is what the next step starts from: values that differ from their
    rounded masters take the masters' place.  step() and state_dict() look for that by
    the parameter's version and address.  A write through ``.data`` changes neither, and the
    replay of a captured step looks for nothing: call refresh() after the one and
    before the other.
    """

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, *, bits=32, master=True,
                 max_norm=None):
        if isinstance(params, torch.Tensor):
            raise TypeError("params must be a list of tensors, not one, whose rows have no gradients")
        self.params = list(params)
        if not self.params:
            raise ValueError("no parameters")
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        for p in self.params:
            if not p.is_contiguous():
                raise ValueError("parameters must be contiguous")
        self.lr, self.betas, self.eps, self.weight_decay = lr, betas, eps, weight_decay
        self.bits, self.max_norm = bits, max_norm
        device = self.params[0].device
        self.count = torch.zeros(1, dtype=torch.int64, device=device)
        kind = torch.float8_e4m3fn if bits == 8 else torch.float32
        # One buffer for each average; the tensors' parts begin at whole blocks.
        block = gear.GEAR_STEP_BLOCK
        blocks = [(p.numel() + block - 1) // block for p in self.params]
        self._avg, self._scale = [], []
        for _ in range(2):
            flat = torch.zeros(sum(blocks) * block, dtype=torch.uint8 if bits == 8 else kind, device=device).view(kind)
            self._avg.append([c[:p.numel()] for c, p in zip(flat.split([b * block for b in blocks]), self.params)])
            if bits == 8:
                self._scale.append(list(torch.zeros(sum(blocks), device=device).split(blocks)))
        self._master = [p.detach().float() if master and p.dtype != torch.float32 else None for p in self.params]
        # Parameters with masters, where they lie and their versions, as the masters were last in line with them.
        self._held = [i for i, m in enumerate(self._master) if m is not None]
        self._places, self._versions = [p.data_ptr() for p in self.params], _versions(self.params)

    def refresh(self):
        """Takes what was written to parameters since the last step into their masters."""
        self._refresh(self._held)

    def _refresh(self, at):
        with torch.no_grad():
            for i in at:
                p, m = self.params[i], self._master[i]
                m.copy_(torch.where(m.to(p.dtype) == p, m, p.float()))
                self._places[i], self._versions[i] = p.data_ptr(), _versions([p])[0]

    def _refresh_changed(self):
        held = [self.params[i] for i in self._held]
        places, versions = [p.data_ptr() for p in held], _versions(held)
        self._refresh([i for i, place, version in zip(self._held, places, versions)
                       if version != self._versions[i] or place != self._places[i]])

    def step(self, scale=1.0):
        """Steps every parameter that has a gradient, the gradients times `scale` (1
        over a loss scale).  Returns their norm after that, on the device, where
        max_norm or scale ask for it, else None."""
        at = [i for i, p in enumerate(self.params) if p.grad is not None]
        if not at:
            return None
        self._refresh_changed()
        params = [self.params[i].detach() for i in at]
        grads = [self.params[i].grad.contiguous() for i in at]
        norm = factor = None
        if self.max_norm is not None or scale != 1.0:
            norm, factor = gear.grad_norm(grads, max_norm=self.max_norm, scale=scale)
        pick = lambda v: [v[i] for i in at]  # noqa: E731
        gear.adamw(params, grads, pick(self._avg[0]), pick(self._avg[1]), self.count, lr=self.lr, betas=self.betas,
                   eps=self.eps, weight_decay=self.weight_decay,
                   scales=(pick(self._scale[0]), pick(self._scale[1])) if self.bits == 8 else None,
                   master=pick(self._master), factor=factor)
        if self._held:
            self._versions = _versions(self.params)  # which the step counted up
        return norm

    def zero_grad(self):
        for p in self.params:
            p.grad = None

    def _state(self):
        names = {"exp_avg": self._avg[0], "exp_avg_sq": self._avg[1], "master": self._master}
        if self.bits == 8:
            names.update(exp_avg_scale=self._scale[0], exp_avg_sq_scale=self._scale[1])
        return names

    def state_dict(self):
        """Copies of the count of steps, averages, scales and masters; not lr and its like."""
        self._refresh_changed()
        state = {k: [None if t is None else t.clone() for t in v] for k, v in self._state().items()}
        return dict(state, count=self.count.clone())

    def load_state_dict(self, state):
        """Takes what state_dict() of an optimizer over like parameters gave.  The parameters
        stay as they are, and count where they differ from their rounded masters: load
        the model's state too, before or after."""
        mine = dict(self._state(), count=[self.count])
        state = dict(state, count=[state["count"]])
        if set(mine) != set(state):
            raise ValueError("the state is of an optimizer with other averages")
        for k, v in mine.items():
            same = len(v) == len(state[k]) and all(
                (a is None) == (b is None) and (a is None or (a.dtype, a.shape) == (b.dtype, b.shape))
                for a, b in zip(v, state[k]))
            if not same:
                raise ValueError("the state is of an optimizer over other parameters")
        with torch.no_grad():
            for k, v in mine.items():
                for a, b in zip(v, state[k]):
                    if a is not None:
                        a.copy_(b)
        self._places = [None] * len(self.params)  # masters may differ from the parameters' last ones
