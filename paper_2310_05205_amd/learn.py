"""The learner's operators as differentiable torch functions.

``recurrence`` and ``policy_loss`` here take what their namesakes in ``gear``
take and record a gradient; every step, forward and backward, runs in the HIP
library.  ``advantages`` and ``action_logp`` need no gradient: see ``gear``.
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
