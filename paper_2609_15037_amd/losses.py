"""Losses of a training step for torch models over the library's operators: log-probabilities of given tokens, losses
of paired responses and of a clipped policy over them, and the load-balancing loss of expert routing.

    logp = token_logps(model(tokens)[:, :-1], tokens[:, 1:])            # batch x tokens, differentiable in the logits
    loss, rewards, about = preference_loss(M.moara_preference_default_config(beta=0.1), logp, ref_logp, mask=mask)
    loss.backward()

    logp, entropy = token_logps(logits, labels, entropy=True)
    cfg = M.moara_policy_default_config(kl_coef=0.04, entropy_coef=0.01, sequence_advantages=1)
    loss, about = policy_loss(cfg, logp, advantages, old_logp=old, ref_logp=ref, entropy=entropy, mask=mask)

Sequences are rows, or packed one after another with their offsets (sequences + 1 integers). A mask is bool or integers, of
any layout (`mask[:, 1:]` beside `logits[:, :-1]`); a token with 0 is left out. Losses are scalars on the GPU; nothing is
copied to the host, and a step can be captured into a graph, its backward pass too. As with any torch operator, first drop
what was computed eagerly from the same parameters (losses of warm-up steps that are still held): their gradients'
accumulation belongs to the stream of that time, which a capture cannot wait for.
Gradients of the gradients are refused.
"""
from __future__ import annotations

import functools
from typing import Optional, Tuple

import torch

from . import moara as M


def _plain(t: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """A tensor without a gradient, float32 and contiguous."""
    return None if t is None else _rows(t.detach() if t.requires_grad else t)


def _rows(t: torch.Tensor) -> torch.Tensor:
    return t if t.dtype is torch.float32 and t.is_contiguous() else t.float().contiguous()


def _mask(mask: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """A mask as the library takes it: contiguous, bool or uint8. Integers are live where they are not 0; of floating point 0
    could as well be what is added to a live token's score."""
    if mask is None or (mask.dtype in (torch.bool, torch.uint8) and mask.is_contiguous()):
        return mask
    if mask.is_floating_point() or mask.is_complex():
        raise ValueError(f"mask: need bool or integers, got {mask.dtype}")
    return (mask if mask.dtype is torch.bool else mask.ne(0)).contiguous()


def _offsets(offsets: Optional[torch.Tensor]) -> Optional[torch.Tensor]:
    """Offsets as the library takes them: contiguous, int64."""
    if offsets is None or (offsets.dtype is torch.int64 and offsets.is_contiguous()) or offsets.is_floating_point():
        return offsets          # the library refuses the last
    return offsets.to(torch.int64).contiguous()


class _Last(torch.autograd.Function):
    """A gradient that may be used, but not differentiated again."""
    @staticmethod
    def forward(ctx, grad, source):
        return grad.view_as(grad)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("the library's losses have no gradient of their gradient")


def _once(backward):
    """For a backward pass that has none of its own. Where a second one may be asked for (create_graph), asking is an error,
    also if what came in is a constant: the gradient is none."""
    @functools.wraps(backward)
    def call(ctx, *grads):
        if not torch.is_grad_enabled():
            return backward(ctx, *grads)
        with torch.no_grad():
            out = backward(ctx, *grads)
        source = torch.zeros((), requires_grad=True)
        last = lambda g: None if g is None else _Last.apply(g, source)      # noqa: E731
        return tuple(map(last, out)) if isinstance(out, tuple) else last(out)
    return call


class _TokenLogps(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, labels, scale, entropy):
        logp, bits, stats = M.moara_token_logps(logits, labels, scale=scale, entropy=entropy)
        ctx.scale = scale
        ctx.set_materialize_grads(False)
        ctx.save_for_backward(logits, labels, stats, bits)
        return (logp, bits) if entropy else logp

    @staticmethod
    @_once
    def backward(ctx, grad_logp, grad_entropy=None):
        if grad_logp is None and grad_entropy is None:
            return None, None, None, None
        logits, labels, stats, bits = ctx.saved_tensors
        g = stats.new_zeros(labels.shape) if grad_logp is None else grad_logp.contiguous()
        h = None if grad_entropy is None else grad_entropy.contiguous()
        grad = M.moara_token_logps_backward(logits, labels, stats, g, scale=ctx.scale, entropy=None if h is None else bits,
                                            grad_entropy=h)
        return grad, None, None, None


def token_logps(logits: torch.Tensor, labels: torch.Tensor, temperature: float = 1.0, entropy: bool = False):
    """Log-probabilities (float32) of the labels under logits / temperature, and with `entropy` the distributions'
    entropies: both of the labels' shape, the logits' without the last axis. Differentiable in the logits (float32 or
    bfloat16; a view such as `logits[:, :-1]` is not copied). A label outside the vocabulary, e.g. -100, has 0 and no
    gradient: all the logits with such labels where a token is not wanted spare the copy that a view's gradient is put
    into the whole logits' with."""
    if labels.shape != logits.shape[:-1]:
        raise ValueError(f"labels: shape {tuple(labels.shape)}, the logits have {tuple(logits.shape)}")
    flat = logits if logits.dim() in (2, 3) else logits.reshape(-1, logits.shape[-1])
    at = labels
    if at.dtype is not torch.int64 or flat is not logits or not at.is_contiguous():
        at = at.to(torch.int64).reshape(flat.shape[:-1]).contiguous()
    out = _TokenLogps.apply(flat, at, 1.0 / temperature, entropy)
    if flat is logits:
        return out
    return tuple(x.reshape(labels.shape) for x in out) if entropy else out.reshape(labels.shape)


class _Preference(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logp, cfg, ref_logp, offsets, mask):
        cfg = M.moara_preference_config.from_buffer_copy(cfg)       # the caller may change its own before the backward pass
        loss = logp.new_empty(())           # by itself: callers may change it in place
        out, rewards, slope = M.moara_preference_loss(cfg, logp, ref_logp, offsets=offsets, mask=mask, loss=loss)
        ctx.cfg = cfg
        ctx.save_for_backward(logp, slope, offsets, mask)
        ctx.mark_non_differentiable(rewards, out)
        return loss, rewards, out

    @staticmethod
    @_once
    def backward(ctx, grad, *_):
        logp, slope, offsets, mask = ctx.saved_tensors
        return M.moara_preference_loss_backward(ctx.cfg, logp, slope, grad.contiguous(), offsets=offsets, mask=mask), \
            None, None, None, None


def preference_loss(cfg: M.moara_preference_config, logp: torch.Tensor, ref_logp: Optional[torch.Tensor] = None,
                    offsets: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None) \
        -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(loss, rewards, about) of pairs of responses, sequences 2p (chosen) and 2p + 1 (rejected); differentiable in logp.
    rewards: one for each sequence; about: loss, share of the pairs with the chosen one ahead, mean difference of their
    rewards. logp, ref_logp, mask: sequences x length, or flat with offsets."""
    return _Preference.apply(_rows(logp), cfg, _plain(ref_logp), _offsets(offsets), _mask(mask))


class _Policy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logp, entropy, cfg, advantages, old_logp, ref_logp, offsets, mask):
        cfg = M.moara_policy_config.from_buffer_copy(cfg)
        loss = logp.new_empty(())
        out, weight = M.moara_policy_loss(cfg, logp, advantages, old_logp=old_logp, ref_logp=ref_logp, entropy=entropy,
                                          offsets=offsets, mask=mask, loss=loss)
        ctx.cfg = cfg
        ctx.save_for_backward(logp, entropy, advantages, weight, old_logp, ref_logp, offsets, mask)
        ctx.mark_non_differentiable(out)
        return loss, out

    @staticmethod
    @_once
    def backward(ctx, grad, _):
        logp, entropy, advantages, weight, old_logp, ref_logp, offsets, mask = ctx.saved_tensors
        if not ctx.needs_input_grad[1]:
            entropy = None
        g, h = M.moara_policy_loss_backward(ctx.cfg, logp, advantages, weight, grad.contiguous(), old_logp=old_logp,
                                            ref_logp=ref_logp, entropy=entropy, offsets=offsets, mask=mask)
        return g, h, None, None, None, None, None, None


def policy_loss(cfg: M.moara_policy_config, logp: torch.Tensor, advantages: torch.Tensor,
                old_logp: Optional[torch.Tensor] = None, ref_logp: Optional[torch.Tensor] = None,
                entropy: Optional[torch.Tensor] = None, offsets: Optional[torch.Tensor] = None,
                mask: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(loss, about) of a clipped policy; differentiable in logp and entropy. about: loss, policy term, distance to the
    reference, entropy, share of clipped tokens, distance to the old policy. logp, old_logp (None: the policy is the one
    that sampled), ref_logp, entropy, mask: sequences x length, or flat with offsets; advantages alike, or one for each
    sequence where cfg.sequence_advantages."""
    return _Policy.apply(_rows(logp), None if entropy is None else _rows(entropy), cfg, _plain(advantages), _plain(old_logp),
                         _plain(ref_logp), _offsets(offsets), _mask(mask))


class _Balance(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, cfg, index, offsets, mask, load, sequences):
        cfg = M.moara_balance_config.from_buffer_copy(cfg)
        loss = logits.new_empty((), dtype=torch.float32)
        out, counts, slope = M.moara_balance_loss(cfg, logits, index, offsets=offsets, mask=mask, load=load, sequences=sequences,
                                                  loss=loss)
        ctx.cfg, ctx.sequences = cfg, sequences
        ctx.save_for_backward(logits, slope, offsets, mask)
        ctx.mark_non_differentiable(counts, out)
        return loss, counts, out

    @staticmethod
    @_once
    def backward(ctx, grad, *_):
        logits, slope, offsets, mask = ctx.saved_tensors
        return M.moara_balance_loss_backward(ctx.cfg, logits, slope, grad.contiguous(), offsets=offsets, mask=mask,
                                             sequences=ctx.sequences), None, None, None, None, None, None


def balance_loss(cfg: M.moara_balance_config, logits: torch.Tensor, index: torch.Tensor,
                 offsets: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None,
                 load: Optional[torch.Tensor] = None, sequences: Optional[int] = None) \
        -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(loss, counts, about) of the routing of tokens to experts; differentiable in the logits. index: as routing gave it;
    counts: each expert's tokens by sequence (int64); about: loss, mean balance, z. Each of the packed (offsets) or equal
    (`sequences`) sequences is balanced for itself; without either all tokens together. load: counts that take the
    place of this call's, e.g. those of all ranks."""
    return _Balance.apply(logits, cfg, index, _offsets(offsets), _mask(mask), load, sequences)
