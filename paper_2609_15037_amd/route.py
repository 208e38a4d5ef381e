"""Expert routing for torch models over the library's operators (moara_route, its backward pass and the
balancing bias's step).

    router = ExpertRouter(d_model, experts=64, top_k=6)
    index, weight = router(x)               # tokens x top_k; differentiable in x and the router's weight
    load = router.load()                    # tokens of each expert since the last balance(), on the host (training)
    loss.backward(); opt.step()
    router.balance(1e-3)                    # moves the bias, starts the counts again

An expert without tokens has no gradient: the MoARa optimizer skips its matrices. Data-parallel ranks add up
`router.counts` (int64) before balance().
"""
from __future__ import annotations

from typing import Optional, Tuple

import numpy as np
import torch

from . import moara as M


class _Route(torch.autograd.Function):
    @staticmethod
    def forward(ctx, logits, cfg, bias, mask, counts):
        cfg = M.moara_route_config.from_buffer_copy(cfg)        # the caller may change its own before the backward pass
        index, weight = M.moara_route(cfg, logits, bias=bias, mask=mask, counts=counts)
        ctx.cfg = cfg
        ctx.save_for_backward(logits, index)
        ctx.mark_non_differentiable(index)
        return index, weight

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, _, grad_weight):
        logits, index = ctx.saved_tensors
        grad = M.moara_route_backward(ctx.cfg, logits, index, grad_weight.float().contiguous())
        return grad, None, None, None, None


def route(logits: torch.Tensor, cfg: M.moara_route_config, bias: Optional[torch.Tensor] = None,
          mask: Optional[torch.Tensor] = None, counts: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Indices and weights (tokens x top_k) of the experts of each row of logits; differentiable in the logits."""
    return _Route.apply(logits, cfg, bias, mask, counts)


class ExpertRouter(torch.nn.Module):
    """A linear router: fp32 logits of each token, its top_k experts and their weights.

    Keyword arguments are moara_route_config's (groups, top_groups, group_best, score, renormalise, scale).
    `bias` (a buffer) only takes part in the choice; it moves with balance(). `counts` are those of training: evaluation
    passes (`eval()`) and the forward passes that activation checkpointing repeats in a backward pass add nothing."""

    def __init__(self, d_model: int, experts: int, top_k: int, **config):
        super().__init__()
        self.cfg = M.moara_route_default_config(experts=experts, top_k=top_k, **config)
        self.weight = torch.nn.Parameter(torch.randn(experts, d_model) * d_model ** -0.5)
        self.register_buffer("bias", torch.zeros(experts, dtype=torch.float32))
        # a tensor but no buffer: DistributedDataParallel gives every rank the first one's buffers at each forward
        # pass, and a rank's counts are its own
        self.counts = torch.zeros(experts, dtype=torch.int64)

    def _apply(self, fn, recurse=True):
        """Casts of the model (`.bfloat16()`, `.to(dtype)`) leave the bias in fp32: it moves by 1e-3 a step."""
        bias = self.bias
        super()._apply(fn, recurse)
        if self.bias.dtype != torch.float32:
            self.bias = bias.to(self.bias.device)
        at = self.bias.device
        self.counts = torch.zeros_like(self.counts, device=at) if self.counts.is_meta else self.counts.to(at)
        return self

    def _save_to_state_dict(self, destination, prefix, keep_vars):
        super()._save_to_state_dict(destination, prefix, keep_vars)
        destination[prefix + "counts"] = self.counts

    def _load_from_state_dict(self, state_dict, prefix, local_metadata, strict, missing_keys, unexpected_keys, error_msgs):
        super()._load_from_state_dict(state_dict, prefix, local_metadata, strict, missing_keys, unexpected_keys, error_msgs)
        key = prefix + "counts"
        if key in unexpected_keys:
            unexpected_keys.remove(key)
        saved = state_dict.get(key)
        if saved is None:
            if strict:
                missing_keys.append(key)
        elif saved.shape != self.counts.shape:
            error_msgs.append(f"size mismatch for {key}: {tuple(saved.shape)}, the router has {tuple(self.counts.shape)}")
        elif local_metadata.get("assign_to_params_buffers", False):
            self.counts = saved
        else:
            self.counts.copy_(saved)

    def forward(self, x: torch.Tensor, mask: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
        """x: tokens x d_model; mask: tokens, False where a token is not routed. An index is -1 (weight 0)
        where there is no expert."""
        with torch.autocast(x.device.type, enabled=False):      # the choice is sensitive to the logits' rounding
            logits = torch.nn.functional.linear(x.float(), self.weight.float())
        if self.counts.device != x.device:      # where buffers are moved one by one
            self.counts = self.counts.to(x.device)
        again = torch._C._current_graph_task_id() != -1         # inside a backward pass
        return route(logits, self.cfg, self.bias, mask, self.counts if self.training and not again else None)

    def load(self) -> np.ndarray:
        """Tokens of each expert in training since the last balance() (waits for the GPU)."""
        return self.counts.cpu().numpy()

    def balance(self, rate: float) -> None:
        """Moves the bias by `rate` towards an even load and sets the counts to zero."""
        M.moara_route_balance(self.counts, self.bias, rate)
