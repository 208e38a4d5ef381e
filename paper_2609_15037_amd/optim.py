"""torch.optim integration of the MoARa library (training-loop use).

MoARa updates the projected weights: the attention q/k/v/o and MLP gate/up/down
matrices of every layer (and MoE experts), each with its module's rank, by the
library's step (`moara_step`: decomposition, projection, Adam on the projected
moments and the magnitudes, back-projection, scaled update, projector refresh
every `refresh_interval` steps). Every other parameter (embeddings, norms, the
output head) takes plain AdamW with the same betas and eps, as in the paper's
training setup (Appendix D: AdamW beta = (0.9, 0.999), eps = 1e-6, zero weight
decay, bias correction, GaLore scale 0.25 and T = 200).

The learning rate of both groups comes from `param_groups`, so torch's LR
schedulers drive it; `warmup_cosine` gives the paper's schedule (10 % linear
warmup, cosine decay to 0.1 of the peak). Gradient clipping (the paper clips at
1.0 for 7B) is the training loop's (`torch.nn.utils.clip_grad_norm_`, before
`step()`), or `step()`'s own with `max_grad_norm`: the library's norm over every
gradient, without a copy to the host.

The AdamW step of the other parameters is torch's by default. `adamw_bits = 32` or
`8` takes the library's instead: all tensors in a launch or two, moments in fp32
whatever the parameters' type, or in 8 bits (2.06 bytes a parameter for both).

    targets, others = moara_targets(model)          # [(param, module id)], [param]
    opt = MoARa(targets, others, lr=1e-2, rank_table=..., block_size=64)
    sched = torch.optim.lr_scheduler.LambdaLR(opt, warmup_cosine(total_steps))
    loss.backward(); opt.step(); sched.step(); opt.zero_grad()

Gradients of a bf16 model's projected weights go to the library as they are, with fp32
buffers the optimizer owns for the kernels that take fp32 only. The library's
kernels do all the work on the projected weights; this module only marshals.
"""
from __future__ import annotations

import copy
import math
from typing import Dict, Iterable, List, Optional, Sequence, Tuple

import numpy as np
import torch

from . import moara as M

# module ids of the usual Llama / Qwen / DeepSeek parameter names (last two name parts);
# MLP projections inside an MoE expert ("...experts.3.gate_proj.weight",
# "...shared_experts.up_proj.weight") take the expert types
_MODULE_OF = {
    "q_proj": M.MOARA_Q, "k_proj": M.MOARA_K, "v_proj": M.MOARA_V, "o_proj": M.MOARA_O,
    "gate_proj": M.MOARA_GATE, "up_proj": M.MOARA_UP, "down_proj": M.MOARA_DOWN,
}
_EXPERT_OF = {M.MOARA_GATE: M.MOARA_EXP_GATE, M.MOARA_UP: M.MOARA_EXP_UP, M.MOARA_DOWN: M.MOARA_EXP_DOWN}


def moara_targets(model: torch.nn.Module) -> Tuple[List[Tuple[torch.nn.Parameter, int]], List[torch.nn.Parameter]]:
    """Split a model's trainable parameters into MoARa targets, (weight, module id) for the
    q/k/v/o/gate/up/down projection weights (`*.q_proj.weight` and so on; expert types for
    MLP projections under a module path containing "expert"), and the rest."""
    targets, others = [], []
    for name, p in model.named_parameters():
        if not p.requires_grad:
            continue
        parts = name.split(".")
        mod = _MODULE_OF.get(parts[-2]) if len(parts) >= 2 and parts[-1] == "weight" and p.dim() >= 2 else None
        if mod is not None and any("expert" in q for q in parts[:-2]):
            mod = _EXPERT_OF.get(mod, mod)
        if mod is None:
            others.append(p)
        else:
            targets.append((p, mod))
    return targets, others


def warmup_cosine(total_steps: int, warmup_frac: float = 0.1, min_ratio: float = 0.1):
    """LR factor for torch.optim.lr_scheduler.LambdaLR: linear warmup over the first
    `warmup_frac` of the steps, then cosine decay from 1 to `min_ratio` (Appendix D)."""
    warm = max(1, int(round(warmup_frac * total_steps)))

    def f(step: int) -> float:
        if step < warm:
            return (step + 1) / warm
        t = min(1.0, (step - warm) / max(1, total_steps - warm))
        return min_ratio + (1.0 - min_ratio) * 0.5 * (1.0 + math.cos(math.pi * t))
    return f


def _order(t_shape: Sequence[int], stride: Sequence[int]) -> List[int]:
    """What says in which order the elements of a tensor without gaps lie: the strides of its axes, those of one
    element aside."""
    return [s for n, s in zip(t_shape, stride) if n != 1]


class _AdamW:
    """The library's AdamW over a list of parameters: their moments, and each one's step count (parameters
    without a gradient are not stepped).

    Moments lie in the order that the parameter's elements had when they were made (`form`: its shape and strides;
    saved with them). A parameter whose strides are others by now is stepped through a copy in that order: 8-bit
    moments share a scale with their neighbours in memory and cannot be moved without rounding them again."""

    def __init__(self, params: Sequence[torch.nn.Parameter], cfg: M.moara_adamw_config, weight_decay: float, seed: int):
        self.params, self.cfg, self.weight_decay, self.seed = list(params), cfg, float(weight_decay), int(seed)
        self.steps = np.zeros(len(self.params), dtype=np.int64)
        self.calls = 0
        self.state = None
        self.form: List[Tuple[Tuple[int, ...], Tuple[int, ...]]] = []

    def _make(self) -> None:
        if self.state is None:
            form = [(tuple(p.shape), p.stride()) for p in self.params]
            for i, p in enumerate(self.params):
                if not M._dense(p):
                    raise ValueError(f"parameter {i}: strides {p.stride()} of shape {tuple(p.shape)} leave gaps")
            self.state, self.form = [M.moara_adamw_state(p, self.cfg.bits) for p in self.params], form

    def step(self, lr: float, clip: Optional[torch.Tensor]) -> None:
        self._make()
        params, grads, copies = list(self.params), [p.grad for p in self.params], []
        strided = torch.strided
        for i, (p, g) in enumerate(zip(self.params, grads)):    # the usual case is a few attribute reads
            if g is None:
                continue
            stride = p.stride()
            if stride != self.form[i][1]:
                shape, made = self.form[i]
                if p.shape != shape:
                    raise ValueError(f"parameter {i} has shape {tuple(p.shape)}, its moments {shape}")
                if _order(shape, stride) != _order(shape, made):
                    params[i] = p = torch.empty_strided(shape, made, dtype=p.dtype, device=p.device).copy_(p)
                    stride = made
                    copies.append(i)
            if g.layout is not strided or g.stride() != stride:
                grads[i] = torch.empty_like(p, dtype=g.dtype).copy_(g if g.layout is strided else g.to_dense())
        args = M.AdamWArgs(params, grads, *([s[k] for s in self.state] for k in (0, 1)),
                           scales=[s[2] for s in self.state] if self.cfg.bits == 8 else None,
                           weight_decay=[self.weight_decay if p.dim() > 1 else 0.0 for p in self.params])
        self.steps += np.array([g is not None for g in grads])
        self.calls += 1
        M.moara_adamw_step(args, self.cfg, lr, np.maximum(self.steps, 1), clip=clip,
                           seed=(self.seed << 32) + self.calls)
        for i in copies:
            self.params[i].copy_(params[i])

    def state_dict(self) -> Dict:
        self._make()
        return {"bits": self.cfg.bits, "steps": self.steps.tolist(), "calls": self.calls, "seed": self.seed,
                "form": [[list(shape), list(stride)] for shape, stride in self.form],
                "state": [[None if t is None else t.cpu().clone() for t in s] for s in self.state]}

    def load_state_dict(self, sd: Dict) -> None:
        if sd["bits"] != self.cfg.bits or len(sd["state"]) != len(self.params):
            raise ValueError(f"the state is of {len(sd['state'])} parameters with moments of {sd['bits']} bits, the optimizer "
                             f"has {len(self.params)} with {self.cfg.bits}")
        self._make()
        # a state without its form is in the order of the parameters' elements
        form = [(tuple(shape), tuple(stride)) for shape, stride in
                sd.get("form") or [(p.shape, p.stride()) for p in self.params]]
        # all of it is looked at before any of it is taken
        if len(form) != len(self.params) or len(sd["steps"]) != len(self.params):
            raise ValueError("the state's steps or shapes are not one for each parameter")
        for i, (s, saved) in enumerate(zip(self.state, sd["state"])):
            if form[i][0] != tuple(self.params[i].shape):
                raise ValueError(f"the state of parameter {i} is of shape {form[i][0]}, the parameter of "
                                 f"{tuple(self.params[i].shape)}")
            if [None if t is None else t.shape for t in s] != [None if x is None else x.shape for x in saved]:
                raise ValueError(f"the state of parameter {i} has not as many elements as its moments")
        for s, saved in zip(self.state, sd["state"]):
            for t, x in zip(s, saved):
                if t is not None:
                    t.copy_(x)
        self.form = form
        self.steps[:] = sd["steps"]
        self.calls, self.seed = int(sd["calls"]), int(sd["seed"])


class MoARa(torch.optim.Optimizer):
    """MoARa for the projected weights (C library), AdamW for the other parameters.

    targets: [(weight parameter, module id MOARA_Q .. MOARA_EXP_DOWN)], weights of
             dtype fp32 or bf16 (all the same), at least two axes (flattened by the
             first axis, Appendix B.1).
    others:  the remaining parameters (AdamW).
    adamw_bits: None: torch.optim.AdamW steps the others; 32 or 8: the library's AdamW, its
             moments of that many bits (parameters fp32 or bf16).
    adamw_weight_decay: of the library's AdamW, on parameters of two axes or more (not on norms and biases).
    adamw_seed: of the random rounding of its 8-bit moments.
    max_grad_norm: None, or the norm that step() clips the gradients of all parameters to. Gradients
             of the targets are scaled in place, so are the others' with torch's AdamW. A norm that is
             not finite clears the gradients that are scaled: the targets, and with torch's AdamW the
             others, take a step of zero gradients (their moments decay, and move them). The library's
             AdamW leaves the others and their moments as they are.
             `grad_norm` holds the last step's norm, on the GPU.
    rank_table: per-module ranks r_tau (MOARA_NUM_MODULES entries, 0 = unused); see
             moara_allocate_ranks for the Phase 3 rule.
    Other keyword arguments go to moara_default_config (block_size, scale,
    refresh_interval, operand_dtype, refresh_oversample, ...).
    """

    def __init__(self, targets: Sequence[Tuple[torch.nn.Parameter, int]], others: Iterable[torch.nn.Parameter],
                 lr: float = 1e-2, betas=(0.9, 0.999), eps: float = 1e-6, rank_table: Sequence[int] = (),
                 block_size: int = 64, scale: float = 0.25, refresh_interval: int = 200,
                 adamw_bits: Optional[int] = None, adamw_weight_decay: float = 0.0, adamw_seed: int = 0,
                 max_grad_norm: Optional[float] = None, **config):
        if adamw_bits not in (None, 8, 32):
            raise ValueError(f"adamw_bits must be None, 8 or 32, got {adamw_bits}")
        if adamw_weight_decay and adamw_bits is None:
            raise ValueError("adamw_weight_decay needs adamw_bits 8 or 32")
        if max_grad_norm is not None and not max_grad_norm > 0:
            raise ValueError(f"max_grad_norm must be positive, got {max_grad_norm}")
        targets = list(targets)
        others = list(others)
        if not targets:
            raise ValueError("MoARa needs at least one target weight")
        wdt = {t.dtype for t, _ in targets}
        if len(wdt) != 1 or next(iter(wdt)) not in (torch.float32, torch.bfloat16):
            raise ValueError(f"target weights must all be fp32 or all bf16, got {wdt}")
        if adamw_bits is not None:      # here, not in a step that has already moved the targets
            for p in others:
                if p.dtype not in (torch.float32, torch.bfloat16):
                    raise ValueError(f"the library's AdamW steps fp32 and bf16 parameters, got {p.dtype}")
        groups = [{"params": [t for t, _ in targets], "moara": True}]
        if others:
            groups.append({"params": others, "moara": False})
        super().__init__(groups, dict(lr=lr, betas=tuple(betas), eps=eps))
        self._modules = [int(m) for _, m in targets]
        self._weight_bf16 = next(iter(wdt)) == torch.bfloat16
        self._cfg = M.moara_default_config(
            rank_table=list(rank_table), block_size=int(block_size), beta1=float(betas[0]),
            beta2=float(betas[1]), adam_eps=float(eps), scale=float(scale), refresh_interval=int(refresh_interval),
            weight_dtype=M.MOARA_BF16 if self._weight_bf16 else M.MOARA_F32, **config)
        self._descs = M.make_descs([(tuple(t.shape), m) for t, m in targets])
        self._st: Optional[M.State] = None
        self._g32: List[Optional[torch.Tensor]] = [None] * len(targets)
        self._adamw = self._own = None
        if others and adamw_bits is None:
            self._adamw = torch.optim.AdamW(others, lr=lr, betas=tuple(betas), eps=eps, weight_decay=0.0)
        elif others:
            self._own = _AdamW(others, M.moara_adamw_default_config(beta1=float(betas[0]), beta2=float(betas[1]),
                                                                   eps=float(eps), bits=adamw_bits),
                               adamw_weight_decay, adamw_seed)
        self._max_norm = max_grad_norm
        self._norm_args: Optional[M.GradArgs] = None
        self.grad_norm: Optional[torch.Tensor] = None

    def _device(self):
        """The target weights' GPU as the current device: the library's calls act on the
        current device, and the state lives on the one that was current at its creation."""
        return torch.cuda.device(self.param_groups[0]["params"][0].device)

    @property
    def moara_state(self) -> Optional[M.State]:
        """The library state (created at the first step), e.g. for moara_alignment."""
        return self._st

    def _grads(self) -> List[Optional[torch.Tensor]]:
        """Contiguous fp32 or bf16 gradients of the targets; None where a target has no gradient
        (e.g. a routed expert no token reached this step: it is skipped, its state kept).
        The library's step runs on the default stream: a bf16 gradient is handed to it there only,
        elsewhere it is copied on the current stream first, which its memory belongs to."""
        out = []
        on_default = torch.cuda.current_stream().cuda_stream == 0
        bf16, strided = torch.bfloat16, torch.strided
        for i, p in enumerate(self.param_groups[0]["params"]):
            if p.grad is None:
                out.append(None)
                continue
            g = p.grad
            if g.dtype != torch.float32 or not g.is_contiguous():
                if self._g32[i] is None:
                    self._g32[i] = torch.empty(p.shape, dtype=torch.float32, device=p.device)
                if not (on_default and g.dtype == bf16 and g.layout == strided and g.is_contiguous()):
                    self._g32[i].copy_(g)
                    g = self._g32[i]
            out.append(g)
        return out

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        tg = self.param_groups[0]
        coef = self._clip() if self._max_norm is not None else None
        with self._device():
            if self._st is None:
                self._st = M.moara_create_state(self._cfg, self._descs)
            grads = self._grads()
            active = [g is not None for g in grads]
            if any(active):
                # torch's side streams and the default one do not wait for each other by themselves: gradients (and
                # their copies) are made on the current stream, weights and gradients used or freed on it afterwards
                here = torch.cuda.current_stream()
                default = torch.cuda.default_stream() if here.cuda_stream != 0 else None
                if default is not None:
                    default.wait_stream(here)
                M.moara_step_mixed(self._st, tg["params"], grads, self._g32, lr=float(tg["lr"]),
                                   active=None if all(active) else active)
                if default is not None:
                    here.wait_stream(default)
        if self._adamw is not None:
            og = self.param_groups[1]
            for g in self._adamw.param_groups:   # the schedule drives both groups
                g["lr"] = og["lr"]
            self._adamw.step()
        if self._own is not None:
            self._own.step(float(self.param_groups[1]["lr"]), coef)
        return loss

    def _clip(self) -> torch.Tensor:
        """Norm of all gradients; the targets' (with torch's AdamW all) scaled to the limit in place. Returns the
        coefficient. Runs on the current stream."""
        params = [p for g in self.param_groups for p in g["params"]]
        grads = [p.grad for p in params]
        for i, g in enumerate(grads):       # what cannot be scaled in place (sparse, or with gaps) is replaced
            if g is not None and (g.layout != torch.strided or not M._dense(g)):
                params[i].grad = grads[i] = (g.to_dense() if g.layout != torch.strided else g).contiguous()
        with self._device():
            here = torch.cuda.current_stream()
            if self._norm_args is None or here != self._norm_stream:    # its workspace is used by one stream at a time
                self._norm_args, self._norm_stream = M.GradArgs([]), here
            self._norm_args.set_grads(grads)
            norm = M.moara_grad_norm(None, self._max_norm, args=self._norm_args)
            targets = len(self.param_groups[0]["params"])
            M.moara_grad_scale(None, norm[1:], args=self._norm_args,
                               first=None if self._own is None else sum(g is not None for g in grads[:targets]))
            self._norm_args.set_grads([])       # the gradients are the caller's: none outlives its zero_grad() here
        self.grad_norm = norm[0]
        return norm[1:]

    def state_dict(self) -> Dict:
        """Library state (projectors, moments, magnitude moments, step counters) as CPU
        tensors, plus the AdamW state of the other parameters and the group settings."""
        lib = None
        if self._st is not None:
            with self._device():
                lib = []
                for i in range(len(self._modules)):
                    d = {"step": int(M.moara_get_tensor(self._st, i, M.MOARA_T_STEP))}
                    for name, which in (("P", M.MOARA_T_P), ("exp_avg", M.MOARA_T_EXP_AVG),
                                        ("exp_avg_sq", M.MOARA_T_EXP_AVG_SQ), ("mag_avg", M.MOARA_T_MAG_AVG),
                                        ("mag_avg_sq", M.MOARA_T_MAG_AVG_SQ)):
                        try:
                            d[name] = torch.from_numpy(np.array(M.moara_get_tensor(self._st, i, which)))
                        except M.MoaraError as e:   # no projector yet: nothing to save for P
                            if which != M.MOARA_T_P or e.status != M.MOARA_E_STATE:
                                raise
                    lib.append(d)
        # the AdamW part is copied: torch's state_dict hands out the live moment tensors, and
        # loading those into another optimizer would alias the two
        out = {"moara": lib, "adamw": copy.deepcopy(self._adamw.state_dict()) if self._adamw else None,
               "lr": [g["lr"] for g in self.param_groups]}
        if self._own is not None:
            out["adamw_own"] = self._own.state_dict()
        return out

    def load_state_dict(self, sd: Dict) -> None:
        if (self._own is not None and sd.get("adamw") is not None) or (self._adamw is not None and "adamw_own" in sd):
            raise ValueError("the state is of the other AdamW (adamw_bits) than this optimizer's")
        if self._adamw is not None and sd["adamw"] is not None:
            self._adamw.load_state_dict(sd["adamw"])
        if self._own is not None and sd.get("adamw_own") is not None:
            self._own.load_state_dict(sd["adamw_own"])
        for g, lr in zip(self.param_groups, sd["lr"]):      # after what may be refused
            g["lr"] = lr
        if sd["moara"] is None:
            return
        with self._device():
            if self._st is None:
                self._st = M.moara_create_state(self._cfg, self._descs)
            for i, d in enumerate(sd["moara"]):
                for name, which in (("P", M.MOARA_T_P), ("exp_avg", M.MOARA_T_EXP_AVG),
                                    ("exp_avg_sq", M.MOARA_T_EXP_AVG_SQ), ("mag_avg", M.MOARA_T_MAG_AVG),
                                    ("mag_avg_sq", M.MOARA_T_MAG_AVG_SQ)):
                    if name in d:
                        M.moara_set_tensor(self._st, i, which, d[name].numpy())
                M.moara_set_tensor(self._st, i, M.MOARA_T_STEP, np.int64(d["step"]))
