"""torch.optim adapter: MALT / MALTER for matrix parameters through libmalt,
AdamW for every other parameter.

Algorithm 1 (MALT) and Algorithm 2 (MALTER) update matrix parameters; the
paper trains embeddings, norms and biases with AdamW.  This optimizer routes
every 2-D parameter (or those `matrix_filter` selects) of a parameter group
into one libmalt plan per group, so one `step()` is one grouped `malt_step`
per group, and hands the remaining parameters to an inner AdamW.

Variants:
  "malt"    Algorithm 1
  "malter"  Algorithm 2 (noise-adaptive stepsize)
  "muon"    Algorithm 1 with L = R = I: Muon's update (Sec. 3.1), the
            baseline the paper compares against

Conventions
  * Matrix parameters must be contiguous float32 CUDA tensors; their
    gradients are made contiguous float32 before the step.  A matrix
    parameter without a gradient is stepped with a zero gradient (the plan
    steps all of its matrices together).
  * The remaining parameters go to torch's AdamW, or with adamw_bits=32 or 8 to this
    module's (moments in that many bits), one launch for a hundred of them.
  * `lr` is the matrix learning rate eta; schedulers that change a group's
    "lr" scale the group's AdamW learning rate by the same factor.
  * `state_dict()` holds each plan's state buffer (M, l, r, nu as float32)
    and step count t, and the inner AdamW's state; `load_state_dict` resumes
    bitwise.
"""
from __future__ import annotations

import itertools
from typing import Callable, Dict, List, Optional, Tuple

import torch

from . import libmalt as lm

VARIANTS = ("malt", "malter", "muon")


def is_matrix(p: torch.Tensor) -> bool:
    """Default selection of matrix parameters: every 2-D tensor."""
    return p.dim() == 2


class AdamW(torch.optim.Optimizer):
    """AdamW on ops.adamw_step: all parameters of a group in one launch for each 108 of
    them.  Parameters and gradients are float32 or bfloat16 CUDA tensors, parameters
    contiguous.

    bits: of the moments.  8 keeps those of parameters of at least `min_8bit` elements in
    8 bits (a scale for each 256), the others in 32; their rounding is random, by `seed`, step and
    place.  A parameter without a gradient is left out of a step and does not count it."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                 bits: int = 32, min_8bit: int = 4096, seed: int = 0):
        if bits not in (8, 32):
            raise ValueError(f"bits must be 8 or 32 (got {bits})")
        if not 0 <= seed < 1 << 32:
            raise ValueError(f"seed must be in [0, 2^32) (got {seed})")
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay))
        self.bits, self.min_8bit, self.seed = bits, min_8bit, int(seed)

    def __getstate__(self):
        # torch's keeps the defaults, the state and the groups: copies and pickles would lack the rest.
        return {**super().__getstate__(), "bits": self.bits, "min_8bit": self.min_8bit, "seed": self.seed}

    @torch.no_grad()
    def step(self, closure=None):
        from . import ops
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        # A captured launch keeps its step count, so that replays would repeat this step.
        if torch.cuda.is_available() and torch.cuda.is_current_stream_capturing():
            raise RuntimeError("AdamW.step cannot be captured: its step count is an argument")
        for k, g in enumerate(self.param_groups):
            calls: Dict[tuple, list] = {}   # parameters of a device that have stepped as often
            for p in g["params"]:
                if p.grad is None:
                    continue
                st = self.state[p]
                if not st:
                    st["step"] = 0
                    st["moments"] = ops.adamw_state(p, 8 if self.bits == 8 and p.numel() >= self.min_8bit else 32)
                calls.setdefault((p.device, st["step"] + 1), []).append(p)
            place = {id(p): i for i, p in enumerate(g["params"])}
            for (_, t), ps in calls.items():
                # No other call has this group, first parameter and step count of it.
                noise = (t * 0x9E3779B1 + k * 0xBB67AE85 + place[id(ps[0])] * 0xA54FF53B) & 0xFFFFFFFF
                ops.adamw_step(ps, [p.grad for p in ps], [self.state[p]["moments"] for p in ps], lr=g["lr"],
                               betas=g["betas"], eps=g["eps"], weight_decay=g["weight_decay"], step=t,
                               seed=self.seed << 32 | noise)
                for p in ps:
                    self.state[p]["step"] = t
        return loss

    def state_dict(self) -> Dict:
        return {**super().state_dict(), "seed": self.seed}

    def _loaded(self, state_dict: Dict) -> List[Tuple[torch.Tensor, dict]]:
        """The state's entries by parameter; ValueError where one is no state of this optimizer for it."""
        ids = itertools.chain.from_iterable(g["params"] for g in state_dict["param_groups"])
        entries = []
        for i, p in zip(ids, itertools.chain.from_iterable(g["params"] for g in self.param_groups)):
            st = state_dict["state"].get(i)
            if not st:
                continue
            if set(st) != {"step", "moments"}:
                raise ValueError(f"parameter {i}: {sorted(st)} are not the step and moments of this AdamW")
            try:
                step = int(st["step"])
            except (TypeError, ValueError):
                step = -1
            if step < 0:
                raise ValueError(f"parameter {i}: the step is {st['step']}")
            m, n = st["moments"], p.numel()
            # 8 bits: two codes for each place of whole blocks of 256, and two scales for each block.
            shape = {torch.float32: (2, n), torch.uint8: (-(-n // 256) * 520,)}
            if not isinstance(m, torch.Tensor) or tuple(m.shape) != shape.get(m.dtype):
                raise ValueError(f"parameter {i} of {n} elements: moments must be float32 {shape[torch.float32]} or uint8 "
                                 f"{shape[torch.uint8]} (got {f'{m.dtype} {tuple(m.shape)}' if isinstance(m, torch.Tensor) else type(m).__name__})")
            entries.append((p, {"step": step, "moments": m}))
        return entries

    def load_state_dict(self, state_dict: Dict) -> None:
        """Takes a state of this class over, its seed too, or raises ValueError and leaves everything as it was."""
        entries = self._loaded(state_dict)
        seed = state_dict.get("seed", self.seed)
        if not isinstance(seed, int) or not 0 <= seed < 1 << 32:
            raise ValueError(f"the state's seed must be in [0, 2^32) (got {seed})")
        super().load_state_dict(state_dict)   # refuses other groups than these
        self.seed = seed
        # Moments keep the type they were saved in, whatever the parameter's.
        for p, st in entries:
            m = st["moments"].detach().to(p.device).clone(memory_format=torch.contiguous_format)
            self.state[p] = {"step": st["step"], "moments": m}


class MALT(torch.optim.Optimizer):
    def __init__(self, params, lr: float = 1.3e-3, mu1: float = 0.95, mu2: float = 0.99, eps: float = 1e-8,
                 weight_decay: float = 0.0, variant: str = "malt", ns_steps: int = 5,
                 adamw_lr: Optional[float] = None, adamw_betas=(0.9, 0.95), adamw_eps: float = 1e-8,
                 adamw_weight_decay: float = 0.0,
                 matrix_filter: Optional[Callable[[torch.Tensor], bool]] = None,
                 adamw_bits: Optional[int] = None):
        if variant not in VARIANTS:
            raise ValueError(f"variant must be one of {VARIANTS}")
        if adamw_bits not in (None, 8, 32):
            raise ValueError(f"adamw_bits must be 8, 32 or None (got {adamw_bits})")
        defaults = dict(lr=lr, mu1=mu1, mu2=mu2, eps=eps, weight_decay=weight_decay, ns_steps=ns_steps,
                        adamw_lr=lr if adamw_lr is None else adamw_lr, adamw_betas=tuple(adamw_betas),
                        adamw_eps=adamw_eps, adamw_weight_decay=adamw_weight_decay)
        super().__init__(params, defaults)
        self.variant = variant
        self._filter = matrix_filter or is_matrix
        self._plans: List[Optional[lm.Plan]] = [None] * len(self.param_groups)
        self._resume: List[Optional[dict]] = [None] * len(self.param_groups)
        # Split each group into matrix parameters (libmalt) and the rest (AdamW).
        self._mats: List[List[torch.Tensor]] = []
        adam_groups = []
        for g in self.param_groups:
            mats = [p for p in g["params"] if self._filter(p)]
            rest = [p for p in g["params"] if not self._filter(p)]
            for p in mats:
                if p.dim() != 2:
                    raise ValueError("matrix_filter selected a parameter that is not 2-D")
            self._mats.append(mats)
            g["lr0"] = g["lr"]
            adam_groups.append(dict(params=rest, lr=g["adamw_lr"], betas=g["adamw_betas"], eps=g["adamw_eps"],
                                    weight_decay=g["adamw_weight_decay"]))
        self._adam_lr0 = [ag["lr"] for ag in adam_groups]
        self._adam = None
        if any(ag["params"] for ag in adam_groups):
            self._adam = torch.optim.AdamW(adam_groups) if adamw_bits is None else AdamW(adam_groups, bits=adamw_bits)

    # ------------------------------------------------------------------ helpers
    def _hparams(self, g: dict):
        return lm.make_hparams(lr=g["lr"], mu1=g["mu1"], mu2=g["mu2"], eps=g["eps"],
                               weight_decay=g["weight_decay"], ns_steps=g["ns_steps"],
                               precond_identity=1 if self.variant == "muon" else 0)

    def _plan(self, k: int) -> Optional[lm.Plan]:
        mats = self._mats[k]
        if not mats:
            return None
        if self._plans[k] is None:
            for p in mats:
                if not (p.is_cuda and p.dtype == torch.float32 and p.is_contiguous()):
                    raise ValueError("matrix parameters must be contiguous float32 CUDA tensors")
            shapes = [tuple(p.shape) for p in mats]
            variant = "malter" if self.variant == "malter" else "malt"
            res = self._resume[k]
            if res is not None:
                state = res["state"].to(mats[0].device)
                self._plans[k] = lm.Plan(shapes, variant, device=mats[0].device, state=state,
                                         from_existing=True, step=int(res["t"]))
                self._resume[k] = None
            else:
                self._plans[k] = lm.Plan(shapes, variant, device=mats[0].device)
        return self._plans[k]

    # --------------------------------------------------------------------- step
    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        stream = torch.cuda.current_stream()
        for k, g in enumerate(self.param_groups):
            plan = self._plan(k)
            if plan is None:
                continue
            grads = []
            for p in self._mats[k]:
                gr = p.grad
                if gr is None:
                    gr = torch.zeros_like(p)
                elif gr.dtype != torch.float32 or not gr.is_contiguous():
                    gr = gr.float().contiguous()
                grads.append(gr)
            plan.step(self._mats[k], grads, self._hparams(g), stream=stream)
        if self._adam is not None:
            for k, g in enumerate(self.param_groups):   # follow the group's schedule
                self._adam.param_groups[k]["lr"] = self._adam_lr0[k] * (g["lr"] / g["lr0"]) if g["lr0"] else 0.0
            self._adam.step()
        return loss

    def zero_grad(self, set_to_none: bool = True):
        super().zero_grad(set_to_none=set_to_none)

    # ---------------------------------------------------------------- state I/O
    def state_dict(self) -> Dict:
        plans = []
        for k in range(len(self.param_groups)):
            p = self._plans[k]
            if p is None:
                plans.append(self._resume[k])
            else:
                torch.cuda.current_stream().synchronize()
                plans.append({"state": p.state[: p.state_bytes].detach().cpu().clone(), "t": p.t,
                              "shapes": list(p.shapes), "variant": self.variant})
        groups = [{k: v for k, v in g.items() if k != "params"} for g in self.param_groups]
        return {"variant": self.variant, "plans": plans, "groups": groups,
                "adamw": self._adam.state_dict() if self._adam is not None else None}

    def load_state_dict(self, sd: Dict) -> None:
        if sd["variant"] != self.variant:
            raise ValueError(f"state is for variant {sd['variant']}, optimizer is {self.variant}")
        if len(sd["plans"]) != len(self.param_groups):
            raise ValueError("parameter group count differs")
        for k, pl in enumerate(sd["plans"]):
            if pl is not None and [tuple(s) for s in pl["shapes"]] != [tuple(p.shape) for p in self._mats[k]]:
                raise ValueError(f"group {k}: matrix shapes differ from the saved state")
        # The other parameters first: what does not fit there raises, and nothing has changed.
        if self._adam is not None and sd.get("adamw") is not None:
            if not isinstance(self._adam, AdamW) and any("moments" in st for st in sd["adamw"]["state"].values()):
                raise ValueError("the state was saved with adamw_bits: it is not one of torch's AdamW")
            self._adam.load_state_dict(sd["adamw"])
        for k, pl in enumerate(sd["plans"]):
            if self._plans[k] is not None:
                self._plans[k].close()
                self._plans[k] = None
            self._resume[k] = pl
        for g, s in zip(self.param_groups, sd["groups"]):
            g.update(s)

    @torch.no_grad()
    def precond_condition(self) -> Dict[torch.Tensor, Tuple[float, float]]:
        """kappa(diag l) and kappa(diag r) of every matrix parameter that has
        stepped, as the paper's analysis of the diagonal preconditioners
        (Sec. 5.4) reports them per layer and module.  One small kernel per
        parameter group, then one copy to the host."""
        out: Dict[torch.Tensor, Tuple[float, float]] = {}
        for k in range(len(self.param_groups)):
            plan = self._plans[k]
            if plan is None:
                continue
            kap = plan.precond_condition(stream=torch.cuda.current_stream()).cpu()
            for p, (kl, kr) in zip(self._mats[k], kap.tolist()):
                out[p] = (kl, kr)
        return out

    def matrix_plan(self, group: int = 0) -> Optional[lm.Plan]:
        """The libmalt plan of a parameter group (built at its first step)."""
        return self._plan(group)
