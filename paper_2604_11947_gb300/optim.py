"""AdamW over libresbm.so (resbm_adamw_step, resbm_grad_norm) as a torch optimizer.

The whole step is one launch for up to 448 tensors of the same types, plus two for the gradients' norm where they are
clipped; nothing is copied to the device or waited for. States are fp32, or e4m3 codes with a scale per 256 elements
(state_bits = 8: 2.03 bytes a parameter instead of 8).
"""
from __future__ import annotations

import torch

from . import resbm

_STATES = ("exp_avg", "exp_avg_sq")
_COLUMNS = _STATES + ("exp_avg_scale", "exp_avg_sq_scale", "master")   # (in AdamWPlan's order)


class AdamW(torch.optim.Optimizer):
    """AdamW with decoupled weight decay on fp32 or bf16 CUDA parameters.

    state_bits      32 or 8 (e4m3 codes of the first moment and of the second's root, with fp32 scales). With 8 bits a second
                    moment follows gradients that change against their block of 256 at a beta2 of about 0.95, not at 0.99 and
                    over, where every step's change is under half a step of e4m3 and lost
    master          fp32 master copies of bf16 parameters, which then are what the step updates
    max_grad_norm   clips the norm of all gradients together; it is left in `grad_norm` (norm and coefficient, on the
                    device). A step whose norm is not finite changes no parameter and no moment (it still counts).

    Parameters without a gradient are left alone. The step count is the host's, so a step cannot be captured into a CUDA
    graph (resbm.resbm_adamw_step with step_dev can)."""

    def __init__(self, params, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2, state_bits=32, master=False,
                 max_grad_norm=None):
        if state_bits not in (8, 32):
            raise ValueError("state_bits is 8 or 32: got %r" % (state_bits,))
        if max_grad_norm is not None and not 0 < max_grad_norm < float("inf"):
            raise ValueError("max_grad_norm is positive and finite, or None: got %r" % (max_grad_norm,))
        if not (lr >= 0 and eps >= 0 and weight_decay >= 0 and all(0 <= b < 1 for b in betas)):
            raise ValueError("lr, eps and weight_decay are not negative, betas lie in [0, 1)")
        self.state_bits, self.master, self.max_grad_norm = state_bits, bool(master), max_grad_norm
        self.grad_norm = None
        self._plans, self._ws = {}, None
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay))

    def __getstate__(self):
        return {**super().__getstate__(), "state_bits": self.state_bits, "master": self.master, "max_grad_norm": self.max_grad_norm}

    def __setstate__(self, state):
        super().__setstate__(state)
        self.grad_norm, self._plans, self._ws = None, {}, None

    def load_state_dict(self, state_dict):
        """As torch's, but the moments keep their own types (torch would cast them to the parameters')."""
        saved = state_dict["state"]
        for st in saved.values():
            if not ("bf16" in st and "exp_avg" in st and "exp_avg_sq" in st) or \
                    (st["exp_avg"].element_size() == 1) != (self.state_bits == 8) or ("master" in st) != (self.master and st["bf16"]):
                raise ValueError("the state has other moments or master copies than this optimizer keeps")
        super().load_state_dict(state_dict)
        for g, s in zip(self.param_groups, state_dict["param_groups"]):
            for p, i in zip(g["params"], s["params"]):
                if i in saved:
                    self.state[p] = {k: v.detach().to(p.device, copy=True) if torch.is_tensor(v) else v for k, v in saved[i].items()}
        self._plans = {}

    def _init_state(self, p):
        st = self.state[p]
        st["step"], st["bf16"] = 0, p.dtype == torch.bfloat16
        for k in _STATES:
            if self.state_bits == 32:
                st[k] = torch.zeros_like(p, dtype=torch.float32, memory_format=torch.contiguous_format)
            else:
                st[k] = torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn)
                st[k + "_scale"] = torch.zeros(-(-p.numel() // resbm.RESBM_STATE_BLOCK), device=p.device)
        self._init_master(p)

    def _init_master(self, p):
        if self.master and p.dtype == torch.bfloat16:
            self.state[p].update(bf16=True, master=p.detach().float())

    def _plan(self, key, params):
        """The plan of a list of parameters: the last step's where it is still of these tensors (parameters and states where they
        were), with other gradients where only they moved."""
        grads = [p.grad if p.grad.is_contiguous() else p.grad.contiguous() for p in params]
        states = [self.state[p] for p in params]
        columns = {k: [st[k] for st in states] for k in _COLUMNS if k in states[0]}
        tensors = [t for column in (params, *columns.values()) for t in column]
        where = [t.data_ptr() for t in tensors] + [t.nbytes for t in tensors]
        gwhere = [g.data_ptr() for g in grads]
        plan, *old = self._plans.pop(key, (None, None, None))   # (back once it is sound)
        if plan is None or old[0] != where:
            plan = resbm.AdamWPlan([p.detach() for p in params], grads, *[columns.get(k) for k in _COLUMNS])
        elif old[1] != gwhere:
            plan.set_grads(grads)
        else:
            plan._fields["g"] = grads
        self._plans[key] = (plan, where, gwhere)
        return plan

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("the step count is the host's: capture resbm.resbm_adamw_step with step_dev instead")
        work = {}
        for i, group in enumerate(self.param_groups):
            for p in group["params"]:
                if p.grad is None:
                    continue
                if not p.is_cuda or p.grad.is_sparse or not p.is_contiguous():
                    raise ValueError("parameters are dense and contiguous, on the GPU")
                if not self.state[p]:
                    self._init_state(p)
                elif "master" not in self.state[p]:
                    self._init_master(p)   # (a parameter that was fp32 before)
                work.setdefault((i, p.dtype, p.grad.dtype, self.state[p]["step"] + 1), []).append(p)
        plans, kept = [], {}
        try:
            for (i, dtype, g_dtype, step), params in work.items():
                key = (i, dtype, g_dtype, *map(id, params))
                plans.append((self.param_groups[i], step, params, self._plan(key, params)))
                kept[key] = self._plans[key]
            self._plans = kept   # (those of other lists than this step's are let go)
            self._launch(plans)
        finally:   # (zero_grad frees the gradients, a program may drop or move the states; what was launched is on the stream)
            for *_, plan in plans:
                plan.release()
        return loss

    def _launch(self, plans):
        scale = None
        if self.max_grad_norm is not None and plans:
            each = [plan for *_, plan in plans]
            need = resbm.resbm_grad_norm_workspace_bytes(each)
            device = plans[0][2][0].device
            if self._ws is None or self._ws.numel() < need or self._ws.device != device:
                self._ws = torch.empty(max(need, 1), dtype=torch.uint8, device=device)
            self.grad_norm = torch.empty(2, device=device)
            resbm.resbm_grad_norm(each, self.max_grad_norm, self.grad_norm, self._ws)
            scale = self.grad_norm[1:]
        for group, step, params, plan in plans:
            b1, b2 = group["betas"]
            resbm.resbm_adamw_step(plan, lr=float(group["lr"]), beta1=b1, beta2=b2, eps=group["eps"], weight_decay=group["weight_decay"],
                                   step=step, grad_scale=scale)
            torch.autograd.graph.increment_version(params)   # (a backward through what they were raises, as after torch's steps)
            for p in params:
                self.state[p]["step"] = step
