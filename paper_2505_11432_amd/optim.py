"""Gradient clipping and the AdamW update over lists of tensors: a table of the tensors is made once, then one or two launches per
step whatever their number.  The tensors stay where they are (the handle keeps them), so a step can be captured into a graph."""
from __future__ import annotations

import torch

from . import binding as B


class GradClip:
    """norm = sqrt(sum of all gradients squared), coef = min(1, max_norm / (norm + 1e-6)), and out = coef * gradients where asked.

    grads: bf16 or fp32 tensors.  out: None (the norm and the factor only, for an update that takes the factor), or a tensor for each
    gradient; the gradients themselves clip in place.  An out shares no memory with another tensor (the gradient of a shared weight comes once).
    Buffers: norm, coef [1] fp32 on the device."""

    def __init__(self, grads, max_norm: float, out=None, device=None):
        self.grads, self.out, self.max_norm = list(grads), None if out is None else list(out), float(max_norm)
        device = device or (self.grads[0].device if self.grads else "cuda:0")
        self.total = sum(g.numel() for g in self.grads)
        self.table = B.moe_grad_clip_table(self.grads, self.out)
        self.workspace = torch.empty((B.moe_grad_clip_workspace_bytes(),), dtype=torch.uint8, device=device)
        self.norm = torch.zeros((1,), dtype=torch.float32, device=device)
        self.coef = torch.ones((1,), dtype=torch.float32, device=device)

    def clip(self):
        """norm and coef of the gradients as they are now; the clipped gradients go to `out`."""
        B.moe_grad_clip(self.table, len(self.grads), self.total, self.max_norm, self.out is not None, self.norm, self.coef, self.workspace)
        return self.norm


class AdamW:
    """In place: fp32 parameters and moments from bf16 or fp32 gradients (a list may have both), and the parameters rounded to bf16 into `weights`.

    params, grads, m, v (and weights): lists of one length; what is written shares no memory (a shared weight comes once).
    lr: a float, or a [1] fp32 device tensor that a schedule writes.
    step: a [1] int32 device tensor with the updates taken so far (made at 0 if not given)."""

    def __init__(self, params, grads, m, v, weights=None, lr=1e-3, betas=(0.9, 0.95), eps=1e-8, weight_decay=0.1, step=None, device=None):
        self.params, self.grads, self.m, self.v = list(params), list(grads), list(m), list(v)
        self.weights = None if weights is None else list(weights)
        device = device or (self.params[0].device if self.params else "cuda:0")
        self.total = sum(p.numel() for p in self.params)
        self.table = B.moe_adamw_table(self.params, self.grads, self.m, self.v, self.weights)
        self.grad_dt = B.adamw_grad_type(self.grads)
        self.lr = lr if isinstance(lr, torch.Tensor) else torch.full((1,), float(lr), dtype=torch.float32, device=device)
        self.step_count = step if step is not None else torch.zeros((1,), dtype=torch.int32, device=device)
        assert self.lr.dtype == torch.float32 and self.lr.numel() == 1, "lr is one fp32 number"
        assert self.step_count.dtype == torch.int32 and self.step_count.numel() == 1, "step is one int32 number"
        self.betas, self.eps, self.weight_decay = betas, eps, weight_decay
        self.workspace = torch.zeros((B.ADAMW_WS_BYTES,), dtype=torch.uint8, device=device)

    def step(self, coef=None):
        """One update; coef: a [1] fp32 device tensor that every gradient is multiplied by (GradClip.coef).  A factor that is NaN leaves the update out:
        nothing changes, the step count neither."""
        assert coef is None or (coef.dtype == torch.float32 and coef.numel() == 1), "coef is one fp32 number"
        B.moe_adamw(self.table, len(self.params), self.total, self.grad_dt, self.lr, self.step_count, coef, self.betas[0], self.betas[1],
                    self.eps, self.weight_decay, self.workspace)
