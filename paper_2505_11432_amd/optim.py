"""Gradient clipping and the AdamW update over lists of tensors: a table of the tensors is made once, then one or two launches per
step whatever their number.  The tensors stay where they are (the handle keeps them), so a step can be captured into a graph.

Muon, for the matrices among them: the update is the momentum orthogonalised by Newton-Schulz steps, one call per tensor (a batch of matrices)."""
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


def _piece(batch: int, rows: int, cols: int, max_bytes: int) -> int:
    """Matrices at a time whose workspace stays within max_bytes (one at least)."""
    assert batch >= 0 and rows > 0 and cols > 0, "matrices have rows and columns"
    assert B.moe_orthogonal_workspace_bytes(1, rows, cols) > 0, f"unsupported matrices: {rows} x {cols}"
    piece = max(1, min(batch, 32768))
    while piece > 1 and not 0 < B.moe_orthogonal_workspace_bytes(batch, rows, cols, piece) <= max_bytes:
        piece -= (piece + 15) // 16
    return piece


class Orthogonal:
    """out = x / |x| after Newton-Schulz steps, for a batch of matrices: singular values near 1 (0.7 to 1.2 with the default steps), the singular
    vectors as they are.

    coefficients: a row (a, b, c) per step X <- a X + b (X X^T) X + c (X X^T)^2 X.  Roundings of matrices of low rank grow by |a| a step: lists with a product of
    |a| above 8192 (with a side of at most 64: 262144) are refused, as are those that leave the range of 16 bits.
    max_bytes bounds the workspace: matrices are taken in pieces (how many at a time can change the bits of the sums, not their exactness).
    Buffer: out [batch, rows, cols] in out_dtype (bf16 or fp32)."""

    def __init__(self, batch: int, rows: int, cols: int, out_dtype=torch.bfloat16, coefficients=B.COEFFICIENTS, max_bytes: int = 8 << 30, device="cuda:0"):
        assert out_dtype in (torch.bfloat16, torch.float32), "results are bf16 or fp32"
        self.batch, self.rows, self.cols = batch, rows, cols
        self.coefficients = B._coefficients(coefficients)
        self.piece = _piece(batch, rows, cols, max_bytes)
        self.workspace = torch.empty((B.moe_orthogonal_workspace_bytes(batch, rows, cols, self.piece),), dtype=torch.uint8, device=device)
        self.out = torch.empty((batch, rows, cols), dtype=out_dtype, device=device)

    def apply(self, x):
        """x [batch, rows, cols], bf16 or fp32."""
        assert tuple(x.shape) == (self.batch, self.rows, self.cols), "x does not fit these matrices"
        B.moe_orthogonalize(x, self.out, self.workspace, self.coefficients, self.piece)
        return self.out


class Muon:
    """In place, for lists of fp32 parameters [..., rows, cols] that are matrices, or batches of them:
    m = momentum m + coef grad,  u = coef grad + momentum m (nesterov; else m),  p = p (1 - lr weight_decay) - lr scale O(u),
    O(u) as in `Orthogonal` but of u / max(|u|, eps), and the parameters rounded to bf16 into `weights`.

    grads: bf16 or fp32 (a list may have both).  What is written shares no memory (a shared weight comes once).
    scale: None: 0.2 sqrt(max(rows, cols)), with which an update is as large as AdamW's (root mean square about 0.2) and both take one learning
    rate; or a number for all of them.  eps: norm below which an update fades, as that of an expert without tokens does.  lr: a float, or a [1] fp32 device tensor that a schedule writes.  coefficients, max_bytes: as in `Orthogonal`;
    the tensors share one workspace."""

    def __init__(self, params, grads, m, weights=None, lr=1e-3, momentum=0.95, nesterov=True, weight_decay=0.1, scale=None, coefficients=B.COEFFICIENTS,
                 max_bytes: int = 8 << 30, device=None, eps=B.MUON_EPS):
        self.params, self.grads, self.m = list(params), list(grads), list(m)
        self.weights = [None] * len(self.params) if weights is None else list(weights)
        assert len(self.params) == len(self.grads) == len(self.m) == len(self.weights), "lists of one length"
        device = device or (self.params[0].device if self.params else "cuda:0")
        for p in self.params:
            assert p.dim() >= 2 and p.shape[-1] > 0 and p.shape[-2] > 0, "parameters are matrices, or batches of them"
        lists = [B._List(t) for t in (self.params, self.m, self.weights, self.grads)]
        assert lists[0].like(lists[0], B.F32) and lists[1].like(lists[0], B.F32), "parameters and momentum are fp32, of one size"
        assert lists[2].like(lists[0], B.BF16), "weights are bf16, of their parameters' sizes"
        assert lists[3].sizes_like(lists[0]), "gradients have their parameters' sizes"
        assert B._apart(lists[:3], lists[3:]), "parameters, momentum and weights share no memory with each other or with a gradient"
        self.lr = lr if isinstance(lr, torch.Tensor) else torch.full((1,), float(lr), dtype=torch.float32, device=device)
        assert self.lr.dtype == torch.float32 and self.lr.numel() == 1, "lr is one fp32 number"
        self.momentum, self.nesterov, self.weight_decay, self.eps = momentum, nesterov, weight_decay, eps
        self.coefficients = B._coefficients(coefficients)
        self.calls, size = [], 256
        for p, g, v, w in zip(self.params, self.grads, self.m, self.weights):
            rows, cols = p.shape[-2:]
            view = [None if t is None else t.view(-1, rows, cols) for t in (p, g, v, w)]
            batch = view[0].shape[0]
            if batch == 0:
                continue
            piece = _piece(batch, rows, cols, max_bytes)
            size = max(size, B.moe_orthogonal_workspace_bytes(batch, rows, cols, piece))
            self.calls.append((*view, 0.2 * max(rows, cols) ** 0.5 if scale is None else float(scale), piece))
        self.workspace = torch.empty((size,), dtype=torch.uint8, device=device)

    def step(self, coef=None):
        """One update; coef: a [1] fp32 device tensor that every gradient is multiplied by (GradClip.coef).  A factor that is NaN leaves the update out."""
        assert coef is None or (coef.dtype == torch.float32 and coef.numel() == 1), "coef is one fp32 number"
        for p, g, m, w, scale, piece in self.calls:
            B.moe_muon(p, g, m, w, self.lr, coef, self.momentum, self.nesterov, self.weight_decay, scale, self.workspace, self.coefficients, piece, self.eps)
