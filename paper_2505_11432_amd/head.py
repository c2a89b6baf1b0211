"""Loss of hidden rows over a vocabulary, on one GPU: buffers allocated once, then one C-ABI call per pass.

The layer's output y (with whatever the model adds to it) goes in as x, and `dx` comes out as the dy of the layer's backward.
Like `MoELayer` this owns device memory and does no arithmetic of its own.
"""
from __future__ import annotations

import torch

from . import binding as B


class VocabLoss:
    """loss[t] = log sum_v exp(x[t] . w[v]) - x[t] . w[target[t]], its mean or weighted sum, and the gradients of x and w.

    T rows of width d, V words.  dtype: of x, w and dx (bf16 or fp32); grad_dtype: of d_w (fp32, or bf16 for bf16 data).
    gradients = False: `score` only, without the buffers of a gradient.
    piece_bytes: the softmax gradient (V elements of the data's type per row; for fp32 data the logits before it) is kept for as many rows
    at a time as fit; the default, 1.4 % of a GPU's memory, takes 16384 rows of 128 k words in bf16 in one piece.

    Buffers: loss, lse [T] fp32 (0 where the target is left out), total [1] fp32, dx [T, d], d_w [V, d]."""

    def __init__(self, T: int, d: int, V: int, dtype=torch.bfloat16, grad_dtype=torch.float32, device="cuda:0",
                 gradients: bool = True, piece_bytes: int = 4 << 30):
        assert T >= 0 and d > 0 and V > 0, "sizes are positive"
        assert dtype in (torch.bfloat16, torch.float32), "rows are bf16 or fp32"
        assert grad_dtype in (torch.float32, dtype), "the vocabulary gradient is fp32 or of the data's type"
        self.T, self.d, self.V, self.dtype, self.gradients = T, d, V, dtype, gradients
        row = (V + 63) // 64 * 64 * (2 if dtype == torch.bfloat16 else 4)
        fit = max(1, piece_bytes // row)
        # whole row tiles, a power of two of them where several pieces are needed, so that the matrix cores fill in whole rounds
        self.piece_rows = 0 if fit >= T else max(256, 1 << (fit.bit_length() - 1))
        dt, gdt = B.dtype_code(dtype), B.dtype_code(grad_dtype)
        size = max(B.moe_vocab_workspace_bytes(T, d, V, dt, gdt, self.piece_rows, g) for g in ((0, 1) if gradients else (0,)))
        assert size > 0, f"unsupported sizes: T {T}, d {d} (a multiple of 16), V {V}"
        f32 = dict(dtype=torch.float32, device=device)
        self.workspace = torch.empty((size,), dtype=torch.uint8, device=device)
        self.loss = torch.zeros((T,), **f32)
        self.lse = torch.zeros((T,), **f32)
        if gradients:
            self.total = torch.zeros((1,), **f32)
            self.dx = torch.empty((T, d), dtype=dtype, device=device)
            self.d_w = torch.zeros((V, d), dtype=grad_dtype, device=device)

    def _rows(self, x, w):
        assert tuple(x.shape) == (self.T, self.d) and x.dtype == self.dtype, "x does not fit this loss"
        assert tuple(w.shape) == (self.V, self.d), "w does not fit this loss"

    def score(self, x, w, target):
        """(loss, lse) of every row.  target [T] int32; outside 0..V-1: left out."""
        self._rows(x, w)
        B.moe_vocab_score(x, w, target, self.piece_rows, self.loss, self.lse, self.workspace)
        return self.loss, self.lse

    def step(self, x, w, target, token_w=None, accumulate: bool = False):
        """total = sum_t c[t] loss[t] with its gradients in dx and d_w; c = token_w [T] fp32, or 1 / (rows that count).  accumulate adds
        into d_w (a micro-batch after the first)."""
        assert self.gradients, "made without gradients"
        self._rows(x, w)
        if self.T == 0:                     # nothing is enqueued: an empty batch adds nothing
            if not accumulate:
                self.d_w.zero_()
            return self.total
        B.moe_vocab_loss(x, w, target, token_w, self.piece_rows, self.total, self.loss, self.lse, self.dx, self.d_w, accumulate,
                         self.workspace)
        return self.total
