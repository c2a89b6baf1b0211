"""Norms before and after a block on the residual stream, with the block's gate and the stream's scale, and all gradients: one C-ABI call per pass."""
from __future__ import annotations

import torch

from . import binding as B


class BlockNorm:
    """The end of one block and the start of the next:
    n = y / rms(y) * w_after (after; else y),  out = alpha x + gate[t // gate_rows] * n,  h = out / rms(out) * w_before (before).

    T rows of width d, dtype bf16 or fp32; the weights [d] and the gate [ceil(T / gate_rows), d] are fp32.
    residual = False: no block ends here (in front of the first one): h is made from x.  gate_rows: tokens that share a row of the gate (T: one
    vector for all, 1: a row per token, a sequence's length: a row per sequence); 0: no gate.

    Buffers: out (x where nothing is added), h, dx, dy [T, d]; d_w_after, d_w_before [d] and d_gate fp32; None for what there is not."""

    def __init__(self, T: int, d: int, dtype=torch.bfloat16, eps: float = 1e-6, alpha: float = 1.0, residual: bool = True, after: bool = True,
                 gate_rows: int = 0, before: bool = True, gradients: bool = True, device="cuda:0"):
        assert T >= 0 and d > 0 and gate_rows >= 0, "sizes are positive"
        assert dtype in (torch.bfloat16, torch.float32), "rows are bf16 or fp32"
        assert residual or not (after or gate_rows or alpha != 1.0), "without a residual there is nothing behind a block"
        assert residual or before, "nothing to do"
        self.T, self.d, self.dtype, self.eps, self.alpha, self.gradients = T, d, dtype, float(eps), float(alpha), gradients
        self.residual, self.after, self.gate_rows, self.before = residual, after, gate_rows, before
        size = B.moe_block_norm_workspace_bytes(T, d, B.dtype_code(dtype), after, gate_rows > 0, before)
        assert size > 0, f"unsupported sizes: T {T}, d {d} (a multiple of 16, at most {B.NORM_MAX_WIDTH})"

        def buffer(there, *shape, dt=dtype):
            return torch.zeros(shape, dtype=dt, device=device) if there else None

        self.out = buffer(residual, T, d)
        self.h = buffer(before, T, d)
        f32 = torch.float32
        self.dx = buffer(gradients, T, d)
        self.dy = buffer(gradients and residual, T, d)
        self.d_w_after = buffer(gradients and after, d, dt=f32)
        self.d_gate = buffer(gradients and gate_rows > 0, -(-T // max(gate_rows, 1)), d, dt=f32)
        self.d_w_before = buffer(gradients and before, d, dt=f32)
        self.workspace = torch.empty((size,), dtype=torch.uint8, device=device) if gradients else None

    def _fits(self, y, w_after, gate, w_before):
        assert (y is not None) == self.residual and (w_after is not None) == self.after, "y and w_after as this norm was made"
        assert (gate is not None) == (self.gate_rows > 0) and (w_before is not None) == self.before, "gate and w_before as this norm was made"

    def forward(self, x, y=None, w_after=None, gate=None, w_before=None):
        """(out, h): the stream behind the block and the next block's input."""
        assert tuple(x.shape) == (self.T, self.d) and x.dtype == self.dtype, "x does not fit this norm"
        self._fits(y, w_after, gate, w_before)
        B.moe_block_norm_fwd(x, y, w_after, gate, w_before, self.gate_rows, self.alpha, self.eps, self.out, self.h)
        return (self.out if self.residual else x), self.h

    def backward(self, out, y=None, w_after=None, gate=None, w_before=None, d_out=None, d_h=None, accumulate: bool = False):
        """dx and dy, and the weights' gradients, from the gradients of the stream (None: none comes down it) and of h.  out: the stream as `forward`
        returned it.  accumulate adds into the weights' gradients."""
        assert self.gradients, "made without gradients"
        self._fits(y, w_after, gate, w_before)
        assert (d_h is not None) == self.before, "d_h where there is a norm before the next block"
        assert d_out is not None or d_h is not None, "no gradient"
        B.moe_block_norm_bwd(out, y, w_after, gate, w_before, d_out, d_h, self.gate_rows, self.alpha, self.eps, self.dx, self.dy, self.d_w_after,
                             self.d_gate, self.d_w_before, accumulate, self.workspace)
        return self.dx, self.dy
