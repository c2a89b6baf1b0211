"""Rows of an embedding for a batch of tokens, and its gradient, on one GPU: buffers allocated once, then one C-ABI call per pass."""
from __future__ import annotations

import torch

from . import binding as B


class Embedding:
    """out[t] = scale * table[tokens[t]] and d_table[v] = scale * sum of dy[t] over the tokens t that are v.

    T tokens (int32; outside 0..V-1: padding, a row of zeros without a gradient), V words of width d.  dtype: of the table, its rows and dy (bf16 or
    fp32); grad_dtype: of d_table (fp32, or bf16 for bf16 data).
    d_table: None, or the [V, d] gradient that `backward` writes or adds to (that of a matrix shared with the vocabulary loss).
    gradients = False: `lookup` only, without the buffers of a gradient.

    Buffers: out [T, d], d_table [V, d]."""

    def __init__(self, T: int, d: int, V: int, dtype=torch.bfloat16, grad_dtype=torch.float32, scale: float = 1.0, gradients: bool = True, d_table=None,
                 device="cuda:0"):
        assert T >= 0 and d > 0 and V > 0, "sizes are positive"
        assert dtype in (torch.bfloat16, torch.float32), "rows are bf16 or fp32"
        grad_dtype = d_table.dtype if d_table is not None else grad_dtype
        assert grad_dtype in (torch.float32, dtype), "the gradient is fp32 or of the data's type"
        self.T, self.d, self.V, self.dtype, self.scale, self.gradients = T, d, V, dtype, float(scale), gradients
        size = B.moe_embedding_workspace_bytes(T, d, V)
        assert size > 0, f"unsupported sizes: T {T}, d {d} (a multiple of 16), V {V}"
        self.out = torch.empty((T, d), dtype=dtype, device=device)
        if gradients:
            assert d_table is None or tuple(d_table.shape) == (V, d), "d_table does not fit this embedding"
            self.d_table = d_table if d_table is not None else torch.zeros((V, d), dtype=grad_dtype, device=device)
            self.workspace = torch.empty((size,), dtype=torch.uint8, device=device)

    def lookup(self, table, tokens):
        assert tuple(table.shape) == (self.V, self.d) and table.dtype == self.dtype, "table does not fit this embedding"
        B.moe_embedding_fwd(table, tokens, self.scale, self.out)
        return self.out

    def backward(self, tokens, dy, accumulate: bool = False):
        """d_table from the rows' gradients; accumulate adds to it (a micro-batch after the first, a shared matrix)."""
        assert self.gradients, "made without gradients"
        assert tuple(dy.shape) == (self.T, self.d) and dy.dtype == self.dtype, "dy does not fit this embedding"
        B.moe_embedding_bwd(tokens, dy, self.scale, self.d_table, accumulate, self.workspace)
        return self.d_table
