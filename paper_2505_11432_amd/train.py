"""A training step around the layer on one GPU: MoE layer, residual, vocabulary loss, their backward, clipping, AdamW.

    python -m paper_2505_11432_amd.train                        # a small bf16 model learns a permutation of its vocabulary
    python -m paper_2505_11432_amd.train --dtype f32 --graph    # the same in single precision, every step replayed from one HIP graph

Everything stays on the device: the loss, the norm and the learning rate are device numbers, so a step enqueues its kernels and
returns.  The embedding is a fixed table (the layer's input gradient ends there).
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B
from .head import VocabLoss
from .layer import MoELayer
from .optim import AdamW, GradClip


class TrainStep:
    """hidden = x + MoE(x); loss over the vocabulary; gradients clipped to max_norm; one AdamW update, left out where the norm is infinite or NaN (the
    step count then stays, so the host can see it whenever it looks).

    Master parameters w_r [E, d], w1 [E, 2f, d], w2 [E, d, f] and w_vocab [V, d] are fp32; bf16 models multiply with the copies
    that the update rounds them to.  grad_dtype: of the gradients of w1, w2 and w_vocab (that of w_r is fp32)."""

    def __init__(self, T, d, E, k, f, V, dtype=torch.bfloat16, lr=3e-3, max_norm=1.0, weight_decay=0.0, seed=0, device="cuda:0",
                 grad_dtype=torch.float32):
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, std):
            return torch.randn(shape, dtype=torch.float32, device=device, generator=g) * std

        self.layer = MoELayer(T, d, E, k, f, dtype=dtype, grad_dtype=grad_dtype, device=device)
        self.head = VocabLoss(T, d, V, dtype=dtype, grad_dtype=grad_dtype, device=device)
        self.masters = [normal(E, d, std=0.1), normal(E, 2 * f, d, std=d ** -0.5), normal(E, d, f, std=f ** -0.5), normal(V, d, std=d ** -0.5)]
        self.params = self.masters if dtype == torch.float32 else [p.to(dtype) for p in self.masters]
        grads = [self.layer.d_w_r, self.layer.d_w1, self.layer.d_w2, self.head.d_w]
        moments = [[torch.zeros_like(p) for p in self.masters] for _ in range(2)]
        self.clip = GradClip(grads, max_norm)
        self.left_out = torch.full((1,), float("nan"), dtype=torch.float32, device=device)
        self.lr = torch.full((1,), lr, dtype=torch.float32, device=device)
        self.adamw = AdamW(self.masters, grads, *moments, weights=None if dtype == torch.float32 else self.params, lr=self.lr,
                           weight_decay=weight_decay)
        self.embedding = normal(V, d, std=1.0).to(dtype)
        self.x = torch.empty((T, d), dtype=dtype, device=device)
        self.hidden = torch.empty_like(self.x)
        self.target = torch.empty((T,), dtype=torch.int32, device=device)
        self.graph = None

    def load(self, tokens, target):
        """The batch of the next step: tokens [T] (indices of the embedding), target [T] int32 (outside the vocabulary: left out)."""
        torch.index_select(self.embedding, 0, tokens, out=self.x)
        self.target.copy_(target)

    def _enqueue(self):
        w_r, w1, w2, w_vocab = self.params
        y = self.layer.forward(self.x, w_r, None, w1, w2)
        torch.add(self.x, y, out=self.hidden)
        self.head.step(self.hidden, w_vocab, self.target)
        self.layer.backward(self.x, w_r, w1, w2, self.head.dx)
        self.clip.clip()
        self.adamw.step(coef=torch.where(torch.isfinite(self.clip.norm), self.clip.coef, self.left_out))

    def step(self):
        """Enqueues one step; returns the loss [1] and the gradient norm [1], on the device."""
        if self.graph is None:
            self._enqueue()
        else:
            self.graph.replay()
        return self.head.total, self.clip.norm

    def capture(self):
        """From here on a step is the replay of one graph.  (Recording runs nothing.)"""
        B.moe_init()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            self._enqueue()
        self.graph = graph


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--steps", type=int, default=60)
    p.add_argument("--tokens", type=int, default=512)
    p.add_argument("--vocab", type=int, default=1000)
    p.add_argument("--dtype", choices=("bf16", "f32"), default="bf16")
    p.add_argument("--graph", action="store_true")
    a = p.parse_args()
    model = TrainStep(a.tokens, 256, 8, 2, 320, a.vocab, dtype=torch.float32 if a.dtype == "f32" else torch.bfloat16)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    follow = torch.randperm(a.vocab, device="cuda:0", generator=g)
    for i in range(a.steps):
        tokens = torch.randint(0, a.vocab, (a.tokens,), device="cuda:0", generator=g)
        model.load(tokens, follow[tokens])
        if i == 1 and a.graph:              # (after one eager step: every kernel has been set up)
            model.capture()
        loss, norm = model.step()
        if i % 10 == 0 or i + 1 == a.steps:
            print(f"step {i + 1}: loss {float(loss):.4f}, gradient norm {float(norm):.4f}", flush=True)


if __name__ == "__main__":
    main()
