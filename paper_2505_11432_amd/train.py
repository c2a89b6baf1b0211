"""A training step around the layer on one GPU: MoE layer, residual, vocabulary loss, their backward, clipping, AdamW.

    python -m paper_2505_11432_amd.train                        # a small bf16 model learns a permutation of its vocabulary
    python -m paper_2505_11432_amd.train --dtype f32 --graph    # the same in single precision, every step replayed from one HIP graph
    python -m paper_2505_11432_amd.train --norms --embedding --muon      # a whole block: trained embedding, norms, Muon for the experts

Everything stays on the device: the loss, the norm and the learning rate are device numbers, so a step enqueues its kernels and
returns.  The embedding is a fixed table (the layer's input gradient ends there) unless it is trained as well.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as B
from .embedding import Embedding
from .head import VocabLoss
from .layer import MoELayer
from .norm import BlockNorm
from .optim import AdamW, GradClip, Muon


class TrainStep:
    """hidden = x + MoE(x); loss over the vocabulary; gradients clipped to max_norm; one AdamW update, left out where the norm is infinite or NaN (the
    step count then stays, so the host can see it whenever it looks).

    Master parameters w_r [E, d], w1 [E, 2f, d], w2 [E, d, f] and w_vocab [V, d] are fp32; bf16 models multiply with the copies
    that the update rounds them to.  grad_dtype: of the gradients of w1, w2 and w_vocab (that of w_r is fp32).

    norms: hidden = norm(s) w_out with s = x + gate * norm(MoE(norm(x) w_in)) w_after; w_in, w_after, gate and w_out [d] are trained (fp32, no copies).
    embedding: the table [V, d] is trained (x = rows of it); its gradient is fp32.
    muon: the experts' matrices (gate and up projections each a matrix of its own) are updated by Muon with the same learning rate, the rest by AdamW.
    What these add to masters and params follows the first four: the table, then w_in, w_after, gate, w_out."""

    def __init__(self, T, d, E, k, f, V, dtype=torch.bfloat16, lr=3e-3, max_norm=1.0, weight_decay=0.0, seed=0, device="cuda:0",
                 grad_dtype=torch.float32, norms=False, embedding=False, muon=False):
        g = torch.Generator(device=device).manual_seed(seed)

        def normal(*shape, std):
            return torch.randn(shape, dtype=torch.float32, device=device, generator=g) * std

        self.layer = MoELayer(T, d, E, k, f, dtype=dtype, grad_dtype=grad_dtype, device=device)
        self.head = VocabLoss(T, d, V, dtype=dtype, grad_dtype=grad_dtype, device=device)
        self.masters = [normal(E, d, std=0.1), normal(E, 2 * f, d, std=d ** -0.5), normal(E, d, f, std=f ** -0.5), normal(V, d, std=d ** -0.5)]
        grads = [self.layer.d_w_r, self.layer.d_w1, self.layer.d_w2, self.head.d_w]
        table = normal(V, d, std=1.0)
        self.embed = None
        if embedding:
            self.embed = Embedding(T, d, V, dtype=dtype, device=device)
            self.masters.append(table)
            grads.append(self.embed.d_table)
        copied = len(self.masters)               # the others are used in fp32
        self.first = self.last = None
        if norms:
            self.first = BlockNorm(T, d, dtype=dtype, residual=False, after=False, device=device)
            self.last = BlockNorm(T, d, dtype=dtype, gate_rows=max(T, 1), device=device)
            self.masters += [torch.ones((d,), dtype=torch.float32, device=device) for _ in range(2)]
            self.masters += [torch.ones((1, d), dtype=torch.float32, device=device), torch.ones((d,), dtype=torch.float32, device=device)]
            grads += [self.first.d_w_before, self.last.d_w_after, self.last.d_gate, self.last.d_w_before]
        self.params = [p.to(dtype) if i < copied else p for i, p in enumerate(self.masters)]         # (fp32: the masters themselves)
        moments = [[torch.zeros_like(p) for p in self.masters] for _ in range(2)]
        copies = [None if dtype == torch.float32 or i >= copied else p for i, p in enumerate(self.params)]
        self.clip = GradClip(grads, max_norm)
        self.left_out = torch.full((1,), float("nan"), dtype=torch.float32, device=device)
        self.lr = torch.full((1,), lr, dtype=torch.float32, device=device)
        self.muon = None
        by_adamw = list(range(len(self.masters)))
        if muon:
            by_adamw = [i for i in by_adamw if i not in (1, 2)]
            as_matrices = lambda t: None if t is None else t.view(2 * E, f, d)           # noqa: E731  (w1 and what belongs to it)
            lists = [[as_matrices(t[1]), t[2]] for t in (self.masters, grads, moments[0], copies)]
            self.muon = Muon(*lists[:3], weights=lists[3], lr=self.lr, weight_decay=weight_decay)
        pick = lambda t: [t[i] for i in by_adamw]         # noqa: E731
        self.adamw = AdamW(pick(self.masters), pick(grads), pick(moments[0]), pick(moments[1]), weights=None if dtype == torch.float32 else pick(copies),
                           lr=self.lr, weight_decay=weight_decay)
        self.embedding = table.to(dtype) if self.embed is None else self.params[4]
        self.x = torch.empty((T, d), dtype=dtype, device=device) if self.embed is None else self.embed.out
        self.hidden = torch.empty_like(self.x) if self.last is None else self.last.h
        self.tokens = torch.zeros((T,), dtype=torch.int32, device=device)
        self.target = torch.empty((T,), dtype=torch.int32, device=device)
        self.graph = None

    def load(self, tokens, target):
        """The batch of the next step: tokens [T] (indices of the embedding), target [T] int32 (outside the vocabulary: left out)."""
        if self.embed is None:
            torch.index_select(self.embedding, 0, tokens, out=self.x)
        else:
            self.tokens.copy_(tokens)
        self.target.copy_(target)

    def _enqueue(self):
        w_r, w1, w2, w_vocab = self.params[:4]
        if self.embed is not None:
            self.embed.lookup(self.embedding, self.tokens)
        if self.last is None:
            layer_in = self.x
            y = self.layer.forward(layer_in, w_r, None, w1, w2)
            torch.add(self.x, y, out=self.hidden)
            self.head.step(self.hidden, w_vocab, self.target)
            self.layer.backward(layer_in, w_r, w1, w2, self.head.dx)
            if self.embed is not None:           # (the layer's input is the stream itself)
                torch.add(self.layer.dx, self.head.dx, out=self.layer.dx)
                d_stream = self.layer.dx
        else:
            w_in, w_after, gate, w_out = self.params[-4:]
            _, layer_in = self.first.forward(self.x, w_before=w_in)
            y = self.layer.forward(layer_in, w_r, None, w1, w2)
            out, hidden = self.last.forward(self.x, y, w_after, gate, w_out)
            self.head.step(hidden, w_vocab, self.target)
            d_stream, dy = self.last.backward(out, y, w_after, gate, w_out, None, self.head.dx)
            d_in = self.layer.backward(layer_in, w_r, w1, w2, dy)
            d_stream, _ = self.first.backward(self.x, w_before=w_in, d_out=d_stream, d_h=d_in)
        if self.embed is not None:
            self.embed.backward(self.tokens, d_stream)
        self.clip.clip()
        coef = torch.where(torch.isfinite(self.clip.norm), self.clip.coef, self.left_out)
        if self.muon is not None:
            self.muon.step(coef=coef)
        self.adamw.step(coef=coef)

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
    p.add_argument("--norms", action="store_true", help="norms before and after the layer, and before the loss")
    p.add_argument("--embedding", action="store_true", help="train the embedding too")
    p.add_argument("--muon", action="store_true", help="update the experts' matrices by Muon")
    a = p.parse_args()
    model = TrainStep(a.tokens, 256, 8, 2, 320, a.vocab, dtype=torch.float32 if a.dtype == "f32" else torch.bfloat16, norms=a.norms, embedding=a.embedding,
                      muon=a.muon)
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
