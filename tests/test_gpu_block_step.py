"""The parts around the layer together, as the training step uses them: embedding, norm, MoE layer, norm with gate, norm, vocabulary loss, all gradients,
clipping, Muon for the experts and AdamW for the rest."""
import math

import pytest
import torch

DEV = "cuda:0"


def batches(T, V, n, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    for _ in range(n):
        tokens = torch.randint(0, V, (T,), device=DEV, generator=g)
        tokens[torch.rand((T,), device=DEV, generator=g) < 0.1] = 3                  # a frequent word
        target = torch.randint(0, V, (T,), device=DEV, generator=g)
        target[torch.rand((T,), device=DEV, generator=g) < 0.1] = -100
        yield tokens, target


def make(T, V, dtype, **k):
    from paper_2505_11432_amd.train import TrainStep
    model = TrainStep(T, 128, 4, 2, 144, V, dtype=dtype, **k)
    if k.get("norms"):
        g = torch.Generator(device=DEV).manual_seed(9)
        for p in model.masters[-4:]:
            p.add_(0.3 * torch.randn(p.shape, device=DEV, generator=g))
    return model


def reference(model, tokens, target, norms):
    """Loss and gradients of the step's function in 64 bits, by autograd, with the experts that the step chose."""
    leaves = [p.detach().double().requires_grad_() for p in model.params]
    w_r, w1, w2, w_vocab, table = leaves[:5]
    x = table[tokens.long()]

    def rms(v, w):
        return v / torch.sqrt(v.pow(2).mean(-1, keepdim=True) + 1e-6) * w

    layer_in = rms(x, leaves[-4]) if norms else x
    chosen = model.layer.topk_idx.long()
    share = torch.softmax((layer_in @ w_r.t()).gather(1, chosen), 1)
    f = w2.shape[2]
    y = torch.zeros_like(x)
    for e in range(w_r.shape[0]):
        h = layer_in @ w1[e].t()
        out = (torch.nn.functional.silu(h[:, :f]) * h[:, f:]) @ w2[e].t()
        y = y + (share * (chosen == e)).sum(1, keepdim=True) * out
    stream = x + (rms(y, leaves[-3]) * leaves[-2] if norms else y)
    hidden = rms(stream, leaves[-1]) if norms else stream
    keep = target >= 0
    logp = torch.log_softmax(hidden[keep] @ w_vocab.t(), 1)
    loss = -logp.gather(1, target[keep].long()[:, None]).mean()
    return loss, torch.autograd.grad(loss, leaves)


@pytest.mark.gpu
@pytest.mark.parametrize("norms", [True, False])
def test_gradients_in_single_precision(norms):
    """Every gradient of a step in fp32 against autograd in 64 bits.  The operations between a parameter and the loss are some dozen, each with a relative error
    (2-norm) of a few 2^-24 times the square root of its sums' lengths (144 at most here): 12 * 4 * 12 * 2^-24 < 2^-14."""
    T, V = 210, 150
    model = make(T, V, torch.float32, norms=norms, embedding=True)
    tokens, target = next(batches(T, V, 1))
    model.load(tokens, target)
    before = [p.clone() for p in model.params]
    loss, _ = model.step()
    after = [p.clone() for p in model.params]
    for p, b in zip(model.params, before):
        p.copy_(b)
    want, grads = reference(model, tokens, target, norms)
    assert abs(float(loss) - float(want.detach())) <= 2.0 ** -14 * float(want.detach())
    got = [model.layer.d_w_r, model.layer.d_w1, model.layer.d_w2, model.head.d_w, model.embed.d_table]
    if norms:
        got += [model.first.d_w_before, model.last.d_w_after, model.last.d_gate, model.last.d_w_before]
    assert len(got) == len(grads)
    for i, (a, b) in enumerate(zip(got, grads)):
        assert float((a.double() - b).norm()) <= 2.0 ** -14 * float(b.norm()), i
    for a, b in zip(after, before):
        assert not torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_the_updates(dtype):
    """One step's updates from the gradients that it made: Muon on w1's halves and w2, the masters' copies, AdamW on the rest."""
    from test_gpu_muon import exact
    T, V = 130, 100
    model = make(T, V, dtype, norms=True, embedding=True, muon=True, lr=1e-2, weight_decay=0.1)
    was = [p.clone() for p in model.masters]
    model.load(*next(batches(T, V, 1)))
    _, norm = model.step()
    coef = min(1.0, 1.0 / (float(norm) + 1e-6))
    lr = float(model.lr)
    for i, grad in ((1, model.layer.d_w1.view(8, 144, 128)), (2, model.layer.d_w2)):
        # (the momentum begins at 0: m = g, u = 1.95 g, whose factor the norm takes out.  These gradients have few rows, one per token of an expert: what the
        # roundings leave in the other directions is multiplied by up to 3.4445^5 = 485, so that two runs from u and g, 2^-24 apart, already differ by a share
        # of the operator's own error.  So the update is compared with the formula in 64 bits, within that error)
        p0, got = was[i].view(grad.shape).double(), model.masters[i].view(grad.shape).double()
        for e in range(grad.shape[0]):
            o, tol = exact(grad[e].float() * coef)
            want = p0[e] * (1 - lr * 0.1) - lr * 0.2 * 144 ** 0.5 * o
            # (p in fp32: half a step, and lr, the decay and their products in fp32, some 2^-23 of what they are factors of)
            assert float((got[e] - want).norm()) <= 2.0 ** -22 * float(p0[e].norm()) + lr * 0.2 * 144 ** 0.5 * (tol + 2.0 ** -22 * float(o.norm()))
    for i, grad in ((0, model.layer.d_w_r), (3, model.head.d_w), (4, model.embed.d_table), (5, model.first.d_w_before), (7, model.last.d_gate)):
        c = grad.double() * coef
        want = was[i].double() * (1 - lr * 0.1) - lr * c / (c.abs() + 1e-8)
        assert float((model.masters[i].double() - want).abs().max()) <= 2.0 ** -20 * (float(was[i].abs().max()) + lr)
    if dtype == torch.bfloat16:
        for p, m in list(zip(model.params, model.masters))[:5]:
            assert torch.equal(p, m.to(dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("k", [dict(norms=True, embedding=True, muon=True), dict(embedding=True), dict(norms=True), dict(muon=True)])
def test_replayed_from_a_graph(dtype, k):
    T, V = 300, 200
    eager, graph = make(T, V, dtype, **k), make(T, V, dtype, **k)
    for i, (tokens, target) in enumerate(batches(T, V, 6)):
        for m in (eager, graph):
            m.load(tokens, target)
        if i == 1:
            graph.capture()
        a = [t.clone() for t in eager.step()]
        b = [t.clone() for t in graph.step()]
        torch.cuda.synchronize()
        assert math.isfinite(float(a[0])) and math.isfinite(float(a[1]))
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        for p, q in zip(eager.masters + eager.params, graph.masters + graph.params):
            assert torch.equal(p, q)


@pytest.mark.gpu
def test_a_bad_step_changes_nothing():
    """A gradient that is no number: the norm is none, and neither Muon nor AdamW changes anything."""
    T, V = 100, 80
    model = make(T, V, torch.bfloat16, norms=True, embedding=True, muon=True)
    tokens, target = next(batches(T, V, 1))
    model.load(tokens, target)
    model.step()
    keep = model.embedding[5].clone()
    model.embedding[5] = float("nan")
    tokens[0] = 5
    model.load(tokens, target)
    was = [p.clone() for p in model.masters] + [m.clone() for m in model.muon.m]
    count = int(model.adamw.step_count)
    _, norm = model.step()
    assert not math.isfinite(float(norm)) and int(model.adamw.step_count) == count
    for a, b in zip(was, model.masters + model.muon.m):
        assert torch.equal(a, b)
    model.embedding[5] = keep
    model.load(tokens, target)
    _, norm = model.step()
    assert math.isfinite(float(norm))
    for p in model.masters:
        assert bool(torch.isfinite(p).all())


@pytest.mark.gpu
def test_a_table_shared_with_the_loss():
    """d_table of the embedding is d_w of the loss: its gradient is added behind the loss's."""
    from paper_2505_11432_amd.embedding import Embedding
    from paper_2505_11432_amd.head import VocabLoss
    T, d, V = 120, 64, 90
    g = torch.Generator(device=DEV).manual_seed(2)
    table = torch.randn((V, d), device=DEV, generator=g)
    head = VocabLoss(T, d, V, dtype=torch.float32, device=DEV)
    embed = Embedding(T, d, V, dtype=torch.float32, scale=8.0, d_table=head.d_w, device=DEV)
    tokens, target = next(batches(T, V, 1))
    tokens, target = tokens.to(torch.int32), target.to(torch.int32)
    x = embed.lookup(table, tokens)
    head.step(x, table, target)
    embed.backward(tokens, head.dx, accumulate=True)
    leaf = table.double().requires_grad_()
    keep = target >= 0
    logp = torch.log_softmax((8.0 * leaf[tokens.long()])[keep] @ leaf.t(), 1)
    loss = -logp.gather(1, target[keep].long()[:, None]).mean()
    want, = torch.autograd.grad(loss, leaf)
    assert float((head.d_w.double() - want).norm()) <= 2.0 ** -15 * float(want.norm())
