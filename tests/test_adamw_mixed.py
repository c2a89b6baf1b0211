"""AdamW over a list whose gradients are of both types, as the layer makes them (bf16 of the experts, fp32 of the router)."""
import ctypes

import pytest

P, F32, BF16, E4M3, MIXED = ctypes.c_void_p, 0, 1, 2, 3


@pytest.fixture(scope="module")
def lib():
    from paper_2505_11432_amd.build import LIB_PATH, ensure_built
    ensure_built()
    lib = ctypes.CDLL(LIB_PATH)
    lib.moe_adamw_table_mixed.argtypes = [ctypes.c_int, P, P, P, P, P, P, P, P]
    lib.moe_adamw_table.argtypes = [ctypes.c_int, P, P, P, P, P, P, ctypes.c_int, P]
    return lib


def array(kind, *v):
    return (kind * max(1, len(v)))(*v)


def test_table(lib):
    host, one = (ctypes.c_int64 * 64)(), (ctypes.c_int64 * 64)()
    a, g, n = array(P, 4096, 8192, None), array(P, 4096, 8194, None), array(ctypes.c_int64, 3, 4, 0)
    dt = array(ctypes.c_int32, F32, BF16, F32)
    fill = lambda n_=3, p=a, g=g, dt=dt, m=a, v=a, w=None, numel=n, host=host: lib.moe_adamw_table_mixed(n_, p, g, dt, m, v, w, numel, host)
    assert fill() == 0
    assert [host[6 * i + 5] for i in range(4)] == [0, 3, 7, 7]
    assert [host[6 * i + 1] for i in range(3)] == [4096, 8194 | 1, 0]           # the type in bit 0
    assert lib.moe_adamw_table(2, a, a, a, a, None, n, F32, one) == 0 and [one[6 * i + 1] for i in range(2)] == [4096, 8192]
    assert lib.moe_adamw_table(1, a, a, a, a, None, n, BF16, one) == 0 and one[1] == 4096
    assert fill(n_=0, p=None, g=None, dt=None, m=None, v=None, numel=None) == 0
    assert fill(n_=-1) == fill(p=None) == fill(g=None) == fill(dt=None) == fill(m=None) == fill(v=None) == fill(numel=None) == fill(host=None) == -1
    assert fill(g=array(P, 4096, None, None)) == -1
    assert fill(dt=array(ctypes.c_int32, F32, E4M3, F32)) == fill(dt=array(ctypes.c_int32, F32, F32, F32)) == fill(g=array(P, 4098, 8194, None)) == -2
    assert fill(g=array(P, 4096, 8193, None)) == -2


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [[5, 7], [40_003, 0, 17, 100_000], [1] * 40, [3_000_001, 1_500_007, 9]])
def test_against_lists_of_one_type(sizes):
    """The same bits as from two lists of one type each."""
    import torch

    from paper_2505_11432_amd.optim import AdamW
    dev = "cuda:0"
    gen = torch.Generator(device=dev).manual_seed(3)

    def normal(n, offset, scale):
        return (torch.randn((n + offset,), device=dev, generator=gen) * scale)[offset:]

    p, m, v = ([normal(n, i % 3, 0.02) for i, n in enumerate(sizes)] for _ in range(3))
    v = [t.square_() for t in v]
    g = [normal(n, i % 2, 1e-3) if i % 2 == 0 else torch.cat([torch.zeros((1,), device=dev), normal(n, 0, 1e-3)]).to(torch.bfloat16)[1:]
         for i, n in enumerate(sizes)]
    w = [torch.zeros((n,), dtype=torch.bfloat16, device=dev) if i % 3 else None for i, n in enumerate(sizes)]
    pick = lambda x, k: [None if t is None else t.clone() for t in x[k::2]]
    apart = [AdamW(pick(p, k), pick(g, k), pick(m, k), pick(v, k), weights=pick(w, k)) for k in (0, 1)]
    op = AdamW(p, g, m, v, weights=w)
    coef = torch.full((1,), 0.625, device=dev)
    for t in (1, 2):
        for o in (op, *apart):
            o.step(coef=coef)
        assert int(op.step_count) == t
    for k in (0, 1):
        for a, b in ((p, apart[k].params), (m, apart[k].m), (v, apart[k].v), (w, apart[k].weights)):
            assert all(x is None or torch.equal(x, y) for x, y in zip(a[k::2], b))


@pytest.mark.gpu
def test_training_step_with_bf16_gradients():
    """The layer's own list: w_r in fp32, the others in bf16."""
    import math

    import torch

    from paper_2505_11432_amd.train import TrainStep
    T, V = 400, 300
    model = TrainStep(T, 128, 4, 2, 144, V, grad_dtype=torch.bfloat16)
    assert {t.dtype for t in model.adamw.grads} == {torch.bfloat16, torch.float32}
    g = torch.Generator(device="cuda:0").manual_seed(1)
    follow = torch.randperm(V, device="cuda:0", generator=g)
    losses = []
    for i in range(40):
        tokens = torch.randint(0, V, (T,), device="cuda:0", generator=g)
        model.load(tokens, follow[tokens])
        if i == 2:
            model.capture()
        loss, _ = model.step()
        losses.append(float(loss))
    assert losses[0] > math.log(V) - 1.0 and losses[-1] < losses[0] / 2 and int(model.adamw.step_count) == 40
