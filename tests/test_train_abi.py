"""Host-only checks of the entry points behind the layer: sizes, tables and refused arguments.  Nothing here reaches a stream."""
import ctypes

import pytest

P, I, Z, D = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_double
FAKE, NULL = P(4096), P(0)
F32, BF16, E4M3 = 0, 1, 2


@pytest.fixture(scope="module")
def lib():
    from paper_2505_11432_amd.build import LIB_PATH, ensure_built
    ensure_built()
    lib = ctypes.CDLL(LIB_PATH)
    lib.moe_vocab_workspace_bytes.restype = Z
    lib.moe_vocab_score.argtypes = [P, P, P, I, I, I, I, I, P, P, P, Z, P]
    lib.moe_vocab_loss.argtypes = [P, P, P, P, I, I, I, I, I, P, P, P, P, P, I, I, P, Z, P]
    lib.moe_grad_clip_table_bytes.restype = lib.moe_grad_clip_workspace_bytes.restype = lib.moe_adamw_table_bytes.restype = Z
    lib.moe_grad_clip_table.argtypes = [I, P, P, P, P, P]
    lib.moe_grad_clip.argtypes = [P, I, ctypes.c_int64, D, I, P, P, P, Z, P]
    lib.moe_adamw_table.argtypes = [I, P, P, P, P, P, P, I, P]
    lib.moe_adamw.argtypes = [P, I, ctypes.c_int64, I, P, P, P, D, D, D, D, P, Z, P]
    return lib


def test_workspace(lib):
    size = lib.moe_vocab_workspace_bytes
    # one piece: the kept elements of every row and the gathered rows at least
    assert size(8192, 4096, 32000, BF16, BF16, 0, 1) >= 8192 * 32000 * 2 + 8192 * 4096 * 2
    # pieces bound it, and several of them sum the gradient of bf16 data in fp32
    assert size(8192, 4096, 32000, BF16, F32, 2048, 1) < size(8192, 4096, 32000, BF16, F32, 0, 1) / 2
    assert size(8192, 4096, 32000, BF16, BF16, 2048, 1) >= 2048 * 32000 * 2 + 32000 * 4096 * 4
    # the score of bf16 data keeps no element
    assert size(8192, 4096, 32000, BF16, BF16, 0, 0) < 8192 * 4096 * 2 + (1 << 25)
    assert size(0, 64, 100, BF16, BF16, 0, 1) > 0
    for bad in ((-1, 64, 100, BF16, BF16, 0, 1), (8, 60, 100, BF16, BF16, 0, 1), (8, 64, 0, BF16, BF16, 0, 1), (8, 64, 100, E4M3, F32, 0, 1),
                (8, 64, 100, F32, BF16, 0, 1), (8, 64, 100, BF16, BF16, -1, 1), (8, 0, 100, BF16, BF16, 0, 1), (8, 64, (1 << 24) + 1, BF16, BF16, 0, 1)):
        assert size(*bad) == 0, bad


def test_vocab_arguments(lib):
    need = lib.moe_vocab_workspace_bytes(8, 64, 100, BF16, F32, 0, 1)

    def step(x=FAKE, w=FAKE, target=FAKE, token_w=NULL, dt=BF16, T=8, d=64, V=100, piece=0, total=FAKE, loss=FAKE, lse=FAKE, dx=FAKE, d_w=FAKE, gdt=F32,
             acc=0, ws=FAKE, n=need):
        return lib.moe_vocab_loss(x, w, target, token_w, dt, T, d, V, piece, total, loss, lse, dx, d_w, gdt, acc, ws, n, None)

    for k in ("x", "w", "target", "total", "loss", "lse", "dx", "d_w"):
        assert step(**{k: NULL}) == -1, k
    assert step(T=-1) == step(V=0) == step(d=0) == step(piece=-1) == -1
    assert step(d=72) == step(dt=E4M3) == step(gdt=E4M3) == step(dt=F32, gdt=BF16) == -2
    assert step(x=P(4104)) == step(w=P(4104)) == step(dx=P(4104)) == step(d_w=P(4104)) == step(target=P(4098)) == step(token_w=P(4098)) == -2
    assert step(ws=NULL) == step(n=need - 1) == step(ws=P(4104)) == -3
    assert step(T=0, x=NULL, w=NULL, ws=NULL, n=0) == 0
    need0 = lib.moe_vocab_workspace_bytes(8, 64, 100, BF16, BF16, 0, 0)
    score = lambda x=FAKE, dt=BF16, T=8, d=64, ws=FAKE, n=need0, lse=FAKE: lib.moe_vocab_score(x, FAKE, FAKE, dt, T, d, 100, 0, FAKE, lse, ws, n, None)
    assert score(x=NULL) == score(T=-1) == score(lse=NULL) == -1
    assert score(dt=E4M3) == score(d=40) == score(x=P(4104)) == -2
    assert score(ws=NULL) == score(n=need0 - 1) == -3
    assert score(T=0, x=NULL, ws=NULL) == 0


def array(kind, *v):
    return (kind * max(1, len(v)))(*v)


def test_clip_table_and_arguments(lib):
    size = lib.moe_grad_clip_table_bytes
    assert size(0) > 0 and size(3) == 4 * size(0) and size(-1) == 0
    host = (ctypes.c_int64 * 64)()
    g, o = array(P, 4096, 8194, None), array(P, 4096, None, None)
    fill = lambda n=3, g=g, o=o, numel=array(ctypes.c_int64, 5, 7, 0), dt=array(ctypes.c_int32, F32, BF16, F32), host=host: lib.moe_grad_clip_table(n, g, o, numel, dt, host)
    assert fill() == 0
    rows = [host[4 * i + 2] for i in range(4)]           # first elements
    assert rows == [0, 5, 12, 12] and host[0] == host[1] == 4096 and host[4] == 8194 and host[5] == 0
    assert fill(o=None) == 0 and fill(n=0, g=None, o=None, numel=None, dt=None) == 0
    assert fill(n=-1) == fill(g=None) == fill(host=None) == fill(numel=array(ctypes.c_int64, 5, -1, 0)) == -1
    assert fill(g=array(P, 4096, None, None)) == -1      # seven elements nowhere
    assert fill(numel=array(ctypes.c_int64, 1 << 62, 1 << 62, 0)) == -1
    assert fill(dt=array(ctypes.c_int32, F32, E4M3, F32)) == fill(g=array(P, 4098, 8194, None)) == fill(g=array(P, 4096, 8193, None)) == -2
    ws = lib.moe_grad_clip_workspace_bytes()
    clip = lambda table=FAKE, n=1, total=5, limit=1.0, norm=FAKE, coef=FAKE, w=FAKE, b=ws: lib.moe_grad_clip(table, n, total, limit, 1, norm, coef, w, b, None)
    assert clip(table=NULL) == clip(n=-1) == clip(total=-1) == clip(limit=-1.0) == clip(limit=float("nan")) == clip(norm=NULL) == clip(coef=NULL) == -1
    assert clip(table=P(4100)) == clip(norm=P(4098)) == -2
    assert clip(w=NULL) == clip(b=ws - 1) == -3


def test_adamw_table_and_arguments(lib):
    size = lib.moe_adamw_table_bytes
    assert size(1) == 2 * size(0) > 0 and size(-1) == 0
    host = (ctypes.c_int64 * 64)()
    a = array(P, 4096, 8192)
    n2 = array(ctypes.c_int64, 3, 4)
    fill = lambda n=2, p=a, g=a, m=a, v=a, w=None, numel=n2, dt=F32, host=host: lib.moe_adamw_table(n, p, g, m, v, w, numel, dt, host)
    assert fill() == 0 and [host[6 * i + 5] for i in range(3)] == [0, 3, 7]
    assert fill(w=array(P, 4098, None)) == 0 and host[4] == 4098
    assert fill(p=None) == fill(g=None) == fill(m=None) == fill(v=None) == fill(numel=None) == fill(n=-1) == fill(p=array(P, 4096, None)) == -1
    assert fill(dt=E4M3) == fill(p=array(P, 4098, 8192)) == fill(g=array(P, 4098, 8192)) == fill(w=array(P, 4097, None)) == -2
    assert fill(g=array(P, 4098, 8192), dt=BF16) == 0
    step = lambda table=FAKE, n=1, total=5, dt=F32, lr=FAKE, st=FAKE, coef=NULL, b1=0.9, b2=0.95, eps=1e-8, wd=0.1, ws=FAKE, b=16: lib.moe_adamw(
        table, n, total, dt, lr, st, coef, b1, b2, eps, wd, ws, b, None)
    assert step(table=NULL) == step(n=-1) == step(total=-1) == step(lr=NULL) == step(st=NULL) == -1
    assert step(b1=1.0) == step(b2=-0.1) == step(b1=float("nan")) == step(eps=-1.0) == step(wd=float("nan")) == -1
    assert step(dt=E4M3) == step(lr=P(4098)) == step(coef=P(4098)) == step(table=P(4100)) == -2
    assert step(ws=NULL) == step(b=8) == -3


def test_vocab_outputs_lie_apart(lib):
    """x, w, dx and d_w of 8 x 64, 100 x 64 bf16 (d_w fp32): refused where an output touches an operand or the other output."""
    need = lib.moe_vocab_workspace_bytes(8, 64, 100, BF16, F32, 0, 1)
    at = {"x": 1 << 20, "w": 2 << 20, "dx": 3 << 20, "d_w": 4 << 20}

    def step(**k):
        a = {**at, **k}
        return lib.moe_vocab_loss(P(a["x"]), P(a["w"]), FAKE, NULL, BF16, 8, 64, 100, 0, FAKE, FAKE, FAKE, P(a["dx"]), P(a["d_w"]), F32, 0, FAKE, need, None)

    x_bytes, w_bytes, d_w_bytes = 8 * 64 * 2, 100 * 64 * 2, 100 * 64 * 4
    assert step(dx=at["x"]) == step(dx=at["x"] + x_bytes - 16) == step(dx=at["w"] + w_bytes - 16) == -1
    assert step(d_w=at["w"]) == step(d_w=at["w"] - d_w_bytes + 16) == step(d_w=at["x"]) == step(d_w=at["dx"] - 16) == -1


def test_vocab_size_limits(lib):
    size = lib.moe_vocab_workspace_bytes
    assert size(1 << 24, 16, 1 << 18, BF16, BF16, 0, 0) > 0
    assert size(1 << 24, 16, 1 << 20, BF16, BF16, 0, 0) == 0            # more tiles than are counted
    # the statistics of a score are those of a piece of rows
    assert size(1 << 22, 64, 131072, BF16, BF16, 0, 0) < 1 << 30
    assert lib.moe_vocab_score(FAKE, FAKE, FAKE, BF16, 1 << 24, 16, 1 << 20, 0, FAKE, FAKE, FAKE, 1 << 40, None) == -2
