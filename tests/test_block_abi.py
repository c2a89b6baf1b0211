"""Host-only checks of the entry points around the layer: sizes and refused arguments.  Nothing here reaches a stream."""
import ctypes

import pytest

P, I, Z, D = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_double
NULL = P(0)
F32, BF16, E4M3 = 0, 1, 2
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    from paper_2505_11432_amd.build import LIB_PATH, ensure_built
    ensure_built()
    lib = ctypes.CDLL(LIB_PATH)
    lib.moe_embedding_workspace_bytes.restype = lib.moe_block_norm_workspace_bytes.restype = lib.moe_orthogonal_workspace_bytes.restype = Z
    lib.moe_embedding_fwd.argtypes = [P, P, I, I, I, I, D, P, P]
    lib.moe_embedding_bwd.argtypes = [P, P, I, I, I, I, D, P, I, I, P, Z, P]
    lib.moe_block_norm_fwd.argtypes = [P, P, P, P, P, I, I, I, I, D, D, P, P, P]
    lib.moe_block_norm_bwd.argtypes = [P] * 7 + [I, I, I, I, D, D] + [P] * 5 + [I, P, Z, P]
    lib.moe_orthogonalize.argtypes = [P, I, I, I, I, I, P, I, P, I, P, Z, P]
    lib.moe_muon.argtypes = [P, P, I, P, P, I, I, I, P, P, D, I, D, D, I, P, I, P, Z, P]
    return lib


def test_embedding(lib):
    size = lib.moe_embedding_workspace_bytes
    assert size(0, 64, 100) > 0 and size(8192, 4096, 32000) >= 8192 * 8
    for bad in ((-1, 64, 100), (8, 0, 100), (8, 72, 100), (8, 64, 0), (8, 64, (1 << 24) + 1), ((1 << 24) + 1, 64, 100), (1 << 24, 1 << 13, 100)):
        assert size(*bad) == 0, bad

    def fwd(table=P(MB), tokens=P(2 * MB), dt=BF16, T=8, d=64, V=100, out=P(3 * MB)):
        return lib.moe_embedding_fwd(table, tokens, dt, T, d, V, 1.0, out, None)

    assert fwd(table=NULL) == fwd(tokens=NULL) == fwd(out=NULL) == fwd(T=-1) == fwd(V=0) == fwd(d=0) == -1
    assert fwd(dt=E4M3) == fwd(d=72) == fwd(table=P(MB + 8)) == fwd(out=P(MB + 8)) == fwd(tokens=P(MB + 2)) == fwd(V=(1 << 24) + 1) == -2
    assert fwd(out=P(MB)) == fwd(out=P(MB + 100 * 64 * 2 - 16)) == fwd(out=P(MB - 8 * 64 * 2 + 16)) == fwd(out=P(2 * MB)) == -1
    assert fwd(T=0, table=NULL, tokens=NULL, out=NULL) == 0
    need = size(8, 64, 100)

    def bwd(tokens=P(2 * MB), dy=P(MB), dt=BF16, T=8, d=64, V=100, d_table=P(3 * MB), gdt=F32, acc=0, ws=P(4 * MB), n=need):
        return lib.moe_embedding_bwd(tokens, dy, dt, T, d, V, 1.0, d_table, gdt, acc, ws, n, None)

    assert bwd(tokens=NULL) == bwd(dy=NULL) == bwd(d_table=NULL) == bwd(T=-1) == -1
    assert bwd(dt=E4M3) == bwd(gdt=E4M3) == bwd(dt=F32, gdt=BF16) == bwd(d=8) == bwd(dy=P(MB + 8)) == bwd(d_table=P(MB + 8)) == -2
    assert bwd(ws=NULL) == bwd(n=need - 1) == bwd(ws=P(4 * MB + 8)) == -3
    assert bwd(d_table=P(MB)) == bwd(d_table=P(MB - 100 * 64 * 4 + 16)) == bwd(d_table=P(2 * MB)) == -1
    assert bwd(T=0, tokens=NULL, dy=NULL, d_table=NULL, acc=1, ws=NULL) == 0


def test_block_norm(lib):
    size = lib.moe_block_norm_workspace_bytes
    assert size(0, 64, BF16, 1, 1, 1) > 0
    assert size(8192, 4096, BF16, 1, 1, 1) > size(8192, 4096, BF16, 1, 0, 1) > size(8192, 4096, BF16, 0, 0, 1)
    for bad in ((-1, 64, BF16), (8, 0, BF16), (8, 72, BF16), (8, 16400, BF16), (8, 64, E4M3)):
        assert size(*bad, 1, 1, 1) == 0, bad

    def fwd(x=P(MB), y=P(2 * MB), wa=P(3 * MB), gate=P(4 * MB), wb=P(5 * MB), dt=BF16, T=8, d=64, rows=4, alpha=1.0, eps=1e-6, out=P(6 * MB), h=P(7 * MB)):
        return lib.moe_block_norm_fwd(x, y, wa, gate, wb, dt, T, d, rows, alpha, eps, out, h, None)

    nan = float("nan")
    assert fwd(x=NULL) == fwd(y=NULL) == fwd(out=NULL) == fwd(h=NULL) == fwd(wb=NULL) == fwd(T=-1) == fwd(d=0) == fwd(rows=0) == fwd(eps=-1.0) == fwd(eps=nan) == -1
    assert fwd(alpha=nan) == fwd(y=NULL, out=NULL) == fwd(y=NULL, out=NULL, wa=NULL, gate=NULL, alpha=0.5) == -1
    assert fwd(y=NULL, out=NULL, wa=NULL, gate=NULL, wb=NULL, h=NULL) == -1
    assert fwd(dt=E4M3) == fwd(d=72) == fwd(d=16400) == fwd(x=P(MB + 8)) == fwd(gate=P(MB + 4)) == fwd(h=P(MB + 8)) == -2
    rows = 8 * 64 * 2
    assert fwd(out=P(7 * MB)) == fwd(out=P(MB + 16)) == fwd(h=P(MB)) == fwd(h=P(2 * MB)) == fwd(out=P(3 * MB)) == fwd(h=P(4 * MB + 2 * 64 * 4 - 16)) == -1
    assert fwd(h=P(6 * MB + rows - 16)) == -1
    assert fwd(T=0, x=NULL, y=NULL, out=NULL, h=NULL) == 0
    need = size(8, 64, BF16, 1, 1, 1)

    def bwd(out=P(MB), y=P(2 * MB), wa=P(3 * MB), gate=P(4 * MB), wb=P(5 * MB), d_out=P(6 * MB), d_h=P(7 * MB), dt=BF16, T=8, d=64, rows=4, alpha=1.0, dx=P(8 * MB),
            dy=P(9 * MB), dwa=P(10 * MB), dg=P(11 * MB), dwb=P(12 * MB), ws=P(13 * MB), n=need):
        return lib.moe_block_norm_bwd(out, y, wa, gate, wb, d_out, d_h, dt, T, d, rows, alpha, 1e-6, dx, dy, dwa, dg, dwb, 0, ws, n, None)

    for k in ("out", "y", "wa", "gate", "wb", "d_h", "dx", "dy", "dwa", "dg", "dwb"):
        assert bwd(**{k: NULL}) == -1, k
    assert bwd(wb=NULL, d_h=NULL, dwb=NULL, d_out=NULL) == bwd(T=-1) == bwd(rows=0) == -1
    assert bwd(dt=E4M3) == bwd(d=40) == bwd(dx=P(MB + 8)) == bwd(dwa=P(MB + 8)) == -2
    assert bwd(ws=NULL) == bwd(n=need - 1) == bwd(ws=P(13 * MB + 4)) == -3
    assert bwd(dx=P(MB)) == bwd(dy=P(MB)) == bwd(dx=P(9 * MB)) == bwd(dx=P(6 * MB + 16)) == bwd(dwa=P(3 * MB)) == bwd(dg=P(4 * MB)) == bwd(dwb=P(10 * MB)) == -1
    assert bwd(T=0, out=NULL, y=NULL, d_out=NULL, d_h=NULL, dx=NULL, dy=NULL, ws=NULL) == 0


def test_orthogonal(lib):
    size = lib.moe_orthogonal_workspace_bytes
    one = size(1, 100, 200, 0)
    assert one > 0 and size(0, 100, 200, 0) > 0 and size(7, 100, 200, 1) == one < size(7, 100, 200, 0) == size(7, 100, 200, 9)
    for bad in ((-1, 8, 8, 0), (1, 0, 8, 0), (1, 8, 0, 0), (1, 8, 8, -1), (1, (1 << 20) + 1, 8, 0), (1, 1 << 20, 1 << 20, 0), (30000, 4096, 4096, 0)):
        assert size(*bad) == 0, bad
    need = size(2, 8, 8, 0)
    coefs = lambda *v: ctypes.cast((D * len(v))(*v), P)

    def orth(x=P(MB), dt=F32, batch=2, rows=8, cols=8, steps=1, c=NULL, piece=0, out=P(2 * MB), odt=BF16, ws=P(3 * MB), n=need):
        return lib.moe_orthogonalize(x, dt, batch, rows, cols, steps, c, piece, out, odt, ws, n, None)

    assert orth(x=NULL) == orth(out=NULL) == orth(batch=-1) == orth(rows=0) == orth(steps=0) == orth(steps=17) == orth(piece=-1) == -1
    assert orth(dt=E4M3) == orth(odt=E4M3) == orth(x=P(MB + 2)) == orth(out=P(MB + 1)) == orth(batch=30000, rows=4096, cols=4096) == -2
    assert orth(c=coefs(20.0, 0.0, 0.0)) == orth(steps=2, c=coefs(1.0, 0.0, 0.0, float("inf"), 0.0, 0.0)) == orth(c=coefs(1.0, float("nan"), 0.0)) == -2
    assert orth(ws=NULL) == orth(n=need - 1) == orth(ws=P(3 * MB + 8)) == -3
    assert orth(out=P(MB)) == orth(out=P(MB + 2 * 64 * 4 - 2)) == orth(out=P(MB + 4), odt=F32) == -1
    assert orth(batch=0, x=NULL, out=NULL, ws=NULL) == 0

    def muon(p=P(MB), g=P(2 * MB), gdt=F32, m=P(3 * MB), w=P(4 * MB), batch=2, rows=8, cols=8, lr=P(5 * MB), coef=NULL, mu=0.9, wd=0.1, scale=1.0, steps=5, ws=P(6 * MB),
             n=need):
        return lib.moe_muon(p, g, gdt, m, w, batch, rows, cols, lr, coef, mu, 1, wd, scale, steps, NULL, 0, ws, n, None)

    for k in ("p", "g", "m", "lr"):
        assert muon(**{k: NULL}) == -1, k
    nan = float("nan")
    assert muon(mu=1.0) == muon(mu=-0.1) == muon(mu=nan) == muon(wd=-1.0) == muon(scale=nan) == muon(batch=-1) == muon(steps=17) == -1
    assert muon(gdt=E4M3) == muon(p=P(MB + 2)) == muon(g=P(MB + 2)) == muon(w=P(MB + 1)) == muon(lr=P(MB + 2)) == -2
    assert muon(ws=NULL) == muon(n=need - 1) == -3
    assert muon(m=P(MB)) == muon(g=P(MB)) == muon(w=P(MB + 16)) == muon(lr=P(MB)) == muon(coef=P(3 * MB + 8)) == -1
    assert muon(batch=0, p=NULL, g=NULL, m=NULL, ws=NULL) == 0
