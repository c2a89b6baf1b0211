"""Host-only checks of arguments of the calls around the layer, beside those of test_block_abi.  Nothing here reaches a stream."""
import ctypes

import pytest

P, I, Z, D = ctypes.c_void_p, ctypes.c_int, ctypes.c_size_t, ctypes.c_double
NULL = P(0)
F32, BF16 = 0, 1
MB = 1 << 20


@pytest.fixture(scope="module")
def lib():
    from paper_2505_11432_amd.build import LIB_PATH, ensure_built
    ensure_built()
    lib = ctypes.CDLL(LIB_PATH)
    lib.moe_embedding_workspace_bytes.restype = lib.moe_block_norm_workspace_bytes.restype = lib.moe_orthogonal_workspace_bytes.restype = Z
    lib.moe_muon_eps.argtypes = [P, P, I, P, P, I, I, I, P, P, D, I, D, D, D, I, P, I, P, Z, P]
    return lib


def test_muon_eps(lib):
    need = lib.moe_orthogonal_workspace_bytes(2, 8, 8, 0)

    def muon(eps, batch=2, p=P(MB), steps=5, n=need):
        return lib.moe_muon_eps(p, P(2 * MB), F32, P(3 * MB), NULL, batch, 8, 8, P(5 * MB), NULL, 0.9, 1, 0.1, 1.0, eps, steps, NULL, 0, P(6 * MB), n, None)

    assert muon(-1e-9) == muon(float("nan")) == muon(1e-7, p=NULL) == muon(1e-7, steps=0) == -1
    assert muon(1e-7, n=need - 1) == muon(0.0, n=need - 1) == -3
    assert muon(1e-7, batch=0) == muon(0.0, batch=0) == 0


def test_gain_of_the_steps(lib):
    """Lists whose small singular values, and roundings with them, are multiplied by more than 8192, or 262144 with a side of at most 64, are refused: -2.  Others
    go on to the workspace, which is too small here: -3."""
    lib.moe_orthogonalize.argtypes = [P, I, I, I, I, I, P, I, P, I, P, Z, P]
    lib.moe_muon.argtypes = [P, P, I, P, P, I, I, I, P, P, D, I, D, D, I, P, I, P, Z, P]

    def both(rows, cols, steps, c=None):
        c = NULL if c is None else ctypes.cast((D * (3 * steps))(*[v for row in c for v in row]), P)
        a = lib.moe_orthogonalize(P(64 * MB), F32, 1, rows, cols, steps, c, 0, P(128 * MB), F32, P(256 * MB), 16, None)
        b = lib.moe_muon(P(64 * MB), P(128 * MB), F32, P(192 * MB), NULL, 1, rows, cols, P(MB), NULL, 0.9, 1, 0.1, 1.0, steps, c, 0, P(256 * MB), 16, None)
        assert a == b
        return a

    for rows, cols in ((65, 65), (65, 4000), (4000, 65)):
        assert both(rows, cols, 7) == -3 and both(rows, cols, 8) == both(rows, cols, 16) == -2
    for rows, cols in ((64, 64), (64, 4000), (4000, 64), (1, 1)):
        assert both(rows, cols, 10) == -3 and both(rows, cols, 11) == both(rows, cols, 16) == -2
    slow, still = (2.0, -1.5, 0.5), (0.5, 0.0, 0.0)
    assert both(100, 100, 13, [slow] * 13) == -3 and both(100, 100, 14, [slow] * 14) == -2
    assert both(60, 100, 14, [slow] * 14) == -3 and both(60, 100, 16, [slow] * 16) == -3
    # (what a later step makes smaller again was large on the way; what an earlier one made smaller is no gain)
    assert both(100, 100, 15, [slow] * 14 + [still]) == -2
    assert both(100, 100, 14, [still] + [slow] * 13) == -3 and both(100, 100, 15, [still] + [slow] * 14) == -2
    assert both(100, 100, 16, [(1.5, -0.5, 0.0)] * 16) == -3
