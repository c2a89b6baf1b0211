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
