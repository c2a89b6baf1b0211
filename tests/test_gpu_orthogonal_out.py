"""Orthogonalised matrices in bf16 from large tiles, whole and cut along the sums, against the formula (a result in bf16 adds half a step, 2^-8 of each element, to the
tolerance of test_gpu_muon's model), and in place of their inputs."""
import pytest
import torch

from test_gpu_muon import DEV, exact, in_pairs, matrices

LARGE = [(1, 1990, 2100), (16, 1024, 1000), (9, 900, 1030), (1, 520, 9000), (1, 3000, 3200), (1, 7100, 1500), (9, 900, 2500)]


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["flat", "falling"])
@pytest.mark.parametrize("batch,rows,cols", LARGE + [(3, 50, 900), (2, 300, 1000)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_bf16(batch, rows, cols, kind, dtype):
    from paper_2505_11432_amd.optim import Orthogonal
    x = matrices(batch, rows, cols, kind, dtype=dtype)
    op = Orthogonal(batch, rows, cols, out_dtype=torch.bfloat16, device=DEV)
    op.out.fill_(float("nan"))
    out = op.apply(x)
    for i in (0, batch - 1):
        want, tol = exact(x[i], pairs=in_pairs(batch, rows, cols))
        assert float((out[i].double() - want).norm()) <= tol * (1 + 2.0 ** -8) + 2.0 ** -8 * float(want.norm())


@pytest.mark.gpu
@pytest.mark.parametrize("batch,rows,cols,piece", [(1, 1990, 2100, 0), (1, 520, 9000, 0), (5, 900, 2500, 2), (3, 50, 900, 0), (3, 900, 50, 2), (2, 300, 1000, 1), (4, 70, 90, 3)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_in_place(batch, rows, cols, piece, dtype):
    from paper_2505_11432_amd import binding as B
    x = matrices(batch, rows, cols, "falling", dtype=dtype)
    workspace = torch.empty((B.moe_orthogonal_workspace_bytes(batch, rows, cols, piece),), dtype=torch.uint8, device=DEV)
    want = torch.empty_like(x)
    B.moe_orthogonalize(x, want, workspace, piece=piece)
    B.moe_orthogonalize(x, x, workspace, piece=piece)
    assert torch.equal(x, want)


@pytest.mark.gpu
@pytest.mark.parametrize("batch,rows,cols,piece", [(1, 65, 65, 0), (1, 300, 1000, 0), (1, 520, 9000, 0), (2, 520, 9000, 0), (3, 520, 9000, 2), (8, 128, 16384, 0), (1, 1990, 2100, 0),
                                                   (9, 900, 1030, 0), (9, 900, 2500, 4), (1, 1500, 7100, 0), (3, 50, 900, 0)])
def test_nothing_behind_the_workspace(batch, rows, cols, piece):
    """A workspace of exactly the size that is asked for: what lies behind it stays as it was."""
    from paper_2505_11432_amd import binding as B
    size = B.moe_orthogonal_workspace_bytes(batch, rows, cols, piece)
    buffer = torch.full((size + (32 << 20),), 77, dtype=torch.uint8, device=DEV)
    x = matrices(batch, rows, cols, "falling")
    out = torch.empty_like(x)
    B.moe_orthogonalize(x, out, buffer[:size], piece=piece)
    assert bool((buffer[size:] == 77).all())
    want, tol = exact(x[-1], pairs=in_pairs(piece or batch, rows, cols))
    assert float((out[-1].double() - want).norm()) <= tol
