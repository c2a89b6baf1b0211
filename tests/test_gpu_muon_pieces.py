"""Orthogonalised matrices taken together, one by one, and in pieces with a smaller last one: each within the tolerance of test_gpu_muon's model (another number of
matrices at a time may cut the sums elsewhere and give other bits), and the same bits for the same call whatever lay in the workspace."""
import pytest
import torch

from test_gpu_muon import DEV, exact, in_pairs, matrices


@pytest.mark.gpu
@pytest.mark.parametrize("batch,rows,cols,piece", [(3, 520, 9000, 1), (3, 520, 9000, 2), (8, 128, 16384, 1), (8, 128, 16384, 5), (5, 900, 2500, 3), (7, 60, 5000, 2),
                                                   (9, 300, 129, 4), (3, 1500, 4100, 2)])
def test_pieces(batch, rows, cols, piece):
    from paper_2505_11432_amd import binding as B
    x = matrices(batch, rows, cols, "falling", seed=batch)
    for take in (0, piece):
        size = B.moe_orthogonal_workspace_bytes(batch, rows, cols, take)
        outs = []
        for fill in (255, 0):
            workspace = torch.full((size,), fill, dtype=torch.uint8, device=DEV)
            out = torch.empty_like(x)
            B.moe_orthogonalize(x, out, workspace, piece=take)
            outs.append(out)
        assert torch.equal(*outs)
        for i in (0, batch - 1):
            together = take or batch
            want, tol = exact(x[i], pairs=in_pairs(together, rows, cols))
            assert float((outs[0][i].double() - want).norm()) <= tol, (take, i)
