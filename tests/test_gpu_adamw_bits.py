"""An update's bits do not depend on where its tensors begin (elements in front of a line go one by one, the others four at a time)."""
import pytest
import torch

DEV = "cuda:0"


@pytest.mark.gpu
@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
def test_any_alignment(grad_dtype):
    from paper_2505_11432_amd.optim import AdamW
    n = 40_003
    g = torch.Generator(device=DEV).manual_seed(1)
    base = [torch.randn((n,), device=DEV, generator=g) * s for s in (0.02, 1e-3, 3e-4, 1e-3)]
    base[3].square_()
    coef = torch.full((1,), 0.625, device=DEV)

    def run(offset):
        p, grad, m, v = (torch.cat([torch.zeros((offset,), device=DEV), t])[offset:] for t in base)
        grad = torch.cat([torch.zeros((offset,), device=DEV), base[1]]).to(grad_dtype)[offset:]
        w = torch.zeros((n,), dtype=torch.bfloat16, device=DEV)
        op = AdamW([p], [grad], [m], [v], weights=[w])
        for _ in range(3):
            op.step(coef=coef)
        return p, m, v, w

    want = run(0)
    for offset in (1, 2, 3, 17, 31):
        assert all(torch.equal(a, b) for a, b in zip(want, run(offset))), offset
