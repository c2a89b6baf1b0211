"""Another default type of torch changes nothing: what is fp32 by contract is made so."""
import pytest
import torch

DEV = "cuda:0"


@pytest.fixture(params=[torch.float64, torch.bfloat16])
def default_dtype(request):
    torch.set_default_dtype(request.param)
    yield request.param
    torch.set_default_dtype(torch.float32)


@pytest.mark.gpu
def test_learning_rate_as_a_number(default_dtype):
    from paper_2505_11432_amd.optim import AdamW
    p, g, m, v = (torch.full((100,), x, dtype=torch.float32, device=DEV) for x in (1.0, 0.5, 0.0, 0.0))
    AdamW([p], [g], [m], [v], lr=0.25, weight_decay=0.0, eps=0.0).step()
    assert float((p - 0.75).abs().max()) <= 2.0 ** -22


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_training_step(default_dtype, dtype):
    from paper_2505_11432_amd.train import TrainStep
    model = TrainStep(64, 128, 4, 2, 144, 200, dtype=dtype)
    model.load(torch.arange(64, device=DEV), torch.arange(64, device=DEV))
    loss, norm = model.step()
    assert bool(torch.isfinite(loss)) and bool(torch.isfinite(norm)) and int(model.adamw.step_count) == 1
