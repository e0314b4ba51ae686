"""AdamW where float32 ends."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def optim(gpu_lib):
    from paper_2211_15601_amd import optim
    return optim


@pytest.mark.parametrize("n", [1001, 300_001])
@pytest.mark.parametrize("max_norm", [None, 1e9])
def test_eps_below_float32(optim, n, max_norm):
    """0 / (sqrt(0) + eps) is 0 for every eps above 0: elements without gradients stay where they are."""
    p = torch.linspace(1, 2, n, device=DEV)
    g = torch.zeros(n, device=DEV)
    g[::3] = 1.0
    before = p.clone()
    opt = optim.AdamW([p], grads=[g], lr=0.25, eps=1e-60, weight_decay=0.0, max_norm=max_norm)
    for _ in range(2):
        opt.step()
    rest = torch.ones(n, dtype=torch.bool, device=DEV)
    rest[::3] = False
    assert torch.equal(p[rest], before[rest])
    # m = v = 1 after the corrections, within the roundings of a step of 0.25 at values below 2: 2 steps of some 10 roundings each
    assert ((before - p)[~rest] - 0.5).abs().max() <= 20 * 2.0 ** -24 * 2
