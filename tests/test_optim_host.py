"""Host code of optim.py without a GPU (fake_lists.py): what it hands to the library, and when."""
import pytest

import fake_lists


@pytest.fixture
def gpu(monkeypatch):
    return fake_lists.Machine(monkeypatch)


def test_settings_that_are_changed_in_place(gpu):
    (p,) = params = gpu.params(10)
    opt = gpu.adamw(params, grads=gpu.grads(params), betas=[0.9, 0.999])
    opt.step()
    opt.betas[0] = 0.5
    opt.step()
    opt.betas[1] = 0.25
    opt.step()
    assert [(r["args"][0]["beta1"], r["args"][0]["beta2"]) for r in gpu.ran] == [(0.9, 0.999), (0.5, 0.999), (0.5, 0.25)]
