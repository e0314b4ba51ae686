"""The rates of fit.py's training loop."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("field, share, given", [("grid", 0.02, 0.05), ("network", 0.5, 2e-3)])
def test_the_shifts_go_by_a_fraction_of_the_rate(gpu_lib, field, share, given):
    from paper_2211_15601_amd import fit
    for lr in (None, 0.1, 1e-4, 0.0):
        _, _, _, opt = fit.train(steps=1, n_points=256, n_poses=2, lr=lr, field=field)
        assert opt.lr == (given if lr is None else lr)
        scales = list(opt._handle.columns["lr_scale"])
        assert scales[-2:] == [np.float32(share)] * 2 and set(scales[:-2]) == {1.0}
