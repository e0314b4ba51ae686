"""The training loop of paper_2211_15601_amd.fit: correspondence search, its backward, clipped AdamW steps."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


def test_a_skinning_field_is_learned(gpu_lib):
    from paper_2211_15601_amd import fit
    losses, norms, peaks, opt = fit.train(steps=80, n_points=2048, n_poses=2)
    first, last = sum(losses[:2]) / 2, sum(losses[-2:]) / 2
    assert last < 0.5 * first, (first, last)
    assert all(math.isfinite(n) and n > 0 for n in norms) and int(opt.step_count) == 80
    assert all(math.isfinite(p) and p > 0 for p in peaks)
    # the norm is that of the last step's gradients in both parameters that it had: the field and one pose's shift
    moved = [s for s in opt.params[1:] if s.abs().max() > 0]
    assert len(moved) == 2


def test_a_limit_bounds_the_first_moment(gpu_lib):
    from paper_2211_15601_amd import fit
    _, norms, _, opt = fit.train(steps=3, n_points=512, n_poses=1, max_norm=1e-3)
    assert min(norms) > 1e-3
    # after three steps of gradients of norm 1e-3: at most (1 - 0.9^3) of that, up to fp32 rounding of the entries
    first = math.sqrt(sum(float(m.double().square().sum()) for m in opt.exp_avgs))
    assert 0 < first <= (1 - 0.9 ** 3) * 1e-3 * (1 + 1e-5)
