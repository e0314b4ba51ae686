"""The coefficient comes from the norm in 64 bits, not from the norm as it is given out.

Gradients are integers, so their squares add up exactly in any order; square root, quotient, and the roundings to float32 of coefficient
and product are correctly rounded: the results are known to the bit."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SIZES = [[700], [5, 3000], [9, 70_001, 4096]]              # one kernel; one kernel; two


@pytest.fixture(scope="module")
def optim(gpu_lib):
    from paper_2211_15601_amd import optim
    return optim


def _lists(sizes, count=24):
    gen = torch.Generator().manual_seed(len(sizes))
    for k in range(count):
        yield [torch.randint(-1000, 1001, (n,), generator=gen).float() for n in sizes], 0.1 * (k + 1), (1.0, 1.0 / 3.0)[k % 2]


def _norm(host, kind, scale):
    flat = torch.cat(host).double()
    return (float(flat.abs().max()) if kind == "max" else float(np.sqrt((flat * flat).sum().item()))) * scale


def _coef(norm, max_norm, scale):
    return np.float32(min(1.0, max_norm / (norm + 1e-6)) * scale)


@pytest.mark.parametrize("sizes", SIZES)
@pytest.mark.parametrize("kind", ["l2", "max"])
@pytest.mark.parametrize("inplace", [False, True])
def test_clip(optim, sizes, kind, inplace):
    for host, max_norm, scale in _lists(sizes):
        g = [x.to(DEV) for x in host]
        outs = g if inplace else [torch.zeros_like(x) for x in g]
        norm = _norm(host, kind, scale)
        got = optim.TensorList(g, outs=None if inplace else outs).clip_grads(max_norm, kind=kind, grad_scale=scale)
        assert float(got) == float(np.float32(norm))
        c = _coef(norm, max_norm, scale)
        for x, y in zip(host, outs):
            assert np.array_equal(y.cpu().numpy(), x.numpy() * c)


@pytest.mark.parametrize("sizes", SIZES)
def test_adamw(optim, sizes):
    """With beta1 = 0 the first moment is the scaled gradient."""
    for host, max_norm, scale in _lists(sizes):
        opt = optim.AdamW([torch.zeros(x.numel(), device=DEV) for x in host], grads=[x.to(DEV) for x in host], betas=(0.0, 0.9), max_norm=max_norm, grad_scale=scale)
        norm = _norm(host, "l2", scale)
        assert float(opt.step()) == float(np.float32(norm))
        c = _coef(norm, max_norm, scale)
        for x, m in zip(host, opt.exp_avgs):
            assert np.array_equal(m.cpu().numpy(), x.numpy() * c)


@pytest.mark.parametrize("n", [4096, 300_000])
def test_norms_beyond_float32(optim, n):
    """Finite gradients whose norm float32 cannot hold: given out as infinity, but clipped and learned from."""
    g = torch.full((n,), 2.0 ** 127, device=DEV)
    norm = 2.0 ** 127 * float(np.sqrt(float(n)))
    c = _coef(norm, 2.0 ** 20, 1.0)
    want = np.float32(2.0 ** 127) * c
    assert 0.0 < want < 2.0 ** 20
    out = torch.zeros_like(g)
    assert float(optim.TensorList([g], outs=[out]).clip_grads(2.0 ** 20)) == float("inf")
    assert (out == float(want)).all()
    p = torch.zeros(n, device=DEV)
    opt = optim.AdamW([p], grads=[g], lr=0.5, betas=(0.0, 0.9), weight_decay=0.0, max_norm=2.0 ** 20, skip_nonfinite=True)
    assert float(opt.step()) == float("inf")
    assert int(opt.step_count) == 1 and (opt.exp_avgs[0] == float(want)).all() and (p < 0).all()
    # what is not finite is skipped as before
    before = p.clone()
    for bad in (float("inf"), float("nan")):
        g[n - 1] = bad
        opt.step()
        assert int(opt.step_count) == 1 and torch.equal(p, before)
    # a norm that is given is taken as it is
    g[n - 1] = 0.0
    opt.step(norm=torch.full((1,), float("inf"), device=DEV))
    assert int(opt.step_count) == 1 and torch.equal(p, before)
    opt.step(norm=torch.full((1,), 2.0 ** 21, device=DEV))
    assert int(opt.step_count) == 2
