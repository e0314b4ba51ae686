"""Layers together: the network of net.py against the same in 64 bits, and the training loop of fit.py on it."""
import math

import pytest
import torch

import net_ref as ref

pytestmark = pytest.mark.gpu
F64 = torch.float64


def wide(network, x, words):
    """The network's outputs in 64 bits, with gradients."""
    params = [p.detach().cpu().to(F64).requires_grad_(True) for p in network.params]
    x = x.detach().cpu().to(F64).requires_grad_(True)
    h = x
    for i in range(network.hidden):
        z = h @ params[2 * i].T + params[2 * i + 1]
        b = network.how["beta"]
        a = torch.logaddexp(torch.zeros_like(z), b * z) / b
        if words is not None:
            seed, offset = (v % 2 ** 64 for v in words[i].tolist())
            a = a * ref.factor(a.shape, network.dropout, (seed, offset))
        h = a + h if i else a
    return h @ params[-2].T + params[-1], [x, *params]


def test_network(gpu_lib):
    from paper_2211_15601_amd import net
    network = net.Network(3, 64, 3, 24, dropout=0.1, seed=3)
    with torch.no_grad():
        network.params[-2].normal_(0.0, 0.125)
    x = (torch.rand(5000, 3, device="cuda") * 2 - 1).requires_grad_(True)
    g = torch.randn(5000, 24, device="cuda")
    words = torch.tensor([[1, 2], [1, 3], [-4, 4]], device="cuda")
    for w in (None, words):
        y = network(x, w)
        grads = torch.autograd.grad(y, [x, *network.params], g)
        Y, leaves = wide(network, x, w)
        wanted = torch.autograd.grad(Y, leaves, g.cpu().to(F64))
        # Every layer adds errors of 8 sqrt(6 64) 2^-24 = 1e-5 of its products' magnitudes at most (net_ref.product), which are about 8 times their sums
        # of 64 terms of either sign; there and back through 4 layers: 8 8e-5 = 6.4e-4 of the norm at most, softplus' slope at 10 z adding 2.5 times its argument's.
        for got, want in zip([y, *grads], [Y, *wanted]):
            want = want.detach()
            off = (got.detach().cpu().to(F64) - want).norm() / want.norm()
            assert float(off) < 2e-3, float(off)
    with pytest.raises(ValueError, match="words"):
        network(x, words[:2])


def test_a_network_is_learned(gpu_lib):
    from paper_2211_15601_amd import fit
    for dropout in (0.0, 0.1):
        losses, norms, peaks, opt = fit.train(steps=12, n_points=1024, n_poses=2, field="network", dropout=dropout)
        assert all(math.isfinite(v) for v in losses + norms + peaks) and all(n > 0 for n in norms) and int(opt.step_count) == 12
        assert len(opt.params) == 2 * 4 + 2 and all(bool(p.isfinite().all()) for p in opt.params)
        # the first step moves the last layer alone (its weight starts at zero), the later ones every layer
        assert all(float(m.abs().max()) > 0 for m in opt.exp_avgs[:8])


def test_the_fields_gradient(gpu_lib):
    """dL/dparameters of a step through softmax, search and network: the network's backward on what the search's gives, against 64 bits."""
    from paper_2211_15601_amd import binding, fit, net, workloads as wl
    from paper_2211_15601_amd.autograd import CorrespondenceSearch
    dims = (16, 16, 4)
    W_true, data = fit.poses(0, dims, 2048, 1)
    B, xq, x = data[0]
    network, at = net.Network(3, 64, 2, wl.N_BONES, seed=1), fit.nodes(dims)
    with torch.no_grad():
        network.params[-2].normal_(0.0, 0.05)
    fs = binding.Context(dims, wl.N_BONES, wl.BOX_LO, wl.BOX_HI)
    logits = network(at)
    W = torch.softmax(0.25 * (W_true + 1e-4).log() + logits, dim=-1)
    roots, conv = CorrespondenceSearch.apply(fs, W, B, xq, None)
    loss = (((roots - x) ** 2).sum(1) * (conv != 0)).sum() / conv.numel()
    (g,) = torch.autograd.grad(loss, logits, retain_graph=True)
    grads = torch.autograd.grad(loss, network.params)
    Y, leaves = wide(network, at, None)
    wanted = torch.autograd.grad(Y, leaves[1:], g.cpu().to(F64))
    assert float(g.abs().max()) > 0
    for got, want in zip(grads, wanted):
        assert float((got.cpu().to(F64) - want).norm() / want.norm()) < 2e-3          # as in test_network
