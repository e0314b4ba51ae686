"""fp32 results that are no finite numbers: what they are, and what they cost."""
import math

import pytest
import torch

import net_ref as ref
from test_gpu_net import SEED, make, net, run, whole  # noqa: F401

pytestmark = pytest.mark.gpu
F64 = torch.float64
SIZES = [(3, 70, 40), (20, 700, 33), (32, 4100, 20), (70, 24, 40), (9000, 97, 128), (20001, 128, 24), (300, 200, 130), (65, 1000, 77), (1500, 640, 1100), (5000, 130, 140)]


def same_kind(name, got, want):
    """NaN where that is, infinities too, and finite numbers elsewhere."""
    got = got.detach().to(F64)
    assert torch.equal(got.isnan(), want.isnan()), (name, int((got.isnan() != want.isnan()).sum()))
    inf = want.isinf()
    assert torch.equal(got[inf], want[inf]) and bool(got[~inf & ~want.isnan()].isfinite().all()), name


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_what_they_are(net, size):  # noqa: F811
    """NaN, infinities, zeros beside them, the largest numbers and least ones, scattered over all inputs: whole numbers elsewhere, so that finite results are exact."""
    rows, inputs, outputs = size
    gen = torch.Generator(device="cuda").manual_seed(sum(size))
    x, w, g = (whole(m, n, torch.float32, gen, 1) for m, n in ((rows, inputs), (outputs, inputs), (rows, outputs)))
    special = [math.inf, -math.inf, math.nan, math.inf]

    def scatter(t, step):
        t = t.clone()
        for i, v in enumerate(special):
            t[(step * (3 * i + 1)) % t.shape[0], (5 + 7 * i * step) % t.shape[1]] = v
        return t

    x, w, g = scatter(x, 5), scatter(w, 2), scatter(g, 11)
    leaves = [t.requires_grad_(True) for t in (x, w)]
    y = net.linear(*leaves)
    dx, dw = torch.autograd.grad(y, leaves, g)
    X, W, G = (t.detach().to(F64) for t in (x, w, g))
    for name, got, want in (("y", y, X @ W.t()), ("dx", dx, G @ W), ("dweight", dw, G.t() @ X)):
        same_kind(name, got, want)
        finite = want.isfinite()
        assert torch.equal(got.detach()[finite], want[finite].float()), name
        assert bool(finite.any()) and not bool(finite.all()), name


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_the_largest_numbers(net, size):  # noqa: F811
    """Products beyond 2^128 are infinities of their sign; the largest numbers themselves, whose first part rounds up to one, come through times 1 and times 2^-10."""
    rows, inputs, outputs = size
    top = torch.finfo(torch.float32).max
    x, w, g = (torch.zeros(m, n, device="cuda") for m, n in ((rows, inputs), (outputs, inputs), (rows, outputs)))
    x[0, 0], x[rows - 1, inputs - 1], x[rows // 2, 3] = top, -top, -top
    w[0, 0], w[1, 0], w[outputs - 1, inputs - 1], w[0, 3] = 1.0, 2.0 ** -10, 2.0, top
    g[0, 0], g[1, 0], g[rows - 1, 1], g[rows // 2, outputs - 1] = top, 1.0, 1.0, -top
    leaves = [t.requires_grad_(True) for t in (x, w)]
    y = net.linear(*leaves)
    dx, dw = torch.autograd.grad(y, leaves, g)
    X, W, G = (t.detach().to(F64) for t in (x, w, g))
    for name, got, want in (("y", y, X @ W.t()), ("dx", dx, G @ W), ("dweight", dw, G.t() @ X)):
        assert torch.equal(got.detach(), want.float()), name


def test_slopes_and_dropout_beside_them(net):  # noqa: F811
    for size in ((70, 24, 40), (9000, 97, 128), (300, 200, 130)):
        x, w, b, r, g = make(*size, torch.float32, seed=3, pad=1)
        x, w = x.abs() + 0.1, w.abs() + 0.1
        g[2, 3], g[size[0] - 1, 5], g[size[0] // 2, 0] = math.inf, -math.inf, math.nan
        out = run(net, x, w, b, r, g, "softplus", 2.0, 0.25, SEED)
        X, W, B, G = (t.cpu().to(F64) for t in (x, w, b, g))
        f = ref.factor(G.shape, 0.25, SEED)
        dz = torch.where(f != 0, G * ref.slope(X @ W.T + B, "softplus", 2.0) * f, 0.0)
        for name, want in (("dx", dz @ W), ("dweight", dz.T @ X), ("dbias", dz.sum(0))):
            same_kind(name, out[name].cpu(), want)


def best_of(f, n=5):
    times = []
    for _ in range(n):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        f()
        b.record()
        b.synchronize()
        times.append(a.elapsed_time(b))
    return min(times)


@pytest.mark.parametrize("size", [(8, 4096, 512), (1024, 512, 512), (32768, 128, 128), (300, 2048, 300)], ids=str)
def test_what_they_cost(net, size):  # noqa: F811
    """A batch of NaN, as of a step that diverged, takes some times as long as another (a scalar sum for each result took hundreds of times)."""
    x, w, b, r, g = make(*size, torch.float32)
    took = {}
    for kind in ("none", "silu"):
        for bad in (False, True):
            v = [t.detach().clone().requires_grad_(True) for t in (x, w, b)]
            G = g.clone()
            if bad:
                with torch.no_grad():
                    v[0].fill_(math.nan)
                    G.fill_(math.nan)
            y = net.linear(*v, activation=kind)
            took[kind, bad] = best_of(lambda: net.linear(*v, activation=kind)), best_of(lambda: torch.autograd.grad(y, v, G, retain_graph=True))
            if bad:
                assert all(bool(t.isnan().all()) for t in (y, *torch.autograd.grad(y, v, G)))
        print(size, kind, *(f"{c:.3f} {d:.3f} ms" for c, d in zip(took[kind, False], took[kind, True])), flush=True)
        for clean, spoiled in zip(took[kind, False], took[kind, True]):
            assert spoiled < 25 * clean + 0.05, (kind, clean, spoiled)
