"""fp16's range in the layers' backward pass: gradients far below and near the largest number."""
import math

import pytest
import torch

import net_ref as ref
from test_gpu_net import SEED, make, net, run  # noqa: F401

pytestmark = pytest.mark.gpu
F64, T = torch.float64, torch.float16
# dZ in two parts and in one by the narrow layers' kernel; in one by the others, and in parts of a long contraction
SIZES = [(70, 24, 40), (1, 10, 40), (1000, 128, 128), (2000, 128, 128), (40001, 17, 97), (300, 200, 130), (9000, 130, 140), (33, 500, 700)]


def two_parts(size):
    return max(size[1:]) <= 128 and size[0] * size[2] <= 1 << 17


def check(out, t, g, kind, beta, p, parts):
    """Against the same numbers in fp32, and what dZ's rounding adds.  It goes in times the power of two that takes the largest |g| / (1 - p) to 2^14 .. 2^15, so that what is
    rounded off is half a step of it (or, in two parts, of its half step) or half of fp16's least number, 2^-25, which is 2^-39 of that largest."""
    x, w, b, r = (v.float() for v in t)
    want = ref.linear(x, w, b, r, g.float(), kind, beta, p, SEED)
    X, W, B, G = (v.cpu().to(F64) for v in (x, w, b, g))
    dz = (G * ref.slope(X @ W.T + B, kind, beta) * ref.factor(G.shape, p, SEED)).abs()
    half = torch.finfo(T).eps / 2
    left = dz * 1.1 * (half ** 2 if parts else half) + float(G.abs().max()) / (1.0 - p) * 2.0 ** -39
    for name, more in (("dx", left @ W.abs()), ("dweight", left.T @ X.abs())):
        value, bound = want[name]
        ref.assert_close(name, out[name], (value, bound + more + ref.rounded(value, T) * 1.01))
    value, bound = want["dbias"]
    ref.assert_close("dbias", out["dbias"], (value, bound + ref.rounded(value, T) * 1.01))


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("kind", ["none", "relu", "silu", "softplus"])
def test_small_gradients(net, size, kind):  # noqa: F811
    """As of a loss that is a mean: g about 1e-5, of which fp16's own steps leave 7 bits, and one row of ordinary size beside them."""
    x, w, b, r, g = make(*size, T, seed=sum(size), pad=1)
    x, w = x * 16, w * 64                              # gradients that do not vanish themselves
    for p, lone in ((0.25, False), (0.0, False), (0.25, True)):
        small = (g.float() * 1e-5).to(T)
        if lone:
            small[0] = g[0]
        check(run(net, x, w, b, r, small, kind, 1.0, p, SEED), (x, w, b, r), small, kind, 1.0, p, two_parts(size))


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("kind", ["none", "gelu", "silu"])
def test_large_gradients(net, size, kind):  # noqa: F811
    """|g| / (1 - p) beyond 65504, of either sign; some weights are 0."""
    x, w, b, r, g = make(*size, T, seed=sum(size), pad=1)
    g = (torch.sign(g.float()) * (40000 + 25000 * torch.rand(g.shape, generator=torch.Generator().manual_seed(1)).cuda())).to(T)
    x, w = (x.float() / (64 * math.sqrt(size[0]))).to(T), (w.float() / 64).to(T)
    w[:, ::3] = 0.0
    for p in (0.5, 0.9):
        out = run(net, x, w, b, r, g, kind, 1.0, p, SEED)
        assert out["dx"].isfinite().all() and out["dweight"].isfinite().all() and not out["dx"][:, ::3].any()
        # dbias may pass 65504 itself
        out["dbias"] = out["dbias"].float()
        x2, w2, b2, r2 = (v.float() for v in (x, w, b, r))
        want = ref.linear(x2, w2, b2, r2, g.float(), kind, 1.0, p, SEED)
        value, bound = want["dbias"]
        fits = (value.abs() + bound) < 65504
        assert bool((out["dbias"].cpu().to(F64)[~fits & (value.abs() - bound > 65520)]).isinf().all())
        out["dbias"] = torch.where(fits.cuda(), out["dbias"], value.cuda().float())
        check(out, (x, w, b, r), g, kind, 1.0, p, two_parts(size))


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_infinities_beside_what_is_scaled(net, size):  # noqa: F811
    """One NaN or infinity in g goes where the formulas send it, and the others' gradients stay finite."""
    rows, inputs, outputs = size
    for at, v in (((0, 1), math.inf), ((rows - 1, outputs - 1), -math.inf), ((rows // 2, 0), math.nan)):
        x, w, b, r, g = make(*size, T, seed=4, pad=3)
        x, w = x.abs() + 1, w.abs() + 0.125
        g[at] = v
        out = run(net, x, w, None, r, g, "softplus", 1.0, 0.0, None)
        X, W, G = (t.cpu().to(F64) for t in (x, w, g))
        dz = G * ref.slope(X @ W.T, "softplus", 1.0)
        for name, want in (("dx", dz @ W), ("dweight", dz.T @ X)):
            got = out[name].cpu().to(F64)
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got[want.isinf()], want[want.isinf()]), (name, v)
            assert got[want.abs() < 60000].isfinite().all(), name


def test_graphs_of_scaled_layers(net):  # noqa: F811
    """What dZ is scaled by is found anew at each replay; wide layers, narrow ones, and products in two parts, on gradients of other sizes each time."""
    layers = [make(*size, T, seed=sum(size)) for size in ((300, 200, 130), (2000, 128, 128), (70, 24, 40), (4, 3, 500))]
    gs = [t[4].clone() for t in layers]

    def step():
        out = []
        for (x, w, b, r, _), g in zip(layers, gs):
            leaves = [t.detach().requires_grad_(True) for t in (x, w, b)]
            out += torch.autograd.grad(net.linear(*leaves, activation="silu", dropout=0.25, seed=SEED), leaves, g)
        return out

    step()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    for k, size in enumerate((1.0, 1e-6, 3e4, 1.0, 2.0 ** -20, 1e-3)):
        for g, t in zip(gs, layers):
            g.copy_(t[4].float().clamp(-2.0, 2.0) * size)
        want = step()
        graph, out = graphs[k % 2]
        graph.replay()
        torch.cuda.synchronize() if k % 3 == 0 else None
        assert all(torch.equal(a, b) for a, b in zip(out, want)) and all(bool(v.any()) for v in want), size
