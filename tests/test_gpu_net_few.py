"""Gradients of 16 bits with few results, or from few values of dZ: dZ's rounding does not average out there, and goes in as two parts."""
import pytest
import torch

import net_ref as ref
from test_gpu_net import SEED, make, net, run  # noqa: F401

pytestmark = pytest.mark.gpu
F64, FEW = torch.float64, 4096
SIZES = [(1, 200, 216), (4, 1, 3655), (2, 300, 150), (3, 1300, 4), (380289, 8, 8), (5000, 10, 200), (20000, 200, 3), (3, 129, 700), (4096, 1, 128), (100000, 64, 64), (1, 4096, 1),
         (7, 500, 585), (9, 140, 455), (1000, 130, 4)]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kind, p", [("silu", 0.25), ("none", 0.25), ("softplus", 0.0)])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_few_gradients_are_rounded_once(net, size, kind, p, dtype):  # noqa: F811
    """Bounds: those of the same numbers in fp32; what two parts of dZ leave, half a step of half a step of it, and half of fp16's least number after scaling (2^-39 of the largest
    |g| / (1 - p)); the result's own rounding.  And as a whole: within a tenth of the result's own rounding's size."""
    T = ref.TYPES[dtype]
    rows, inputs, outputs = size
    x, w, b, r, g = make(*size, T, seed=5 + sum(size), pad=1)
    out = run(net, x, w, b, r, g, kind, 1.0, p, SEED)
    x, w, b, r, g = (v.float() for v in (x, w, b, r, g))
    want = ref.linear(x, w, b, r, g, kind, 1.0, p, SEED)
    X, W, B, G = (v.cpu().to(F64) for v in (x, w, b, g))
    dz = (G * ref.slope(X @ W.T + B, kind, 1.0) * ref.factor(G.shape, p, SEED)).abs()
    left = dz * 1.1 * (torch.finfo(T).eps / 2) ** 2 + float(G.abs().max()) / (1.0 - p) * 2.0 ** -39
    few = {"dx": min(rows * outputs, rows * inputs) <= FEW, "dweight": min(rows * outputs, outputs * inputs) <= FEW}
    assert any(few.values())
    for name, more in (("dx", left @ W.abs()), ("dweight", left.T @ X.abs())):
        value, bound = want[name]
        if few[name]:
            ref.assert_close(name, out[name], (value, bound + more + ref.rounded(value, T) * 1.01))
            off, own = ((v.cpu().to(F64) - value).norm() for v in (out[name], value.to(T)))
            assert float(off) <= 1.1 * float(own) + float((bound + more).norm()), (name, float(off / own))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("size", [(4, 1, 3655), (5000, 10, 200), (20000, 200, 3), (3, 129, 700), (1, 200, 216)], ids=str)
def test_infinities_beside_parts(net, size, dtype):  # noqa: F811
    """A rest of 0 beside an infinity is no NaN."""
    T = ref.TYPES[dtype]
    rows, inputs, outputs = size
    for where in range(3):
        x, w, _, r, g = make(*size, T, seed=rows + where)
        x, w, g = (t.abs() + 1 for t in (x, w, g))
        (x, w, g)[where][-1, 0] = float("inf")
        leaves = [t.detach().requires_grad_(True) for t in (x, w)]
        # everything is kept, times 1 / (1 - 2^-33), which is 1 in fp32: dZ is made, and is g
        dx, dw = torch.autograd.grad(net.linear(*leaves, dropout=2.0 ** -40, seed=SEED), leaves, g)
        X, W, G = (t.cpu().to(F64) for t in (x, w, g))
        for name, got, v in (("dx", dx, G @ W), ("dweight", dw, G.T @ X)):
            got = got.cpu().to(F64)
            assert not got.isnan().any() and torch.equal(got[v.isinf()], v[v.isinf()]), (name, where)
            assert bool(got[v < 60000].isfinite().all()), (name, where)
