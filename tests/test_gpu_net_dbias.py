"""dbias of columns that cancel: sums over the rows in 64 bits."""
import pytest
import torch

import net_ref as ref
from test_gpu_net import SEED, net  # noqa: F401

pytestmark = pytest.mark.gpu
F64 = torch.float64
SIZES = [(104, 332, 1), (12596, 1857, 1), (7207, 45, 1), (20001, 17, 8), (65536, 128, 128), (37578, 344, 8), (3000, 20, 300), (300001, 40, 24), (2, 3, 5)]


@pytest.mark.parametrize("dtype", list(ref.TYPES))
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_columns_that_cancel(net, size, dtype):  # noqa: F811
    """Pairs of rows that are one another's negative but for a small rest.  dZ is g itself, or g where z > 0 (the same in all rows), or g / (1 - p) as fp32 has it: what is left is
    the rounding of the sum to fp32, 2^-24, and sums of n numbers in 64 bits, each addition 2^-53 of at most sum |g|."""
    rows, inputs, outputs = size
    T, gen = ref.TYPES[dtype], torch.Generator().manual_seed(rows)
    g = torch.randn(rows, outputs, generator=gen) * 100
    half = rows // 2
    g[half:2 * half] = -g[:half] + 0.01 * torch.randn(half, outputs, generator=gen)
    g = g.to(T)
    x, w = torch.ones(rows, inputs, dtype=T, device="cuda"), torch.ones(outputs, inputs, dtype=T, device="cuda")
    for kind, p in (("none", 0.0), ("relu", 0.0), ("none", 0.5)):
        b = torch.zeros(outputs, device="cuda", requires_grad=True)
        (db,) = torch.autograd.grad(net.linear(x, w, b, activation=kind, dropout=p, seed=SEED), b, g.cuda())
        dz = g.to(F64) * ref.factor(g.shape, p, SEED)
        want = dz.sum(0)
        off = (db.cpu().to(F64) - want).abs()
        assert bool((off <= want.abs() * 2.0 ** -24 * 1.01 + rows * 2.0 ** -53 * dz.abs().sum(0)).all()), (kind, p, float((off / want.abs()).max()))
