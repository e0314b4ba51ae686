"""Narrow layers whose blocks take several groups of 32 rows, and gradients through broadcast and repeated tensors, by their values."""
import math

import pytest
import torch

import net_ref as ref
from test_gpu_net import SEED, check, make, net, run, whole  # noqa: F401

pytestmark = pytest.mark.gpu
F64 = torch.float64
SIZES = [((20001, 128, 24), "f32"), ((20001, 97, 128), "f32"), ((24640, 1, 128), "f32"), ((60001, 128, 40), "bf16"), ((60001, 128, 40), "f16"), ((50000, 33, 128), "bf16"),
         ((131072, 10, 9), "f16"), ((130999, 8, 1), "bf16"), ((300001, 128, 9), "bf16"), ((262149, 40, 24), "f16")]


@pytest.mark.parametrize("size, dtype", SIZES, ids=str)
def test_whole_numbers(net, size, dtype):  # noqa: F811
    """Exact: sums of whole numbers below 2^24 in fp32; 64-bit sums on the GPU."""
    rows, inputs, outputs = size
    T, gen = ref.TYPES[dtype], torch.Generator(device="cuda").manual_seed(rows)
    x, w, g = (whole(m, n, T, gen, 3) for m, n in ((rows, inputs), (outputs, inputs), (rows, outputs)))
    b = torch.zeros(outputs, device="cuda")
    leaves = [t.detach().requires_grad_(True) for t in (x, w, b)]
    f = ref.factor((rows, outputs), 0.5, SEED).cuda()
    X, W, G = (t.to(F64) for t in (x, w, g))
    for kind in ("none", "relu"):
        grads = torch.autograd.grad(net.linear(*leaves, activation=kind, dropout=0.5, seed=SEED), leaves, g)
        dz = G * f * ((X @ W.t() > 0) if kind == "relu" else 1.0)
        assert float((dz.t().abs() @ X.abs()).max()) < 2 ** 24
        for name, got, want in zip(("dx", "dweight", "dbias"), grads, (dz @ W, dz.t() @ X, dz.sum(0))):
            off = got != want.to(got.dtype)
            assert not bool(off.any()), (kind, name, int(off.sum()), off.nonzero()[:4].tolist())


@pytest.mark.parametrize("size, dtype", SIZES, ids=str)
def test_against_64_bits(net, size, dtype):  # noqa: F811
    t = make(*size, ref.TYPES[dtype], seed=sum(size), pad=1)
    check(run(net, *t, "silu", 1.0, 0.25, SEED), *t, "silu", 1.0, 0.25, SEED)


@pytest.mark.parametrize("size, dtype", SIZES, ids=str)
def test_an_infinity_in_a_late_row(net, size, dtype):  # noqa: F811
    rows, inputs, outputs = size
    T, gen = ref.TYPES[dtype], torch.Generator(device="cuda").manual_seed(rows)
    for where in range(2):
        x, w, g = (whole(m, n, T, gen).abs() + 1 for m, n in ((rows, inputs), (outputs, inputs), (rows, outputs)))
        (x, g)[where][rows - 7, 0] = -math.inf
        leaves = [t.detach().requires_grad_(True) for t in (x, w)]
        dx, dw = torch.autograd.grad(net.linear(*leaves), leaves, g)
        X, W, G = (t.to(F64) for t in (x, w, g))
        for name, got, want in (("dx", dx, G @ W), ("dweight", dw, G.t() @ X)):
            assert torch.equal(got, want.to(T)), (name, where)


def test_a_row_that_is_broadcast(net):  # noqa: F811
    """Its gradient is the sum over the rows that it is seen as: of whole numbers, exact."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    for T in ref.TYPES.values():
        for rows, inputs, outputs in ((60, 24, 40), (500, 300, 200)):
            row, w, res, g = (whole(m, n, T, gen) for m, n in ((1, inputs), (outputs, inputs), (1, outputs), (rows, outputs)))
            leaves = [t.detach().requires_grad_(True) for t in (row, w, res)]
            y = net.linear(leaves[0].expand(rows, inputs), leaves[1], residual=leaves[2].expand(rows, outputs))
            drow, dw, dres = torch.autograd.grad(y, leaves, g)
            R, W, G = (t.to(F64) for t in (row, w, g))
            each = (G @ W).to(T)                       # rounded, then added up by PyTorch
            assert torch.equal(drow, each.sum(0, keepdim=True)) and torch.equal(dres, g.sum(0, keepdim=True)) and torch.equal(dw, (G.t() @ R.expand(rows, inputs)).to(T))
            assert torch.equal(y.detach(), ((R @ W.t()) + res.to(F64)).expand(rows, outputs).to(T))


def test_one_tensor_as_input_and_weight(net):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(5)
    for T in ref.TYPES.values():
        for n, k in ((64, 64), (20, 160), (300, 200), (1100, 1100)):
            v, g = whole(n, k, T, gen), whole(n, n, T, gen)
            leaf = v.detach().requires_grad_(True)
            y = net.linear(leaf, leaf)
            (d,) = torch.autograd.grad(y, leaf, g)
            V, G = v.to(F64), g.to(F64)
            # two gradients, each rounded, added up by PyTorch
            assert torch.equal(y.detach(), (V @ V.t()).to(T)) and torch.equal(d, (G @ V).to(T) + (G.t() @ V).to(T))
