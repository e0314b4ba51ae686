"""Z beyond what fp16 holds, kept in fp16."""
import pytest
import torch

from test_gpu_net import net  # noqa: F401

pytestmark = pytest.mark.gpu
F64, T = torch.float64, torch.float16


@pytest.mark.parametrize("size", [(6, 4, 5), (2000, 17, 97), (300, 200, 130)], ids=str)
@pytest.mark.parametrize("kind", ["relu", "gelu", "silu", "softplus"])
def test_z_beyond_fp16(net, monkeypatch, size, kind):  # noqa: F811
    """Z of +-70144, and of 2^-26, kept in 16 bits as in layers of more than 2^22 values: slopes are 1, 0, and those at 0 (of relu 1: it is positive)."""
    rows, inputs, outputs = size
    monkeypatch.setattr(net, "_Z_FULL", 0)
    net._plan.cache_clear()
    try:
        x, w = (torch.zeros(n, inputs, dtype=T, device="cuda") for n in (rows, outputs))
        x[0::3, 0], x[1::3, 0], x[2::3, 1] = 256.0, -256.0, 2.0 ** -13
        w[:, 0], w[:, 1] = 274.0, 2.0 ** -13
        x, w = x.requires_grad_(True), w.requires_grad_(True)
        y = net.linear(x, w, activation=kind, beta=100.0 if kind == "softplus" else 1.0)
        assert torch.equal(y[0::3].isinf(), torch.ones_like(y[0::3], dtype=torch.bool)) and not y[1::3].any()
        g = torch.full((rows, outputs), 2.0 ** -10, dtype=T, device="cuda")
        dx, dw = torch.autograd.grad(y, [x, w], g)
        slope = torch.tensor([1.0, 0.0, 1.0 if kind == "relu" else 0.5], dtype=F64)[torch.arange(rows) % 3]
        want = (g.cpu().to(F64) * slope[:, None]) @ w.detach().cpu().to(F64)
        # one rounding of dz (of the slope at 0: 0.5 + 2^-26), fp32 sums, one of the result
        assert float(((dx.cpu().to(F64) - want).abs() - want.abs() * 2.0 ** -9).max()) <= 2.0 ** -24
        want = (g.cpu().to(F64) * slope[:, None]).T @ x.detach().cpu().to(F64)
        assert float(((dw.cpu().to(F64) - want).abs() - want.abs() * 2.0 ** -9).max()) <= 2.0 ** -24
    finally:
        net._plan.cache_clear()


def test_a_flat_softplus(net, monkeypatch):  # noqa: F811
    """beta = 1e-5: Z of +-400000 has slopes of its own, 1 / (1 + e^-+4), which +-65504 would not give."""
    monkeypatch.setattr(net, "_Z_FULL", 0)
    net._plan.cache_clear()
    try:
        x = torch.tensor([[640.0], [-640.0], [0.0]], dtype=T, device="cuda").repeat(40, 1).requires_grad_(True)
        w = torch.full((150, 1), 625.0, dtype=T, device="cuda").requires_grad_(True)
        g = torch.full((120, 150), 2.0 ** -13, dtype=T, device="cuda")
        dx, dw = torch.autograd.grad(net.linear(x, w, activation="softplus", beta=1e-5), [x, w], g)
        slope = torch.sigmoid(1e-5 * x.detach().cpu().to(F64) * 625.0)
        want = 2.0 ** -13 * slope * 625.0 * 150
        # one rounding of dz, of a slope good to fp32, and one of the result: 2^-11 each
        assert float(((dx.cpu().to(F64) - want).abs() / want).max()) <= 2.1 * 2.0 ** -11
        want = (2.0 ** -13 * slope * x.detach().cpu().to(F64)).sum()
        assert float(((dw.cpu().to(F64) - want).abs() / want).max()) <= 2.1 * 2.0 ** -11
    finally:
        net._plan.cache_clear()
