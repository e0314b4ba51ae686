"""Layers in programs that torch.compile takes: it goes round their calls, forward and backward."""
import pytest
import torch

from test_gpu_net import net  # noqa: F401

pytestmark = pytest.mark.gpu


def test_compiled_programs(net):  # noqa: F811
    gen = torch.Generator(device="cuda").manual_seed(1)
    one = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    x, w, b, g = one(40, 24).requires_grad_(True), one(24, 24).requires_grad_(True), one(24).requires_grad_(True), one(40, 24)

    def f(t):
        return net.linear(net.dropout(t * 2, 0.3, (1, 2)), w, b, residual=t, activation="gelu", dropout=0.2, seed=(3, 4)) * 2

    want = f(x)
    grads = torch.autograd.grad(want, [x, w, b], g)
    torch.compiler.reset()
    try:
        compiled = torch.compile(f, backend="aot_eager")
        y = compiled(x)
        # the same kernels on the same numbers, between operations of PyTorch's own that are exact
        assert torch.equal(y, want) and all(torch.equal(a, c) for a, c in zip(torch.autograd.grad(y, [x, w, b], g), grads))
        with torch.no_grad():
            assert torch.equal(compiled(x), want)
    finally:
        torch.compiler.reset()
