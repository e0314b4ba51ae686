"""net.py where PyTorch looks on: forward-mode derivatives and traces, which the calls do not offer, are refused and not lost."""
import pytest
import torch
import torch.autograd.forward_ad as forward_ad

from test_net_host import OnGpu, fake, on_gpu  # noqa: F401

CALLS = (lambda net, x: net.linear(x, on_gpu(6, 6)), lambda net, x: net.linear(on_gpu(4, 6), on_gpu(6, 6), residual=x, activation="silu"), lambda net, x: net.dropout(x, 0.5, (1, 2)),
         lambda net, x: net.dropout(on_gpu(4, 6), 0.5, (1, 2), residual=x))


@pytest.mark.parametrize("call", CALLS)
def test_tangents_are_not_lost(fake, call):  # noqa: F811
    from paper_2211_15601_amd import net
    with forward_ad.dual_level():
        dual = forward_ad.make_dual(torch.zeros(4, 6), torch.ones(4, 6)).as_subclass(OnGpu)
        for enabled in (True, False):
            with torch.set_grad_enabled(enabled), pytest.raises(NotImplementedError, match="jvp"):
                call(net, dual)
        assert not fake.calls
        call(net, on_gpu(4, 6))                          # without a tangent it is a call as any other
    assert len(fake.calls) == 1


@pytest.mark.parametrize("call", CALLS)
def test_traces_are_refused(fake, call):  # noqa: F811
    from torch.fx.experimental.proxy_tensor import make_fx
    from paper_2211_15601_amd import net
    for before in (False, True):
        with pytest.raises(RuntimeError, match="cannot be traced"):
            make_fx(lambda t: call(net, t), pre_dispatch=before)(on_gpu(4, 6))
    with pytest.raises(RuntimeError, match="cannot be traced"):
        torch.jit.trace(lambda t: call(net, t), (on_gpu(4, 6),), check_trace=False)
    assert not fake.calls


def test_other_modes_are_none_of_its_business(fake):  # noqa: F811
    """A mode that only looks on (a counter of operations, a log) sees the call run."""
    from torch.utils._python_dispatch import TorchDispatchMode
    from paper_2211_15601_amd import net

    class Log(TorchDispatchMode):
        def __torch_dispatch__(self, func, types, args=(), kwargs=None):
            return func(*args, **(kwargs or {}))

    with Log():
        net.dropout(on_gpu(4, 6), 0.5, (1, 2))
    assert len(fake.calls) == 1


def test_values_that_are_negated_lazily(fake):  # noqa: F811
    """The imaginary part of a conjugate has its sign kept beside the tensor; what the library reads has to have it."""
    import ctypes
    from paper_2211_15601_amd import net
    read = lambda p: ctypes.c_float.from_address(p).value
    seen = []
    fake.fs_linear_forward = lambda layer, x, ldx, w, ldw, b, r, ldr, y, *a: seen.append([read(p) for p in (x, w, b, r)]) or 0
    fake.fs_dropout = lambda kind, rows, columns, drop, x, ldx, r, ldr, *a: seen.append([read(p) for p in (x, r)]) or 0
    negated = lambda *shape: torch.complex(torch.zeros(shape), torch.ones(shape)).conj().imag.as_subclass(OnGpu)
    assert negated(3, 1).is_neg() and negated(3, 1).stride(0) == 2
    net.linear(negated(3, 1), negated(1, 1), negated(1), residual=negated(3, 1))
    net.dropout(negated(3, 1), 0.5, (1, 2), residual=negated(3, 1))
    net.dropout(negated(3, 2), 0.5, (1, 2), residual=negated(3, 2))
    assert seen == [[-1.0] * 4, [-1.0] * 2, [-1.0] * 2]


def test_second_derivatives_are_not_lost(fake):  # noqa: F811
    """A penalty on a gradient (of a field's normals, say): the gradients of x, weight and bias depend on x and weight, also where the loss is a sum and its own gradient constant."""
    from paper_2211_15601_amd import net
    leaf = lambda *shape: on_gpu(*shape).requires_grad_(True)
    for act in ("none", "softplus"):
        for of in range(3):
            leaves = [leaf(4, 6), leaf(8, 6), leaf(8)]
            y = net.linear(*leaves, activation=act)
            (d,) = torch.autograd.grad(y.sum(), leaves[of], create_graph=True)
            assert d.shape == leaves[of].shape and d.requires_grad
            with pytest.raises(RuntimeError, match="no second derivatives"):
                (y.sum() + d.square().sum()).backward()
    # a gradient that is only looked at, beside others; the residual's is y's own
    leaves, r = [leaf(4, 6), leaf(8, 6), leaf(8)], leaf(4, 8)
    y = net.linear(*leaves, residual=r)
    g = on_gpu(4, 8, fill=3.0).requires_grad_(True)
    grads = torch.autograd.grad(y, [*leaves, r], g, create_graph=True)
    assert [d.shape for d in grads] == [t.shape for t in (*leaves, r)]
    (again,) = torch.autograd.grad(grads[3].square().sum(), g)
    assert torch.equal(again, 2 * g.detach())
    y.sum().backward()
    assert all(t.grad is not None and not t.grad.requires_grad for t in leaves)


@pytest.mark.parametrize("act", ["none", "silu"])
def test_second_derivatives_towards_every_input(fake, act):  # noqa: F811
    """Also where only some inputs' derivatives are asked for, and those that are not found may be left out, as torch.autograd.functional does."""
    from paper_2211_15601_amd import net
    for wanted in range(1, 8):
        leaves = [on_gpu(*shape).requires_grad_(bool(wanted >> i & 1)) for i, shape in enumerate(((4, 6), (8, 6), (8,)))]
        asked = [t for t in leaves if t.requires_grad]
        g = on_gpu(4, 8, fill=1.0).requires_grad_(True)
        for first in asked:
            for second in (*asked, g):
                y = net.linear(*leaves, activation=act)
                (d,) = torch.autograd.grad(y, first, g, create_graph=True)
                with pytest.raises(RuntimeError, match="no second derivatives"):
                    torch.autograd.grad(d.sum(), second, allow_unused=True)
    for f in (lambda t: torch.autograd.functional.hessian(lambda v: net.linear(v, on_gpu(8, 6), activation=act).sum(), t), lambda t: torch.autograd.functional.jvp(lambda v: net.linear(v, on_gpu(8, 6), activation=act), t, t)):
        with pytest.raises(RuntimeError, match="no second derivatives"):
            f(on_gpu(4, 6))


def test_dropout_is_its_own_derivative(fake, monkeypatch):  # noqa: F811
    """Its gradient is dropout of y's gradient, and is differentiated as such."""
    import ctypes
    from paper_2211_15601_amd import net
    words = on_gpu(2, dtype=torch.int64)

    def double(kind, rows, columns, drop, x, ldx, r, ldr, y, ldy, stream):
        """stands for drop(): twice of everything"""
        for i in range(rows):
            for j in range(columns):
                at = lambda p, ld: ctypes.c_float.from_address(p + 4 * (i * ld + j))
                at(y, ldy).value = 2.0 * at(x, ldx).value + (at(r, ldr).value if r else 0.0)
        return 0

    class Any:                                         # PyTorch's own gradients here are CPU tensors, without an index
        __ne__ = lambda self, other: False

    monkeypatch.setattr(torch._C, "_cuda_getDevice", Any)
    fake.fs_dropout = double
    for seed in ((1, 2), words):
        x, r = on_gpu(3, 4, fill=3.0).requires_grad_(True), on_gpu(3, 4, fill=1.0).requires_grad_(True)
        y = net.dropout(x, 0.5, seed, residual=r)
        dx, dr = torch.autograd.grad(y.square().sum(), [x, r], create_graph=True)     # y = 2 x + r: 4 y and 2 y
        assert bool((dx == 28.0).all()) and bool((dr == 14.0).all())
        assert bool((torch.autograd.grad(dx.sum() + dr.sum(), x, retain_graph=True)[0] == 8.0 + 4.0).all())
        assert bool((torch.autograd.grad(dx.sum(), r)[0] == 4.0).all())


@pytest.mark.parametrize("call", CALLS)
@pytest.mark.parametrize("grad", [False, True])
def test_compiled_programs_go_round_the_calls(fake, call, grad):  # noqa: F811
    from paper_2211_15601_amd import net
    x = on_gpu(4, 6).requires_grad_(grad)
    torch.compiler.reset()
    try:
        y = torch.compile(lambda t: call(net, t) + 1, backend="eager")(x)
        assert len(fake.calls) == 1 and y.shape == (4, 6) and y.requires_grad == grad
    finally:
        torch.compiler.reset()
