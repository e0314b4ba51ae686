"""Host code of net.py without a GPU: what it refuses, and what it hands to the library (a fake one that writes down its arguments)."""
import contextlib
import ctypes

import pytest
import torch

GPU = torch.device("cuda", 0)


class OnGpu(torch.Tensor):
    """A CPU tensor that is taken for one on the GPU."""
    device = property(lambda self: GPU)
    is_cuda = property(lambda self: True)


def on_gpu(*shape, dtype=torch.float32, fill=None):
    t = torch.zeros(shape, dtype=dtype) if fill is None else torch.full(shape, fill, dtype=dtype)
    return t.as_subclass(OnGpu)


class Fake:
    def __init__(self, binding):
        self.binding, self.calls, self.asked = binding, [], 0

    def fs_linear_bytes(self, layer, backward):
        self.asked += 1
        return 256 if backward else 0

    def _note(self, name, layer, args):
        l = self.binding.Linear()
        ctypes.pointer(l)[0] = layer._obj
        self.calls.append((name, l, args))
        return 0

    def fs_linear_forward(self, layer, *args):
        return self._note("forward", layer, args)

    def fs_linear_backward(self, layer, *args):
        return self._note("backward", layer, args)

    def fs_dropout(self, kind, rows, columns, drop, *args):
        self.calls.append(("dropout", (kind, rows, columns, drop._obj.p, drop._obj.seed, drop._obj.offset, drop._obj.d_seed), args))
        return 0

    def fs_net_error(self):
        return b"no"


@pytest.fixture
def fake(monkeypatch):
    from paper_2211_15601_amd import binding, net
    f = Fake(binding)
    monkeypatch.setattr(binding, "load", lambda: f)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 5, raising=False)
    monkeypatch.setattr(torch.cuda, "device", lambda d: contextlib.nullcontext())
    net._plan.cache_clear()
    yield f
    net._plan.cache_clear()


def test_refusals(fake):
    from paper_2211_15601_amd import net
    x, w, b, r = on_gpu(4, 6), on_gpu(8, 6), on_gpu(8), on_gpu(4, 8)
    half = lambda t: t.to(torch.bfloat16).as_subclass(OnGpu)
    for kind, match, f in (
            (TypeError, "x: expected a tensor", lambda: net.linear([1.0], w)),
            (TypeError, "x: torch.float64", lambda: net.linear(on_gpu(4, 6, dtype=torch.float64), w)),
            (ValueError, "must be on a GPU", lambda: net.linear(torch.zeros(4, 6), w)),
            (ValueError, "x needs a dimension", lambda: net.linear(on_gpu(), w)),
            (TypeError, "weight: expected a tensor", lambda: net.linear(x, None)),
            (TypeError, "weight: torch.bfloat16", lambda: net.linear(x, half(w))),
            (ValueError, "weight: on cpu", lambda: net.linear(x, torch.zeros(8, 6))),
            (ValueError, "weight: shape", lambda: net.linear(x, on_gpu(6, 8))),
            (ValueError, "weight: shape", lambda: net.linear(x, on_gpu(6))),
            (ValueError, "bias: shape", lambda: net.linear(x, w, on_gpu(7))),
            (TypeError, "bias: torch.bfloat16", lambda: net.linear(x, w, half(b))),
            (TypeError, "bias: torch.float16", lambda: net.linear(half(x), half(w), b.to(torch.float16).as_subclass(OnGpu))),
            (ValueError, "residual: shape", lambda: net.linear(x, w, b, residual=on_gpu(1, 8))),
            (TypeError, "residual: torch.bfloat16", lambda: net.linear(x, w, b, residual=half(r))),
            (ValueError, "activation must be", lambda: net.linear(x, w, activation="tanh")),
            (ValueError, "beta must be", lambda: net.linear(x, w, activation="softplus", beta=0.0)),
            (ValueError, "beta must be", lambda: net.linear(x, w, activation="softplus", beta=float("nan"))),
            (ValueError, "dropout must be", lambda: net.linear(x, w, dropout=1.5, seed=(1, 2))),
            (ValueError, "dropout must be", lambda: net.linear(x, w, dropout=float("nan"), seed=(1, 2))),
            (ValueError, "needs a seed", lambda: net.linear(x, w, dropout=0.5)),
            (ValueError, "needs a seed", lambda: net.linear(x, w, dropout=0.5, seed=(1, -2))),
            (ValueError, "needs a seed", lambda: net.linear(x, w, dropout=0.5, seed=(1, 2 ** 64))),
            (ValueError, "needs a seed", lambda: net.linear(x, w, dropout=0.5, seed=7)),
            (TypeError, "seed: torch.float32", lambda: net.linear(x, w, dropout=0.5, seed=on_gpu(2))),
            (ValueError, "seed: on cpu", lambda: net.linear(x, w, dropout=0.5, seed=torch.zeros(2, dtype=torch.int64))),
            (ValueError, "two words", lambda: net.linear(x, w, dropout=0.5, seed=on_gpu(3, dtype=torch.int64))),
            (ValueError, "two words", lambda: net.linear(x, w, dropout=0.5, seed=on_gpu(2, 2, dtype=torch.int64)[:, 0])),
            (ValueError, "p must be", lambda: net.dropout(x, -0.1, (1, 2))),
            (ValueError, "needs a seed", lambda: net.dropout(x, 0.5)),
            (ValueError, "residual: shape", lambda: net.dropout(x, 0.5, (1, 2), residual=on_gpu(6))),
            (TypeError, "residual: torch.bfloat16", lambda: net.dropout(x, 0.5, (1, 2), residual=half(x))),
            (ValueError, "a network needs", lambda: net.Network(3, 8, 0, 2)),
            (ValueError, "activation must be", lambda: net.Network(3, 8, 1, 2, activation="sin")),
            (ValueError, "dropout must be", lambda: net.Network(3, 8, 1, 2, dropout=2.0))):
        with pytest.raises(kind, match=match):
            f()
    assert not fake.calls


def test_what_the_library_gets(fake):
    from paper_2211_15601_amd import net
    x, w, b, r = on_gpu(2, 3, 6), on_gpu(8, 10)[:, :6], on_gpu(8), on_gpu(2, 3, 8)
    y = net.linear(x, w, b, residual=r, activation="softplus", beta=3.0, dropout=0.25, seed=(7, 9))
    ((name, l, args),) = fake.calls
    assert name == "forward" and (l.rows, l.inputs, l.outputs, l.type, l.bias_type, l.act, l.beta) == (6, 6, 8, 0, 0, 4, 3.0)
    assert (l.drop.p, l.drop.seed, l.drop.offset, l.drop.d_seed) == (0.25, 7, 9, None)
    assert args == (x.data_ptr(), 6, w.data_ptr(), 10, b.data_ptr(), r.data_ptr(), 8, y.data_ptr(), 8, None, 8, None, 0, 5)
    assert y.shape == (2, 3, 8)
    words = on_gpu(2, dtype=torch.int64)
    net.linear(x, w, dropout=0.25, seed=words)
    _, l, args = fake.calls[-1]
    assert l.drop.d_seed == words.data_ptr() and args[4] is None and args[5] is None
    # the same sizes: the plan is that of before; a seed that is not asked for is not looked at
    before = fake.asked
    for _ in range(3):
        net.linear(x, w, dropout=0.0, seed="nothing")
    assert fake.asked == before + 2
    # rows that do not lie apart evenly, or whose elements do, are copied
    for t in (on_gpu(6, 2, 3).permute(1, 2, 0), on_gpu(2, 3, 12)[..., ::2], on_gpu(3, 4, 6)[:, :2].transpose(0, 1)):
        net.linear(t, w)
        assert fake.calls[-1][1].rows == 6 and fake.calls[-1][2][1] == 6
    net.linear(on_gpu(6).expand(5, 6), w)
    assert fake.calls[-1][2][1] == 0                 # one row, seen five times
    fake.calls.clear()
    net.dropout(on_gpu(4, 10)[:, :7], 0.5, (1, 2 ** 64 - 1), residual=on_gpu(4, 7))
    ((name, how, args),) = fake.calls
    assert how == (0, 4, 7, 0.5, 1, 2 ** 64 - 1, None) and args[1] == 10 and args[3] == 7 and args[5] == 7


def test_errors_are_raised(fake):
    from paper_2211_15601_amd import net
    fake.fs_linear_forward = lambda *a: 2
    with pytest.raises(fake.binding.FsError, match="FS_E_SHAPE: no"):
        net.linear(on_gpu(4, 6), on_gpu(8, 6))
    net._plan.cache_clear()
    fake.fs_linear_bytes = lambda *a: -1
    with pytest.raises(fake.binding.FsError, match="FS_E_SHAPE: no"):
        net.linear(on_gpu(4, 6), on_gpu(8, 6))


def test_another_device_than_the_current_one(fake, monkeypatch):
    """The call is made with the tensors' device current, on that device's stream, and the other one is current again afterwards."""
    from paper_2211_15601_amd import net
    now, seen = [3], []

    @contextlib.contextmanager
    def device(d):
        before, now[0] = now[0], d if isinstance(d, int) else d.index
        yield
        now[0] = before

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 100 + i, raising=False)
    monkeypatch.setattr(torch.cuda, "device", device)
    fake.fs_linear_forward = lambda *a: seen.append((now[0], a[-1])) or 0
    fake.fs_dropout = lambda *a: seen.append((now[0], a[-1])) or 0
    net.linear(on_gpu(4, 6), on_gpu(8, 6))
    net.dropout(on_gpu(4, 6), 0.5, (1, 2))
    assert seen == [(0, 100), (0, 100)] and now == [3]


@pytest.mark.parametrize("rows, act, kind, bias_kind, full", [
    (6, "gelu", torch.bfloat16, torch.bfloat16, True), (6, "silu", torch.float16, None, True), (1 << 19, "softplus", torch.float16, None, True),
    ((1 << 19) + 1, "softplus", torch.float16, None, False), (6, "relu", torch.bfloat16, None, False), (6, "none", torch.bfloat16, None, False),
    (6, "gelu", torch.float32, None, False), (6, "gelu", torch.bfloat16, torch.float32, False)])
def test_where_z_is_kept_in_fp32(fake, rows, act, kind, bias_kind, full):
    net = __import__("paper_2211_15601_amd.net", fromlist=["net"])
    plan = net._plan(0, rows, 6, 8, net._TYPES[kind], net._TYPES[bias_kind or kind], net._ACTS[act], 1.0, 0.0)
    assert plan.z_full == full and plan.bare.act == net._ACTS[act] + 256 * full
