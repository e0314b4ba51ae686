"""optim.py without a GPU: a library that keeps what every list holds on the device instead of launching kernels, streams that record
graphs, and tensors on the CPU that say they are on a GPU.

Eager calls take effect at once, calls on a stream that records do when their graph is replayed.  A call that runs looks at the list as it is
on the device then, and notes which scratch it uses."""
import contextlib
import ctypes

import numpy as np
import torch

GPU = torch.device("cuda", 0)


class OnGpu(torch.Tensor):
    """A CPU tensor that is taken for one on the GPU."""
    device = property(lambda self: GPU)
    used_on = []                                 # (address, stream), of all of them

    def record_stream(self, stream):
        OnGpu.used_on.append((self.data_ptr(), stream.cuda_stream))


def on_gpu(t):
    return torch.as_tensor(t).as_subclass(OnGpu)


class Graph:
    def __init__(self):
        self.todo = []

    def replay(self):
        for f in self.todo:
            f()


class Stream:
    def __init__(self, machine, number):
        self.machine, self.cuda_stream = machine, number

    def wait_stream(self, other):
        self.machine.waits.append((self.cuda_stream, other.cuda_stream))


class Machine:
    """The fake library (its functions are the library's), the current stream, what has run."""

    def __init__(self, monkeypatch):
        from paper_2211_15601_amd import binding, optim
        self.optim, self.binding = optim, binding
        self.stream, self.device, self.lists, self.ran, self.waits, self.destroyed = 5, 0, {}, [], [], []
        self.captures = {}                       # stream: (number of the capture, graph)
        self.count = 0
        monkeypatch.setattr(binding, "load", lambda: self)
        monkeypatch.setattr(optim, "_device_of", lambda tensors, device=None: GPU)
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: self.stream in self.captures)
        monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: self.stream)
        monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: Stream(self, self.stream))
        monkeypatch.setattr(torch.cuda, "current_device", lambda: self.device)
        monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: self.device)
        monkeypatch.setattr(torch.cuda, "device", self.on_device)
        empty = torch.empty
        monkeypatch.setattr(torch, "empty", lambda *size, device=None, **k: on_gpu(empty(*size, **k)) if device == GPU else empty(*size, device=device, **k))

    @contextlib.contextmanager
    def on_device(self, device):
        before, self.device = self.device, torch.device(device).index if not isinstance(device, int) else device
        yield
        self.device = before

    @contextlib.contextmanager
    def on(self, stream):
        before, self.stream = self.stream, stream
        yield
        self.stream = before

    @contextlib.contextmanager
    def capture(self, stream=9):
        self.count += 1
        graph = Graph()
        self.captures[stream] = (self.count, graph)
        with self.on(stream):
            yield graph
        del self.captures[stream]

    def do(self, h, f):
        s = self.lists[h]["stream"]
        (self.captures[s][1].todo.append if s in self.captures else lambda f: f())(f)

    def here(self, h):
        return self.captures.get(self.lists[h]["stream"], (0,))[0]

    # ---- the library ----
    def _put(self, h, array, count):
        at = array if isinstance(array, int) else ctypes.addressof(array)
        given = np.frombuffer((ctypes.c_char * max(1, count * 72)).from_address(at), dtype=self.optim._COLUMNS, count=count).copy()
        x = self.lists[h]
        x["host"], x["put_in"] = given, self.here(h)
        self.do(h, lambda: x.update(device=given))
        return self.binding.FS_OK

    def _new(self, array, count, stream, out, scratch):
        self.count += 1
        h = self.count
        self.lists[h] = {"stream": stream, "device": None, "scratch": scratch or h}
        out._obj.value = h
        return self._put(h, array, count)

    def fs_tensors_create(self, array, count, stream, out):
        return self._new(array, count, stream, out, None)

    def fs_tensors_create_noalloc(self, array, count, stream, workspace, size, out):
        return self._new(array, count, stream, out, ("workspace", workspace))

    def fs_tensors_bytes(self, count):
        return 100 + count

    def fs_tensors_update(self, h, array, count):
        return self._put(h.value, array, count) if self.device == GPU.index else self.binding.FS_E_DEVICE

    def fs_tensors_set_stream(self, h, stream):
        self.lists[h.value]["stream"] = stream
        return self.binding.FS_OK

    def fs_tensors_ready(self, h):
        x = self.lists[h.value]
        return self.binding.FS_E_STATE if x["put_in"] and x["put_in"] != self.here(h.value) else self.binding.FS_OK

    def fs_tensors_destroy(self, h):
        self.destroyed.append(h.value)
        return self.binding.FS_OK

    def fs_tensors_error(self, h):
        return b"refused"

    def _call(self, name, h, *args):
        h = h.value
        if self.device != GPU.index:
            return self.binding.FS_E_DEVICE
        x = self.lists[h]
        if x["put_in"] and x["put_in"] != self.here(h):
            return self.binding.FS_E_STATE
        host = x["host"]
        self.do(h, lambda: self.ran.append({"call": name, "list": x["device"], "fits": x["device"] is not None and np.array_equal(x["device"], host),
                                            "scratch": x["scratch"], "args": args}))
        return self.binding.FS_OK

    def fs_grad_norm(self, h, *args):
        return self._call("norm", h, *args)

    def fs_grad_clip(self, h, *args):
        return self._call("clip", h, *args)

    def fs_adamw_step(self, h, how, step, norm):
        return self._call("adamw", h, {name: getattr(how._obj, name) for name, _ in how._obj._fields_}, step, norm)

    # ---- what a test makes ----
    def params(self, *sizes, dtype=torch.float32):
        return [on_gpu(torch.ones(n, dtype=dtype)).requires_grad_(True) for n in sizes]

    def adamw(self, params, **k):
        return self.optim.AdamW(params, step=on_gpu(torch.zeros(1, dtype=torch.int64)), **k)

    def grads(self, params):
        """New gradients, at other places than any before."""
        for p in params:
            p.grad = on_gpu(torch.ones_like(p.detach().as_subclass(torch.Tensor)))
        return [p.grad for p in params]
