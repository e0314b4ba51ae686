"""What a training program does with its gradients, over the C ABI of include/fastsnarf_train.h: the global norm of a list of
tensors, clipping, and the AdamW step.

    norm = TensorList([p.grad for p in params]).clip_grads(1.0)          # scales the gradients where they are

    opt = AdamW(params, lr=1e-3, weight_decay=0.01, max_norm=1.0)        # clips inside the step: no gradient is rewritten
    loss.backward(); norm = opt.step(); opt.zero_grad()

Tensors are float32, bfloat16 or float16 on one GPU, of any size and alignment, dense (any order of dimensions, without
gaps); moments and masters are float32.  Results stay on the GPU and nothing waits for it.  Calls run on the stream that is current
when they are made, and can be captured into graphs of torch.cuda (after the list was made, or used once, outside of them), which may be replayed in any order,
beside one another and beside eager calls.  Argument marshalling only: the arithmetic runs in the HIP kernels.  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Sequence

import numpy as np
import torch

from . import binding

# an fs_tensor, for whole columns of a list at once
_COLUMNS = np.dtype([(n, np.uint64) for n in ("grad", "out", "param", "master", "exp_avg", "exp_avg_sq")] +
                    [("n", np.uint64), ("grad_type", np.int32), ("param_type", np.int32), ("lr_scale", np.float32), ("decay_scale", np.float32)])
_TYPES = {torch.float32: binding.FS_FLOAT_FULL, torch.bfloat16: binding.FS_FLOAT_BRAIN, torch.float16: binding.FS_FLOAT_HALF}
_BYTES = np.array([4, 2, 2], dtype=np.uint64)          # of an element, by type
_KINDS = {"l2": binding.FS_NORM_TWO, "max": binding.FS_NORM_MAX}


def _dense(t: torch.Tensor) -> bool:
    """Does the tensor's memory hold its elements one after another, in some order of the dimensions?"""
    if t.is_contiguous():
        return True
    at = 1
    for stride, size in sorted((st, sz) for st, sz in zip(t.stride(), t.shape) if sz != 1):
        if stride != at:
            return False
        at *= size
    return True


def _order(t: torch.Tensor):
    return [st for st, sz in zip(t.stride(), t.shape) if sz != 1]


def _check(what: str, i: int, t: torch.Tensor, like: Optional[torch.Tensor], device, types):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}[{i}]: expected a tensor, got {type(t).__name__}")
    if t.dtype not in types:
        raise TypeError(f"{what}[{i}]: {t.dtype} is not supported here, expected {' or '.join(str(k) for k in types)}")
    if t.device != device:
        raise ValueError(f"{what}[{i}]: on {t.device}, the list is on {device}")
    if like is None:
        if t.layout != torch.strided or not _dense(t):
            raise ValueError(f"{what}[{i}]: elements must lie one after another in memory (use .contiguous())")
    elif t.shape != like.shape or not (t.is_contiguous() and like.is_contiguous()) and t.numel() and _order(t) != _order(like):
        raise ValueError(f"{what}[{i}]: shape {tuple(t.shape)} and strides {t.stride()}, expected {tuple(like.shape)} and {like.stride()}")


def _overlap():
    raise ValueError("tensors of the list overlap in memory")


def _apart(begin, size):
    """No two of these arrays may share memory: calls write them, block by block in no order.  Returns where they lie, for _untouched()."""
    begin, size = begin[size > 0], size[size > 0]
    order = begin.argsort()
    begin = begin[order]
    end = begin + size[order]
    if (begin[1:] < end[:-1]).any():
        _overlap()
    # with an array of nothing at either end, so that every place has one before it (the one before the first is the last)
    return np.concatenate([_ENDS[:1], begin, _ENDS[1:]]), np.concatenate([_ENDS[:1], end, _ENDS[:1]])


_ENDS = np.array([0, 2 ** 64 - 1], dtype=np.uint64)


def _untouched(begin, size, written):
    """None of these arrays, which may share memory with one another, may share any with the written ones."""
    last = written[0].searchsorted(begin + size) - 1             # the last one that begins before this one's end
    if (written[1][last] > begin).any():
        _overlap()


def _check_apart(arrays):
    arrays = [t for t in arrays if t is not None]
    _apart(np.array(_places(arrays), dtype=np.uint64), np.array([t.nbytes for t in arrays], dtype=np.uint64))


class _OnDevice:
    """An fs_tensors: the list on the device, the scratch of its calls, their stream."""

    def __init__(self, L, h, version, stream, workspace=None):
        self.L, self.h, self.version, self.stream, self.raw, self.workspace = L, h, version, stream, stream.cuda_stream, workspace

    def __del__(self):
        try:
            # a list with memory of its own is not freed while a graph is captured, which that would void
            if self.workspace is None and torch.cuda.is_current_stream_capturing() or self.L.fs_tensors_destroy(self.h) != binding.FS_OK:
                _later.append(self.h)
        except Exception:
            pass


_later = []                            # lists that could not be freed when they went


def _free_later(L):
    for _ in range(len(_later)):
        h = _later.pop(0)
        if L.fs_tensors_destroy(h) != binding.FS_OK:
            _later.append(h)


class _Handle:
    """A list on the host, and on the device once for eager calls and once for the graph that is captured now, or was last.  Holds no tensors.

    A graph is replayed where and when its owner likes, so its calls have a list and scratch of their own, in memory of the graph's pool, and
    the graph brings the list there whenever it runs: what other calls and other graphs use, it neither reads nor writes."""

    def __init__(self, count: int, device: torch.device):
        self.L = binding.load()
        if device.type != "cuda":
            raise ValueError(f"tensors must be on a GPU, got {device}")
        self.device = device if device.index is not None else torch.device("cuda", torch.cuda.current_device())
        self.count, self.index = count, self.device.index
        self.list = (binding.Tensor * max(1, count))()
        self.columns = np.frombuffer(self.list, dtype=_COLUMNS)[:count]
        self.columns["lr_scale"] = self.columns["decay_scale"] = 1.0
        self.version = 0               # of the columns; who changes them counts it up
        self.eager = self.graph = None

    def call(self, f, *args):
        """A call on the list, on its device's current stream."""
        if torch._C._cuda_getDevice() != self.index:
            with torch.cuda.device(self.device):
                return self.call(f, *args)
        # the current stream's number; asking for the stream itself makes an object, 2 us of the 7 that a call then takes the host
        raw = torch._C._cuda_getCurrentRawStream(self.index)
        if raw != 0 and torch.cuda.is_current_stream_capturing():              # the default stream is none that can be captured
            x = self.in_graph(raw)
        else:
            x = self.eager
            if x is None or x.version != self.version:
                x = self.put()
            elif raw != x.raw:
                self.to_stream(x)
        st = f(x.h, *args)
        if st != binding.FS_OK:
            self.fail(x, st)

    def first(self):
        with torch.cuda.device(self.device):
            self.put()

    def put(self):
        """Hands the list over for eager calls: the first time, or after it has changed."""
        x = self.eager
        if x is None:
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("a list has to be made, or used once, before a graph is captured")
            x = self.eager = self.make()
        else:
            if torch._C._cuda_getCurrentRawStream(self.index) != x.raw:
                self.to_stream(x)
            self.update(x)
        return x

    def in_graph(self, raw):
        x = self.graph
        if self.eager is None:
            raise RuntimeError("a list has to be made, or used once, before a graph is captured")
        before = None
        if x is not None and raw != x.raw:
            before = x.stream
            self.to_stream(x)
        if x is None or self.L.fs_tensors_ready(x.h) != binding.FS_OK:         # none yet, or of an earlier graph
            workspace = torch.empty(self.L.fs_tensors_bytes(self.count), dtype=torch.uint8, device=self.device)
            x = self.graph = self.make(workspace)
            return x
        if before is not None:
            x.stream.wait_stream(before)       # another stream of the same graph
            x.workspace.record_stream(x.stream)
        if x.version != self.version:
            self.update(x)
        return x

    def update(self, x):
        st = self.L.fs_tensors_update(x.h, self.list, self.count)
        if st != binding.FS_OK:
            self.fail(x, st)
        x.version = self.version

    def make(self, workspace=None):
        h = ctypes.c_void_p()
        stream = torch.cuda.current_stream(self.device)
        if workspace is None:
            _free_later(self.L)
            st = self.L.fs_tensors_create(self.list, self.count, stream.cuda_stream, ctypes.byref(h))
        else:
            st = self.L.fs_tensors_create_noalloc(self.list, self.count, stream.cuda_stream, workspace.data_ptr(), workspace.nbytes, ctypes.byref(h))
        if st != binding.FS_OK:
            raise binding.FsError(st, "fs_tensors_create failed")
        return _OnDevice(self.L, h, self.version, stream, workspace)

    def fail(self, x, st):
        raise binding.FsError(st, self.L.fs_tensors_error(x.h).decode())

    def to_stream(self, x):
        now = torch.cuda.current_stream(self.device)
        if x is self.eager:
            now.wait_stream(x.stream)          # the scratch is one: this stream's calls come after those of the stream before
        x.stream, x.raw = now, now.cuda_stream
        self.L.fs_tensors_set_stream(x.h, x.raw)

    def norm(self, norm):
        """Where a call's norm goes or comes from."""
        if norm is None:
            return torch.empty(1, dtype=torch.float32, device=self.device)
        _check("norm", 0, norm, None, self.device, [torch.float32])
        if norm.numel() != 1:
            raise ValueError("norm must have one element")
        return norm


def _lists(n: int, **lists):
    """Every argument as a list of n entries."""
    out = []
    for name, v in lists.items():
        v = [None] * n if v is None else list(v)
        if len(v) != n:
            raise ValueError(f"{name}: {len(v)} entries, expected {n}")
        out.append(v)
    return out


def _device_of(tensors, device=None) -> torch.device:
    some = next((t for t in tensors if isinstance(t, torch.Tensor)), None)
    return torch.device(device) if device is not None else some.device if some is not None else torch.device("cuda")


def _places(tensors):
    return [0 if t is None else t.data_ptr() for t in tensors]


def _aliases(tensors):
    """The same memory, which stays theirs whatever becomes of the tensors."""
    return [None if t is None else t.detach() for t in tensors]


_PLACE, _SIZE, _TYPE = torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.dtype.__get__


def _look_at_params(params):
    """What parameters could have other than those before them: the place; and at the same place (memory that was freed and taken again, another view
    of it) the size and the type."""
    return [*map(_PLACE, params), *map(_SIZE, params), *map(_TYPE, params)]


def _sizes(tensors):
    return [0 if t is None else t.numel() for t in tensors]


def _types(tensors):
    return [0 if t is None else _TYPES[t.dtype] for t in tensors]


class TensorList:
    """A list of gradients, and where their clipped values go (`outs`; without: in place).  Entries of `grads` may be None: they
    are left out.  The list is of the memory that the tensors have when it is made, and keeps it alive: a tensor that gets other memory later
    (`.grad` made anew, `.data` replaced) needs another list."""

    def __init__(self, grads: Sequence[Optional[torch.Tensor]], outs: Optional[Sequence[Optional[torch.Tensor]]] = None, device=None):
        grads = list(grads)
        (outs,) = _lists(len(grads), outs=outs)
        h = self._handle = _Handle(len(grads), _device_of(grads, device))
        for i, g in enumerate(grads):
            if g is not None:
                _check("grads", i, g, None, h.device, _TYPES)
        for i, (g, o) in enumerate(zip(grads, outs)):
            if g is not None and o is not None:
                _check("outs", i, o, g, h.device, [g.dtype])
        grads, outs = _aliases(grads), _aliases([None if g is None else o for g, o in zip(grads, outs)])
        _check_apart(grads + [o for o, g in zip(outs, grads) if o is not None and o.data_ptr() != g.data_ptr()])
        self._grads, self._written = grads, [o if o is not None else g for o, g in zip(outs, grads) if g is not None]
        c = h.columns
        c["grad"], c["out"], c["n"], c["grad_type"] = _places(grads), _places(outs), _sizes(grads), _types(grads)
        h.first()

    def grad_norm(self, kind: str = "l2", grad_scale: float = 1.0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Global norm of the gradients times grad_scale, float32 [1]: "l2", or "max", the largest magnitude."""
        h = self._handle
        out = h.norm(out)
        h.call(h.L.fs_grad_norm, _kind(kind), grad_scale, out.data_ptr())
        return out

    def clip_grads(self, max_norm: float, kind: str = "l2", grad_scale: float = 1.0, norm: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Gradients times grad_scale min(1, max_norm / (norm + 1e-6)).  Returns the norm; one that is given (of gradients that are
        spread over several GPUs, say) is taken as it is."""
        h = self._handle
        d = h.norm(norm)
        h.call(h.L.fs_grad_clip, _kind(kind), max_norm, grad_scale, norm is not None, d.data_ptr())
        torch.autograd.graph.increment_version(self._written)
        return d


class AdamW:
    """AdamW with decoupled weight decay over a list of parameters, one or two launches a step whatever their number.

      params       float32, bfloat16 or float16 tensors on one GPU
      grads        their gradients, by the memory that they have now; without: each parameter's .grad at the time of the step (None: the
                   parameter stays as it is)
      lr           a number, or a float32 tensor of one element on the GPU that is read at every step (a schedule under graph capture)
      max_norm     limit of the gradients' global 2-norm; None: no clipping
      grad_scale   factor on all gradients before anything else (the inverse of a loss scale)
      skip_nonfinite  a step whose norm (in 64 bits, where it is computed here) is NaN or infinite changes nothing but the norm, and is not counted
      masters      True: 16-bit parameters get float32 masters, which are what is updated; or a list (None: no master)
      lr_scales, decay_scales   factors per parameter on lr and weight_decay
      exp_avgs, exp_avg_sqs, step   state to go on from: float32 tensors like the parameters, and an int64 tensor of one element

    State: .step_count, and .masters, .exp_avgs, .exp_avg_sqs, by the memory that they have now (updated in place; other values come
    by load_state_dict())."""

    def __init__(self, params: Sequence[torch.Tensor], grads=None, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2,
                 max_norm: Optional[float] = None, grad_scale: float = 1.0, skip_nonfinite: bool = False, masters=None, lr_scales=None,
                 decay_scales=None, exp_avgs=None, exp_avg_sqs=None, step: Optional[torch.Tensor] = None):
        self.params = list(params)
        n = len(self.params)
        h = self._handle = _Handle(n, _device_of(self.params))
        self.lr, self.betas, self.eps, self.weight_decay = lr, betas, eps, weight_decay
        self.max_norm, self.grad_scale, self.skip_nonfinite = max_norm, grad_scale, skip_nonfinite
        for i, p in enumerate(self.params):
            _check("params", i, p, None, h.device, _TYPES)
        if masters is True:
            masters = [p.detach().to(torch.float32, memory_format=torch.preserve_format) if p.dtype != torch.float32 else None for p in self.params]
        zeros = lambda: [torch.zeros_like(p, dtype=torch.float32, memory_format=torch.preserve_format, requires_grad=False) for p in self.params]
        (masters,) = _lists(n, masters=masters or None)
        moments = _lists(n, exp_avgs=zeros() if exp_avgs is None else exp_avgs, exp_avg_sqs=zeros() if exp_avg_sqs is None else exp_avg_sqs)
        lr_scales, decay_scales = _lists(n, lr_scales=[1.0] * n if lr_scales is None else lr_scales, decay_scales=[1.0] * n if decay_scales is None else decay_scales)
        for name, v in (("masters", masters), ("exp_avgs", moments[0]), ("exp_avg_sqs", moments[1])):
            for i, (t, p) in enumerate(zip(v, self.params)):
                if t is not None or name != "masters":
                    _check(name, i, t, p, h.device, [torch.float32])
        # not the tensors themselves: whoever has them may give them other memory, and the list goes on with this
        self._masters, self._exp_avgs, self._exp_avg_sqs = _aliases(masters), _aliases(moments[0]), _aliases(moments[1])
        self.step_count = step if step is not None else torch.zeros(1, dtype=torch.int64, device=h.device)
        self._counter = None
        self._check_counter()
        self._given = None
        if grads is not None:
            (given,) = _lists(n, grads=grads)
            for i, (g, p) in enumerate(zip(given, self.params)):
                if g is not None:
                    _check("grads", i, g, p, h.device, _TYPES)
            self._given = _aliases(given)
        self._params_look = self._grads_look = self._orders = None
        self._how, self._set_to = binding.AdamW(), None
        self._how_at = ctypes.byref(self._how)
        c = h.columns
        c["master"], c["exp_avg"], c["exp_avg_sq"] = _places(self._masters), _places(self._exp_avgs), _places(self._exp_avg_sqs)
        c["lr_scale"], c["decay_scale"] = lr_scales, decay_scales
        _check_apart(self.params + self._masters + self._exp_avgs + self._exp_avg_sqs + (self._given or []))
        if self._given is not None:
            self._put(self._given, _look_at_params(self.params), None)
            h.first()

    masters = property(lambda self: _aliases(self._masters))
    exp_avgs = property(lambda self: _aliases(self._exp_avgs))
    exp_avg_sqs = property(lambda self: _aliases(self._exp_avg_sqs))

    def _check_counter(self):
        _check("step", 0, self.step_count, None, self._handle.device, [torch.int64])
        if self.step_count.numel() != 1:
            raise ValueError("step must have one element")
        self._counter = self.step_count

    def _put(self, grads, params_look, grads_look):
        h, c = self._handle, self._handle.columns
        _lists(h.count, params=self.params)
        # parameters may have another type or size now; or another order, and then their gradients have, too
        orders = [x and x[2] for x in grads_look] if grads_look is not None else None
        anew = params_look != self._params_look or orders != self._orders
        self._params_look = None
        for i, (g, p) in enumerate(zip(grads, self.params)):
            if anew:
                _check("params", i, p, None, h.device, _TYPES)
                _check("exp_avgs", i, self._exp_avgs[i], p, h.device, [torch.float32])
            if g is not None:
                _check("grads", i, g, p, h.device, _TYPES)
        c["grad"], c["n"], c["grad_type"] = _places(grads), _sizes(grads), _types(grads)
        if anew:
            c["param"], c["param_type"] = params_look[:h.count], _types(self.params)
            n, kind = c["n"], c["param_type"]
            written = [c["param"], *(c[name] for name in ("master", "exp_avg", "exp_avg_sq"))]
            self._written = _apart(np.concatenate(written), np.concatenate([n * _BYTES[kind]] + [n * (at > 0) * _BYTES[0] for at in written[1:]]))
        _untouched(c["grad"], c["n"] * _BYTES[c["grad_type"]], self._written)
        h.version += 1
        self._params_look, self._grads_look, self._orders = params_look, grads_look, orders

    def step(self, norm: Optional[torch.Tensor] = None) -> Optional[torch.Tensor]:
        """One step.  Returns the gradients' global norm, float32 [1] (None where neither max_norm nor skip_nonfinite asks for it); a
        `norm` that is given is taken as it is (one over several GPUs, say)."""
        h, how = self._handle, self._how
        params_look, grads, grads_look = _look_at_params(self.params), self._given, None
        if grads is None:
            # the same of gradients that are not held here; their shape is prescribed by the parameters
            grads = [p.grad for p in self.params]
            grads_look = [None if g is None else (g.data_ptr(), g.dtype, g.is_contiguous() or g.stride()) for g in grads]
        if params_look != self._params_look or grads_look != self._grads_look:
            self._put(grads, params_look, grads_look)
        asked = norm is not None or self.max_norm is not None or self.skip_nonfinite
        d = h.norm(norm) if asked else None
        lr = self.lr
        if isinstance(lr, torch.Tensor):
            _check("lr", 0, lr, None, h.device, [torch.float32])
            if lr.numel() != 1:
                raise ValueError("lr must have one element")
            how.d_lr, lr = lr.data_ptr(), 0.0
        else:
            how.d_lr = None
        set_to = (lr, *self.betas, self.eps, self.weight_decay, self.grad_scale, self.max_norm, self.skip_nonfinite, norm is not None)
        if set_to != self._set_to:
            self._set_to = None
            how.lr, (how.beta1, how.beta2) = lr, self.betas
            how.eps, how.weight_decay, how.grad_scale = self.eps, self.weight_decay, self.grad_scale
            how.max_norm = math.inf if self.max_norm is None else self.max_norm
            how.norm_given, how.skip_nonfinite = norm is not None, bool(self.skip_nonfinite)
            self._set_to = set_to
        if self.step_count is not self._counter:
            self._check_counter()
        h.call(h.L.fs_adamw_step, self._how_at, self.step_count.data_ptr(), d.data_ptr() if asked else None)
        torch._C._increment_version(self.params)                  # autograd has to notice that they have changed
        return d

    def zero_grad(self, set_to_none: bool = False):
        """Gradients to zero, in the memory that they have; or away with them (the next step then finds others)."""
        grads = [g for g in (self._given if self._given is not None else [p.grad for p in self.params]) if g is not None]
        if set_to_none and self._given is None:
            for p in self.params:
                p.grad = None
        elif grads:
            torch._foreach_zero_(grads)

    def state_dict(self):
        return {"step": self.step_count, "masters": self.masters, "exp_avgs": self.exp_avgs, "exp_avg_sqs": self.exp_avg_sqs}

    def load_state_dict(self, state):
        """Copies a state in; the parameters are the caller's to load."""
        new = [state["masters"], state["exp_avgs"], state["exp_avg_sqs"]]
        for name, mine, theirs in zip(("masters", "exp_avgs", "exp_avg_sqs"), (self._masters, self._exp_avgs, self._exp_avg_sqs), new):
            if len(theirs) != len(mine) or any((a is None) != (b is None) or (a is not None and a.shape != b.shape) for a, b in zip(mine, theirs)):
                raise ValueError(f"{name} do not fit")
        with torch.no_grad():
            for mine, theirs in zip((self._masters, self._exp_avgs, self._exp_avg_sqs), new):
                for a, b in zip(mine, theirs):
                    if a is not None:
                        a.copy_(b)
            self.step_count.copy_(state["step"])


def _kind(kind):
    if kind not in _KINDS:
        raise ValueError(f"kind must be one of {', '.join(_KINDS)}, got {kind!r}")
    return _KINDS[kind]
