"""The layers of the networks on either side of the search (the skinning network, the occupancy network), over the C ABI of
include/fastsnarf_net.h: matrix products with bias, activation, dropout and residual in one pass, and dropout alone, both with gradients.

    y = linear(x, weight, bias, activation="softplus", beta=100.0)                  # x [..., inputs], weight [outputs, inputs]
    y = linear(y, weight, bias, residual=y, activation="gelu", dropout=0.1, seed=words)
    y = dropout(y, 0.1, words)

    field = Network(3, 64, 2, n_bones, dropout=0.1)                                 # layers of them: the skinning network of fit.py
    logits = field(nodes, words)

Tensors are float32, bfloat16 or float16 on one GPU, all of one type but the bias, which may be float32.  Dropout draws its numbers from a counter:
`seed` is a pair of integers (seed, offset), or an int64 tensor of those two words on the GPU, which is read when the kernels run (a captured graph that
counts the offset up drops other elements at each replay).  The same words drop the same elements, so every call of a step gets an offset of its own.
The mask is not stored: the backward pass makes it anew.

Calls run on the stream that is current when they are made, wait for nothing, keep nothing but what autograd saves, and can be captured into graphs of torch.cuda.
A captured backward pass needs its forward pass in the same capture, and no eager graph of the same leaves alive.  Forward-mode derivatives, second derivatives of
linear() and traces are refused (torch.compile goes round the calls).  There is no CPU fallback."""
from __future__ import annotations

import ctypes
import functools
import math
from typing import Optional, Sequence, Tuple, Union

import torch
import torch.autograd.forward_ad as forward_ad

from . import binding

_TYPES = {torch.float32: binding.FS_FLOAT_FULL, torch.bfloat16: binding.FS_FLOAT_BRAIN, torch.float16: binding.FS_FLOAT_HALF}
_ACTS = {"none": binding.FS_ACT_NONE, "relu": binding.FS_ACT_RELU, "gelu": binding.FS_ACT_GELU, "silu": binding.FS_ACT_SILU, "softplus": binding.FS_ACT_SOFTPLUS}

Seed = Union[torch.Tensor, Tuple[int, int]]


def _check(what: str, t: torch.Tensor, like: torch.Tensor, types):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}: expected a tensor, got {type(t).__name__}")
    if t.dtype not in types:
        raise TypeError(f"{what}: {t.dtype} is not supported here, expected {' or '.join(str(k) for k in types)}")
    if t.device != like.device:
        raise ValueError(f"{what}: on {t.device}, expected {like.device}")
    if t.layout != torch.strided:
        raise ValueError(f"{what}: expected a dense tensor, got {t.layout}")


def _check_input(x):
    # The library writes through addresses: a trace would hold a result that nothing computes.
    # (torch.compile stops at those addresses, and has the call made.)
    if not torch.compiler.is_compiling() and (torch._C._is_tracing() or torch._C._dispatch_tls_is_dispatch_key_included(torch._C.DispatchKey.PreDispatch) or
                                              torch._C._len_torch_dispatch_stack() and torch._C._get_dispatch_mode(torch._C._TorchDispatchModeKey.PROXY) is not None):
        raise RuntimeError("layers cannot be traced (torch.jit.trace, make_fx, torch.export): their calls leave no operations behind")
    if not isinstance(x, torch.Tensor):
        raise TypeError(f"x: expected a tensor, got {type(x).__name__}")
    if x.dtype not in _TYPES:
        raise TypeError(f"x: {x.dtype} is not supported here, expected {' or '.join(str(k) for k in _TYPES)}")
    if not x.is_cuda:
        raise ValueError(f"tensors must be on a GPU, got {x.device}")
    if x.layout != torch.strided:
        raise ValueError(f"x: expected a dense tensor, got {x.layout}")


def _check_tangents(*tensors):
    """Those of forward mode would be lost in a call."""
    if any(t is not None and forward_ad.unpack_dual(t).tangent is not None for t in tensors):
        raise NotImplementedError("layers have no forward-mode derivatives (jvp)")


def _check_p(what, p):
    if not 0.0 <= p <= 1.0:
        raise ValueError(f"{what} must be in 0 .. 1, got {p}")


def _check_seed(seed, x):
    if isinstance(seed, torch.Tensor):
        _check("seed", seed, x, (torch.int64,))
        if seed.shape != (2,) or not seed.is_contiguous():
            raise ValueError("seed must hold two words, one after another")
        if seed.requires_grad:
            raise ValueError("seed cannot require a gradient")
    elif not (isinstance(seed, Sequence) and len(seed) == 2 and all(isinstance(v, int) and 0 <= v < 2 ** 64 for v in seed)):
        raise ValueError("dropout needs a seed: two integers in 0 .. 2^64 - 1, or an int64 tensor of two words on the GPU")


def _rows(t: torch.Tensor) -> torch.Tensor:
    """[rows, columns] with a row's elements one after another: a view where the strides allow one, else a copy."""
    if t.is_neg():                     # its sign stands beside the tensor: the imaginary part of a conjugate
        t = t.resolve_neg()
    if t.dim() != 2:
        t = t.reshape(1, -1) if t.dim() < 2 else t.reshape(math.prod(t.shape[:-1]), t.shape[-1])
    return t if t.stride(1) == 1 or t.shape[1] <= 1 else t.contiguous()


def _drop(p, seed) -> binding.Drop:
    if p == 0.0:
        return binding.Drop()
    if isinstance(seed, torch.Tensor):
        return binding.Drop(p, 0, 0, seed.data_ptr())
    return binding.Drop(p, seed[0], seed[1], None)


def _call(index, f, *args):
    """A call on a device's current stream."""
    if torch._C._cuda_getDevice() != index:
        with torch.cuda.device(index):
            return _call(index, f, *args)
    st = f(*args, torch._C._cuda_getCurrentRawStream(index))
    if st != binding.FS_OK:
        raise binding.FsError(st, binding.load().fs_net_error().decode())


# Activations whose slope changes with Z.  Up to _Z_FULL values Z is kept in float32 for them: few values do not average out what 16 bits round off, and the
# bytes, 8 MB more at most, are few beside the calls themselves.
_BENT = (binding.FS_ACT_GELU, binding.FS_ACT_SILU, binding.FS_ACT_SOFTPLUS)
_Z_FULL = 1 << 22
# float16 keeps Z within +-65504.  The slope of softplus is 0 or 1 there (to e^-32) from this beta on; below it Z is kept in float32 too, whatever its size.
_FLAT = 2.0 ** -11


class _Plan:
    """What calls of the same sizes share: the layer as the library takes it, without a seed, and the bytes that its calls work in."""

    def __init__(self, index, rows, inputs, outputs, kind, bias_kind, act, beta, p):
        L = binding.load()
        flat = kind == binding.FS_FLOAT_HALF and act == binding.FS_ACT_SOFTPLUS and beta < _FLAT
        keep = binding.FS_Z_FULL if act in _BENT and bias_kind != binding.FS_FLOAT_FULL and (rows * outputs <= _Z_FULL or flat) else 0
        self.z_full = bool(keep)
        self.index, self.bare = index, binding.Linear(rows, inputs, outputs, kind, bias_kind, act | keep, beta, binding.Drop(p, 0, 0, None))
        self.at = ctypes.byref(self.bare)
        self.forward, self.backward = L.fs_linear_forward, L.fs_linear_backward
        with torch.cuda.device(index):
            self.bytes = L.fs_linear_bytes(self.at, 0), L.fs_linear_bytes(self.at, 1)
        if min(self.bytes) < 0:
            raise binding.FsError(binding.FS_E_SHAPE, L.fs_net_error().decode())

    def layer(self, seed):
        if seed is None:
            return self.at
        b = self.bare
        return ctypes.byref(binding.Linear(b.rows, b.inputs, b.outputs, b.type, b.bias_type, b.act, b.beta, _drop(b.drop.p, seed)))


_plan = functools.lru_cache(maxsize=1024)(_Plan)


def _forward(plan, shape, x, weight, bias, residual, keep_z, seed):
    """Y (of `shape`: no view, so that a program may change it in place), and Z where it is kept."""
    x, w = _rows(x), _rows(weight)
    r = None if residual is None else _rows(residual)
    y = x.new_empty(shape)
    z = x.new_empty(shape, dtype=torch.float32 if plan.z_full else x.dtype if bias is None else bias.dtype) if keep_z else None
    n, outputs = plan.bytes[0], w.shape[0]
    work = x.new_empty(n, dtype=torch.uint8) if n else None
    b = None if bias is None else bias.resolve_neg().contiguous()
    _call(plan.index, plan.forward, plan.layer(seed), x.data_ptr(), x.stride(0), w.data_ptr(), w.stride(0), None if b is None else b.data_ptr(),
          None if r is None else r.data_ptr(), 0 if r is None else r.stride(0), y.data_ptr(), outputs, None if z is None else z.data_ptr(), outputs,
          None if work is None else work.data_ptr(), n)
    return y, z


class _Last(torch.autograd.Function):
    """Gradients that have none themselves.  Who differentiates them is told so; PyTorch would take them for constants, although they depend on y's gradient `g` and, by way of
    the layer's `mark`, on its inputs."""

    @staticmethod
    def forward(ctx, mark, g, *grads):
        return tuple(None if g is None else g.view_as(g) for g in grads)

    @staticmethod
    def backward(ctx, *_):
        raise RuntimeError("layers have no second derivatives")


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, residual, plan, shape, seed):
        need_x, need_w, need_b = ctx.needs_input_grad[:3]
        own = need_x or need_w or need_b               # the residual's gradient is y's
        y, z = _forward(plan, shape, x, weight, bias, residual, own and plan.bare.act != binding.FS_ACT_NONE, seed)
        words = seed if isinstance(seed, torch.Tensor) else None
        ctx.plan, ctx.seed, ctx.shape, ctx.bias_type = plan, None if words is not None else seed, x.shape, None if bias is None else bias.dtype
        mark = torch.empty(0) if own else None         # a second result, of nothing: what _Last knows the layer by
        ctx.save_for_backward(x if need_w else None, weight if need_x else None, z, words if own else None, mark)
        ctx.set_materialize_grads(False)
        return y, mark

    @staticmethod
    def backward(ctx, g, _):
        if g is None:
            return (None,) * 7
        need_x, need_w, need_b, need_r = ctx.needs_input_grad[:4]
        dx = dw = db = None
        if need_x or need_w or need_b:
            x, weight, z, words, mark = ctx.saved_tensors
            plan = ctx.plan
            G, w, X = _rows(g), None if weight is None else _rows(weight), None if x is None else _rows(x)
            outputs, inputs = plan.bare.outputs, plan.bare.inputs
            dx = g.new_empty(ctx.shape) if need_x else None
            dw = g.new_empty((outputs, inputs)) if need_w else None
            db = g.new_empty(outputs, dtype=ctx.bias_type) if need_b else None
            n = plan.bytes[1]
            work = g.new_empty(n, dtype=torch.uint8) if n else None
            _call(plan.index, plan.backward, plan.layer(ctx.seed if words is None else words), G.data_ptr(), G.stride(0), None if X is None else X.data_ptr(),
                  0 if X is None else X.stride(0), None if w is None else w.data_ptr(), 0 if w is None else w.stride(0), None if z is None else z.data_ptr(), outputs, None if dx is None else dx.data_ptr(), inputs,
                  None if dw is None else dw.data_ptr(), inputs, None if db is None else db.data_ptr(), None if work is None else work.data_ptr(), n)
            if torch.is_grad_enabled():                # create_graph
                dx, dw, db = _Last.apply(mark, g, dx, dw, db)
        return dx, dw, db, g if need_r else None, None, None, None


def linear(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, activation: str = "none",
           beta: float = 1.0, dropout: float = 0.0, seed: Optional[Seed] = None) -> torch.Tensor:
    """residual + drop(act(x weight^T + bias)), [..., outputs], with gradients for x, weight, bias and residual.

      x            [..., inputs], of any strides (rows whose elements do not lie one after another are copied)
      weight       [outputs, inputs];  bias [outputs], float32 or of the tensors' type;  residual [..., outputs]
      activation   "none", "relu", "gelu", "silu", or "softplus": ln(1 + e^(beta z)) / beta
      dropout      the chance of an activation to be dropped (those that are kept are divided by 1 - dropout), of the numbers that `seed` gives"""
    _check_input(x)
    kind, device, shape = x.dtype, x.device, x.shape
    if not shape:
        raise ValueError("x needs a dimension")
    _check("weight", weight, x, (kind,))
    if weight.dim() != 2 or weight.shape[1] != shape[-1]:
        raise ValueError(f"weight: shape {tuple(weight.shape)}, expected [outputs, {shape[-1]}]")
    outputs = weight.shape[0]
    bias_kind, y_shape = kind, (*shape[:-1], outputs)
    if bias is not None:
        _check("bias", bias, x, (kind, torch.float32))
        if bias.shape != (outputs,):
            raise ValueError(f"bias: shape {tuple(bias.shape)}, expected ({outputs},)")
        bias_kind = bias.dtype
    if residual is not None:
        _check("residual", residual, x, (kind,))
        if residual.shape != y_shape:
            raise ValueError(f"residual: shape {tuple(residual.shape)}, expected {y_shape}")
    act = _ACTS.get(activation)
    if act is None:
        raise ValueError(f"activation must be one of {', '.join(_ACTS)}, got {activation!r}")
    if act != binding.FS_ACT_SOFTPLUS:
        beta = 1.0
    elif not (beta > 0.0 and math.isfinite(beta)):
        raise ValueError(f"beta must be positive and finite, got {beta}")
    _check_p("dropout", dropout)
    if dropout > 0.0:
        _check_seed(seed, x)
    else:
        seed = None
    plan = _plan(device.index, math.prod(shape[:-1]), shape[-1], outputs, _TYPES[kind], _TYPES[bias_kind], act, float(beta), float(dropout))
    if forward_ad._current_level >= 0:
        _check_tangents(x, weight, bias, residual)
    if torch.is_grad_enabled() and (x.requires_grad or weight.requires_grad or bias is not None and bias.requires_grad or residual is not None and residual.requires_grad):
        return _Linear.apply(x, weight, bias, residual, plan, y_shape, seed)[0]
    return _forward(plan, y_shape, x, weight, bias, residual, False, seed)[0]


def _dropped(x, residual, p, seed):
    y, drop = x.new_empty(x.shape), _drop(p, seed)
    x, r = _rows(x), None if residual is None else _rows(residual)
    rows, columns = x.shape
    _call(x.device.index, binding.load().fs_dropout, _TYPES[x.dtype], rows, columns, ctypes.byref(drop), x.data_ptr(), x.stride(0), None if r is None else r.data_ptr(),
          0 if r is None else r.stride(0), y.data_ptr(), columns)
    return y


class _Dropout(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, p, seed):
        ctx.how = p, None if isinstance(seed, torch.Tensor) else seed
        ctx.save_for_backward(seed if isinstance(seed, torch.Tensor) and ctx.needs_input_grad[0] else None)
        ctx.set_materialize_grads(False)
        return _dropped(x, residual, p, seed)

    @staticmethod
    def backward(ctx, g):
        if g is None:
            return None, None, None, None
        (words,) = ctx.saved_tensors
        p, seed = ctx.how
        seed = seed if words is None else words
        dx = None
        if ctx.needs_input_grad[0]:                    # dropout again, and differentiated as that where gradients of gradients are asked for
            dx = _Dropout.apply(g, None, p, seed) if torch.is_grad_enabled() and g.requires_grad else _dropped(g, None, p, seed)
        return dx, g if ctx.needs_input_grad[1] else None, None, None


def dropout(x: torch.Tensor, p: float, seed: Optional[Seed] = None, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """residual + drop(x), with gradients for both: elements of x are dropped with a chance of p, those that are kept divided by 1 - p.  Which
    ones goes by their place in the tensor's order and by `seed`: linear(..., dropout=p, seed=seed) drops the same."""
    _check_input(x)
    _check_p("p", p)
    if p > 0.0:
        _check_seed(seed, x)
    else:
        seed = None
    if residual is not None:
        _check("residual", residual, x, (x.dtype,))
        if residual.shape != x.shape:
            raise ValueError(f"residual: shape {tuple(residual.shape)}, expected {tuple(x.shape)}")
    if forward_ad._current_level >= 0:
        _check_tangents(x, residual)
    if torch.is_grad_enabled() and (x.requires_grad or residual is not None and residual.requires_grad):
        return _Dropout.apply(x, residual, p, seed)
    return _dropped(x, residual, p, seed)


class Network:
    """Layers of linear(): `inputs` to `width`, `hidden` - 1 times `width` to `width` with the layer's input as residual, then `width` to `outputs` without an
    activation.  .params: weights and biases in turn, leaves that require gradients; the last weight starts at zero, so that the network does.

    network(x, words): x [..., inputs]; words: with dropout, where it is wanted, one row of two words (seed, offset) for every hidden layer (an int64
    tensor [hidden, 2] on the GPU); None: nothing is dropped."""

    def __init__(self, inputs: int, width: int, hidden: int, outputs: int, activation: str = "softplus", beta: float = 10.0, dropout: float = 0.0,
                 dtype: torch.dtype = torch.float32, device="cuda", seed: int = 0):
        if min(inputs, width, hidden, outputs) < 1:
            raise ValueError("a network needs a hidden layer or more, and sizes of 1 or more")
        if activation not in _ACTS:
            raise ValueError(f"activation must be one of {', '.join(_ACTS)}, got {activation!r}")
        _check_p("dropout", dropout)
        gen = torch.Generator().manual_seed(seed)
        self.hidden, self.how, self.dropout, self.params = hidden, dict(activation=activation, beta=beta), dropout, []
        sizes = [inputs] + [width] * hidden + [outputs]
        for i, (k, n) in enumerate(zip(sizes, sizes[1:])):
            w = torch.randn(n, k, generator=gen) * (math.sqrt(2.0 / k) if i < hidden else 0.0)
            self.params += [w.to(device, dtype).requires_grad_(True), torch.zeros(n, dtype=dtype, device=device, requires_grad=True)]

    def __call__(self, x: torch.Tensor, words: Optional[torch.Tensor] = None) -> torch.Tensor:
        if words is not None and self.dropout > 0.0 and tuple(words.shape) != (self.hidden, 2):
            raise ValueError(f"words: shape {tuple(words.shape)}, expected ({self.hidden}, 2)")
        p = 0.0 if words is None else self.dropout
        for i in range(self.hidden):
            x = linear(x, *self.params[2 * i:2 * i + 2], residual=x if i else None, dropout=p, seed=words[i] if p > 0.0 else None, **self.how)
        return linear(x, *self.params[-2:])
