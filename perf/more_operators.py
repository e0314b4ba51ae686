"""The layers of the networks around the weight grid (the skinning network before it, the occupancy network behind the search), as cases
that can be timed and compared.

A case is one pass through one operator whose tensors are resident on the GPU:

  linear   y = residual + drop(act(x w^T + b)), and where `train`, the gradients of x, w, b and the residual from the one of y
  dropout  y = residual + drop(x), and where `train`, the gradients of x and the residual

drop() keeps element e = row * columns + column where word e mod 4 of Philox4x32-10 with counter (e div 4, offset) and key `seed` is at least
round(p 2^32), and divides it by 1 - p.  `pad` > 0: rows are that many elements further apart than they are long (views into wider buffers).

`own` false computes the operators from their definitions with elementary torch operations in 32 bits; `own` true calls the framework.
"""
import math

import torch

own = False

DEV = "cuda:0"
F32, F64 = torch.float32, torch.float64
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LOW = 0xFFFFFFFF


def _linear(name, type, rows, inputs, outputs, act="none", beta=1.0, bias=True, bias32=False, residual=False, p=0.0, train=False, pad=0):
    return {"name": name, "call": "linear", "type": type, "rows": rows, "inputs": inputs, "outputs": outputs, "act": act, "beta": beta,
            "bias": bias, "bias32": bias32, "residual": residual, "p": p, "train": train, "pad": pad}


def _dropout(name, type, rows, columns, p, residual, train=True, pad=0):
    return {"name": name, "call": "dropout", "type": type, "rows": rows, "outputs": columns, "p": p, "residual": residual, "train": train, "pad": pad}


def listed():
    return [
        # a single row through a large layer, as in serving one query at a time: the weights are all there is to read
        _linear("linear_token", "bf16", 1, 4096, 16384, act="silu", bias=False),
        # a small batch of rows through a square layer with a residual
        _linear("linear_batch", "f16", 24, 4096, 4096, act="gelu", residual=True),
        # a hidden layer of an occupancy network, evaluated at the roots of a frame of 200 thousand points
        _linear("linear_roots", "f32", 200_003, 256, 256, act="softplus", beta=100.0),
        # nothing is a multiple of anything: sizes, and rows of views
        _linear("linear_odd", "f16", 1537, 1003, 777, act="gelu", residual=True, pad=5),
        # a wide layer of a large network, forward alone
        _linear("linear_wide", "bf16", 8192, 4096, 16384, act="gelu"),
        # the tiny configuration's nodes (16x16x4) through a narrow hidden layer: latency
        _linear("train_tiny", "f32", 16 * 16 * 4, 64, 64, act="softplus", beta=100.0, residual=True, train=True),
        # the training configuration's nodes (64x64x16) through a hidden layer of a skinning network
        _linear("train_nodes", "f32", 64 * 64 * 16, 128, 128, act="softplus", beta=100.0, train=True),
        # its last layer: the logits of 24 bones
        _linear("train_logits", "f32", 64 * 64 * 16, 128, 24, train=True),
        # the multi-pose configuration's nodes (128x128x32) in 16 bits, biases in 32
        _linear("train_grid", "bf16", 128 * 128 * 32, 256, 256, act="silu", bias32=True, residual=True, p=0.1, train=True),
        # a square layer of a large network
        _linear("train_large", "bf16", 8192, 4096, 4096, act="gelu", residual=True, p=0.1, train=True),
        # odd rows of views, short
        _dropout("dropout_odd", "f16", 1537, 777, 0.2, True, pad=5),
        # the activations of a large network
        _dropout("dropout_large", "bf16", 65536, 2048, 0.1, True),
    ]


def _spread(rng, low, high):
    return int(math.exp(rng.uniform(math.log(low), math.log(high + 0.999))))


def draw(rng):
    kind = rng.choice(["f32", "bf16", "f16"])
    train = rng.random() < 0.5
    rows, outputs = _spread(rng, 1, 524288), _spread(rng, 1, 16384)
    pad = rng.choice([0, 0, 0, 1, 5, 8])
    p = rng.choice([0.0, 0.0, 0.1, 0.25, 0.5])
    if rng.random() < 0.25:
        rows = max(1, min(rows, 130_000_000 // outputs))
        c = _dropout("", kind, rows, outputs, p or 0.3, rng.random() < 0.5, train, pad)
    else:
        inputs = _spread(rng, 1, 16384)
        if rng.random() < 0.5:      # most layers' sizes are multiples of 8
            inputs, outputs = -(-inputs // 8) * 8, -(-outputs // 8) * 8
        most = min(1e12 / (6.0 if train else 2.0) / (inputs * outputs), 250e6 / (inputs + outputs))
        rows = max(1, min(rows, int(most)))
        act = rng.choice(["none", "relu", "gelu", "silu", "softplus"])
        c = _linear("", kind, rows, inputs, outputs, act, rng.choice([1.0, 100.0]) if act == "softplus" else 1.0, rng.random() < 0.8,
                    rng.random() < 0.3, rng.random() < 0.5, p if train else 0.0, train, pad)
    del c["name"]
    return c


# ------------------------------------------------------------------------------------------------ inputs

def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    kind, rows, n, pad = TYPES[case["type"]], case["rows"], case["outputs"], case["pad"]

    def matrix(m, width, scale):
        wide = torch.empty(m, width + pad, dtype=kind, device=DEV)
        view = wide[:, :width]
        view.copy_(torch.randn(m, width, generator=gen, device=DEV).mul_(scale))
        return view

    # numbers that a program counts up from step to step: a seed of its own per run, an offset per call
    words = torch.randint(0, 2 ** 62, (2,), generator=gen, device=DEV, dtype=torch.int64)
    s = {"case": case, "words": words, "residual": matrix(rows, n, 1.0) if case["residual"] else None}
    if case["call"] == "linear":
        k = case["inputs"]
        s["x"], s["weight"] = matrix(rows, k, 1.0), matrix(n, k, 1.0 / math.sqrt(k))
        s["bias"] = torch.randn(n, generator=gen, device=DEV).mul_(0.1).to(F32 if case["bias32"] else kind) if case["bias"] else None
    else:
        s["x"] = matrix(rows, n, 1.0)
    if case["train"]:
        s["grad"] = matrix(rows, n, 1.0)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if own and case["train"]:
        s["leaves"] = [s[k].requires_grad_(True) for k in ("x", "weight", "bias", "residual") if s.get(k) is not None]
    return s


# ------------------------------------------------------------------------------------------------ the pass

def _times(a, b):
    """The two halves (high, low) of the product of a 32-bit constant and 32-bit words that are held in 64 bits."""
    product = b * a
    return (product >> 32) & LOW, product & LOW


def _kept(s, rows, columns):
    """Which elements drop() keeps."""
    low, high = (s["words"] & LOW).unbind(0), (s["words"] >> 32 & LOW).unbind(0)
    count = rows * columns
    index = torch.arange(-(-count // 4), device=DEV)
    a, b, c, d = index & LOW, index >> 32, low[1].expand_as(index), high[1].expand_as(index)
    k0, k1 = low[0], high[0]
    for _ in range(10):
        (h0, l0), (h1, l1) = _times(0xD2511F53, a), _times(0xCD9E8D57, c)
        a, b, c, d = h1 ^ b ^ k0, l1, h0 ^ d ^ k1, l0
        k0, k1 = k0 + 0x9E3779B9 & LOW, k1 + 0xBB67AE85 & LOW
    t = int(math.floor(s["case"]["p"] * 2.0 ** 32 + 0.5))
    return (torch.stack([a, b, c, d], 1).flatten()[:count] >= t).view(rows, columns)


def _drop(v, kept, p):
    return v if kept is None else torch.where(kept, v * (1.0 / (1.0 - p)), 0.0)


def _act(z, act, beta):
    if act == "relu":
        return z.clamp(min=0.0)
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    if act == "softplus":
        return z.clamp(min=0.0) + torch.log1p(torch.exp(-(z * beta).abs())) / beta
    return z


def _slope(z, act, beta):
    if act == "relu":
        return (z > 0.0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) / math.sqrt(2.0 * math.pi)
    if act == "silu":
        sigmoid = 1.0 / (1.0 + torch.exp(-z))
        return sigmoid * (1.0 + z * (1.0 - sigmoid))
    return 1.0 / (1.0 + torch.exp(-z * beta))


def _own(s):
    from paper_2211_15601_amd import net
    case = s["case"]
    seed = s["words"] if case["p"] > 0.0 else None
    if case["call"] == "linear":
        y = net.linear(s["x"], s["weight"], s["bias"], residual=s["residual"], activation=case["act"], beta=case["beta"], dropout=case["p"], seed=seed)
        names = [k for k in ("x", "weight", "bias", "residual") if s[k] is not None]
    else:
        y = net.dropout(s["x"], case["p"], seed, residual=s["residual"])
        names = [k for k in ("x", "residual") if s[k] is not None]
    if not case["train"]:
        return {"y": y}
    grads = torch.autograd.grad(y, s["leaves"], s["grad"])
    return {"y": y.detach()} | {"d" + k: g for k, g in zip(names, grads)}


def run(s):
    if own:
        return _own(s)
    case, kind, p = s["case"], TYPES[s["case"]["type"]], s["case"]["p"]
    kept = _kept(s, case["rows"], case["outputs"]) if p > 0.0 else None
    x = s["x"].float()
    if case["call"] == "linear":
        w = s["weight"].float()
        z = x @ w.t()
        if s["bias"] is not None:
            z = z + s["bias"].float()
        y = _drop(_act(z, case["act"], case["beta"]), kept, p)
    else:
        y = _drop(x, kept, p)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    out = {"y": y.to(kind)}
    if not case["train"]:
        return out
    g = _drop(s["grad"].float(), kept, p)
    if s["residual"] is not None:
        out["dresidual"] = s["grad"]
    if case["call"] == "dropout":
        return out | {"dx": g.to(kind)}
    dz = g if case["act"] == "none" else g * _slope(z, case["act"], case["beta"])
    if s["bias"] is not None:
        out["dbias"] = dz.sum(0, dtype=F64).to(s["bias"].dtype)
    return out | {"dx": (dz @ w).to(kind), "dweight": (dz.t() @ x).to(kind)}


# ------------------------------------------------------------------------------------------------ in 64 bits

def _words(block, offset, key):
    """Philox4x32-10 of counters (block, offset), the products from 16-bit halves so that none passes 2^63."""
    def product(m, v):
        ml, mh, vl, vh = m & 0xFFFF, m >> 16, v & 0xFFFF, v >> 16
        middle = mh * vl + (ml * vl >> 16)
        cross = ml * vh + (middle & 0xFFFF)
        return mh * vh + (middle >> 16) + (cross >> 16), ((cross & 0xFFFF) << 16) + (ml * vl & 0xFFFF)

    ctr = [block & LOW, block >> 32, torch.full_like(block, offset & LOW), torch.full_like(block, offset >> 32)]
    for r in range(10):
        round_key = (key & LOW) + r * 0x9E3779B9 & LOW, (key >> 32) + r * 0xBB67AE85 & LOW
        p0, p1 = product(0xD2511F53, ctr[0]), product(0xCD9E8D57, ctr[2])
        ctr = [p1[0] ^ ctr[1] ^ round_key[0], p1[1], p0[0] ^ ctr[3] ^ round_key[1], p0[1]]
    return ctr


def exact(case, seed):
    """The definition in 64 bits."""
    s = _inputs(case, seed)
    wide = {k: v.to(F64) for k, v in s.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    rows, n = case["rows"], case["outputs"]
    factor = None
    if case["p"] > 0.0:
        key, offset = s["words"].tolist()
        words = _words(torch.arange((rows * n + 3) // 4, device=DEV), offset, key)
        word = torch.empty(4 * len(words[0]), dtype=torch.int64, device=DEV)
        for i, w in enumerate(words):
            word[i::4] = w
        least = round(case["p"] * 2 ** 32)
        factor = (word[:rows * n].reshape(rows, n) >= least).to(F64).div_(1.0 - case["p"])
        del words, word
    value, slope = wide["x"], None
    if case["call"] == "linear":
        z = torch.mm(wide["x"], wide["weight"].T.contiguous())
        if "bias" in wide:
            z += wide["bias"]
        act, zero = case["act"], torch.zeros((), dtype=F64, device=DEV)
        if act == "none":
            value, slope = z, torch.ones_like(z)
        elif act == "relu":
            value, slope = torch.maximum(z, zero), torch.heaviside(z, zero)
        elif act == "gelu":
            phi = 0.5 * torch.erfc(z * -(0.5 ** 0.5))
            value, slope = z * phi, phi + z * torch.exp(z.square() * -0.5) * (2.0 * math.pi) ** -0.5
        elif act == "silu":
            gate = torch.exp(-torch.logaddexp(zero, -z))
            value, slope = z * gate, gate + z * gate * torch.exp(-torch.logaddexp(zero, z))
        else:
            t = z * case["beta"]
            value, slope = torch.logaddexp(zero, t) / case["beta"], torch.exp(-torch.logaddexp(zero, -t))
        del z
    y = value if factor is None else value * factor
    if "residual" in wide:
        y = y + wide["residual"]
    out = {"y": y}
    if case["train"]:
        g = wide["grad"]
        if "residual" in wide:
            out["dresidual"] = g
        dz = g if factor is None else g * factor
        if case["call"] == "dropout":
            return out | {"dx": dz}
        dz = dz * slope
        if "bias" in wide:
            out["dbias"] = dz.sum(0)
        out["dx"], out["dweight"] = torch.mm(dz, wide["weight"]), torch.mm(dz.T.contiguous(), wide["x"])
    return out


def work(case):
    """Bytes: inputs (and the gradient of y) read once, outputs written once; the residual's gradient is the one of y.  Operations: the products;
    of dropout a multiplication and an addition."""
    size, m, n = (4 if case["type"] == "f32" else 2), case["rows"], case["outputs"]
    k, linear = case.get("inputs", n), case["call"] == "linear"
    values = m * k + m * n + (m * n if case["residual"] else 0)
    if case["train"]:
        values += m * n + m * k
    total, flops = 0, 2 * m * n * (2 if case["train"] else 1)
    if linear:
        values += n * k * (2 if case["train"] else 1)
        if case["bias"]:
            total += n * (4 if case["bias32"] else size) * (2 if case["train"] else 1)
        flops = 2 * m * n * k * (3 if case["train"] else 1)
    return {"bytes": total + values * size, "flops": flops}
