"""The networks' layers in 64 bits on the CPU, with bounds of what fp32 sums and roundings to the type may change.

Bounds.  `half` is half a step of the type, relative to the value: eps / 2.  Sums of n products in fp32: each of up to n additions rounds by 2^-24 of a
partial sum that is at most S = sum |x w|; such roundings are as often up as down, so their sum stays within L sqrt(n) 2^-24 S but for one result in
exp(L^2 / 2) / 2, 4e13 for L = 8.  fp32 operands go in as three bf16 parts, six products each (n is 6 times as large), and what is left out is at most
2^-23 of each product, 2^-24 more for each operand's rest: 2^-22 S together."""
import math

import numpy as np
import torch

F64 = torch.float64
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ACTS = ["none", "relu", "gelu", "silu", "softplus"]


def philox(block, offset, seed):
    """Philox4x32-10 with the counter (block, offset), both 64 bits: four words for every entry of the array `block`."""
    m32 = np.uint64(0xFFFFFFFF)
    block = np.asarray(block, dtype=np.uint64)
    c = [block & m32, block >> np.uint64(32), np.full_like(block, offset & 0xFFFFFFFF), np.full_like(block, offset >> 32)]
    key = [seed & 0xFFFFFFFF, seed >> 32]
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> np.uint64(32)) ^ c[1] ^ np.uint64(key[0]), q & m32, (p >> np.uint64(32)) ^ c[3] ^ np.uint64(key[1]), p & m32]
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, axis=-1)


def factor(shape, p, seed, first=0):
    """0 where drop() drops and 1 / (1 - p) elsewhere, of elements from `first` on."""
    n = math.prod(shape)
    if p == 0.0 or n == 0:
        return torch.ones(shape, dtype=F64)
    b0 = first // 4
    words = philox(np.arange(b0, (first + n + 3) // 4, dtype=np.uint64), seed[1], seed[0]).reshape(-1)[first - 4 * b0:][:n]
    kept = torch.from_numpy(words >= math.floor(p * 2 ** 32 + 0.5))
    return (kept.to(F64) / (1.0 - p) if p < 1.0 else torch.zeros(n, dtype=F64)).reshape(shape)


def act(z, kind, beta):
    if kind == "relu":
        return z.clamp(min=0)
    if kind == "gelu":
        return z * 0.5 * torch.erfc(-z / math.sqrt(2.0))
    if kind == "silu":
        return z * torch.sigmoid(z)
    if kind == "softplus":
        return torch.logaddexp(torch.zeros_like(z), beta * z) / beta
    return z


def slope(z, kind, beta):
    if kind == "relu":
        return (z > 0).to(F64)
    if kind == "gelu":
        return 0.5 * torch.erfc(-z / math.sqrt(2.0)) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if kind == "silu":
        s = torch.sigmoid(z)
        return s + z * s * (1 - s)
    if kind == "softplus":
        return torch.sigmoid(beta * z)
    return torch.ones_like(z)


def bend(kind, beta):
    """The largest second derivative."""
    return {"none": 0.0, "relu": 0.0, "gelu": 0.8, "silu": 0.5, "softplus": beta / 4}[kind]


def half(dtype):
    return torch.finfo(dtype).eps / 2


def rounded(v, dtype):
    """How far rounding to the type may take a value (the least step of fp16 is that of its smallest numbers)."""
    return v.abs() * half(dtype) + (2.0 ** -25 if dtype == torch.float16 else 0.0)


def product(a, b, dtype):
    """a b^T in 64 bits, and the bound of what fp32 sums of it are off."""
    size = a.abs() @ b.abs().T
    n = a.shape[1] * (6 if dtype == torch.float32 else 1)
    return a @ b.T, size * (8 * math.sqrt(n + 1) * 2.0 ** -24 + (2.0 ** -22 if dtype == torch.float32 else 0.0))


def linear(x, w, b, r, g, kind, beta, p, seed):
    """{name: (value, bound)} of y, and with g of dx, dweight, dbias."""
    dtype = x.dtype
    wide = lambda t: None if t is None else t.detach().cpu().to(F64)
    X, W, B, R, G = wide(x), wide(w), wide(b), wide(r), wide(g)
    z, ez = product(X, W, dtype)
    if B is not None:
        z = z + B
        ez = ez + z.abs() * 2.0 ** -23
    f = factor(z.shape, p, seed)
    a = act(z, kind, beta)
    # functions in fp32 to some units of the last place; the argument of e^-z^2/2 is off by its own rounding times z^2
    ea = 1.2 * ez + (a.abs() * (16 + 4 * z * z) + (1.0 / beta if kind == "softplus" else 0.0)) * 2.0 ** -24
    y, ey = a * f, ea * f + (a * f).abs() * 2.0 ** -23
    if R is not None:
        y = y + R
        ey = ey + y.abs() * 2.0 ** -23
    out = {"y": (y, ey + rounded(y, dtype) * 1.01)}
    if G is None:
        return out
    s = slope(z, kind, beta)
    kept = rounded(z, dtype if B is None else b.dtype)
    es = bend(kind, beta) * (ez + kept) + 2.0 ** -20
    if kind == "relu":
        es = (z.abs() <= ez + 2.0 ** -25).to(F64)
    dz = G * s * f
    edz = (G * f).abs() * (es + 2.0 ** -22 * s.abs())
    if B is not None:
        size = dz.abs().sum(0)
        db = dz.sum(0)
        out["dbias"] = db, edz.sum(0) + 8 * math.sqrt(dz.shape[0] + 1) * 2.0 ** -24 * size + rounded(db, b.dtype) * 1.01
    if dtype != torch.float32 and (kind != "none" or p > 0.0):
        edz = edz + rounded(dz, dtype)
    for name, (u, v, eu) in {"dx": (dz, W.T, edz), "dweight": (dz.T, X.T, edz.T)}.items():
        d, ed = product(u, v.contiguous(), dtype)
        out[name] = d, ed + eu @ v.abs().T + rounded(d, dtype) * 1.01
    return out


def assert_close(name, got, want):
    value, bound = want
    got = got.detach().cpu().to(F64)
    assert got.shape == value.shape, (name, got.shape, value.shape)
    if got.numel() == 0:
        return
    off = (got - value).abs() / (bound + 1e-300)
    i = int(off.argmax())
    assert bool((off <= 1.0).all()), f"{name}: {int((~(off <= 1.0)).sum())} of {off.numel()} off, most {float(off.max()):.3g} of the bound at {i}: {float(got.flatten()[i])} for {float(value.flatten()[i])}"
