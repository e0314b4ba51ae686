"""The formulas of include/fastsnarf_train.h in 64 bits, and how far a computation in 32 bits may be from them.

A rounding to n bits of precision is off by at most half a step: U = 2^-24 of the value in float32, finfo.eps / 2 in the 16-bit types;
below the normal range, half the smallest subnormal.  The bounds count the roundings of each result to first order; SLACK covers the
products of two of them."""
import math

import torch

U = 2.0 ** -24
SLACK = 1.0 + 1e-3
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}
TINY = {t: torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2 for t in HALF}


def norm(grads, kind="l2", scale=1.0):
    """As a Python float."""
    flat = [g.double().reshape(-1) for g in grads if g is not None and g.numel()]
    if kind == "max":
        return max([float(f.abs().max()) for f in flat], default=0.0) * scale
    return math.sqrt(sum(float(f @ f) for f in flat)) * scale


def coef(norm, max_norm, scale=1.0):
    return scale * min(1.0, max_norm / (norm + 1e-6)) if max_norm is not None and not math.isinf(max_norm) else scale


def clip(g, c):
    """(g c, bound): the norm is rounded once, the coefficient once, the product once and the result, in 16 bits, once more."""
    want = g.double() * c
    roundings = 3 * U + (HALF[g.dtype] if g.dtype != torch.float32 else 0.0)
    return want, (want.abs() * roundings + TINY[g.dtype] + TINY[torch.float32]) * SLACK


def adamw(p, g, m, v, t, c, lr, betas, eps, decay, lr_scale=1.0, decay_scale=1.0, master=None):
    """One step from the state of the tensors given: {name: (value, bound)}; t is the number of this step, c the coefficient."""
    b1, b2 = betas
    dtype, master = p.dtype, p if master is None else master
    old, m0, v0 = master.double(), m.double(), v.double()
    x = g.double() * c
    low = TINY[torch.float32] * 4
    # x carries the roundings of norm, coefficient and product
    new_m = b1 * m0 + (1 - b1) * x
    off_m = U * (b1 * m0.abs() + (3 + 2) * (1 - b1) * x.abs() + new_m.abs()) + low
    new_v = b2 * v0 + (1 - b2) * x * x
    off_v = U * (b2 * v0 + (2 * 3 + 3) * (1 - b2) * x * x + new_v) + low
    l = lr * lr_scale
    step = l / -math.expm1(t * math.log(b1)) if b1 else l
    root = 1.0 / math.sqrt(-math.expm1(t * math.log(b2)) if b2 else 1.0)
    # the square root of v + off is at most off / (2 sqrt(v)) and at most sqrt(off) away
    r = new_v.sqrt()
    off_r = torch.minimum(off_v / (2 * r).clamp_min(1e-300), off_v.sqrt()) + U * r
    below = r * root + eps
    off_below = off_r * root + U * (r * root + eps + below)
    up = step * new_m / below
    # off_below against the smallest value that the denominator can have
    least = (below - off_below).clamp_min(eps * (1 - 4 * U) if eps else 1e-300)
    # lr, its scale, the bias correction and their products: 5; times m, divided: 2
    off_up = abs(step) * off_m / least + up.abs() * off_below / least * 1.0 + 7 * U * up.abs() + low
    fade = l * decay * decay_scale * old
    change = fade + up
    new_p = old - change
    off_p = off_up + 6 * U * fade.abs() + U * change.abs() + U * new_p.abs() + low
    out = {"exp_avg": (new_m, off_m * SLACK), "exp_avg_sq": (new_v, off_v * SLACK), "master": (new_p, off_p * SLACK)}
    more = HALF[dtype] * (new_p.abs() + off_p) + TINY[dtype] if dtype != torch.float32 else 0.0
    # beyond the type's range the rounding gives infinity
    stored = torch.where(new_p.abs() >= torch.finfo(dtype).max * (1 + HALF[dtype]), torch.copysign(torch.full_like(new_p, math.inf), new_p), new_p)
    return out | {"param": (stored, (off_p + more) * SLACK)}


def near(got, want, bound, what=""):
    got = got.detach().to(want.device).double()
    bad = ~((got == want) | ((got - want).abs() <= bound))
    if bad.any():
        i = int(torch.nonzero(bad.reshape(-1))[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} outside; [{i}] {got.reshape(-1)[i]} for {want.reshape(-1)[i]}, bound {bound.reshape(-1)[i]}")
