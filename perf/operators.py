"""What a training program does with the gradients that the backward pass leaves, as cases that can be timed and compared.

A case is one pass through one operator over a list of tensors that is resident on the GPU:

  norm   the global norm of all gradients (the 2-norm, or the largest magnitude)
  clip   that norm, and the gradients scaled down where it is above `max_norm`, into buffers of their own or in place
  adamw  a training step: the norm, the scaled gradients' moments, and the parameters' update with decoupled weight decay

The tensors of a case are views into one flat buffer per type, as data-parallel training keeps them: packed without gaps
(`align` 1: odd offsets follow from odd sizes), or each on a boundary of `align` elements as an allocator would place them.
The gaps hold zeros and stay zero.  Sizes: tensor i of a list gets a share of `elements` in proportion to (i + 1) ** -`skew`.

`own` false computes the operators from their definitions with elementary torch operations on the flat buffers; `own` true
calls the framework with the lists of tensors.
"""
import math

import torch

own = False

DEV = "cuda:0"
F32, F64 = torch.float32, torch.float64
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
LR, BETA1, BETA2, EPS, DECAY = 1e-3, 0.9, 0.999, 1e-8, 0.01
NORM_EPS = 1e-6            # added to the norm that max_norm is divided by


def _case(name, call, types, tensors, elements, skew=0.0, align=64, kind="l2", clipped=True, inplace=False, masters=False,
          grads32=False, scale=1.0, step=1000):
    return {"name": name, "call": call, "types": types, "tensors": tensors, "elements": elements, "skew": skew, "align": align,
            "kind": kind, "clipped": clipped, "inplace": inplace, "masters": masters, "grads32": grads32, "scale": scale, "step": step}


def listed():
    return [
        # the tiny configuration's weight grid (16x16x4 nodes, 24 bones) and its bone transforms: latency only
        _case("norm_tiny", "norm", "f32", 2, 16 * 16 * 4 * 24 + 24 * 12, skew=6.4),
        # a network of some hundred layers in 16 bits, its gradients packed into one bucket, all sizes odd
        _case("norm_bucket", "norm", "bf16", 300, 45_000_000, skew=0.8, align=1),
        # largest magnitude of half-precision gradients under a loss scale: the check for overflow of a scaled step
        _case("norm_peak", "norm", "f16", 37, 13_000_001, skew=0.5, align=1, kind="max", scale=1.0 / 1024),
        # the gradients of a large model on one GPU
        _case("norm_large", "norm", "f32", 64, 400_000_000, skew=0.3),
        # the training configuration's weight grid (64x64x16 nodes) and one pose's bones, a spike clipped
        _case("clip_grid", "clip", "f32", 2, 64 * 64 * 16 * 24 + 24 * 12, skew=12.4),
        # a network with 16-bit matrices and 32-bit vectors, packed
        _case("clip_bucket", "clip", "mixed", 120, 20_000_000, skew=0.9, align=1),
        # what most steps after the first are: the norm is below the limit and the gradients stay as they are
        _case("clip_calm", "clip", "bf16", 80, 80_000_000, skew=0.4, clipped=False, inplace=True),
        # a large model's 32-bit accumulated gradients
        _case("clip_large", "clip", "f32", 48, 250_000_000, skew=0.3),
        # first step of the tiny configuration: fresh moments
        _case("adamw_tiny", "adamw", "f32", 2, 16 * 16 * 4 * 24 + 24 * 12, skew=6.4, step=0),
        # the multi-pose configuration's weight grid (128x128x32 nodes) and the bones of 8 poses
        _case("adamw_grid", "adamw", "f32", 2, 128 * 128 * 32 * 24 + 8 * 24 * 12, skew=12.4),
        # 16-bit parameters with 32-bit masters, packed, all sizes odd
        _case("adamw_bucket", "adamw", "bf16", 200, 30_000_000, skew=0.8, align=1, masters=True),
        # a large model on one GPU, 16-bit matrices and 32-bit vectors
        _case("adamw_large", "adamw", "mixed", 96, 250_000_000, skew=0.3, masters=True),
    ]


def draw(rng):
    call = rng.choice(["norm", "clip", "adamw"])
    types = rng.choice(["f32", "f32", "bf16", "f16", "mixed"])
    most = {"norm": 400e6, "clip": 250e6, "adamw": 200e6}[call]
    elements = int(math.exp(rng.uniform(math.log(1000), math.log(most))))
    tensors = int(math.exp(rng.uniform(0, math.log(400))))
    clipped = rng.random() < 0.7
    half = types != "f32"
    return {"call": call, "types": types, "tensors": max(1, min(tensors, elements // 8)), "elements": elements,
            "skew": round(rng.uniform(0.0, 1.5), 2), "align": rng.choice([1, 1, 64]),
            "kind": "max" if call != "adamw" and rng.random() < 0.3 else "l2", "clipped": clipped,
            "inplace": call == "clip" and not clipped and rng.random() < 0.5,
            "masters": call == "adamw" and half and rng.random() < 0.6, "grads32": call == "adamw" and half and rng.random() < 0.3,
            "scale": rng.choice([1.0, 1.0 / 1024]) if types == "f16" else 1.0, "step": rng.choice([0, 7, 1000, 100000])}


# ------------------------------------------------------------------------------------------------ inputs

def _groups(case):
    """The lists of a case by type: [(type of the parameters, type of the gradients, sizes, places, length of the flat buffer)]."""
    n, total, a = case["tensors"], case["elements"], case["align"]
    share = [(i + 1.0) ** -case["skew"] for i in range(n)]
    f = total / sum(share)
    sizes = [total] if n == 1 else [max(1, int(x * f)) | (1 if a == 1 else 0) for x in share]
    kinds = [("bf16" if i % 4 else "f32") if case["types"] == "mixed" else case["types"] for i in range(n)]
    return [_group(kind, F32 if case["grads32"] else TYPES[kind], [x for x, k in zip(sizes, kinds) if k == kind], a) for kind in sorted(set(kinds))]


def _group(kind, grad_type, sizes, align):
    places = [0] + torch.tensor([-(-n // align) * align for n in sizes], dtype=torch.int64).cumsum(0).tolist()
    return TYPES[kind], grad_type, sizes, places[:-1], places[-1]


def _views(flat, group):
    return [flat[at:at + n] for n, at in zip(group[2], group[3])]


def _no_gaps(flat, group, align):
    """Zeros between the tensors."""
    if align == 1:
        return flat
    inside = torch.zeros(group[4] + 1, dtype=torch.int8, device=DEV)
    inside[torch.tensor(group[3], device=DEV)] += 1
    inside[torch.tensor([at + n for n, at in zip(group[2], group[3])], device=DEV)] -= 1
    return flat.mul_(inside.cumsum(0, dtype=torch.int8)[:-1])


def _flats(case, group, gen):
    """The flat buffers of one type."""
    n, a = group[4], case["align"]
    new = lambda make, **k: make(n, generator=gen, device=DEV, **k)  # noqa: E731
    # every tensor's gradients have a size of their own, over four decades, and half of them are zero (nodes that no root touched)
    size = 10.0 ** (-4.0 * torch.rand(len(group[2]), generator=gen, device=DEV))
    lengths = torch.tensor([q - p for p, q in zip(group[3], group[3][1:] + [n])], device=DEV)
    size = torch.repeat_interleave(size, lengths, output_size=n)
    grad = _no_gaps(new(torch.randn).mul_(size), group, a).mul_(new(torch.rand) < 0.5)
    f = {"grad": grad.div_(case["scale"]).to(group[1])}
    if case["call"] == "clip":
        f["out"] = f["grad"] if case["inplace"] else torch.zeros_like(f["grad"])
    if case["call"] == "adamw":
        p = _no_gaps(new(torch.randn).mul_(0.05), group, a)
        f["param"] = p.to(group[0])
        f["master"] = p if case["masters"] and group[0] != F32 else None
        fresh = case["step"] == 0
        f["m"] = torch.zeros(n, device=DEV) if fresh else _no_gaps(new(torch.randn).mul_(0.1).mul_(size), group, a)
        f["v"] = torch.zeros(n, device=DEV) if fresh else _no_gaps(new(torch.rand).mul_(0.9).add_(0.1).mul_(size).mul_(size), group, a)
    return f


def _inputs(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(int(seed))
    groups = _groups(case)
    flats = [_flats(case, g, gen) for g in groups]
    s = {k: [f[k] for f in flats] for k in flats[0]}
    # a limit that all but the smallest lists exceed, or one that such gradients never reach
    limit = (0.25 if case["kind"] == "l2" else 0.01) if case["clipped"] else 1e9
    return s | {"case": case, "groups": groups, "max_norm": limit, "step": torch.full((1,), case["step"], dtype=torch.int64, device=DEV)}


def prepare(case, seed):
    s = _inputs(case, seed)
    if own:
        from paper_2211_15601_amd import optim
        lists = lambda flats: [v for f, g in zip(flats, s["groups"]) for v in ([None] * len(g[2]) if f is None else _views(f, g))]  # noqa: E731
        if case["call"] == "adamw":
            s["handle"] = optim.AdamW(lists(s["param"]), grads=lists(s["grad"]), lr=LR, betas=(BETA1, BETA2), eps=EPS, weight_decay=DECAY,
                                      max_norm=s["max_norm"], grad_scale=case["scale"], masters=lists(s["master"]) if case["masters"] else None,
                                      exp_avgs=lists(s["m"]), exp_avg_sqs=lists(s["v"]), step=s["step"])
        else:
            s["handle"] = optim.TensorList(lists(s["grad"]), outs=lists(s["out"]) if case["call"] == "clip" and not case["inplace"] else None)
    return s


# ------------------------------------------------------------------------------------------------ the pass

def _norm(s):
    """The global norm as a 64-bit scalar; magnitudes are squared in 32 bits and added in 64."""
    if s["case"]["kind"] == "max":
        top = [g.float().abs().amax() for g in s["grad"]]
        return torch.stack(top).amax().double() * s["case"]["scale"]
    squares = [g.float().square().sum(dtype=F64) for g in s["grad"]]
    return torch.stack(squares).sum().sqrt() * s["case"]["scale"]


def _scaled(s, norm):
    """The clipped gradients in 32 bits."""
    coef = ((s["max_norm"] / (norm + NORM_EPS)).clamp(max=1.0) * s["case"]["scale"]).float()
    return [g.float() * coef for g in s["grad"]]


def _update(p, m, v, g, c1, c2):
    """The new parameters in 32 bits; moments are changed in place."""
    m.mul_(BETA1).add_(g * (1 - BETA1))
    v.mul_(BETA2).add_(g * g * (1 - BETA2))
    return p * (1 - LR * DECAY) - (m / c1) / ((v / c2).sqrt() + EPS) * LR


def _stored(p, new, master):
    """Keeps the new values, rounded to the parameters' type, and whole in the master where there is one."""
    p.copy_(new)
    return p if master is None else master.copy_(new)


def _answer(s, norm):
    case = s["case"]
    if case["call"] == "norm":
        return {"norm": norm}
    if case["call"] == "clip":
        return {"norm": norm, "out": s["out"]}
    return {"norm": norm, "param": s["param"], "master": [t for t in s["master"] if t is not None], "m": s["m"], "v": s["v"], "step": s["step"]}


def run(s):
    case = s["case"]
    if own:
        h = s["handle"]
        if case["call"] == "norm":
            norm = h.grad_norm(kind=case["kind"], grad_scale=case["scale"])
        elif case["call"] == "clip":
            norm = h.clip_grads(s["max_norm"], kind=case["kind"], grad_scale=case["scale"])
        else:
            norm = h.step()
        return _answer(s, norm)
    norm = _norm(s)
    if case["call"] == "clip":
        [o.copy_(g) for o, g in zip(s["out"], _scaled(s, norm))]
    if case["call"] == "adamw":
        s["step"] += 1
        t = s["step"].double()
        c1, c2 = (1 - BETA1 ** t).float(), (1 - BETA2 ** t).float()
        masters = s["master"]
        olds = [p.float() if w is None else w for p, w in zip(s["param"], masters)]
        news = [_update(p, m, v, g, c1, c2) for p, m, v, g in zip(olds, s["m"], s["v"], _scaled(s, norm))]
        [_stored(p, new, w) for p, new, w in zip(s["param"], news, masters)]
    return _answer(s, norm.float().reshape(1))


def exact(case, seed):
    """One pass in 64 bits, tensor by tensor of the definition: the answer that both sides approximate."""
    s = _inputs(case, seed)
    grads = [g.to(F64).mul_(case["scale"]) for g in s["grad"]]
    if case["kind"] == "max":
        norm = max(float(g.abs().max()) for g in grads)
    else:
        norm = math.sqrt(math.fsum(float(torch.dot(g, g)) for g in grads))
    shrink = 1.0 if norm + NORM_EPS <= s["max_norm"] else s["max_norm"] / (norm + NORM_EPS)
    out = {"norm": torch.tensor([norm], dtype=F64)}
    if case["call"] == "clip":
        out["out"] = [g.mul_(shrink) for g in grads]
    if case["call"] == "adamw":
        t = case["step"] + 1
        bias1, bias2 = -math.expm1(t * math.log(BETA1)), -math.expm1(t * math.log(BETA2))
        out |= {"param": [], "master": [], "m": [], "v": [], "step": torch.tensor([t])}
        for i, g in enumerate(grads):
            g.mul_(shrink)
            m = s["m"][i].to(F64)
            m += (g - m) * (1 - BETA1)
            v = s["v"][i].to(F64)
            v += (g.square_() - v) * (1 - BETA2)
            master = s["master"][i]
            p = (s["param"][i] if master is None else master).to(F64)
            p -= LR * DECAY * p
            p.addcdiv_(m, (v / bias2).sqrt_().add_(EPS), value=-LR / bias1)
            out["param"].append(p)
            out["m"].append(m)
            out["v"].append(v)
            if master is not None:
                out["master"].append(p)
    return out


def work(case):
    """Bytes: gradients, parameters (masters in their place) and moments read once; scaled gradients (none where nothing is
    to be scaled in place), parameters, masters and moments written once."""
    size = {F32: 4, torch.bfloat16: 2, torch.float16: 2}
    total = flops = 0
    for param, grad, sizes, _, _ in _groups(case):
        n = sum(sizes)
        total += n * size[grad] + 4
        flops += 2 * n
        if case["call"] == "clip" and not case["inplace"]:
            total += n * size[grad]
            flops += n
        if case["call"] == "adamw":
            own_master = case["masters"] and param != F32
            total += n * (16 + (8 + size[param] if own_master else 2 * size[param]))
            flops += 15 * n
    return {"bytes": total, "flops": flops}
