"""Gradient norm, clipping and the AdamW step over lists of tensors, against the formulas in 64 bits (train_ref.py)."""
import itertools
import math

import pytest
import torch

import train_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
# lengths around the unit of 2048 elements and the 4 and 8 elements of a load; zero and one
# (without the last ones the list is short enough for kernels of its own)
LENGTHS = [0, 1, 2, 3, 5, 7, 8, 9, 31, 255, 1023, 1024, 1025, 2047, 2048, 2049, 4093, 8192, 40961]


@pytest.fixture(scope="module")
def optim(gpu_lib):
    from paper_2211_15601_amd import optim
    return optim


def _values(gen, n, dtype, size=1.0):
    return (torch.randn(n, generator=gen) * size).to(dtype)


def _packed(tensors, dtype, lead=0):
    """(flat buffer on the GPU, views): one behind the other without gaps, with `lead` sentinel elements before and after all of them."""
    total = sum(t.numel() for t in tensors)
    flat = torch.full((total + 2 * lead,), 7.0, dtype=dtype, device=DEV)
    views, at = [], lead
    for t in tensors:
        views.append(flat[at:at + t.numel()])
        views[-1].copy_(t)
        at += t.numel()
    return flat, views


def _cpu(tensors):
    return [t.detach().cpu() for t in tensors]


# ---- norm ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["l2", "max"])
def test_norm_of_each_length(optim, dtype, kind):
    gen = torch.Generator().manual_seed(1)
    for n in LENGTHS:
        g = _values(gen, n, dtype)
        for lead in (0, 1, 3):
            _, (view,) = _packed([g], dtype, lead)
            got = float(optim.TensorList([view]).grad_norm(kind=kind, grad_scale=0.5))
            want = ref.norm([g], kind, 0.5)
            # squares and sums in 64 bits: one rounding, to float32
            assert abs(got - want) <= (0.0 if kind == "max" else want * ref.U * ref.SLACK), (n, lead, got, want)


@pytest.mark.parametrize("kind", ["l2", "max"])
def test_norm_of_a_mixed_list(optim, kind):
    gen = torch.Generator().manual_seed(2)
    grads = [_values(gen, n, TYPES[i % 3], 10.0 ** -(i % 5)) for i, n in enumerate(LENGTHS * 3)]
    on = [g.to(DEV) for g in grads]
    on.insert(4, None)
    lst = optim.TensorList(on)
    got = [float(lst.grad_norm(kind=kind)) for _ in range(3)]
    want = ref.norm(grads, kind)
    assert got[0] == got[1] == got[2]
    assert abs(got[0] - want) <= (0.0 if kind == "max" else want * ref.U * ref.SLACK)


@pytest.mark.parametrize("count", [63, 64, 65, 129, 4097, 9001])
def test_norm_of_many_tensors(optim, count):
    gen = torch.Generator().manual_seed(count)
    sizes = torch.randint(1, 40, (count,), generator=gen).tolist()
    sizes[count // 2] = 70001
    grads = [_values(gen, n, F32) for n in sizes]
    _, views = _packed(grads, F32)
    want = ref.norm(grads)
    assert abs(float(optim.TensorList(views).grad_norm()) - want) <= want * ref.U * ref.SLACK


def test_norm_of_nothing(optim):
    assert float(optim.TensorList([]).grad_norm()) == 0.0
    assert float(optim.TensorList([None, torch.empty(0, device=DEV)]).grad_norm(kind="max")) == 0.0


@pytest.mark.parametrize("value", [1e30, 3e38, 1e-30, 1e-44])
def test_norm_where_squares_leave_float32(optim, value):
    g = torch.full((4096,), value)
    want = ref.norm([g])
    if want > torch.finfo(F32).max:
        want = math.inf
    got = float(optim.TensorList([g.to(DEV)]).grad_norm())
    assert got == want or abs(got - want) <= want * ref.U * ref.SLACK + ref.TINY[F32]


@pytest.mark.parametrize("dtype", TYPES)
def test_norm_of_nan_and_infinity(optim, dtype):
    for n, at in ((1, 0), (2049, 2048), (5000, 17)):
        for bad, kind in itertools.product((math.inf, -math.inf, math.nan), ("l2", "max")):
            g = torch.ones(n, dtype=dtype)
            g[at] = bad
            got = float(optim.TensorList([torch.ones(3, device=DEV), g.to(DEV)]).grad_norm(kind=kind))
            assert math.isnan(got) if math.isnan(bad) else got == math.inf
    g = torch.tensor([math.inf, math.nan], dtype=dtype, device=DEV)
    assert math.isnan(float(optim.TensorList([g]).grad_norm(kind="max")))


# ---- clipping ----

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("lengths", [LENGTHS, LENGTHS[:-2]])
@pytest.mark.parametrize("kind,max_norm,scale", [("l2", 0.5, 1.0), ("max", 0.25, 1.0), ("l2", 3.0, 2.0 ** -7), ("l2", 1e9, 0.125), ("l2", 0.0, 1.0)])
def test_clip(optim, dtype, inplace, lengths, kind, max_norm, scale):
    gen = torch.Generator().manual_seed(3)
    grads = [_values(gen, n, dtype) for n in lengths]
    flat, views = _packed(grads, dtype, 5)
    flat_out, outs = _packed([torch.zeros(n) for n in lengths], dtype, 5)
    before = flat.clone()
    got_norm = float(optim.TensorList(views, outs=None if inplace else outs).clip_grads(max_norm, kind=kind, grad_scale=scale))
    norm = ref.norm(grads, kind, scale)
    assert abs(got_norm - norm) <= norm * ref.U * ref.SLACK
    c = ref.coef(norm, max_norm, scale)
    for n, g, out in zip(lengths, grads, views if inplace else outs):
        ref.near(out, *ref.clip(g, c), f"length {n}")
    written = flat if inplace else flat_out
    assert (written[:5] == 7).all() and (written[-5:] == 7).all()
    assert inplace or torch.equal(flat, before)


@pytest.mark.parametrize("dtype", TYPES)
def test_clip_below_the_limit_keeps_the_bits(optim, dtype):
    gen = torch.Generator().manual_seed(4)
    g = _values(gen, 5001, dtype).to(DEV)
    before = g.clone()
    optim.TensorList([g]).clip_grads(1e6)
    assert torch.equal(g, before)
    out = torch.zeros_like(g)
    optim.TensorList([g], outs=[out]).clip_grads(math.inf)
    assert torch.equal(out, before)


def test_clip_with_a_given_norm_and_of_bad_norms(optim):
    g = torch.linspace(-2, 2, 3001)
    on, norm = g.to(DEV), torch.tensor([8.0], device=DEV)
    out = torch.zeros_like(on)
    lst = optim.TensorList([on], outs=[out])
    assert lst.clip_grads(2.0, norm=norm) is norm and float(norm) == 8.0
    ref.near(out, *ref.clip(g, ref.coef(8.0, 2.0)))
    # NaN: everything NaN; infinity: finite gradients become 0, infinite ones NaN; no limit: as they are
    norm.fill_(math.nan)
    lst.clip_grads(2.0, norm=norm)
    assert out.isnan().all()
    on[7] = math.inf
    assert float(lst.clip_grads(2.0)) == math.inf
    assert out[7].isnan() and (out[:7] == 0).all() and (out[8:] == 0).all()
    lst.clip_grads(math.inf)
    assert torch.equal(out, on)


# ---- AdamW ----

def _adam_lists(gen, sizes, ptype, gtype, masters, fresh):
    p = [_values(gen, n, F32) for n in sizes]
    g = [_values(gen, n, gtype, 10.0 ** -(i % 4)) for i, n in enumerate(sizes)]
    for x in g:
        x[::3] = 0.0
    zeros = [torch.zeros(n) for n in sizes]
    m = zeros if fresh else [_values(gen, n, F32, 0.1) for n in sizes]
    v = zeros if fresh else [torch.rand(n, generator=gen) for n in sizes]
    return [x.to(ptype) for x in p], g, m, v, (p if masters else None)


@pytest.mark.parametrize("ptype", TYPES)
@pytest.mark.parametrize("gtype", TYPES)
@pytest.mark.parametrize("masters", [False, True])
@pytest.mark.parametrize("start,sizes", [(0, LENGTHS), (1000, LENGTHS), (0, LENGTHS[:-2])])
def test_adamw(optim, ptype, gtype, masters, start, sizes):
    gen = torch.Generator().manual_seed(5)
    p, g, m, v, w = _adam_lists(gen, sizes, ptype, gtype, masters, start == 0)
    lead = 3
    flats, on = {}, {}
    for name, tensors, dtype in (("p", p, ptype), ("g", g, gtype), ("m", m, F32), ("v", v, F32)) + ((("w", w, F32),) if masters else ()):
        flats[name], on[name] = _packed(tensors, dtype, lead)
    lr_scales = [1.0 if i % 3 else 0.5 for i in range(len(sizes))]
    decay_scales = [float(i % 2) for i in range(len(sizes))]
    how = dict(lr=3e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.1)
    opt = optim.AdamW(on["p"], grads=on["g"], max_norm=2.0, grad_scale=0.5, masters=on.get("w"), exp_avgs=on["m"], exp_avg_sqs=on["v"],
                      step=torch.tensor([start], device=DEV), lr_scales=lr_scales, decay_scales=decay_scales, **how)
    for t in range(start + 1, start + 4):
        before = {k: _cpu(x) for k, x in on.items()}
        norm = ref.norm(before["g"], "l2", 0.5)
        got = float(opt.step())
        assert abs(got - norm) <= norm * ref.U * ref.SLACK
        c = ref.coef(norm, 2.0, 0.5)
        for i, n in enumerate(sizes):
            want = ref.adamw(before["p"][i], before["g"][i], before["m"][i], before["v"][i], t, c, how["lr"], how["betas"], how["eps"],
                             how["weight_decay"], lr_scales[i], decay_scales[i], before["w"][i] if masters else None)
            for key, name in (("exp_avg", "m"), ("exp_avg_sq", "v"), ("param", "p")) + ((("master", "w"),) if masters else ()):
                ref.near(on[name][i], *want[key], f"{key}, length {n}, step {t}")
        assert int(opt.step_count) == t
    for name, flat in flats.items():
        assert (flat[:lead] == 7).all() and (flat[-lead:] == 7).all(), name


@pytest.mark.parametrize("betas,eps,start", [((0.0, 0.0), 1e-3, 0), ((0.0, 0.999), 1e-8, 5), ((0.9, 0.95), 0.0, 0), ((0.99, 0.9999), 1e-8, 10 ** 7)])
def test_adamw_betas_and_late_steps(optim, betas, eps, start):
    gen = torch.Generator().manual_seed(6)
    n = 3001
    p, g = _values(gen, n, F32), _values(gen, n, F32)
    on = [x.to(DEV) for x in (p, g, torch.zeros(n), torch.zeros(n))]
    opt = optim.AdamW([on[0]], grads=[on[1]], lr=1e-2, betas=betas, eps=eps, weight_decay=0.0, exp_avgs=[on[2]], exp_avg_sqs=[on[3]],
                      step=torch.tensor([start], device=DEV))
    assert opt.step() is None
    want = ref.adamw(p, g, torch.zeros(n), torch.zeros(n), start + 1, 1.0, 1e-2, betas, eps, 0.0)
    ref.near(on[2], *want["exp_avg"])
    ref.near(on[3], *want["exp_avg_sq"])
    ref.near(on[0], *want["param"])


def test_adamw_of_zero_gradients_only_decays(optim):
    p = torch.full((2500,), 2.0, device=DEV, requires_grad=True)
    p.grad = torch.zeros_like(p)
    opt = optim.AdamW([p], lr=0.5, weight_decay=0.5, max_norm=1.0)
    assert float(opt.step()) == 0.0
    assert (p == 1.5).all()


@pytest.mark.parametrize("more", [3, 100_000])
def test_adamw_skips_a_step_that_is_not_finite(optim, more):
    gen = torch.Generator().manual_seed(7)
    p = [_values(gen, n, BF16).to(DEV).requires_grad_(True) for n in (7, 5000, more)]
    opt = optim.AdamW(p, lr=0.1, skip_nonfinite=True, masters=True)
    for x in p:
        x.grad = torch.ones_like(x)
    opt.step()
    state = [t.clone() for t in p + opt.masters + opt.exp_avgs + opt.exp_avg_sqs]
    for bad in (math.nan, math.inf):
        p[1].grad[4999] = bad
        assert not math.isfinite(float(opt.step()))
        assert int(opt.step_count) == 1
        assert all(torch.equal(a, b) for a, b in zip(state, p + opt.masters + opt.exp_avgs + opt.exp_avg_sqs))
    p[1].grad[4999] = 1.0
    opt.step()
    assert int(opt.step_count) == 2 and not torch.equal(state[0], p[0])
    # without the flag the formula holds: NaN in one place of the gradients, no clipping
    opt2 = optim.AdamW(p, lr=0.1)
    p[1].grad[4999] = math.nan
    opt2.step()
    assert p[1][4999].isnan() and not p[1][:4999].isnan().any() and not p[0].isnan().any()


def test_adamw_reads_the_rate_and_the_norm_from_the_device(optim):
    gen = torch.Generator().manual_seed(8)
    p, g = _values(gen, 4099, F32), _values(gen, 4099, F32)
    rate, norm = torch.tensor([0.25], device=DEV), torch.tensor([16.0], device=DEV)
    on = p.to(DEV)
    opt = optim.AdamW([on], grads=[g.to(DEV)], lr=rate, weight_decay=0.01, max_norm=4.0)
    assert opt.step(norm=norm) is norm
    zero = torch.zeros(4099)
    ref.near(on, *ref.adamw(p, g, zero, zero, 1, ref.coef(16.0, 4.0), 0.25, (0.9, 0.999), 1e-8, 0.01)["param"])
    now = on.cpu()
    rate.fill_(0.0)
    opt.step(norm=norm)
    assert torch.equal(now, on.cpu())
    # settings that change between steps: a number in its place, then another, no limit
    opt.lr, opt.weight_decay = 1.0, 0.0
    opt.step(norm=norm)
    first = (on.cpu() - now).abs().max()
    opt.lr, opt.max_norm = 0.5, None
    now = on.cpu()
    assert opt.step() is None
    assert 0 < (on.cpu() - now).abs().max() < first


def test_parameters_without_gradients_and_gradients_that_move(optim):
    gen = torch.Generator().manual_seed(9)
    shapes = [(33, 7), (5,), (64, 3, 3, 3), (1,)]
    p = [torch.randn(s, generator=gen).to(DEV).requires_grad_(True) for s in shapes]
    p[2] = p[2].detach().to(memory_format=torch.channels_last).requires_grad_(True)
    opt = optim.AdamW(p, lr=0.1, weight_decay=0.0)
    opt.step()                                               # no gradients at all
    assert int(opt.step_count) == 1 and all((m == 0).all() for m in opt.exp_avgs)
    keep = []
    for t in range(2, 6):
        opt.zero_grad(set_to_none=True)
        keep.append(torch.empty(1000 * t, device=DEV))       # gradients will lie elsewhere
        before, state = _cpu(p), [(_cpu([m])[0], _cpu([v])[0]) for m, v in zip(opt.exp_avgs, opt.exp_avg_sqs)]
        used = [i for i in range(4) if (t + i) % 3]
        loss = sum((p[i] * (i + t)).square().sum() for i in used)
        versions = [x._version for x in p]
        loss.backward()
        opt.step()
        assert all(x._version > n for x, n in zip(p, versions))
        for i in range(4):
            if i not in used:
                assert torch.equal(p[i].detach().cpu(), before[i])
                continue
            want = ref.adamw(before[i], p[i].grad.cpu(), *state[i], t, 1.0, 0.1, (0.9, 0.999), 1e-8, 0.0)
            ref.near(p[i], *want["param"], f"tensor {i}, step {t}")


def test_parameters_that_change_their_type(optim):
    """As Module.bfloat16() does it, between two steps."""
    gen = torch.Generator().manual_seed(14)
    m = torch.nn.Linear(37, 53).to(DEV)
    opt = optim.AdamW(list(m.parameters()), lr=0.1)
    for dtype in (F32, BF16, BF16, F32):
        m.to(dtype)
        x = torch.randn(5, 37, generator=gen).to(DEV, dtype)
        for p in m.parameters():
            p.grad = None
        m(x).square().sum().backward()
        before = [(p.detach().cpu(), a.cpu(), b.cpu()) for p, a, b in zip(m.parameters(), opt.exp_avgs, opt.exp_avg_sqs)]
        t = int(opt.step_count) + 1
        opt.step()
        for p, (old, a, b) in zip(m.parameters(), before):
            ref.near(p, *ref.adamw(old, p.grad.cpu(), a, b, t, 1.0, 0.1, (0.9, 0.999), 1e-8, 0.01)["param"], f"{dtype}, step {t}")


def test_state_goes_on(optim):
    def make():
        p = torch.linspace(-1, 1, 999, device=DEV).to(BF16).requires_grad_(True)
        p.grad = torch.linspace(1, -2, 999, device=DEV).to(BF16)
        return p, optim.AdamW([p], lr=0.01, masters=True, max_norm=0.5)
    (a, x), (b, y) = make(), make()
    for _ in range(3):
        x.step()
    y.load_state_dict(x.state_dict())
    with torch.no_grad():
        b.copy_(a)
    x.step(), y.step()
    assert torch.equal(a, b) and torch.equal(x.masters[0], y.masters[0]) and int(y.step_count) == 4


def test_results_do_not_change_from_call_to_call(optim):
    gen = torch.Generator().manual_seed(10)
    g = [_values(gen, n, F32).to(DEV) for n in (3_000_017, 5, 70_001)]
    lst = optim.TensorList(g)
    assert len({float(lst.grad_norm()) for _ in range(5)}) == 1


def test_many_tensors_are_clipped_and_updated(optim):
    """More than a block keeps the places of, several to a chunk."""
    gen = torch.Generator().manual_seed(15)
    sizes = torch.randint(0, 60, (3000,), generator=gen).tolist()
    sizes[1500] = 400_003
    p, g, m, v, _ = _adam_lists(gen, sizes, F32, F32, False, False)
    on = {k: _packed(x, F32)[1] for k, x in (("p", p), ("g", g), ("m", m), ("v", v))}
    outs = _packed([torch.zeros(n) for n in sizes], F32)[1]
    optim.TensorList(on["g"], outs=outs).clip_grads(1.0)
    opt = optim.AdamW(on["p"], grads=on["g"], lr=0.01, max_norm=1.0, exp_avgs=on["m"], exp_avg_sqs=on["v"], step=torch.tensor([3], device=DEV))
    opt.step()
    c = ref.coef(ref.norm(g), 1.0)
    g, p, m, v = (torch.cat(x) for x in (g, p, m, v))
    ref.near(torch.cat(outs), *ref.clip(g, c))
    want = ref.adamw(p, g, m, v, 4, c, 0.01, (0.9, 0.999), 1e-8, 0.01)
    for key, name in (("exp_avg", "m"), ("exp_avg_sq", "v"), ("param", "p")):
        ref.near(torch.cat(on[name]), *want[key], key)


@pytest.mark.parametrize("dtype,total", [(BF16, 4_000_000), (F32, 9_000_000), (BF16, 30_000_000), (F32, 60_000_000), (F16, 130_000_000)])
def test_large_lists(optim, dtype, total):
    """Sizes that differ in what stays in the caches and in how chunks are dealt out; the reference on the GPU, in 64 bits."""
    gen = torch.Generator(device=DEV).manual_seed(total)
    sizes = [total // 2 + 1, total // 5, 12_345, 1, total // 7 + 3]
    new = lambda n, scale=1.0: torch.randn(n, generator=gen, device=DEV) * scale
    g = [(new(n) * 10.0 ** -i).to(dtype) for i, n in enumerate(sizes)]
    norm = ref.norm(g)
    c = ref.coef(norm, 0.1)
    outs = [torch.zeros_like(x) for x in g]
    lst = optim.TensorList(g, outs=outs)
    assert abs(float(lst.clip_grads(0.1)) - norm) <= norm * ref.U * ref.SLACK
    assert abs(float(lst.grad_norm()) - norm) <= norm * ref.U * ref.SLACK
    for x, y in zip(g, outs):
        ref.near(y, *ref.clip(x, c))
    del outs, lst, y
    p, m, v = [new(n).to(dtype) for n in sizes], [new(n, 0.1) for n in sizes], [new(n).square() for n in sizes]
    w = [x.float() + 0.01 for x in p] if dtype != F32 else None
    before = [[x.clone() for x in t] for t in (p, m, v)] + [[x.clone() for x in w] if w else None]
    opt = optim.AdamW(p, grads=g, lr=0.01, max_norm=0.1, masters=w, exp_avgs=m, exp_avg_sqs=v, step=torch.tensor([99], device=DEV))
    opt.step()
    for i in range(len(sizes)):
        want = ref.adamw(before[0][i], g[i], before[1][i], before[2][i], 100, c, 0.01, (0.9, 0.999), 1e-8, 0.01, master=before[3][i] if w else None)
        ref.near(p[i], *want["param"], "param")
        ref.near(m[i], *want["exp_avg"], "exp_avg")
        ref.near(v[i], *want["exp_avg_sq"], "exp_avg_sq")
        if w:
            ref.near(w[i], *want["master"], "master")


def test_a_long_norm_streams_its_beginning(optim):
    gen = torch.Generator(device=DEV).manual_seed(16)
    g = [torch.randn(n, generator=gen, device=DEV) for n in (150_000_001, 140_000_000, 3)]
    want = ref.norm(g)
    out = [torch.empty_like(x) for x in g]
    lst = optim.TensorList(g, outs=out)
    for got in (lst.grad_norm(), lst.clip_grads(want / 4)):
        assert abs(float(got) - want) <= want * ref.U * ref.SLACK
    assert float(lst.grad_norm(kind="max")) == ref.norm(g, "max")
    for x, y in zip(g, out):
        ref.near(y, *ref.clip(x, ref.coef(want, want / 4)))


# ---- more than 2^31 elements; streams; graphs ----

def test_more_elements_than_32_bits_count(optim):
    n = 2 ** 31 + 4099
    g = torch.zeros(n, dtype=BF16, device=DEV)
    places = [0, 2 ** 31 - 1, 2 ** 31, 2 ** 31 + 2048, n - 1]
    for i, at in enumerate(places):
        g[at] = 3.0 + i
    want = math.sqrt(sum((3.0 + i) ** 2 for i in range(5)))
    lst = optim.TensorList([g])
    assert abs(float(lst.clip_grads(want / 2)) - want) <= want * ref.U * ref.SLACK
    assert float(lst.grad_norm(kind="max")) == 3.5
    assert [float(g[at]) for at in places] == [1.5, 2.0, 2.5, 3.0, 3.5]
    p = torch.zeros(n, dtype=BF16, device=DEV)
    opt = optim.AdamW([p], grads=[g], lr=0.5, weight_decay=0.0)
    opt.step()
    # a first step goes by lr in the gradient's direction
    assert int(torch.count_nonzero(p)) == 5 and all(abs(float(p[at]) + 0.5) < 0.002 for at in places)
    assert all(float(opt.exp_avgs[0][at]) != 0 for at in places)


def test_calls_run_on_the_current_stream(optim):
    gen = torch.Generator().manual_seed(11)
    host = [_values(gen, n, F32) for n in (2_000_003, 77)]
    g = [torch.zeros(x.numel(), device=DEV) for x in host]
    lst = optim.TensorList(g)
    assert float(lst.grad_norm()) == 0.0
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for a, b in zip(g, host):
            a.copy_(b.pin_memory(), non_blocking=True)
            a.mul_(2.0)
        norm = lst.clip_grads(1e9)
    torch.cuda.current_stream().wait_stream(side)
    want = 2 * ref.norm(host)
    assert abs(float(norm) - want) <= want * ref.U * ref.SLACK
    assert abs(float(lst.grad_norm()) - want) <= want * ref.U * ref.SLACK


@pytest.mark.parametrize("sizes", [[70_001, 3, 2048], [5, 9001]])
def test_a_captured_step_is_replayed(optim, sizes):
    gen = torch.Generator().manual_seed(12)
    host = [_values(gen, n, BF16) for n in sizes]

    def make():
        p = [x.to(DEV) for x in host]
        return p, optim.AdamW(p, grads=[torch.zeros(n, dtype=BF16, device=DEV) for n in sizes], lr=torch.tensor([0.01], device=DEV), max_norm=0.5, masters=True)

    (p, opt), (q, eager) = make(), make()
    opt.step()                                              # the list is made before the capture
    eager.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = opt.step()
    assert int(opt.step_count) == 1
    for t in range(2, 7):
        for a, b in zip(opt._given, eager._given):
            new = _values(gen, a.numel(), BF16, 0.1 * t).to(DEV)
            a.copy_(new), b.copy_(new)
        opt.lr.fill_(0.01 / t), eager.lr.fill_(0.01 / t)
        graph.replay()
        want = eager.step()
        torch.cuda.synchronize()
        assert int(opt.step_count) == t == int(eager.step_count)
        assert float(norm) == float(want)
        for a, b in zip(p + opt.masters + opt.exp_avgs + opt.exp_avg_sqs, q + eager.masters + eager.exp_avgs + eager.exp_avg_sqs):
            assert torch.equal(a, b)


@pytest.mark.parametrize("n", [9001, 300_001])
def test_graphs_and_eager_steps_keep_apart(optim, n):
    """Gradients that lie elsewhere in the graph and outside of it: neither works on the other's."""
    p = torch.zeros(n, device=DEV, requires_grad=True)
    opt = optim.AdamW([p], lr=1.0, betas=(0.0, 0.0), eps=0.0, weight_decay=0.0)      # p goes by the gradient's sign
    outside = torch.ones(n, device=DEV)
    p.grad = outside
    opt.step()
    graph = torch.cuda.CUDAGraph()
    p.grad = None
    with torch.cuda.graph(graph):
        (p * -2.0).sum().backward()
        inside = p.grad
        opt.step()
    assert inside.data_ptr() != outside.data_ptr()
    torch.cuda.synchronize()
    assert (p == -1).all()
    p.grad = outside
    opt.step()                                              # before the graph has ever run
    assert (p == -2).all()
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert (p == -1 - k).all()
        opt.step(), opt.step()
        assert (p == -3 - k).all()
    moved = torch.full_like(outside, -1.0)
    p.grad = moved
    opt.step()
    assert (p == -4).all()
    graph.replay()
    torch.cuda.synchronize()
    assert (p == -3).all() and int(opt.step_count) == 13


def test_a_list_is_not_made_while_a_graph_is_captured(optim):
    g = torch.ones(100, device=DEV)
    x = torch.zeros(3, device=DEV)
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        x.add_(1.0)
        with pytest.raises(RuntimeError, match="before a graph is captured"):
            optim.TensorList([g])


def test_arrays_that_are_aligned_differently(optim):
    gen = torch.Generator().manual_seed(13)
    n = 50_003
    for short in (False, True):
        m = n if not short else 5003
        host = {"p": _values(gen, m, BF16), "g": _values(gen, m, F16), "m": _values(gen, m, F32, 0.1), "v": torch.rand(m, generator=gen), "w": _values(gen, m, F32)}
        on = {k: _packed([x], x.dtype, 1 + 2 * i)[1] for i, (k, x) in enumerate(host.items())}
        opt = optim.AdamW(on["p"], grads=on["g"], lr=0.01, max_norm=1.0, masters=on["w"], exp_avgs=on["m"], exp_avg_sqs=on["v"], step=torch.tensor([9], device=DEV))
        opt.step()
        c = ref.coef(ref.norm([host["g"]]), 1.0)
        want = ref.adamw(host["p"], host["g"], host["m"], host["v"], 10, c, 0.01, (0.9, 0.999), 1e-8, 0.01, master=host["w"])
        for key, name in (("exp_avg", "m"), ("exp_avg_sq", "v"), ("param", "p"), ("master", "w")):
            ref.near(on[name][0], *want[key], key)
        out = _packed([torch.zeros(m)], F16, 7)[1]
        optim.TensorList(on["g"], outs=out).clip_grads(1.0)
        ref.near(out[0], *ref.clip(host["g"], c))


# ---- refusals that need tensors on a GPU ----

def test_refusals(optim):
    g = torch.ones(8, 6, device=DEV)
    T = optim.TensorList
    for bad, error in ((g[:, ::2], ValueError), (g.expand(2, 8, 6), ValueError), (g.double(), TypeError), (g.cpu(), ValueError), (3.0, TypeError)):
        with pytest.raises(error, match=r"grads\[1\]"):
            T([torch.ones(3, device=DEV), bad])
    with pytest.raises(ValueError, match="overlap"):
        T([g, g[2:4]])
    with pytest.raises(ValueError, match="overlap"):
        T([g[:4]], outs=[g[2:6]])
    with pytest.raises(ValueError, match=r"outs\[0\]"):
        T([g], outs=[torch.empty(6, 8, device=DEV)])
    with pytest.raises(ValueError, match=r"outs\[0\]"):
        T([g], outs=[torch.empty(6, 8, device=DEV).t()])
    with pytest.raises(TypeError, match=r"outs\[0\]"):
        T([g], outs=[g.half()])
    with pytest.raises(ValueError, match="outs: 0 entries"):
        T([g], outs=[])
    lst = T([g])
    from paper_2211_15601_amd import binding
    for call in (lambda: lst.clip_grads(-1.0), lambda: lst.clip_grads(math.nan), lambda: lst.grad_norm(grad_scale=0.0), lambda: lst.grad_norm(grad_scale=math.inf)):
        with pytest.raises(binding.FsError, match="FS_E_ARG"):
            call()
    with pytest.raises(ValueError, match="kind"):
        lst.grad_norm(kind="l1")
    with pytest.raises(ValueError, match="one element"):
        lst.grad_norm(out=torch.zeros(2, device=DEV))
    with pytest.raises(TypeError, match="norm"):
        lst.clip_grads(1.0, norm=torch.zeros(1, device=DEV, dtype=torch.float64))
    p = torch.ones(8, 6, device=DEV)
    A = optim.AdamW
    with pytest.raises(ValueError, match=r"grads\[0\]"):
        A([p], grads=[g.t().contiguous().t()]).step()
    with pytest.raises(TypeError, match=r"exp_avgs\[0\]"):
        A([p], exp_avgs=[g.half()])
    with pytest.raises(TypeError, match=r"exp_avgs\[0\]"):
        A([p], exp_avgs=[None])
    with pytest.raises(ValueError, match="overlap"):
        A([p, p])
    with pytest.raises(ValueError, match="overlap"):
        A([p], grads=[p])
    with pytest.raises(TypeError, match="step"):
        A([p], step=torch.zeros(1, device=DEV))
    for how in (dict(lr=math.nan), dict(betas=(1.0, 0.9)), dict(betas=(0.9, -0.1)), dict(eps=-1.0), dict(max_norm=-1.0), dict(grad_scale=-2.0), dict(weight_decay=math.inf)):
        with pytest.raises(binding.FsError, match="FS_E_ARG"):
            A([p], grads=[g], **how).step()
    assert (p == 1).all() and (g == 1).all()
