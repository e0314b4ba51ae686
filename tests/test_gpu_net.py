"""The networks' layers on the GPU against their definitions in 64 bits (net_ref.py)."""
import itertools
import math

import numpy as np
import pytest
import torch

import net_ref as ref

pytestmark = pytest.mark.gpu
F64 = torch.float64
SEED = (0x0123456789ABCDEF, 0xFEDCBA9876543210)
# rows, inputs, outputs: single ones, none, a tile and its neighbours, thin and wide, split ranges
SIZES = [(1, 1, 1), (0, 8, 8), (5, 0, 7), (3, 7, 0), (64, 64, 64), (65, 63, 66), (129, 65, 131), (3, 1000, 2), (1000, 24, 257), (257, 1000, 24),
         (2, 9, 700), (16, 2048, 40), (130, 3, 128), (1, 777, 1001), (4100, 20, 36), (31, 129, 33)]


@pytest.fixture(scope="module")
def net(gpu_lib):
    from paper_2211_15601_amd import net
    return net


def make(rows, inputs, outputs, dtype, seed=0, pad=0, whole=False):
    """x, weight, bias, residual, g on the GPU; rows `pad` elements further apart than they are long."""
    gen = torch.Generator().manual_seed(seed)

    def one(m, n, scale):
        v = torch.randint(-2, 3, (m, n), generator=gen).float() if whole else torch.randn(m, n, generator=gen) * scale
        wide = torch.full((m, n + pad), math.nan, dtype=dtype, device="cuda")
        wide[:, :n] = v.to(dtype)
        return wide[:, :n]

    return (one(rows, inputs, 1.0), one(outputs, inputs, 1.0 / math.sqrt(max(1, inputs))), one(1, outputs, 0.5)[0], one(rows, outputs, 1.0), one(rows, outputs, 1.0))


def run(net, x, w, b, r, g, kind, beta, p, seed):
    leaves = [t.detach().requires_grad_(True) if t is not None else None for t in (x, w, b, r)]
    y = net.linear(leaves[0], leaves[1], leaves[2], residual=leaves[3], activation=kind, beta=beta, dropout=p, seed=seed)
    wanted = [t for t in leaves if t is not None]
    grads = iter(torch.autograd.grad(y, wanted, g))
    out = {"y": y}
    for name, t in zip(("dx", "dweight", "dbias", "dresidual"), leaves):
        if t is not None:
            out[name] = next(grads)
    return out


def check(out, x, w, b, r, g, kind, beta, p, seed):
    want = ref.linear(x, w, b, r, g, kind, beta, p, seed)
    for name, v in want.items():
        ref.assert_close(name, out[name], v)
    if r is not None:
        assert torch.equal(out["dresidual"], g)


@pytest.mark.parametrize("dtype", list(ref.TYPES))
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_sizes(net, size, dtype):
    t = make(*size, ref.TYPES[dtype], seed=sum(size))
    for kind, p in (("none", 0.0), ("gelu", 0.25)):
        check(run(net, *t, kind, 1.0, p, SEED), *t, kind, 1.0, p, SEED)


@pytest.mark.parametrize("dtype", list(ref.TYPES))
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_whole_numbers_are_exact(net, size, dtype):
    """Small whole numbers: every sum is exact in fp32, so results are the definition's, rounded once."""
    T = ref.TYPES[dtype]
    x, w, b, r, g = make(*size, T, seed=1 + sum(size), pad=3, whole=True)
    out = run(net, x, w, b, r, g, "none", 1.0, 0.5, SEED)
    X, W, B, R, G = (t.cpu().to(F64) for t in (x, w, b, r, g))
    f = ref.factor(R.shape, 0.5, SEED)
    dz = G * f
    for name, want in (("y", (X @ W.T + B) * f + R), ("dx", dz @ W), ("dweight", dz.T @ X), ("dbias", dz.sum(0))):
        assert torch.equal(out[name].cpu(), want.to(T)), name


@pytest.mark.parametrize("dtype", list(ref.TYPES))
@pytest.mark.parametrize("kind", ref.ACTS)
@pytest.mark.parametrize("pad", [0, 1, 8])
def test_activations(net, kind, dtype, pad):
    T = ref.TYPES[dtype]
    for beta in ((1.0, 100.0) if kind == "softplus" else (1.0,)):
        x, w, b, r, g = make(200, 72, 136, T, seed=7, pad=pad)
        for bias, residual in ((b, r), (None, r), (b.float(), None), (None, None)):
            for p in (0.0, 0.1):
                check(run(net, x, w, bias, residual, g, kind, beta, p, SEED), x, w, bias, residual, g, kind, beta, p, SEED)


@pytest.mark.parametrize("dtype", list(ref.TYPES))
@pytest.mark.parametrize("size", [(1500, 1200, 1100), (9000, 130, 140), (300, 5000, 300)], ids=str)
def test_larger(net, size, dtype):
    t = make(*size, ref.TYPES[dtype], seed=3)
    check(run(net, *t, "silu", 1.0, 0.1, SEED), *t, "silu", 1.0, 0.1, SEED)


def test_inference_is_the_same(net):
    for dtype in ref.TYPES.values():
        x, w, b, r, _ = make(100, 70, 90, dtype)
        kw = dict(residual=r, activation="gelu", dropout=0.3, seed=SEED)
        y = net.linear(x, w, b, **kw)
        assert not y.requires_grad and torch.equal(y, net.linear(x, w.detach().requires_grad_(True), b, **kw))
        with torch.no_grad():
            assert torch.equal(y, net.linear(x.detach().requires_grad_(True), w, b, **kw))


def test_gradients_against_differences(net):
    """Central differences of the definition in 64 bits, at the operator's own inputs."""
    x, w, b, r, g = make(6, 5, 7, torch.float32, seed=11)
    for kind, beta in (("gelu", 1.0), ("silu", 1.0), ("softplus", 3.0), ("none", 1.0)):
        out = run(net, x, w, b, r, g, kind, beta, 0.4, SEED)
        wide = [t.cpu().to(F64) for t in (x, w, b, r)]
        f, G = ref.factor((6, 7), 0.4, SEED), g.cpu().to(F64)
        loss = lambda v: float((G * (ref.act(v[0] @ v[1].T + v[2], kind, beta) * f + v[3])).sum())
        for k, name in enumerate(("dx", "dweight", "dbias", "dresidual")):
            got = out[name].cpu().flatten()
            for i in range(wide[k].numel()):
                h, two = 1e-4, []
                for sign in (1, -1):
                    v = [t.clone() for t in wide]
                    v[k].view(-1)[i] += sign * h
                    two.append(loss(v))
                # third derivatives of these sums are below 1e3: h^2 1e3 / 6 < 2e-6; fp32 sums of 7 terms below 10
                assert abs((two[0] - two[1]) / (2 * h) - float(got[i])) < 2e-5, (kind, name, i)


def test_shapes_and_strides(net):
    T = torch.bfloat16
    x, w, b, r, g = make(60, 24, 40, T, seed=5)
    want = net.linear(x, w, b, residual=r, activation="silu")
    same = lambda y, shape=(60, 40): torch.equal(y.reshape(60, 40), want) and y.shape == shape
    assert same(net.linear(x.view(3, 4, 5, 24), w, b, residual=r.view(3, 4, 5, 40), activation="silu"), (3, 4, 5, 40))
    assert same(net.linear(x.t().contiguous().t(), w.t().contiguous().t(), b, residual=r.t().contiguous().t(), activation="silu"))
    assert same(net.linear(x[:, None].expand(60, 2, 24)[:, 1], w, b, residual=r, activation="silu"))
    one = net.linear(x[3], w, b, residual=r[3], activation="silu")
    assert one.shape == (40,) and torch.equal(one, net.linear(x[3:4], w, b, residual=r[3:4], activation="silu")[0])
    # results are no views: a program may change them
    y = net.linear(x.detach().requires_grad_(True).view(3, 20, 24), w, b)
    assert torch.equal(y.mul_(2.0).detach(), net.linear(x, w, b).view(3, 20, 40) * 2)
    # a row that is broadcast, and a residual that is: their gradients are sums over the rows
    row, res = x[:1].detach().requires_grad_(True), r[:1].detach().requires_grad_(True)
    y = net.linear(row.expand(60, 24), w, b, residual=res.expand(60, 40))
    assert torch.equal(y, net.linear(x[:1].repeat(60, 1), w, b, residual=r[:1].repeat(60, 1)))
    drow, dres = torch.autograd.grad(y, [row, res], g)
    full = net.linear(x[:1].repeat(60, 1).requires_grad_(True), w, b)
    assert torch.equal(dres, g.sum(0, keepdim=True)) and drow.shape == (1, 24)
    # the same weight twice; a sum as the loss, whose gradient is one number seen 2400 times
    weight = w.detach()[:24].clone().requires_grad_(True)
    y = net.linear(net.linear(x, weight, activation="relu"), weight).sum()
    (d,) = torch.autograd.grad(y, weight)
    W = weight.detach().double().requires_grad_(True)
    (D,) = torch.autograd.grad(((x.double() @ W.T).clamp(min=0) @ W.T).sum(), W)
    assert float((d.double() - D).norm() / D.norm()) < 0.01


def test_only_what_is_asked_for(net):
    x, w, b, r, g = make(70, 33, 50, torch.float32)
    every = run(net, x, w, b, r, g, "silu", 1.0, 0.2, SEED)
    for wanted in itertools.product((False, True), repeat=4):
        if not any(wanted):
            continue
        leaves = [t.detach().requires_grad_(n) for t, n in zip((x, w, b, r), wanted)]
        y = net.linear(leaves[0], leaves[1], leaves[2], residual=leaves[3], activation="silu", dropout=0.2, seed=SEED)
        grads = torch.autograd.grad(y, [t for t in leaves if t.requires_grad], g)
        names = [n for n, k in zip(("dx", "dweight", "dbias", "dresidual"), wanted) if k]
        assert torch.equal(y, every["y"]) and all(torch.equal(d, every[n]) for d, n in zip(grads, names))


def test_values_that_are_not_finite(net):
    """Of a row that holds NaN or infinities, that row's results; of every row, those columns of the weight's gradient."""
    for dtype in ref.TYPES.values():
        x, w, b, r, g = make(140, 40, 70, dtype, seed=2)
        clean = run(net, x, w, b, r, g, "none", 1.0, 0.0, None)
        bad = x.clone()
        bad[3, 5], bad[77, 0], bad[100, 39] = math.inf, math.nan, -math.inf
        out = run(net, bad, w, b, r, g, "none", 1.0, 0.0, None)
        rows = [i for i in range(140) if i not in (3, 77, 100)]
        assert torch.equal(out["y"][rows], clean["y"][rows]) and torch.equal(out["dx"], clean["dx"])
        assert out["y"][77].isnan().all()
        assert torch.equal(out["y"][3], torch.where(w[:, 5] > 0, math.inf, -math.inf).to(dtype)), dtype
        assert torch.equal(out["y"][100], torch.where(w[:, 39] > 0, -math.inf, math.inf).to(dtype))
        cols = [i for i in range(40) if i not in (0, 5, 39)]
        assert torch.equal(out["dweight"][:, cols], clean["dweight"][:, cols]) and out["dweight"][:, 0].isnan().all() and out["dweight"][:, 5].isinf().all()
        # dropped elements are 0 whatever they were
        y = net.linear(bad, w, b, dropout=1.0, seed=SEED)
        assert torch.equal(y, torch.zeros_like(y))
    big = torch.full((2, 3), 3.4e38, device="cuda")
    y = net.linear(big, torch.tensor([[1.0, -1.0, 1.0], [0.0, 0.0, 0.25], [1.0, 1.0, 0.0]], device="cuda"))
    assert torch.equal(y[0], torch.tensor([3.4e38, 3.4e38 * 0.25, math.inf], device="cuda"))


@pytest.mark.parametrize("dtype", list(ref.TYPES))
@pytest.mark.parametrize("shape", [(1,), (0, 5), (7,), (3, 5, 7), (33, 1), (1, 1000), (257, 777), (64, 2048), ()], ids=str)
def test_dropout(net, shape, dtype):
    T = ref.TYPES[dtype]
    gen = torch.Generator().manual_seed(4)
    for p, pad in ((0.0, 0), (0.1, 0), (0.5, 3), (0.999, 1), (1.0, 0)):
        def one():
            v = torch.randn(shape, generator=gen).to(T).cuda()
            if pad and v.dim() > 1:
                v = torch.cat([v, torch.full((*shape[:-1], pad), math.nan, dtype=T, device="cuda")], -1)[..., :shape[-1]]
            return v
        x, r, g = one(), one(), one()
        f = ref.factor(shape, p, SEED)
        fp32 = (x.cpu().float() * torch.tensor(1.0 / (1.0 - p) if p < 1 else 0.0, dtype=torch.float32)) * (f != 0)
        for residual in (None, r):
            leaf, res = x.detach().requires_grad_(True), None if residual is None else r.detach().requires_grad_(True)
            y = net.dropout(leaf, p, SEED, residual=res)
            want = fp32 if residual is None else fp32 + r.cpu().float()
            assert y.shape == tuple(shape) and torch.equal(y.cpu(), want.to(T)), (p, pad)
            assert torch.equal(net.dropout(x, p, SEED, residual=residual), y)
            grads = torch.autograd.grad(y, [leaf] if res is None else [leaf, res], g)
            want = (g.cpu().float() * torch.tensor(1.0 / (1.0 - p) if p < 1 else 0.0, dtype=torch.float32)) * (f != 0)
            assert torch.equal(grads[0].cpu(), want.to(T))
            assert res is None or torch.equal(grads[1], g)


def test_dropout_and_linear_draw_the_same(net):
    words = torch.tensor([77, -5], dtype=torch.int64, device="cuda")
    seed = (77, 2 ** 64 - 5)
    for n in (64, 77):
        x, w, b, r, g = make(90, 50, n, torch.float32)
        y = net.linear(x, w, b, activation="silu", dropout=0.3, seed=words)
        assert torch.equal(y, net.dropout(net.linear(x, w, b, activation="silu"), 0.3, seed))
        assert torch.equal(net.linear(x, w, b, residual=r, dropout=0.3, seed=seed), net.linear(x, w, b, residual=r, dropout=0.3, seed=words))
        assert torch.equal(y == 0, ref.factor((90, n), 0.3, seed).cuda() == 0)
    share = float((net.dropout(torch.ones(1 << 20, device="cuda"), 0.3, words) == 0).float().mean())
    assert abs(share - 0.3) < 6 * math.sqrt(0.3 * 0.7 / 2 ** 20)
    words[1] += 1
    assert not torch.equal(y, net.linear(x, w, b, activation="silu", dropout=0.3, seed=words))


def test_a_seed_that_changes_is_noticed(net):
    x, w, *_ = make(8, 8, 8, torch.float32)
    words = torch.tensor([1, 2], device="cuda")
    for f in (lambda t: net.linear(t, w, dropout=0.5, seed=words), lambda t: net.dropout(t, 0.5, words)):
        y = f(x.detach().requires_grad_(True))
        words += 1
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.sum().backward()


def test_same_results_from_call_to_call(net):
    for dtype in ref.TYPES.values():
        t = make(3000, 200, 100, dtype)
        a, b = (run(net, *t, "gelu", 1.0, 0.1, SEED) for _ in range(2))
        assert all(torch.equal(a[k], b[k]) for k in a)


def test_other_streams(net):
    t = make(500, 300, 200, torch.bfloat16)
    want = run(net, *t, "gelu", 1.0, 0.1, SEED)
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = []
    for _ in range(4):
        for s in streams:
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                got.append(run(net, *t, "gelu", 1.0, 0.1, SEED))
    torch.cuda.synchronize()
    assert all(torch.equal(g[k], want[k]) for g in got for k in want)


def test_graphs(net):
    """A captured step of layers and dropout, replayed between eager work, with its words counted up by the graph."""
    x, w, b, r, g = make(300, 64, 64, torch.bfloat16)
    words = torch.tensor([5, 0], device="cuda")

    def step(words):
        leaves = [t.detach().requires_grad_(True) for t in (x, w, b)]
        h = net.linear(leaves[0], leaves[1], leaves[2], residual=leaves[0], activation="gelu", dropout=0.2, seed=words)
        y = net.dropout(net.linear(h, leaves[1]), 0.1, words, residual=h)
        return [y.detach(), *torch.autograd.grad(y, leaves, g)]

    step(words)
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            now = words.clone()
            out = step(now)
            words += 3
        graphs.append((graph, out))
    for k in range(6):
        graph, out = graphs[k % 2]
        before = words.clone()
        want = step(before)
        graph.replay()
        torch.cuda.synchronize() if k % 3 == 0 else None
        assert torch.equal(words, before + 3)
        assert all(torch.equal(a, b) for a, b in zip(out, want)), k


def test_two_graphs_beside_one_another(net):
    t = make(700, 500, 90, torch.float32)
    want = run(net, *t, "silu", 1.0, 0.0, None)
    pairs = []
    for _ in range(2):
        graph, s = torch.cuda.CUDAGraph(), torch.cuda.Stream()
        with torch.cuda.graph(graph, stream=s):
            out = run(net, *t, "silu", 1.0, 0.0, None)
        pairs.append((graph, out, s))
    for _ in range(3):
        for graph, out, s in pairs:
            for name in ("y", "dx", "dweight", "dbias"):
                out[name].detach().zero_()
        torch.cuda.synchronize()
        for graph, _, s in pairs:
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(out[k], want[k]) for _, out, _ in pairs for k in want)


def test_more_than_32_bits_of_elements(net):
    rows, n = (1 << 32) // 56 + 1000, 56
    x = torch.zeros(rows, 3, dtype=torch.bfloat16, device="cuda")
    x[-5:] = torch.randn(5, 3).to(torch.bfloat16).cuda()
    w = torch.randn(n, 3).to(torch.bfloat16).cuda()
    y = net.linear(x, w, dropout=0.25, seed=SEED)
    assert y.numel() > 1 << 32
    f = ref.factor((5, n), 0.25, SEED, first=(rows - 5) * n)
    want = (x[-5:].cpu().to(F64) @ w.cpu().to(F64).T) * f
    ref.assert_close("y", y[-5:], (want, ref.rounded(want, torch.bfloat16) * 1.01 + 1e-6))
    assert int(y[:-5].count_nonzero()) == 0
    leaf = w.detach().requires_grad_(True)
    g = y
    dx, dw = torch.autograd.grad(net.linear(x.requires_grad_(True), leaf), [x, leaf], g)
    X, G = x.detach()[-5:].cpu().to(F64), g[-5:].cpu().to(F64)
    want = G.T @ X
    ref.assert_close("dweight", dw, (want, ref.rounded(want, torch.bfloat16) * 1.01 + 1e-5))
    ref.assert_close("dx", dx[-5:], (G @ w.cpu().to(F64), ref.rounded(G @ w.cpu().to(F64), torch.bfloat16) * 1.01 + 1e-4))
    assert int(dx[:-5].count_nonzero()) == 0
    del dx, dw, x
    z = net.dropout(g, 0.25, SEED)                     # without gaps: one long row
    assert torch.equal(z[-5:].cpu(), (g[-5:].cpu().float() * torch.tensor(1 / 0.75) * (f != 0)).to(torch.bfloat16))
    wide = g.view(-1)[: g.numel() - 56].view(-1, 56)[:, :55]
    z = net.dropout(wide, 0.25, SEED)                  # rows with gaps
    f = ref.factor((4, 55), 0.25, SEED, first=(wide.shape[0] - 4) * 55)
    assert torch.equal(z[-4:].cpu(), (wide[-4:].cpu().float() * torch.tensor(1 / 0.75) * (f != 0)).to(torch.bfloat16))


def whole(rows, cols, dtype, gen, pad=0):
    v = torch.randint(-2, 3, (rows, cols + pad), generator=gen, device="cuda", dtype=torch.int8).to(dtype)
    return v[:, :cols]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("size", [(4100, 584, 4104), (4100, 4104, 584), (584, 4104, 4096), (4096, 1024, 4096), (4099, 600, 4101)], ids=str)
@pytest.mark.parametrize("pad", [0, 8, 3])
def test_large_whole_numbers_are_exact(net, size, pad, dtype):
    """The large tiles, with edges along p, q and t, in each of the three products; 64-bit sums on the GPU."""
    rows, inputs, outputs = size
    T, gen = ref.TYPES[dtype], torch.Generator(device="cuda").manual_seed(rows)
    x, w, g = (whole(m, n, T, gen, pad).requires_grad_(True) for m, n in ((rows, inputs), (outputs, inputs), (rows, outputs)))
    g = g.detach()
    y = net.linear(x, w)
    dx, dw = torch.autograd.grad(y, [x, w], g)
    X, W, G = (t.detach().to(F64) for t in (x, w, g))
    for name, got, want in (("y", y, X @ W.t()), ("dx", dx, G @ W), ("dweight", dw, G.t() @ X)):
        off = got.detach() != want.to(T)
        assert not bool(off.any()), (name, int(off.sum()), off.nonzero()[:4].tolist())


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_long_contractions_in_parts(net, dtype):
    rows, T, gen = 530001, ref.TYPES[dtype], torch.Generator(device="cuda").manual_seed(1)
    x, w, g = (whole(m, n, T, gen).requires_grad_(True) for m, n in ((rows, 256), (256, 256), (rows, 256)))
    b = torch.zeros(256, device="cuda", requires_grad=True)
    # partial sums of whole numbers below 2^24 are exact in fp32
    dw, db = torch.autograd.grad(net.linear(x, w, b, activation="relu"), [w, b], g.detach())
    X, W, G = (t.detach().to(F64) for t in (x, w, g))
    dz = G * (X @ W.t() > 0)
    assert float((dz.t().abs() @ X.abs()).max()) < 2 ** 24
    assert torch.equal(dw, (dz.t() @ X).to(T)) and torch.equal(db, dz.sum(0).float())


def test_every_digit_of_fp32(net):
    """Through a matrix of ones on the diagonal every fp32 number comes as it is: its three parts hold all of it, small, large or infinite."""
    gen = torch.Generator().manual_seed(9)
    for rows, n in ((1, 64), (3, 128), (20, 160), (200, 64), (300, 128), (300, 200), (1100, 1100)):
        v = torch.randn(rows, n, generator=gen) * 2.0 ** torch.randint(-90, 120, (rows, n), generator=gen).float()
        v[0, :4] = torch.tensor([3.4028235e38, -3.4028235e38, math.inf, 2.0 ** -100 * (1 + 2.0 ** -23)])
        x, w = v.cuda().requires_grad_(True), torch.eye(n, device="cuda").requires_grad_(True)
        y = net.linear(x, w)
        # beside an infinity stands 0 times it
        clean = torch.ones(rows, n, dtype=torch.bool)
        clean[0] = False
        assert torch.equal(y.detach().cpu()[clean], v[clean])
        dx, dw = torch.autograd.grad(y, [x, w], torch.eye(rows, n, device="cuda") * 1.2345678)
        assert torch.equal(dx, torch.eye(rows, n, device="cuda") * 1.2345678)
        few = torch.autograd.grad(net.linear(w, w), w, v.cuda()[:n] if rows >= n else torch.cat([v, v.new_zeros(n - rows, n)]).cuda())[0]
        assert few.shape == (n, n)
    v = v[1:]
    x = v.cuda().requires_grad_(True)
    (dx,) = torch.autograd.grad(net.linear(x, torch.eye(1100, device="cuda")), x, v.cuda())
    assert torch.equal(dx.cpu(), v)


def test_small_numbers_of_16_bits(net):
    for T, small in ((torch.float16, 2.0 ** -24), (torch.bfloat16, 2.0 ** -126)):
        for rows in (2, 100):
            x = torch.full((rows, 64), small, dtype=T, device="cuda") * torch.arange(64, device="cuda").to(T)
            y = net.linear(x, torch.eye(64, dtype=T, device="cuda"))
            assert torch.equal(y, x), T


@pytest.mark.parametrize("dtype", list(ref.TYPES))
def test_odd_addresses(net, dtype):
    """Tensors that begin between the multiples of their vectors, rows as well."""
    T, gen = ref.TYPES[dtype], torch.Generator(device="cuda").manual_seed(2)
    for size in ((3, 70, 40), (150, 130, 90), (1500, 640, 1100)):
        rows, inputs, outputs = size

        def odd(m, n):
            flat = torch.randint(-2, 3, (m * (n + 1) + 1,), generator=gen, device="cuda", dtype=torch.int8).to(T)
            return flat[1:].view(m, n + 1)[:, :n]

        x, w, r, g = odd(rows, inputs), odd(outputs, inputs), odd(rows, outputs), odd(rows, outputs)
        b = odd(1, outputs)[0]
        out = run(net, x, w, b, r, g, "none", 1.0, 0.5, SEED)
        X, W, B, R, G = (t.to(F64) for t in (x, w, b, r, g))
        f = ref.factor((rows, outputs), 0.5, SEED).cuda()
        for name, want in (("y", (X @ W.t() + B) * f + R), ("dx", (G * f) @ W), ("dweight", (G * f).t() @ X), ("dbias", (G * f).sum(0))):
            assert torch.equal(out[name].detach(), want.to(T)), (size, name)
        assert torch.equal(net.dropout(x, 0.5, SEED, residual=x), (X * ref.factor((rows, inputs), 0.5, SEED).cuda() + X).to(T))


def test_in_place(gpu_lib):
    """The C calls with Y in the residual's place, or in X's."""
    import ctypes
    L, T = gpu_lib.load(), torch.bfloat16
    s = torch.cuda.current_stream().cuda_stream
    for rows, inputs, outputs in ((5, 40, 72), (300, 72, 90), (90, 3000, 64)):
        x, w, b, r, _ = make(rows, inputs, outputs, T)
        layer = gpu_lib.Linear(rows, inputs, outputs, 1, 1, gpu_lib.FS_ACT_SILU, 1.0, gpu_lib.Drop(0.3, 1, 2, None))
        n = L.fs_linear_bytes(ctypes.byref(layer), 0)
        work = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
        want, z = torch.empty_like(r), torch.empty_like(r)
        go = lambda y, res: L.fs_linear_forward(ctypes.byref(layer), x.data_ptr(), inputs, w.data_ptr(), inputs, b.data_ptr(), res.data_ptr(), outputs, y.data_ptr(), outputs, z.data_ptr(),
                                                outputs, work.data_ptr() if n else None, n, s)
        assert go(want, r) == 0
        same = r.clone()
        assert go(same, same) == 0 and torch.equal(same, want)
    drop = gpu_lib.Drop(0.4, 3, 4, None)
    for shape in ((7, 33), (64, 4096)):
        x, r = torch.randn(shape, device="cuda"), torch.randn(shape, device="cuda")
        want, a, c = torch.empty_like(x), x.clone(), r.clone()
        go = lambda x, r, y: L.fs_dropout(0, *shape, ctypes.byref(drop), x.data_ptr(), shape[1], r.data_ptr(), shape[1], y.data_ptr(), shape[1], s)
        assert go(x, r, want) == 0 and go(a, r, a) == 0 and go(x, c, c) == 0
        assert torch.equal(a, want) and torch.equal(c, want)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kind", ["none", "gelu", "silu", "softplus"])
@pytest.mark.parametrize("size", [(40, 10, 1), (1, 10, 40), (2, 27, 2), (1899, 10, 1), (70, 128, 128), (1, 1, 1), (87983, 1, 1)], ids=str)
def test_small_layers_round_their_gradients_once(net, size, kind, dtype):
    """Neither dZ nor Z is rounded to 16 bits in small layers.  Bounds: those of the same numbers in fp32; what two parts of dZ leave, half a step of half a step of it, and
    half of fp16's least number (2^-25); the result's own rounding."""
    T = ref.TYPES[dtype]
    t = make(*size, T, seed=9 + sum(size), pad=1)
    out = run(net, *t, kind, 1.0, 0.25, SEED)
    x, w, b, r, g = (v.float() for v in t)
    want = ref.linear(x, w, b, r, g, kind, 1.0, 0.25, SEED)
    X, W, B, G = (v.cpu().to(F64) for v in (x, w, b, g))
    dz = (G * ref.slope(X @ W.T + B, kind, 1.0) * ref.factor(G.shape, 0.25, SEED)).abs()
    left = dz * 1.1 * (torch.finfo(T).eps / 2) ** 2 + 2.0 ** -25
    for name, more in (("dx", left @ W.abs()), ("dweight", left.T @ X.abs())):
        value, bound = want[name]
        ref.assert_close(name, out[name], (value, bound + more + ref.rounded(value, T) * 1.01))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("size", [(65, 63, 66), (1100, 128, 128), (2000, 17, 97), (300, 200, 130)], ids=str)
def test_z_in_16_bits(net, monkeypatch, size, dtype):
    """As layers of more than 2^22 values keep it; the second and third have more values of dZ than go in as two parts."""
    T = ref.TYPES[dtype]
    monkeypatch.setattr(net, "_Z_FULL", 0)
    net._plan.cache_clear()
    try:
        for kind in ("gelu", "silu", "softplus"):
            t = make(*size, T, seed=3 + sum(size), pad=2)
            check(run(net, *t, kind, 1.0, 0.25, SEED), *t, kind, 1.0, 0.25, SEED)
    finally:
        net._plan.cache_clear()


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("rows", [70, 1100])
def test_infinities_in_small_layers(net, rows, dtype):
    """One infinity in weight, x or g reaches the results that the formulas send it to, and no others; dZ's parts make no NaN of it."""
    T = ref.TYPES[dtype]
    for where in range(3):
        x, w, b, r, g = make(rows, 24, 128, T, seed=rows + where, whole=True)
        x, w, g = (t.abs() + 1 for t in (x, w, g))
        (x, w, g)[where][1, 2] = math.inf
        leaves = [t.detach().requires_grad_(True) for t in (x, w, b)]
        dx, dw, db = torch.autograd.grad(net.linear(leaves[0], leaves[1], leaves[2]), leaves, g)
        X, W, G = (t.cpu().to(F64) for t in (x, w, g))
        for name, got, want in (("dx", dx, G @ W), ("dweight", dw, G.T @ X), ("dbias", db, G.sum(0))):
            assert torch.equal(got.cpu(), want.to(T)), (name, where)
