"""Gradient norm, clipping and AdamW in several graphs, beside one another and beside eager calls."""
import pytest
import torch

import train_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def optim(gpu_lib):
    from paper_2211_15601_amd import optim
    return optim


@pytest.mark.parametrize("n", [9001, 300_001])
def test_each_of_several_graphs_works_alone(optim, n):
    """Gradients that have moved since the eager call: the graph that is captured last is replayed first, and the first one never."""
    p = torch.zeros(n, device=DEV, requires_grad=True)
    opt = optim.AdamW([p], lr=1.0, betas=(0.0, 0.0), eps=0.0, weight_decay=0.0)      # p goes by the gradient's sign
    p.grad = torch.ones(n, device=DEV)
    opt.step()
    p.grad = torch.full((n,), -2.0, device=DEV)
    graphs = [torch.cuda.CUDAGraph() for _ in range(3)]
    for g in graphs:
        with torch.cuda.graph(g):
            opt.step(), opt.step()
    torch.cuda.synchronize()
    at = -1
    for k in (2, 1, 2, 1):
        assert (p == at).all()
        graphs[k].replay()
        torch.cuda.synchronize()
        at += 2
    assert (p == at).all()
    opt.step()
    assert (p == at + 1).all() and int(opt.step_count) == 10
    del graphs, g
    p.grad = torch.full((n,), 3.0, device=DEV)
    opt.step()
    assert (p == at).all()


@pytest.mark.parametrize("sizes", [[5, 9001], [2_000_003, 77, 4096]])
def test_replays_beside_eager_calls(optim, sizes):
    """All of them only read the gradients, on streams that wait for nobody."""
    gen = torch.Generator().manual_seed(21)
    host = [torch.randn(n, generator=gen) for n in sizes]
    grads = [x.to(DEV) for x in host]
    outs = [torch.zeros_like(x) for x in grads]
    lst = optim.TensorList(grads, outs=outs)
    want = ref.norm(host)
    right = lambda x: abs(float(x) - want) <= want * ref.U * ref.SLACK
    assert right(lst.grad_norm())
    graphs, norms = [], []
    for k in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            norms.append(lst.clip_grads(want / 2) if k == 0 else lst.grad_norm())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        eager = []
        for x in norms + outs:
            x.zero_()
        torch.cuda.synchronize()
        for _ in range(20):
            for g, s in zip(graphs, streams):
                with torch.cuda.stream(s):
                    g.replay()
            eager.append(lst.grad_norm())
        torch.cuda.synchronize()
        assert all(right(x) for x in eager + norms)
        for x, y in zip(host, outs):
            ref.near(y, *ref.clip(x, ref.coef(want, want / 2)))


def test_one_graph_on_two_streams(optim):
    g = torch.full((100_003,), 2.0, device=DEV)
    lst = optim.TensorList([g])
    want = float(lst.grad_norm())
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = lst.grad_norm()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            b = lst.grad_norm(grad_scale=2.0)
        torch.cuda.current_stream().wait_stream(side)
        c = lst.grad_norm(grad_scale=4.0)
    for _ in range(3):
        for x in (a, b, c):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert [float(x) for x in (a, b, c)] == [want, 2 * want, 4 * want]
        assert float(lst.grad_norm()) == want


def test_branches_of_one_graph(optim):
    """Calls that the graph itself leaves unordered: the list's scratch orders them."""
    g = torch.full((3_000_001,), 2.0, device=DEV)
    lst = optim.TensorList([g])
    want = float(lst.grad_norm())
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        side.wait_stream(main)
        a = lst.grad_norm()
        with torch.cuda.stream(side):
            b = lst.grad_norm(grad_scale=2.0)
        c = lst.grad_norm(grad_scale=4.0)
        main.wait_stream(side)
    for _ in range(5):
        for x in (a, b, c):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert [float(x) for x in (a, b, c)] == [want, 2 * want, 4 * want]


def test_lists_that_go_during_a_capture(optim):
    g = torch.full((50_003,), 2.0, device=DEV)
    keep, gone = optim.TensorList([g]), optim.TensorList([g])
    want = float(keep.grad_norm())
    assert float(gone.grad_norm()) == want
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a = keep.grad_norm()
        b = gone.grad_norm(grad_scale=2.0)
        del gone
        c = keep.grad_norm(grad_scale=4.0)
    other = optim.TensorList([g])
    for _ in range(3):
        for x in (a, b, c):
            x.zero_()
        graph.replay()
        assert float(other.grad_norm()) == want
        torch.cuda.synchronize()
        assert [float(x) for x in (a, b, c)] == [want, 2 * want, 4 * want]


def test_a_list_that_goes_during_a_capture_with_branches(optim):
    g = torch.full((3_000_001,), 2.0, device=DEV)
    lst = optim.TensorList([g])
    want = float(lst.grad_norm())
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        main = torch.cuda.current_stream()
        a = lst.grad_norm()
        side.wait_stream(main)
        with torch.cuda.stream(side):
            b = lst.grad_norm(grad_scale=2.0)
        del lst
        rest = [torch.full((26_000,), 7, dtype=torch.uint8, device=DEV) for _ in range(8)]      # of the size of its memory, on the other branch
        main.wait_stream(side)
    for _ in range(5):
        for x in [a, b] + rest:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert [float(x) for x in (a, b)] == [want, 2 * want] and all((x == 7).all() for x in rest)
