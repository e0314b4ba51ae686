"""Host code of optim.py without a GPU (fake_lists.py): what it hands to the library, and when."""
import pytest
import torch

import fake_lists


@pytest.fixture
def gpu(monkeypatch):
    return fake_lists.Machine(monkeypatch)


def test_settings_that_are_changed_in_place(gpu):
    (p,) = params = gpu.params(10)
    opt = gpu.adamw(params, grads=gpu.grads(params), betas=[0.9, 0.999])
    opt.step()
    opt.betas[0] = 0.5
    opt.step()
    opt.betas[1] = 0.25
    opt.step()
    assert [(r["args"][0]["beta1"], r["args"][0]["beta2"]) for r in gpu.ran] == [(0.9, 0.999), (0.5, 0.999), (0.5, 0.25)]


def test_every_graph_brings_the_list_that_it_needs(gpu):
    """Gradients that moved between the eager call and the captures: whichever graph is replayed first, or alone, works on them."""
    params = gpu.params(10, 20)
    opt = gpu.adamw(params)
    gpu.grads(params)
    opt.step()
    moved = [g.data_ptr() for g in gpu.grads(params)]
    graphs = []
    for _ in range(3):
        with gpu.capture() as g:
            opt.step(), opt.step()
        graphs.append(g)
    for g in reversed(graphs):                              # the first one last
        gpu.ran.clear()
        g.replay()
        assert len(gpu.ran) == 2 and all(r["fits"] and r["list"]["grad"].tolist() == moved for r in gpu.ran)
    gpu.ran.clear()
    opt.step()
    assert gpu.ran[0]["fits"] and gpu.ran[0]["list"]["grad"].tolist() == moved


def test_graphs_have_scratch_of_their_own(gpu):
    """Replays are ordered behind nothing that optim.py knows of: beside an eager call, or another graph's replay, they must not share counters."""
    lst = gpu.optim.TensorList([fake_lists.on_gpu(g) for g in (torch.ones(10), torch.ones(20))])
    out = fake_lists.on_gpu(torch.zeros(1))
    params = gpu.params(10, 20)
    opt = gpu.adamw(params, grads=gpu.grads(params))
    for call in (lambda: lst.grad_norm(out=out), lambda: lst.clip_grads(1.0, norm=out), opt.step):
        gpu.ran.clear()
        call()
        graphs = []
        for _ in range(2):
            with gpu.capture() as g:
                call(), call()
            graphs.append(g)
        with gpu.on(6):
            call()
        for g in graphs[::-1]:
            g.replay()
        call()
        assert all(r["fits"] for r in gpu.ran)
        eager, one, two = ({r["scratch"] for r in gpu.ran[a:b]} for a, b in ((0, 2), (2, 4), (4, 6)))
        assert len(eager) == len(one) == len(two) == 1 and len(eager | one | two) == 3 and gpu.ran[6]["scratch"] in eager
        graphs[0].replay()
        assert gpu.ran[-1]["scratch"] in two and gpu.ran[-1]["fits"]


def test_calls_of_one_graph_on_several_streams_come_one_after_another(gpu):
    params = gpu.params(10)
    opt = gpu.adamw(params, grads=gpu.grads(params))
    opt.step()
    with gpu.capture(9) as g:
        opt.step()
        gpu.captures[11] = gpu.captures[9]                  # a stream that has joined the capture
        gpu.waits.clear()
        with gpu.on(11):
            opt.step()
        assert gpu.waits == [(11, 9)]
        opt.step()
        assert gpu.waits == [(11, 9), (9, 11)]
        del gpu.captures[11]
    g.replay()
    assert all(r["fits"] for r in gpu.ran) and len({r["scratch"] for r in gpu.ran[1:]}) == 1
    # the stream of the capture is no stream to wait for outside of it
    gpu.waits.clear()
    opt.step()
    assert gpu.waits == []


def _other_type_at_the_same_place(p, dtype):
    at = p.data_ptr()
    p.data = fake_lists.on_gpu(p.detach().as_subclass(torch.Tensor).view(dtype).reshape(-1)[:p.numel()].view(p.shape))
    assert p.data_ptr() == at and p.dtype == dtype


@pytest.mark.parametrize("given", [False, True])
def test_parameters_of_another_type_at_the_same_place(gpu, given):
    """A block that was freed and taken again, or a view of it in 16 bits: four bytes an element would go past its end."""
    params = gpu.params(10, 20)
    grads = gpu.grads(params)
    opt = gpu.adamw(params, grads=grads if given else None)
    opt.step()
    for dtype, code in ((torch.bfloat16, gpu.binding.FS_FLOAT_BRAIN), (torch.float16, gpu.binding.FS_FLOAT_HALF)):
        params[1].grad = None
        _other_type_at_the_same_place(params[1], dtype)
        if not given:
            params[1].grad = fake_lists.on_gpu(torch.ones(20, dtype=dtype))
        opt.step()
        assert gpu.ran[-1]["fits"] and gpu.ran[-1]["list"]["param_type"].tolist() == [gpu.binding.FS_FLOAT_FULL, code]


@pytest.mark.parametrize("given", [False, True])
def test_parameters_of_another_size_at_the_same_place_are_refused(gpu, given):
    params = gpu.params(10, 20)
    opt = gpu.adamw(params, grads=gpu.grads(params) if given else None)
    opt.step()
    at, whole, grad = params[1].data_ptr(), params[1].data, params[1].grad
    params[1].grad = None
    params[1].data = whole[:5]
    assert params[1].data_ptr() == at
    if not given:
        params[1].grad = fake_lists.on_gpu(torch.ones(5))
    for _ in range(2):
        with pytest.raises(ValueError, match=r"\[1\]: shape"):
            opt.step()
    assert len(gpu.ran) == 1
    params[1].grad = None
    params[1].data = whole
    params[1].grad = grad
    opt.step()
    assert len(gpu.ran) == 2 and gpu.ran[-1]["fits"]


def test_parameters_in_another_order_at_the_same_place_are_refused(gpu):
    p = fake_lists.on_gpu(torch.ones(4, 6)).requires_grad_(True)
    opt = gpu.adamw([p])
    gpu.grads([p])
    opt.step()
    p.grad, p.data = None, p.data.as_strided((4, 6), (1, 4))
    p.grad = fake_lists.on_gpu(torch.ones(6, 4)).t()
    with pytest.raises(ValueError, match=r"exp_avgs\[0\]"):
        opt.step()


def test_state_is_not_exchanged_behind_the_list(gpu):
    """The list has the addresses of the state: what is put in its place later would be ignored, and its memory written to after it was freed."""
    params = gpu.params(10, 20, dtype=torch.bfloat16)
    opt = gpu.adamw(params, grads=gpu.grads(params), masters=[fake_lists.on_gpu(torch.ones(n)) for n in (10, 20)])
    opt.step()
    for name in ("masters", "exp_avgs", "exp_avg_sqs"):
        before = getattr(opt, name)
        at = [t.data_ptr() for t in before]
        assert gpu.ran[-1]["list"][name[:-1]].tolist() == at
        with pytest.raises(AttributeError):
            setattr(opt, name, [torch.zeros_like(t) for t in before])
        changed = getattr(opt, name)
        changed[0] = torch.zeros_like(before[0])
        assert [t.data_ptr() for t in getattr(opt, name)] == at == [t.data_ptr() for t in opt.state_dict()[name]]
        # other memory for the same tensor object: the list goes on with what it has, which is kept
        before[1].data = torch.zeros(20)
    old = [gpu.ran[-1]["list"][name].tolist() for name in ("master", "exp_avg", "exp_avg_sq")]
    new = [fake_lists.on_gpu(torch.ones(20)) for _ in range(16)]
    opt.step()
    assert [gpu.ran[-1]["list"][name].tolist() for name in ("master", "exp_avg", "exp_avg_sq")] == old
    assert not {t.data_ptr() for t in new} & {a for at in old for a in at}


def test_the_step_counter_is_checked_when_it_is_exchanged(gpu):
    params = gpu.params(10)
    opt = gpu.adamw(params, grads=gpu.grads(params))
    opt.step()
    for bad, error in ((fake_lists.on_gpu(torch.zeros(1, dtype=torch.int32)), TypeError), (fake_lists.on_gpu(torch.zeros(2, dtype=torch.int64)), ValueError),
                       (torch.zeros(1, dtype=torch.int64), ValueError), (3, TypeError)):
        opt.step_count = bad
        with pytest.raises(error, match="step"):
            opt.step()
    assert len(gpu.ran) == 1
    opt.step_count = fake_lists.on_gpu(torch.full((1,), 7, dtype=torch.int64))
    opt.step()
    assert gpu.ran[-1]["args"][1] == opt.step_count.data_ptr()


@pytest.mark.parametrize("given", [False, True])
def test_a_number_of_parameters_that_changes_is_refused(gpu, given):
    params = gpu.params(10, 20)
    opt = gpu.adamw(params, grads=gpu.grads(params) if given else None)
    opt.step()
    for change in (lambda: opt.params.pop(), lambda: opt.params.extend(2 * gpu.params(20))):
        change()
        with pytest.raises(ValueError, match="params: . entries, expected 2"):
            opt.step()
    opt.params[:] = params
    opt.step()
    assert len(gpu.ran) == 2 and gpu.ran[0]["list"].tolist() == gpu.ran[1]["list"].tolist()


def test_memory_that_comes_to_overlap_is_refused(gpu):
    """Parameters and gradients may move between steps; what a step writes must not be what it reads or writes elsewhere."""
    params = gpu.params(10, 20)
    opt = gpu.adamw(params)
    gpu.grads(params)
    opt.step()
    good = [p.grad for p in params]
    state = opt.exp_avgs[1]
    for p, bad in ((0, params[1].data[3:13]), (0, opt.exp_avg_sqs[0]), (1, state), (1, params[1].data)):
        params[p].grad = bad.as_subclass(torch.Tensor).as_subclass(fake_lists.OnGpu)
        assert params[p].grad.data_ptr() == bad.data_ptr()
        for _ in range(2):
            with pytest.raises(ValueError, match="overlap"):
                opt.step()
        params[p].grad = good[p]
    opt.step()
    # tied by their memory
    before = params[0].data
    params[0].data = params[1].data[5:15]
    with pytest.raises(ValueError, match="overlap"):
        opt.step()
    params[0].grad = None                                   # not updated: nothing is written twice
    opt.step()
    params[0].data, params[0].grad = before, good[0]
    # gradients are read only, and may share memory
    whole = fake_lists.on_gpu(torch.ones(20))
    params[0].grad, params[1].grad = whole[:10], whole
    opt.step()
    assert all(r["fits"] for r in gpu.ran) and len(gpu.ran) == 4


def test_lists_that_go_while_a_graph_is_captured_are_freed_later(gpu):
    """Freeing memory is nothing that a capture allows."""
    import gc
    new = lambda: gpu.optim.TensorList([fake_lists.on_gpu(torch.ones(10))])
    out = fake_lists.on_gpu(torch.zeros(1))
    keep, a, b = new(), new(), new()
    h = [x._handle.eager.h.value for x in (a, b)]
    with gpu.capture() as g:
        keep.grad_norm(out=out)
        a.grad_norm(out=out)
        own = a._handle.graph.h.value
        del a, b
        gc.collect()
        assert gpu.destroyed == [own]                       # that one has no memory of its own
    g.replay()
    assert all(r["fits"] for r in gpu.ran)
    c = new()
    assert sorted(gpu.destroyed) == sorted(h + [own])
    # the runtime may refuse at other times too (a capture in another thread)
    refuse, at = gpu.binding.FS_E_DEVICE, c._handle.eager.h.value
    ok = gpu.fs_tensors_destroy
    gpu.fs_tensors_destroy = lambda h: refuse
    del c
    gc.collect()
    gpu.fs_tensors_destroy = ok
    assert at not in gpu.destroyed
    new()
    assert at in gpu.destroyed and len(set(gpu.destroyed)) == len(gpu.destroyed)


def test_calls_on_a_list_of_another_gpu_than_the_current_one(gpu):
    params = gpu.params(10, 20)
    out = fake_lists.on_gpu(torch.zeros(1))
    gpu.device = 1
    lst = gpu.optim.TensorList([fake_lists.on_gpu(torch.ones(10))], device="cuda:0")
    opt = gpu.adamw(params)
    lst.grad_norm(out=out)
    for _ in range(2):
        gpu.grads(params)
        opt.step()
    with gpu.capture() as g:
        lst.clip_grads(1.0, norm=out)
        opt.step()
    g.replay()
    assert [r["call"] for r in gpu.ran] == ["norm", "adamw", "adamw", "clip", "adamw"] and all(r["fits"] for r in gpu.ran) and gpu.device == 1


def test_a_graphs_memory_is_known_to_be_used_on_each_of_its_streams(gpu):
    """A list that goes during the capture leaves its memory to what the capture allocates next: not while another branch is still at it."""
    lst = gpu.optim.TensorList([fake_lists.on_gpu(torch.ones(10))])
    out = fake_lists.on_gpu(torch.zeros(1))
    fake_lists.OnGpu.used_on.clear()
    with gpu.capture(9):
        lst.grad_norm(out=out)
        gpu.captures[11] = gpu.captures[9]
        with gpu.on(11):
            lst.grad_norm(out=out)
        assert fake_lists.OnGpu.used_on == [(lst._handle.graph.workspace.data_ptr(), 11)]
        del gpu.captures[11]
