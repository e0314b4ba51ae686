"""Host code of the calls on a list of tensors without a GPU (host_path.py): what they refuse, what they launch, what they give back."""
import pytest
import torch

import host_path

CHILD = """
import math

class Tensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("grad", "out", "param", "master", "m", "v")] + [("n", ctypes.c_int64)] + \\
               [(n, ctypes.c_int32) for n in ("gt", "pt")] + [(n, ctypes.c_float) for n in ("ls", "ds")]

class How(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "b1", "b2", "eps", "wd", "max_norm", "scale")] + \\
               [(n, ctypes.c_int32) for n in ("given", "skip")] + [("d_lr", ctypes.c_void_p)]

L.fs_tensors_error.restype = ctypes.c_char_p

def at(i):
    return 0x300000000000 + (i << 36)

def tensor(n=100, **k):
    t = Tensor(at(1), at(2), at(3), None, at(4), at(5), n, 0, 0, 1.0, 1.0)
    for name, v in k.items():
        setattr(t, name, v)
    return t

def make(tensors, status=OK, count=None):
    h = ctypes.c_void_p(77)
    a = (Tensor * max(1, len(tensors)))(*tensors)
    st = L.fs_tensors_create(a, len(tensors) if count is None else count, None, ctypes.byref(h))
    assert st == status, st
    assert (h.value is None) == (status != OK)
    return h

def error(h):
    return L.fs_tensors_error(h).decode()

def how(**k):
    x = How(1e-3, 0.9, 0.999, 1e-8, 0.01, 1.0, 1.0, 0, 0, None)
    for name, v in k.items():
        setattr(x, name, v)
    return x

D = ctypes.c_double
def norm(h, kind=0, scale=1.0, d=buf(7)):
    return L.fs_grad_norm(h, kind, D(scale), d)
def clip(h, kind=0, max_norm=1.0, scale=1.0, given=0, d=buf(7)):
    return L.fs_grad_clip(h, kind, D(max_norm), D(scale), given, d)
def adamw(h, x, step=buf(8), d=buf(7)):
    return L.fs_adamw_step(h, ctypes.byref(x) if x is not None else None, step, d)
"""


def run(code, tmp_path):
    host_path.run(CHILD + code, tmp_path)


def test_lists_that_are_refused(tmp_path):
    run("""
for bad, status in ((dict(n=-1), E_SHAPE), (dict(n=(1 << 40) + 1), E_SHAPE), (dict(grad=None), E_ARG), (dict(grad=at(1) + 2), E_ARG), (dict(gt=3), E_ARG),
                    (dict(gt=-1), E_ARG), (dict(pt=7), E_ARG), (dict(gt=1, grad=at(1) + 1), E_ARG), (dict(out=at(2) + 1), E_ARG), (dict(m=at(4) + 2), E_ARG),
                    (dict(v=at(5) + 3), E_ARG), (dict(master=at(6) + 2), E_ARG), (dict(out=at(1) + 4), E_ARG), (dict(out=at(1) - 396), E_ARG),
                    (dict(ls=math.nan), E_ARG), (dict(ds=math.inf), E_ARG)):
    make([tensor(), tensor(**bad)], status)
make(4 * [tensor(n=1 << 40, out=None)], E_SHAPE)      # more units than 31 bits count
make([], E_SHAPE, count=-1)
make([], E_SHAPE, count=(1 << 20) + 1)
h = ctypes.c_void_p(77)
assert L.fs_tensors_create(None, 3, None, ctypes.byref(h)) == E_ARG and h.value is None
assert L.fs_tensors_create(None, 0, None, None) == E_ARG
assert S.stub_live_blocks() == 0 and names() == []
# what is allowed: empty tensors whatever their pointers, in place, apart by a hair, 16-bit tensors at even addresses, no parameters
for good in (dict(n=0, grad=None, gt=9), dict(out=None), dict(out=at(1)), dict(out=at(1) + 400), dict(out=at(1) - 400),
             dict(gt=1, grad=at(1) + 2, out=None), dict(param=None, m=None, v=None, pt=9)):
    L.fs_tensors_destroy(make([tensor(**good)]))
assert S.stub_live_blocks() == 0 and S.stub_bad_frees() == 0
assert error(None) == "null list" and L.fs_tensors_destroy(None) == OK
""", tmp_path)


def test_calls_that_are_refused(tmp_path):
    run("""
h = make([tensor(), tensor(out=None)])
S.stub_clear_launches()
for st, what in ((norm(h, 2), "kind"), (norm(h, scale=0.0), "grad_scale"), (norm(h, scale=math.nan), "grad_scale"), (norm(h, d=None), "d_norm"),
                 (norm(h, d=ctypes.c_void_p(at(7) + 2)), "d_norm"), (clip(h, kind=-1), "kind"), (clip(h, max_norm=-1.0), "max_norm"),
                 (clip(h, max_norm=math.nan), "max_norm"), (clip(h, scale=math.inf), "grad_scale"), (clip(h, given=2), "norm_given"), (clip(h, d=None), "d_norm"),
                 (adamw(h, None), "how"), (adamw(h, how(lr=math.nan)), "lr"), (adamw(h, how(wd=math.inf)), "weight_decay"), (adamw(h, how(b1=1.0)), "betas"),
                 (adamw(h, how(b2=-0.1)), "betas"), (adamw(h, how(b2=math.nan)), "betas"), (adamw(h, how(eps=-1.0)), "eps"), (adamw(h, how(max_norm=-0.5)), "max_norm"),
                 (adamw(h, how(scale=-1.0)), "grad_scale"), (adamw(h, how(given=5)), "norm_given"), (adamw(h, how(skip=2)), "skip_nonfinite"),
                 (adamw(h, how(), d=None), "d_norm"), (adamw(h, how(max_norm=math.inf, skip=1), d=None), "d_norm"), (adamw(h, how(max_norm=math.inf, given=1), d=None), "d_norm"),
                 (adamw(h, how(), step=None), "d_step"), (adamw(h, how(), step=ctypes.c_void_p(at(8) + 4)), "d_step"), (adamw(h, how(d_lr=at(9) + 1)), "d_lr")):
    assert st == E_ARG, (st, what)
for st in (norm(h, 2), clip(h, given=2), adamw(h, how(lr=math.nan))):
    pass
assert "lr" in error(h)
for call in (lambda h: norm(h), lambda h: clip(h), lambda h: adamw(h, how()), lambda h: L.fs_tensors_update(h, None, 0), lambda h: L.fs_tensors_set_stream(h, None)):
    assert call(None) == E_ARG
for missing in (dict(param=None, m=None, v=None), dict(m=None), dict(v=None)):
    g = make([tensor(), tensor(**missing)])
    S.stub_clear_launches()
    assert adamw(g, how()) == E_STATE and "exp_avg" in error(g) and names() == []
    assert norm(g) == OK
    L.fs_tensors_destroy(g)
S.stub_clear_launches()
# an update that is refused changes nothing
a = (Tensor * 2)(tensor(), tensor(grad=None))
assert L.fs_tensors_update(h, a, 1) == E_SHAPE and L.fs_tensors_update(h, a, 2) == E_ARG and "tensor 1" in error(h) and L.fs_tensors_update(h, None, 2) == E_ARG
assert names() == []
""", tmp_path)


def test_launches(tmp_path):
    run("""
h = make([])
S.stub_clear_launches()
assert norm(h) == OK and clip(h) == OK and adamw(h, how()) == OK
kinds = lambda ls: [l[0].split("<")[0] for l in ls]
ls = launched()
assert kinds(ls) == ["k_norm_short", "k_clip_short", "k_adamw_short"] and all(l[1][0] == 1 for l in ls)      # norm 0; the step counts
h = make([tensor(n=0, grad=None)] + 100 * [tensor(n=1)])
assert [n for n in names() if n == "k_list_put"] == 3 * ["k_list_put"]       # 40 tensors at a time
assert norm(h, 1) == OK and adamw(h, how(max_norm=math.inf), d=None) == OK and adamw(h, how(given=1)) == OK and clip(h, given=1, kind=9) == OK
ls = launched()
assert kinds(ls) == ["k_norm", "k_adamw", "k_adamw", "k_clip"] and all(1 <= l[1][0] <= 4096 and l[2] == (256, 1, 1) for l in ls)
a = (Tensor * 101)(*(101 * [tensor(n=5)]))
assert L.fs_tensors_update(h, a, 101) == OK and names() == 3 * ["k_list_put"]
# blocks never outnumber the partial sums, however long the list and large the device
h = make([tensor(n=1 << 40, out=None)])
S.stub_clear_launches()
assert norm(h) == OK
assert launched()[0][1][0] <= 4096
""", tmp_path)


def test_failures_leave_nothing_behind(tmp_path):
    run("""
for n in range(2):
    S.stub_fail_allocation(n)
    h = ctypes.c_void_p(77)
    st = L.fs_tensors_create((Tensor * 1)(tensor()), 1, None, ctypes.byref(h))
    assert st == (E_ALLOC if n == 0 else OK)
    if st == OK: L.fs_tensors_destroy(h)
    else: assert h.value is None
    S.stub_fail_allocation(-1)
assert S.stub_live_blocks() == 0
for n in range(2):
    S.stub_fail_launch(n)
    make([tensor()], E_DEVICE)
    S.stub_fail_launch(-1)
assert S.stub_live_blocks() == 0 and S.stub_bad_frees() == 0
h = make([tensor()])
for call in (norm, clip, lambda h: adamw(h, how())):
    S.stub_fail_launch(0)
    assert call(h) == E_DEVICE and "stub" in error(h)
    S.stub_fail_launch(-1)
    assert call(h) == OK
assert S.stub_memsets() == 0
# a list that has not reached the device is not worked on
a = (Tensor * 1)(tensor(n=7))
S.stub_fail_launch(0)
assert L.fs_tensors_update(h, a, 1) == E_DEVICE
S.stub_fail_launch(-1)
S.stub_clear_launches()
for call in (norm, clip, lambda h: adamw(h, how())):
    assert call(h) == E_STATE and "reached" in error(h)
assert names() == []
assert L.fs_tensors_update(h, a, 1) == OK and norm(h) == OK
""", tmp_path)


def test_tensors_on_the_cpu_are_refused():
    from paper_2211_15601_amd import optim
    with pytest.raises(ValueError, match="GPU"):
        optim.TensorList([torch.ones(3)])
    with pytest.raises(ValueError, match="GPU"):
        optim.AdamW([torch.ones(3)])


def test_structs_match_the_header():
    import ctypes
    from paper_2211_15601_amd import binding
    assert ctypes.sizeof(binding.Tensor) == 6 * 8 + 8 + 2 * 4 + 2 * 4 and ctypes.sizeof(binding.AdamW) == 7 * 8 + 2 * 4 + 8
