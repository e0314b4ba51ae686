"""Host code of the calls on a list of tensors beside graphs that are captured, and on devices of other sizes, without a GPU: host_path.py on
host_capture_stub.c."""
import os
import subprocess
import sys

import host_path
from test_host_train import CHILD

STREAMS = """
A, B = ctypes.c_void_p(0x1000), ctypes.c_void_p(0x2000)
def capture(stream, number, failed=0):
    S.stub_capture(stream, ctypes.c_ulonglong(number), failed)
def array(*tensors):
    return (Tensor * len(tensors))(*tensors)
calls = (norm, clip, lambda h: adamw(h, how()))
"""


def run(code, tmp_path):
    stub = os.path.join(str(tmp_path), "host_stub.so")
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                           os.path.join(host_path.HERE, "host_capture_stub.c"), "-o", stub])
    env = dict(os.environ, FS_HOST_STUB=stub, PYTHONPATH=host_path.HERE)
    r = subprocess.run([sys.executable, "-c", "from host_path import *\n" + CHILD + STREAMS + code + "\nprint('CHILD-OK')"], env=env,
                       capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and "CHILD-OK" in r.stdout, (r.stdout + r.stderr)[-3000:]


def test_a_recorded_update_is_of_its_graph_alone(tmp_path):
    """Until the graph is replayed the device has another list than the host: neither eager calls nor other graphs may go by it."""
    run("""
h = make([tensor(n=1 << 20), tensor()])
other = array(tensor(n=5), tensor(n=0, grad=None))
assert L.fs_tensors_set_stream(h, A) == OK and norm(h) == OK
capture(A, 7)
assert norm(h) == OK                                        # recorded, with the list as it was
assert L.fs_tensors_update(h, other, 2) == OK
for call in calls:
    assert call(h) == OK
capture(A, 0)                                               # the capture has ended
S.stub_clear_launches()
for call in calls:
    assert call(h) == E_STATE and "graph" in error(h)
capture(A, 8)                                               # another one
for call in calls:
    assert call(h) == E_STATE and "graph" in error(h)
assert names() == []
assert L.fs_tensors_update(h, other, 2) == OK and names() == ["k_list_put"]
for call in calls:
    assert call(h) == OK
capture(B, 8)                                               # a second stream of the same capture
assert L.fs_tensors_set_stream(h, B) == OK
for call in calls:
    assert call(h) == OK
capture(A, 8, 1), capture(B, 8, 1)                          # it has failed
for call in calls:
    assert call(h) == E_STATE
capture(A, 0), capture(B, 0)
S.stub_clear_launches()
for call in calls:
    assert call(h) == E_STATE
assert names() == []
# an update that runs makes all calls right again, whatever the stream
for stream in (A, None):
    assert L.fs_tensors_set_stream(h, stream) == OK and L.fs_tensors_update(h, other, 2) == OK
    for call in calls:
        assert call(h) == OK
""", tmp_path)


def test_a_list_says_whether_calls_would_find_it(tmp_path):
    run("""
h = make([tensor()])
other = array(tensor(n=5))
ready = L.fs_tensors_ready
assert ready(h) == OK and ready(None) == E_ARG
assert L.fs_tensors_set_stream(h, A) == OK
capture(A, 7)
assert ready(h) == OK and L.fs_tensors_update(h, other, 1) == OK and ready(h) == OK
assert L.fs_tensors_set_stream(h, B) == OK and ready(h) == E_STATE and "graph" in error(h)
capture(B, 7)
assert ready(h) == OK
capture(B, 8)
assert ready(h) == E_STATE
capture(B, 0)
assert ready(h) == E_STATE and L.fs_tensors_update(h, other, 1) == OK and ready(h) == OK
S.stub_fail_launch(0)
assert L.fs_tensors_update(h, other, 1) == E_DEVICE
S.stub_fail_launch(-1)
assert ready(h) == E_STATE and "graph" not in error(h)
""", tmp_path)


def test_a_list_in_memory_of_the_callers(tmp_path):
    run("""
L.fs_tensors_bytes.restype = ctypes.c_int64
need = L.fs_tensors_bytes
assert need(-1) == need((1 << 20) + 1) == 0 and 0 < need(0) <= 27000 and need(1000) <= need(0) + 1000 * 84 + 256

def noalloc(tensors, status=OK, at=buf(20), size=None, count=None):
    h = ctypes.c_void_p(77)
    n = len(tensors) if count is None else count
    st = L.fs_tensors_create_noalloc(array(*tensors, tensor()), n, A, at, ctypes.c_int64(need(n) if size is None else size), ctypes.byref(h))
    assert st == status and (h.value is None) == (status != OK), st
    return h

one = [tensor()]
noalloc(one, E_ARG, at=None), noalloc(one, E_ARG, at=ctypes.c_void_p(buf(20).value + 128)), noalloc(one, E_ARG, size=need(1) - 1), noalloc(one, E_ARG, size=-1)
noalloc([], E_SHAPE, count=-1), noalloc([], E_SHAPE, count=(1 << 20) + 1), noalloc([tensor(n=-1)], E_SHAPE), noalloc([tensor(grad=None)], E_ARG)
h = ctypes.c_void_p(77)
assert L.fs_tensors_create_noalloc(None, 1, A, buf(20), ctypes.c_int64(1 << 20), ctypes.byref(h)) == E_ARG and h.value is None
assert L.fs_tensors_create_noalloc(array(tensor()), 1, A, buf(20), ctypes.c_int64(1 << 20), None) == E_ARG
assert names() == []
S.stub_fail_allocation(0)                                   # it asks for none
capture(A, 3)
for tensors in ([], one, 101 * one):
    h = noalloc(tensors)
    assert names() == max(1, -(-len(tensors) // 40)) * ["k_list_put"]      # the first one clears the counters
    assert norm(h) == OK and clip(h) == OK and adamw(h, how()) == OK
    capture(A, 4)
    assert norm(h) == E_STATE and "graph" in error(h)
    capture(A, 3)
    S.stub_clear_launches()
    assert L.fs_tensors_destroy(h) == OK
S.stub_fail_launch(0)
noalloc(one, E_DEVICE)
S.stub_fail_launch(-1)
assert S.stub_live_blocks() == 0 and S.stub_bad_frees() == 0
""", tmp_path)


def test_a_list_that_cannot_be_freed_stays(tmp_path):
    """As while a graph is captured: the call can be made again."""
    run("""
h = make([tensor()])
S.stub_refuse_free(1)
for _ in range(2):
    assert L.fs_tensors_destroy(h) == E_DEVICE and error(h) and S.stub_live_blocks() == 1
S.stub_refuse_free(0)
assert norm(h) == OK                                        # and no error is left for the next call
assert L.fs_tensors_destroy(h) == OK and S.stub_live_blocks() == 0 and S.stub_bad_frees() == 0
""", tmp_path)


def test_blocks_never_outnumber_the_partial_sums(tmp_path):
    """Whatever the device and the list: 2048 of them lie in front of the counters, and a block of the norm writes one."""
    run("""
sizes = (40 * 2048, 300 * 2048, 4100 * 2048, 20000 * 2048, 66000 * 2048, 1 << 40)
most = 0
for units in (1, 64, 256, 304, 512, 513, 1000, 4096):
    S.stub_compute_units(units)
    for n in sizes:
        for gt in (0, 1):
            h = make([tensor(n=n, gt=gt, out=None)])
            S.stub_clear_launches()
            assert norm(h) == OK and norm(h, 1) == OK and clip(h) == OK and adamw(h, how()) == OK
            ls = launched()
            assert [l[0].split("<")[0] for l in ls] == ["k_norm", "k_norm", "k_norm", "k_clip", "k_norm", "k_adamw"]
            blocks = [l[1][0] for l in ls if l[0].startswith("k_norm")]
            assert all(1 <= b <= 2048 for b in blocks) and all(l[2] == (256, 1, 1) for l in ls), (units, n, blocks)
            most = max([most] + blocks)
            L.fs_tensors_destroy(h)
assert most == 2048                                         # the bound is reached
""", tmp_path)


def test_every_refusal_names_its_reason(tmp_path):
    run("""
h = make([tensor(), tensor(out=None)])
for call, what in ((lambda: norm(h, 2), "kind"), (lambda: norm(h, scale=0.0), "grad_scale"), (lambda: norm(h, d=None), "d_norm"), (lambda: clip(h, kind=-1), "kind"),
                   (lambda: clip(h, max_norm=-1.0), "max_norm"), (lambda: clip(h, scale=math.inf), "grad_scale"), (lambda: clip(h, given=2), "norm_given"),
                   (lambda: clip(h, d=None), "d_norm"), (lambda: adamw(h, None), "how"), (lambda: adamw(h, how(lr=math.nan)), "lr"), (lambda: adamw(h, how(wd=math.inf)), "weight_decay"),
                   (lambda: adamw(h, how(b1=1.0)), "betas"), (lambda: adamw(h, how(b2=math.nan)), "betas"), (lambda: adamw(h, how(eps=-1.0)), "eps"),
                   (lambda: adamw(h, how(max_norm=-0.5)), "max_norm"), (lambda: adamw(h, how(scale=-1.0)), "grad_scale"), (lambda: adamw(h, how(given=5)), "norm_given"),
                   (lambda: adamw(h, how(skip=2)), "skip_nonfinite"), (lambda: adamw(h, how(), d=None), "d_norm"), (lambda: adamw(h, how(), step=None), "d_step"),
                   (lambda: adamw(h, how(d_lr=at(9) + 1)), "d_lr")):
    S.stub_clear_launches()
    assert call() == E_ARG and what in error(h) and names() == [], (what, error(h))
""", tmp_path)
