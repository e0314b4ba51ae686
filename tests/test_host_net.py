"""Host code of the networks' layers without a GPU (host_path.py): what the C calls refuse, what they launch."""
import host_path

CHILD = """
import math

class Drop(ctypes.Structure):
    _fields_ = [("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64), ("d_seed", ctypes.c_void_p)]

class Layer(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int64) for n in ("rows", "inputs", "outputs")] + [(n, ctypes.c_int32) for n in ("type", "bias_type", "act")] + \\
               [("beta", ctypes.c_float), ("drop", Drop)]

L.fs_net_error.restype = ctypes.c_char_p
L.fs_linear_bytes.restype = ctypes.c_int64
i64 = ctypes.c_int64

def at(i, off=0):
    return None if i is None else 0x300000000000 + (i << 40) + off

def layer(rows=1000, inputs=300, outputs=200, type=0, bias_type=None, act=0, beta=1.0, p=0.0, d_seed=None):
    return Layer(rows, inputs, outputs, type, type if bias_type is None else bias_type, act, beta, Drop(p, 1, 2, d_seed))

X, W, B, R, Y, Z, WORK, G, DX, DW, DB = range(1, 12)

def forward(l, x=at(X), ldx=None, w=at(W), ldw=None, b=at(B), r=at(R), ldr=None, y=at(Y), ldy=None, z=at(Z), ldz=None, work=at(WORK), bytes=None):
    n = lambda v, d: i64(d if v is None else v)
    need = L.fs_linear_bytes(ctypes.byref(l), 0)
    p = ctypes.c_void_p
    return L.fs_linear_forward(ctypes.byref(l), p(x), n(ldx, l.inputs), p(w), n(ldw, l.inputs), p(b), p(r), n(ldr, l.outputs), p(y), n(ldy, l.outputs), p(z), n(ldz, l.outputs),
                               p(work), n(bytes, max(0, need)), None)

def backward(l, g=at(G), ldg=None, x=at(X), ldx=None, w=at(W), ldw=None, z=at(Z), ldz=None, dx=at(DX), lddx=None, dw=at(DW), lddw=None, db=at(DB), work=at(WORK), bytes=None):
    n = lambda v, d: i64(d if v is None else v)
    need = L.fs_linear_bytes(ctypes.byref(l), 1)
    p = ctypes.c_void_p
    return L.fs_linear_backward(ctypes.byref(l), p(g), n(ldg, l.outputs), p(x), n(ldx, l.inputs), p(w), n(ldw, l.inputs), p(z), n(ldz, l.outputs), p(dx), n(lddx, l.inputs),
                                p(dw), n(lddw, l.inputs), p(db), p(work), n(bytes, max(0, need)), None)

def dropout(type=0, rows=10, cols=20, p=0.5, x=at(X), ldx=20, r=at(R), ldr=20, y=at(Y), ldy=20, d_seed=None):
    d = Drop(p, 1, 2, d_seed)
    q = ctypes.c_void_p
    return L.fs_dropout(type, i64(rows), i64(cols), ctypes.byref(d), q(x), i64(ldx), q(r), i64(ldr), q(y), i64(ldy), None)

def error():
    return L.fs_net_error().decode()
"""


def run(code, tmp_path):
    host_path.run(CHILD + code, tmp_path)


def test_layers_that_are_refused(tmp_path):
    run("""
for bad, status in ((dict(rows=-1), E_SHAPE), (dict(rows=5 * 10 ** 8 + 1), E_SHAPE), (dict(inputs=-1), E_SHAPE), (dict(inputs=(1 << 24) + 1), E_SHAPE), (dict(outputs=-1), E_SHAPE),
                    (dict(outputs=(1 << 24) + 1), E_SHAPE), (dict(type=3), E_ARG), (dict(type=-1), E_ARG), (dict(type=0, bias_type=1), E_ARG), (dict(type=1, bias_type=2), E_ARG),
                    (dict(act=5), E_ARG), (dict(act=-1), E_ARG), (dict(act=4, beta=0.0), E_ARG), (dict(act=4, beta=math.inf), E_ARG), (dict(act=4, beta=math.nan), E_ARG),
                    (dict(p=-0.1), E_ARG), (dict(p=1.1), E_ARG), (dict(p=math.nan), E_ARG)):
    l = layer(**bad)
    assert L.fs_linear_bytes(ctypes.byref(l), 0) == -1 and L.fs_linear_bytes(ctypes.byref(l), 1) == -1, bad
    for call in (forward, backward):
        assert call(l) == status, (bad, error())
        assert "fs_linear" in error()
assert L.fs_linear_bytes(None, 0) == -1
assert L.fs_linear_forward(*[None] * 15) == E_ARG and L.fs_linear_backward(*[None] * 17) == E_ARG
assert forward(layer(rows=5 * 10 ** 8, outputs=1 << 24)) == E_SHAPE and "too many" in error()      # more tiles than a launch has blocks
assert names() == []
for good in (dict(act=0, beta=math.nan), dict(type=1, bias_type=0), dict(type=2), dict(p=1.0), dict(p=0.0), dict(rows=0), dict(inputs=0), dict(outputs=0)):
    assert forward(layer(**good)) == OK and backward(layer(**good)) == OK, (good, error())
""", tmp_path)


def test_arrays_that_are_refused(tmp_path):
    run("""
for bad in (dict(x=None), dict(w=None), dict(y=None), dict(x=at(X, 2)), dict(w=at(W, 1)), dict(b=at(B, 2)), dict(r=at(R, 3)), dict(y=at(Y, 2)), dict(z=at(Z, 2)),
            dict(y=at(X)), dict(y=at(W, 400)), dict(y=at(B, -4)), dict(z=at(Y, 8)), dict(z=at(R)), dict(y=at(R), ldy=201), dict(y=at(R, 4)), dict(y=at(WORK), work=at(WORK))):
    l = layer(rows=40, inputs=3000, outputs=200)       # in parts: with workspace
    assert L.fs_linear_bytes(ctypes.byref(l), 0) > 0
    assert forward(l, **bad) == E_ARG, (bad, error())
for bad in (dict(ldx=-1), dict(ldy=199), dict(ldz=1), dict(ldr=-5)):
    assert forward(layer(), **bad) == E_SHAPE, (bad, error())
for bad in (dict(work=None), dict(work=at(WORK, 4)), dict(bytes=100)):
    assert forward(layer(rows=40, inputs=3000), **bad) == E_ARG, (bad, error())
    assert backward(layer(), **bad) == E_ARG, (bad, error())
assert forward(layer(p=0.5, d_seed=at(20, 4))) == E_ARG and "d_seed" in error()
for bad in (dict(g=None), dict(x=None), dict(w=None), dict(z=None), dict(g=at(G, 2)), dict(dx=at(DX, 2)), dict(dw=at(DW, 1)), dict(db=at(DB, 3)), dict(dx=at(X)), dict(dx=at(G, 16)),
            dict(dw=at(W)), dict(dw=at(DX)), dict(db=at(DW, 40)), dict(dx=at(Z)), dict(dw=at(WORK))):
    assert backward(layer(act=2), **bad) == E_ARG, (bad, error())
for bad in (dict(lddx=299), dict(lddw=10), dict(ldg=-1)):
    assert backward(layer(act=2), **bad) == E_SHAPE, (bad, error())
assert names() == []
# what is allowed
assert forward(layer(), y=at(R)) == OK                                # in place of the residual
assert forward(layer(), b=None, r=None, z=None) == OK
assert forward(layer(), ldx=0, ldw=0, ldr=0) == OK                    # one row, seen again and again
assert forward(layer(type=1), x=at(X, 2), w=at(W, 2), b=at(B, 2), y=at(Y, 2)) == OK
assert forward(layer(rows=1), ldy=3, ldx=1) == OK                     # what lies between rows does not matter where there is one
assert backward(layer(), z=None) == OK
assert backward(layer(act=1), dx=None, w=None) == OK and backward(layer(act=1), dw=None, x=None) == OK and backward(layer(act=1), dx=None, dw=None, x=None, w=None) == OK
assert backward(layer(rows=0), g=None, x=None, z=None) == OK
""", tmp_path)


def test_dropouts_that_are_refused(tmp_path):
    run("""
assert L.fs_dropout(0, i64(1), i64(1), None, *[None] * 7) == E_ARG
for bad, status in ((dict(type=3), E_ARG), (dict(rows=-1), E_SHAPE), (dict(cols=-1), E_SHAPE), (dict(rows=1 << 30, cols=1 << 20), E_SHAPE), (dict(p=-1.0), E_ARG), (dict(p=math.nan), E_ARG),
                    (dict(x=None), E_ARG), (dict(y=None), E_ARG), (dict(x=at(X, 1)), E_ARG), (dict(r=at(R, 2)), E_ARG), (dict(y=at(X, 4)), E_ARG), (dict(y=at(R, -8)), E_ARG),
                    (dict(ldy=19), E_SHAPE), (dict(ldx=-1), E_SHAPE), (dict(y=at(X), ldx=21), E_ARG), (dict(d_seed=at(20, 4)), E_ARG)):
    assert dropout(**bad) == status, (bad, error())
assert names() == []
for good in (dict(y=at(X)), dict(y=at(R)), dict(r=None), dict(rows=0, x=None, y=None), dict(ldx=0), dict(p=1.0), dict(p=0.0), dict(d_seed=at(20))):
    assert dropout(**good) == OK, (good, error())
""", tmp_path)


def test_what_is_launched(tmp_path):
    run("""
def launches(call, l, **k):
    names()
    assert call(l, **k) == OK, error()
    return [(n, g, b) for n, g, b, _ in launched()]

ends = lambda x: [n.split("<")[0] for n, g, b in x]
# few rows: the weights are read once, by one launch
for rows in (1, 4, 5, 8, 17, 32):
    ((n, g, b),) = launches(forward, layer(rows=rows, inputs=4096, outputs=1000))
    assert n.startswith("k_few") and g == (63, 1, 1) and b[0] % 64 == 0 and b[0] <= 1024
for l in (layer(rows=33, inputs=4096, outputs=1000), layer(rows=9, inputs=4096, outputs=16384), layer(rows=2, inputs=11000, outputs=300)):
    assert ends(launches(forward, l))[0] == "k_product"
assert ends(launches(forward, layer(rows=8, inputs=11000, outputs=16384, type=1))) == ["k_few"]
# large ones of 16 bits: the large tile, where the rows lie at multiples of 16 bytes; smaller ones where they do not
big = layer(rows=8192, inputs=4096, outputs=4096, type=1)
((n, g, b),) = launches(forward, big)
assert n.startswith("k_product_big") and g == (512, 1, 1)
((n, g, b),) = launches(forward, big, ldx=4100)
assert n.startswith("k_product<") and g == (2048, 1, 1)
((n, g, b),) = launches(forward, big, w=at(W, 2))
assert n.startswith("k_product<")
# narrow ones: two launches backward
assert ends(launches(backward, layer(rows=5000, inputs=128, outputs=24, act=4))) == ["k_narrow", "k_narrow_end"]
assert ends(launches(backward, layer(rows=5000, inputs=128, outputs=24), dw=None, db=None)) == ["k_narrow"]
# others: dZ with the sums for dbias, both products, their parts
assert ends(launches(backward, layer(rows=50000, inputs=300, outputs=200, act=1))) == ["k_dz", "k_dbias", "k_product", "k_product", "k_parts"]
assert ends(launches(backward, layer(rows=50000, inputs=300, outputs=200), dw=None, db=None)) == ["k_product"]
# nothing to do, or only zeros
assert launches(forward, layer(rows=0)) == [] and launches(forward, layer(outputs=0)) == []
assert [n for n, g, b in launches(backward, layer(rows=0))] and launches(backward, layer(rows=0, inputs=0, outputs=0)) == []
# every grid is within what a launch may have
for l in (layer(rows=5 * 10 ** 8, inputs=1, outputs=1), layer(rows=5 * 10 ** 8, inputs=300, outputs=200, type=1), layer(rows=1, inputs=1 << 20, outputs=1 << 18, type=1), layer(rows=100, inputs=1 << 24, outputs=3)):
    for call in (forward, backward):
        st = call(l)
        assert st in (OK, E_SHAPE), error()
        for n, g, b, _ in launched():
            assert g[0] * b[0] < 1 << 32 and g[1] <= 65535 and g[2] == 1, (n, g, b)
assert dropout(rows=1, cols=1 << 36, ldx=1 << 36, ldy=1 << 36, r=None) == OK, error()
((n, g, b, _),) = launched()
assert g[0] * b[0] < 1 << 32
# a launch that fails is reported by the call
S.stub_fail_launch(0)
assert forward(layer()) == E_DEVICE and "fs_linear_forward" in error()
assert forward(layer()) == OK
assert S.stub_live_blocks() == 0                        # nothing is allocated
""", tmp_path)


def test_z_in_fp32(tmp_path):
    """FS_Z_FULL goes with every act, and changes what Z's elements are aligned to."""
    run("""
for act in range(5):
    for type in range(3):
        l = layer(act=act + 256, type=type)
        assert forward(l) == OK and backward(l) == OK, (act, type, error())
for act in (256 + 5, 256 - 1, 512, 768, -256, -1):
    assert forward(layer(act=act)) == E_ARG and "bad act" in error(), act
assert forward(layer(act=2, type=1), z=at(Z, 2)) == OK
assert forward(layer(act=2 + 256, type=1), z=at(Z, 2)) == E_ARG and "d_z" in error()
assert backward(layer(act=2 + 256, type=1), z=at(Z, 2)) == E_ARG and "d_z" in error()
""", tmp_path)
