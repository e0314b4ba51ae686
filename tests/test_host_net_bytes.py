"""What the layers' calls ask for as workspace, without a GPU (host_path.py)."""
from test_host_net import run


def test_narrow_layers_ask_for_what_they_use(tmp_path):
    """One pass over the rows: parts of dweight and dbias for each block, at most 1024 of them, and no dZ."""
    run("""
for type in range(3):
    for rows in (1, 1000, 131072) + ((5 * 10 ** 8,) if type == 0 else ()):
        for inputs, outputs in ((128, 128), (1, 128), (128, 1), (3, 64)):
            for act, p in ((0, 0.0), (4, 0.0), (2, 0.5)):
                l = layer(rows=rows, inputs=inputs, outputs=outputs, type=type, act=act, p=p)
                need = L.fs_linear_bytes(ctypes.byref(l), 1)
                assert 0 < need <= 1024 * 4 * outputs * (inputs + 3 + 1) + 512, (type, rows, inputs, outputs, need)
                if rows < 10 ** 6:
                    names()
                    assert backward(l) == OK, error()
                    assert [n.split("<")[0] for n in names()] == ["k_narrow", "k_narrow_end"]
                    assert backward(l, bytes=need - 1) == E_ARG
# the others have dZ, the sums of its columns and the products' parts; also narrow ones that have nothing to go over
l = layer(rows=1000, inputs=300, outputs=200, act=2)
assert L.fs_linear_bytes(ctypes.byref(l), 1) >= 1000 * 200 * 4
for empty in (dict(rows=0), dict(inputs=0), dict(outputs=0)):
    l = layer(**{**dict(rows=100, inputs=20, outputs=30, act=2), **empty})
    need = L.fs_linear_bytes(ctypes.byref(l), 1)
    assert need >= l.rows * l.outputs * 4
    names()
    assert backward(l) == OK, error()
    assert "k_narrow" not in [n.split("<")[0] for n in names()]
""", tmp_path)


def test_where_fp16_is_scaled(tmp_path):
    """The largest |G| is looked for where dZ is made, of fp16 and by itself, in memory of the workspace behind all else."""
    run("""
ends = lambda: [n.split("<")[0] for n in names()]
for type in range(3):
    for act, p in ((0, 0.0), (1, 0.0), (0, 0.5)):
        for rows, outputs in ((5000, 200), (0, 200), (5000, 0)):
            l = layer(rows=rows, inputs=300, outputs=outputs, act=act, p=p, type=type)
            dz = (act != 0 or p > 0.0) and outputs > 0
            names()
            assert backward(l) == OK, error()
            assert ends().count("k_largest") == (dz and type == 2), (type, act, p, rows, outputs)
            assert backward(l, dx=None, dw=None) == OK and "k_largest" not in ends()           # dbias is made from dZ in fp32
sizes = [L.fs_linear_bytes(ctypes.byref(layer(rows=5000, act=1, type=t)), 1) for t in (1, 2)]
assert sizes[1] == sizes[0] + 256 + 4096
""", tmp_path)
