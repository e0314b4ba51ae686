"""How many blocks the narrow layers' backward pass launches: no more than compute units hold at once, from the code objects built here and the launches on the stub runtime."""
import re

from test_host_net import run
from test_net_registers import kernels


def test_narrow_blocks_are_there_at_once(tmp_path):
    run("""
# (the stub's device has as many compute units as it says; rows for more blocks than that)
for type, per_unit in ((0, 1), (1, 2), (2, 2)):
    l = layer(rows=131072, inputs=128, outputs=128, type=type, act=4)
    names()
    assert backward(l) == OK, error()
    (n, g, b, lds) = launched()[0]
    assert n.startswith("k_narrow<") and g[0] % per_unit == 0, n
    open("DIR/units%d" % type, "w").write(str(g[0] // per_unit))
""".replace("DIR", str(tmp_path)), tmp_path)
    units = [int((tmp_path / f"units{t}").read_text()) for t in range(3)]
    assert units[0] == units[1] == units[2]            # compute units
    found = 0
    for n, k in kernels(tmp_path).items():
        m = re.match(r"k_narrow<(\d),128,(\d+),", n)
        if m:
            waves, per_unit = int(m.group(2)), 1 if m.group(1) == "0" else 2
            each = 512 // (-(-k["vgpr_count"] // 8) * 8)                  # waves a SIMD, of four
            assert per_unit * waves <= 4 * each and per_unit * k["group_segment_fixed_size"] <= 160 << 10, (n, k)
            found += 1
    assert found == 5
