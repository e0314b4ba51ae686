"""What the compiler made of the layers' kernels, from the metadata of the code objects built here: none keeps registers in scratch memory, none has more LDS
than a compute unit, and those whose launch rules count on several blocks a compute unit can have them."""
import re
import subprocess

import host_path

LLVM = "/opt/rocm/llvm/bin/"


def kernels(tmp_path):
    """{name with template arguments: {field: number}} of every code object in the library (one for each source file)"""
    fat = str(tmp_path / "fat")
    subprocess.check_call(["objcopy", "-O", "binary", "--only-section=.hip_fatbin", host_path.LIB, fat])
    data = open(fat, "rb").read()
    at = [m.start() for m in re.finditer(b"__CLANG_OFFLOAD_BUNDLE__", data)] + [len(data)]
    out = {}
    for i, (a, b) in enumerate(zip(at, at[1:])):
        one, obj = tmp_path / f"fat{i}", str(tmp_path / f"obj{i}")
        one.write_bytes(data[a:b])
        subprocess.check_call([LLVM + "clang-offload-bundler", "--unbundle", "--type=o", "--input=" + str(one), "--output=" + obj, "--targets=hipv4-amdgcn-amd-amdhsa--gfx950"])
        notes = subprocess.check_output([LLVM + "llvm-readelf", "--notes", obj], text=True)
        for part in notes.split("- .agpr_count:")[1:]:
            name = subprocess.check_output(["c++filt", re.search(r"\.symbol:\s*(\S+)\.kd", part).group(1)], text=True)
            name = re.match(r"(?:void )?fs::(\w+(?:<[^(]*>)?)\(", name)
            if name:
                field = lambda f: int(re.search(rf"\.{f}:\s*(\d+)", part).group(1))
                out[name.group(1).replace(" ", "")] = {f: field(f) for f in ("vgpr_count", "vgpr_spill_count", "private_segment_fixed_size", "group_segment_fixed_size")}
    return out


def test_registers(tmp_path):
    ks = {n: k for n, k in kernels(tmp_path).items() if re.match(r"k_(few|product|product_big|parts|narrow|narrow_end|dz|dbias|dropout)<", n)}
    assert len(ks) > 50
    spilled = {n: k for n, k in ks.items() if k["vgpr_spill_count"] or k["private_segment_fixed_size"]}
    assert not spilled, spilled
    assert all(k["group_segment_fixed_size"] <= 160 << 10 for k in ks.values())
    waves = lambda k: 512 // (-(-k["vgpr_count"] // 8) * 8)
    for n, k in ks.items():
        if n.startswith("k_few<"):                      # blocks of up to 16 waves
            assert waves(k) >= 4, (n, k)
        if re.match(r"k_product<0,true,false,128,128,2,2", n):     # fp32, dX: three blocks of four waves
            assert waves(k) >= 3 and 3 * k["group_segment_fixed_size"] <= 160 << 10, (n, k)
        if re.match(r"k_product<\d,false,false,128,128,2,4", n):   # forward: two blocks of eight
            assert waves(k) >= 3 and 2 * k["group_segment_fixed_size"] <= 160 << 10, (n, k)
        if n.startswith(("k_product_big<", "k_narrow<0")):        # eight waves
            assert waves(k) >= 2, (n, k)
