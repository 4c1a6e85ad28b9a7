"""What the adapters' kernels tell the compiler of their memory accesses: in its intermediate form of csrc/adapters.hip, before it
optimises anything (no GPU)."""
import functools
import os
import re
import subprocess

from paper_2310_03675_amd import build


@functools.lru_cache(None)
def functions():
    """Name -> body of every device function."""
    cmd = [os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), *(f for f in build.HIPCC_FLAGS if f not in ("-shared", "-O3")), "-O1", "-Xclang",
           "-disable-llvm-passes", "--cuda-device-only", "-emit-llvm", "-S", os.path.join(build.CSRC, "adapters.hip"), "-o", "-"]
    text = subprocess.run(cmd, capture_output=True, text=True, check=True).stdout
    return dict(re.findall(r"^define [^\n]*?@(\S+?)\([^\n]*\{\n(.*?)^\}", text, re.S | re.M))


def test_a_waves_turns_in_lds_are_in_order():
    """A step's pieces are there before other lanes of the wave take them, and taken before the next step's are put over them; rows of
    a group are counted 64 after 64."""
    ordered = [body for name, body in functions().items() if name.endswith("wave_in_orderEv")]
    assert len(ordered) == 1
    assert re.search(r'fence syncscope\("wavefront"\) release.*wave\.barrier.*fence syncscope\("wavefront"\) acquire', ordered[0], re.S)
    calls = {name: body.count("wave_in_orderEv()") for name, body in functions().items()}
    # Down<type, tiles of ranks, mode, SHORT>::tile; SHORT goes without LDS
    tiles = {name: re.search(r"4DownILi(\d)ELi(\d)ELi(\d)ELb(\d)EE4tileERKNS0_8DownArgsERKNS0_5GroupEjPc$", name) for name in calls}
    with_lds = [name for name, m in tiles.items() if m and m[4] == "0"]
    assert len(with_lds) == 16 and all(calls[name] == 2 for name in with_lds)
    assert [n for name, n in calls.items() if "12look_through" in name] == [1]


def test_h_is_loaded_from_any_of_its_values_on():
    """Of a rank that is no multiple of a load the last lanes begin at its end minus a load: at 4 or 8 bytes."""
    bodies = [body for name, body in functions().items() if "6load_hI" in name]
    assert len(bodies) == 3
    for body in bodies:
        copies = re.findall(r"@llvm\.memcpy[^(]*\([^,]*, ptr align (\d+) [^,]*, i64 16,", body)
        assert copies == ["4", "4"], copies
