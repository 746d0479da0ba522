"""What the hand-over of a row's sums between workgroups (draw_whole_kernel) counts on: the target it is
compiled for, and the order in which the compiler left its steps in the built library.  Needs no GPU."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2605_29707_amd import binding as bd, build

LLVM = "/opt/rocm/llvm/bin/"


@pytest.mark.parametrize("arch,ok", [("gfx950", True), ("gfx90a", False), ("gfx1100", False)])
def test_other_targets_do_not_compile(tmp_path, arch, ok):
    """Stores that a thread's vector-memory count covers, and that pass the caches of an XCD: this chip's."""
    src = tmp_path / "t.hip"
    src.write_text('#include "common.h"\n__global__ void k(float *p) { st_coherent(p, 1.f); }\n')
    r = subprocess.run([build.hipcc(), "-std=c++17", f"--offload-arch={arch}", "--offload-device-only", "-fsyntax-only",
                        "-I", build.CSRC, str(src)], capture_output=True, text=True)
    assert (r.returncode == 0) == ok and ("gfx950" in r.stderr) == (not ok), r.stderr


def test_sums_are_stored_before_they_are_counted(tmp_path):
    """Both variants: the last store of sums, a wait for all of the thread's stores, the workgroup's barrier, the
    count, a wait for it, and only then the loads of the others' sums; nothing between that moves one past another."""
    if not os.path.exists(LLVM + "llvm-objdump"):
        pytest.skip("no LLVM tools")
    shutil.copy(bd.LIB_PATH, tmp_path / "lib.so")
    subprocess.run([LLVM + "llvm-objdump", "--offloading", "lib.so"], cwd=tmp_path, check=True, capture_output=True)
    found = 0
    for f in sorted(tmp_path.glob("*gfx950*")):
        if b"draw_whole_kernel" not in f.read_bytes():
            continue
        text = subprocess.run([LLVM + "llvm-objdump", "-d", "--no-show-raw-insn", str(f)], capture_output=True, text=True).stdout
        for name, body in re.findall(r"^[0-9a-f]+ <(\S*draw_whole_kernel\S*)>:\n((?:\t.*\n|\n)*)", text, re.M):
            ops = [line.split("//")[0].strip() for line in body.splitlines()]
            adds = [i for i, o in enumerate(ops) if o.startswith("global_atomic_add ")]
            assert len(adds) == 1, (name, adds)
            stores = [i for i, o in enumerate(ops) if o.startswith("global_store_dword") and o.endswith("sc1")]
            loads = [i for i, o in enumerate(ops) if o.startswith("global_load_dword") and o.endswith("sc1")]
            waits = [i for i, o in enumerate(ops) if o.startswith("s_waitcnt") and "vmcnt(0)" in o]
            barriers = [i for i, o in enumerate(ops) if o == "s_barrier"]
            last = max(stores)
            wait = min(i for i in waits if i > last)
            barrier = min(i for i in barriers if i > last)
            assert last < wait < barrier < adds[0], (name, last, wait, barrier, adds)
            counted = min(i for i in waits if i > adds[0])
            assert min(i for i in barriers if i > counted) < min(loads), (name, counted, loads[:3])
            found += 1
    assert found == 2
