"""The alignment of the local memory that an eviction's choice uses, without a GPU: from the object that is built for it."""
import os
import re
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06833_amd", "csrc")


def test_dynamic_local_memory_is_aligned_to_its_accesses(tmp_path):
    """Ranks are stored four at a time (16 bytes) and the words behind them are 64 bits: the array says so itself, whatever static arrays lie before it."""
    (tmp_path / "e.hip").write_text('#include "evict.hpp"\ntemplate <typename T> struct show;\nvoid f() { (void)(void *)ead::k_evict_choose; }\n')
    subprocess.run(["hipcc", "--offload-arch=gfx950", "--offload-device-only", "-O1", "-std=c++17", "-w", "-S", "-emit-llvm", "-Xclang", "-disable-llvm-passes", "-I", CSRC,
                    str(tmp_path / "e.hip"), "-o", str(tmp_path / "e.ll")], check=True)
    text = (tmp_path / "e.ll").read_text()
    arrays = [l for l in text.splitlines() if re.match(r"@\S*lds\S* = external .*addrspace\(3\) global \[0 x i32\]", l)]
    assert len(arrays) == 1 and int(re.search(r"align (\d+)", arrays[0]).group(1)) >= 16, arrays
