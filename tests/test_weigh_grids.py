"""Grids of the simple weighing kernel for page tables and bounds of up to 2^31 positions (csrc/paged_rules.hpp), without a GPU."""
import ctypes as C
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06833_amd", "csrc")


def test_a_launch_counts_its_threads_in_32_bits(tmp_path):
    (tmp_path / "r.cpp").write_text('#include "paged_rules.hpp"\nextern "C" unsigned groups(int held) { return ead::weigh_simple_groups(held); }\n')
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(tmp_path / "r.so"), str(tmp_path / "r.cpp")], check=True)
    groups = C.CDLL(str(tmp_path / "r.so")).groups
    groups.restype = C.c_uint
    for held in (1, 15, 16, 17, 300, 1 << 24, (1 << 24) + 1, 1 << 28, (1 << 28) + 1, 1 << 29, 0x7FFFFF00):
        n = groups(held)
        assert 1 <= n * 256 < 2 ** 32
        assert n * 16 >= held or n == 1 << 20                 # every key has a workgroup, or the workgroups go on past their grid
    # the source launches what the rule says
    text = open(os.path.join(CSRC, "paged_steps.hip")).read()
    assert "dim3 grid(weigh_simple_groups(held)" in text
