"""Which rows go four heads to a group of lanes in rotation and append (csrc/paged_rules.hpp), without a GPU."""
import ctypes as C
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06833_amd", "csrc")


def test_four_heads_to_a_group_only_where_that_is_the_faster(tmp_path):
    (tmp_path / "r.cpp").write_text('#include "paged_rules.hpp"\nextern "C" int wide(long rows, long heads, int hd, int bytes) { return ead::rotate_wide(rows, heads, hd, bytes); }\n')
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(tmp_path / "r.so"), str(tmp_path / "r.cpp")], check=True)
    wide = C.CDLL(str(tmp_path / "r.so")).wide
    wide.argtypes = [C.c_long, C.c_long, C.c_int, C.c_int]
    for rows, heads, hd, bytes_ in ((3272, 40, 128, 2), (6552, 40, 64, 2)):
        assert not wide(rows, heads, hd, bytes_) and wide(rows + 8, heads, hd, bytes_)
    for rows in (1, 3272, 10 ** 5, 10 ** 7):
        assert not wide(rows, 16, 32, 2)                      # short vectors: sines and cosines are few beside what is moved
        assert not any(wide(rows, 40, hd, 4) for hd in (32, 64, 128))
