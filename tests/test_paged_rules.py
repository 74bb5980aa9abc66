"""Host logic of the paged cache without a GPU: how a call is cut into workgroups, and what the C entry points refuse."""
import ctypes as C
import math
import os
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2502_06833_amd", "csrc")

SRC = r"""
#include "paged_rules.hpp"
#include <cstring>
using namespace ead;
extern "C" {
long rules_keys(int tile_rows, int key_tile, int group, int max_kv, int window, int sinks) { return paged_keys(tile_rows, key_tile, group, max_kv, window, sinks); }
void rules_few(int batch, int n_kv, long rows, int nb, int group, int max_kv, long capacity, int window, int sinks, long resident, long *out) {
    const PagedShares p = paged_few(batch, n_kv, rows, nb, group, max_kv, capacity, window, sinks, resident);
    out[0] = p.row_tiles; out[1] = p.pairs; out[2] = p.units; out[3] = p.groups; out[4] = p.parts;
    out[5] = (long)paged_workspace(p.units, p.parts, 16 * nb, 128);
}
void rules_many(int batch, int n_kv, int group, long rows, int max_kv, int window, int sinks, int cus, int hd, long *out) {
    const PagedPlan p = paged_many(batch, n_kv, group, rows, max_kv, window, sinks, cus, hd);
    out[0] = p.tile_rows; out[1] = p.row_tiles; out[2] = p.splits; out[3] = p.split_tiles; out[4] = p.units;
}
int rules_blocks(int f32, long rows, int nb_max, double work, double kv) { return paged_blocks(f32 != 0, rows, nb_max, work, kv); }
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "r.cpp").write_text(SRC)
    out = d / "r.so"
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(out), str(d / "r.cpp")], check=True)
    L = C.CDLL(str(out))
    L.rules_keys.restype = C.c_long
    L.rules_few.argtypes = [C.c_int, C.c_int, C.c_long, C.c_int, C.c_int, C.c_int, C.c_long, C.c_int, C.c_int, C.c_long, C.POINTER(C.c_long)]
    L.rules_many.argtypes = [C.c_int, C.c_int, C.c_int, C.c_long] + [C.c_int] * 5 + [C.POINTER(C.c_long)]
    L.rules_blocks.argtypes = [C.c_int, C.c_long, C.c_int, C.c_double, C.c_double]
    return L


@pytest.mark.parametrize("group", [1, 4, 7])
@pytest.mark.parametrize("window,sinks", [(1, 0), (5, 4), (100, 0), (100, 33), (4096, 16)])
def test_no_tile_of_rows_sees_more_tiles_of_keys_than_planned(rules, group, window, sinks):
    """The bound on key tiles against a count over the rows, for tiles of rows and of keys as both kernels use them."""
    for tile_rows, key_tile in ((16, 32), (64, 32), (128, 64)):
        for kv in (1, 31, 64, 200, 777, 5000):
            bound = math.ceil(rules.rules_keys(tile_rows, key_tile, group, kv, window, sinks) / key_tile)
            tokens = (tile_rows - 1) // group + 2                          # rows of a tile may start inside a token
            for first in {0, max(0, kv - tokens), kv // 2}:
                last = min(first + tokens - 1, kv - 1)
                lo = max(0, first - window + 1)
                tiles = set(range(lo // key_tile, last // key_tile + 1)) | set(range(0, -(-min(sinks, lo) // key_tile)))
                assert len(tiles) <= bound, (tile_rows, kv, first)


def test_shares(rules):
    def few(*a):
        out = (C.c_long * 6)()
        rules.rules_few(*a, out)
        return list(out)
    # a long context of one sequence is cut, short contexts and too many pairs are not
    row_tiles, pairs, units, groups, parts, ws = few(1, 8, 4, 1, 4, 8192, 8192, 0, 0, 512)
    assert (row_tiles, pairs, units) == (1, 1, 8) and 8 < groups <= 512 and parts == 2 * groups
    assert ws == units * 128 + parts * 16 * (8 + 4 * 128)
    assert few(64, 8, 4, 1, 4, 300, 300, 0, 0, 512)[1] == 0
    assert few(2000, 8, 4, 1, 4, 8192, 8192, 0, 0, 512)[1:] == [0, 16000, 16000, 0, 0]
    # the device counts groups in 30 bits whatever the arrays hold: page tables that reach further are not cut
    assert few(1000, 8, 4, 1, 4, 8192, 1 << 31, 0, 0, 512)[1] == 0
    assert few(1, 1, 0, 1, 4, 0, 16, 0, 0, 512)[0] == 1


@pytest.mark.parametrize("hd", [32, 64, 128])
@pytest.mark.parametrize("rows", [65, 1000, 40000])
@pytest.mark.parametrize("kv", [1, 100, 5000, 10 ** 6])
def test_ranges_of_keys(rules, hd, rows, kv):
    out = (C.c_long * 5)()
    for batch in (1, 30):
        rules.rules_many(batch, 8, 4, rows, kv, 0, 0, 256, hd, out)
        tile_rows, row_tiles, splits, split_tiles, units = list(out)
        assert row_tiles * tile_rows >= rows and units == batch * 8 * row_tiles
        assert splits * split_tiles * 64 >= kv and 1 <= splits <= hd // 4
        assert splits == 1 or split_tiles >= 4


def test_blocks_of_rows(rules):
    assert rules.rules_blocks(0, 16, 4, 1e12, 1e9) == 1
    assert rules.rules_blocks(0, 32, 4, 1e12, 1e9) == 2 and rules.rules_blocks(0, 64, 4, 1e12, 1e9) == 4 and rules.rules_blocks(0, 64, 2, 1e12, 1e9) == 2
    assert rules.rules_blocks(0, 64, 4, 1e9, 1e6) == 1 and rules.rules_blocks(0, 64, 4, 1e9, 1e9) == 4
    assert rules.rules_blocks(1, 64, 4, 1e9, 1e6) == 2 and rules.rules_blocks(1, 64, 4, 1e8, 1e6) == 1


# ---- the C entry points, refused before anything reaches a device
def _objects():
    from paper_2502_06833_amd.paged import AttnDesc, BatchDesc, CacheDesc, Rows
    import paper_2502_06833_amd as ead
    cache = CacheDesc(1, 8, 16, 2, 64, 0x1000, 0x2000, None, None)
    batch = BatchDesc(2, 3, 2, 1, 20, 4, 4, 0x3000, 0x4000, 0x5000)
    attn = AttnDesc(4, 1, 0, 0, 0.125)
    rows = Rows(0x6000, 128, 64)
    return ead.lib(), cache, batch, attn, rows


def _set(obj, **kw):
    for k, v in kw.items():
        setattr(obj, k, v)


INVALID, SHAPE = 1, 2


@pytest.mark.parametrize("status,which,change", [
    (INVALID, "cache", dict(dtype=3)), (SHAPE, "cache", dict(n_pages=0)), (SHAPE, "cache", dict(page_size=24)), (SHAPE, "cache", dict(page_size=8)),
    (SHAPE, "cache", dict(page_size=512)), (SHAPE, "cache", dict(head_dim=96)), (SHAPE, "cache", dict(n_kv_heads=0)), (INVALID, "cache", dict(k=None)),
    (INVALID, "cache", dict(k=0x1008)), (INVALID, "cache", dict(dtype=2)), (INVALID, "cache", dict(k_scale=0x7000, v_scale=0x7000)),
    (INVALID, "cache", dict(dtype=2, k_scale=0x7000)),
    (INVALID, "batch", dict(batch=0)), (INVALID, "batch", dict(batch=70000)), (INVALID, "batch", dict(rows=-1)), (INVALID, "batch", dict(max_q=4)),
    (INVALID, "batch", dict(min_q=3)), (INVALID, "batch", dict(max_kv=-1)), (INVALID, "batch", dict(table_width=0)), (INVALID, "batch", dict(table_stride=3)),
    (INVALID, "batch", dict(page_table=None)), (INVALID, "batch", dict(kv_lens=None)), (SHAPE, "batch", dict(rows=1 << 29)),
    (SHAPE, "attn", dict(n_heads=3)), (SHAPE, "attn", dict(n_heads=0)), (SHAPE, "attn", dict(n_heads=130)), (INVALID, "attn", dict(dtype=0)),
    (INVALID, "attn", dict(window=-1)), (INVALID, "attn", dict(sinks=-1)), (INVALID, "attn", dict(scale=0.0)), (INVALID, "attn", dict(scale=math.inf)),
    (INVALID, "attn", dict(scale=math.nan)),
    (INVALID, "rows", dict(data=None)), (INVALID, "rows", dict(data=0x6001)),
])
def test_refusals(status, which, change):
    L, cache, batch, attn, rows = _objects()
    _set({"cache": cache, "batch": batch, "attn": attn, "rows": rows}[which], **change)
    r = C.byref
    bytes_ = C.c_uint64(7)
    calls = [lambda: L.ead_paged_attention(r(cache), r(batch), r(attn), r(rows), r(rows), None, None, 0, None)]
    if which != "attn":
        calls += [lambda: L.ead_paged_write(r(cache), r(batch), 1, r(rows), r(rows), None), lambda: L.ead_paged_read(r(cache), r(batch), 1, r(rows), r(rows), None)]
    if which != "rows":
        calls += [lambda: L.ead_paged_workspace(r(cache), r(batch), r(attn), r(bytes_))]
    for call in calls:
        assert call() == status
        assert L.ead_last_error(None)


def test_null_arguments():
    L, cache, batch, attn, rows = _objects()
    r = C.byref
    assert L.ead_paged_write(None, r(batch), 1, r(rows), r(rows), None) == INVALID
    assert L.ead_paged_write(r(cache), None, 1, r(rows), r(rows), None) == INVALID
    assert L.ead_paged_write(r(cache), r(batch), 2, r(rows), r(rows), None) == INVALID
    assert L.ead_paged_read(r(cache), r(batch), 1, None, r(rows), None) == INVALID
    assert L.ead_paged_attention(r(cache), r(batch), None, r(rows), r(rows), None, None, 0, None) == INVALID
    assert L.ead_paged_attention(r(cache), r(batch), r(attn), r(rows), None, None, None, 0, None) == INVALID
    assert L.ead_paged_workspace(r(cache), r(batch), r(attn), None) == INVALID
