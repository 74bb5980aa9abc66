"""How the steps around a paged cache's attention are cut into workgroups (csrc/paged_rules.hpp), without a GPU."""
import ctypes as C
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_06833_amd", "csrc")

SRC = r"""
#include "paged_rules.hpp"
using namespace ead;
extern "C" {
void rules_logprob(long rows, int vocab, int *out) { const LogprobPlan p = logprob_plan(rows, vocab, 256, 256); out[0] = p.parts; out[1] = p.part_sets; out[2] = kLogprobTickets; }
long rules_units(long q, long k, long v, int each) { return rotate_units(q, k, v, each); }
int rules_tiles(long units, int held) { return weigh_tiles(units, held, 256); }
void rules_weigh(int batch, int n_kv, long rows, int held, int *out) { const WeighPlan p = weigh_many(batch, n_kv, rows, held, 256); out[0] = p.splits; out[1] = p.part_keys; }
void rules_evict(int batch, int n_kv, int held, int keep, int recent, int bytes, int *out) {
    const EvictPlan p = evict_plan(batch, n_kv, held, keep, recent, bytes, 256);
    out[0] = p.threads; out[1] = p.columns; out[2] = p.shares; out[3] = p.shift_threads;
    out[4] = evict_cached(held, kEvictLds); out[5] = evict_words(held); out[6] = kEvictLds; out[7] = evict_cached(held, kEvictPlainLds); out[8] = kEvictPlainLds; out[9] = kEvictMost;
}
}
"""


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "r.cpp").write_text(SRC)
    subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-I", CSRC, "-o", str(d / "r.so"), str(d / "r.cpp")], check=True)
    L = C.CDLL(str(d / "r.so"))
    L.rules_units.restype = C.c_long
    L.rules_units.argtypes = [C.c_long, C.c_long, C.c_long, C.c_int]
    L.rules_tiles.argtypes = [C.c_long, C.c_int]
    L.rules_logprob.argtypes = [C.c_long, C.c_int, C.POINTER(C.c_int)]
    L.rules_weigh.argtypes = [C.c_int, C.c_int, C.c_long, C.c_int, C.POINTER(C.c_int)]
    return L


def test_every_logit_has_a_part(rules):
    rng, out = random.Random(0), (C.c_int * 3)()
    for _ in range(3000):
        rows, vocab = int(2 ** rng.uniform(0, 22)), int(2 ** rng.uniform(0, 24))
        rules.rules_logprob(rows, vocab, out)
        parts, sets = out[0], out[1]
        for shift in (0, 1, 7):                                # elements before the row's first, down to a 16-byte boundary
            need = -(-(-(-(vocab + shift) // 8)) // 256)
            assert parts * sets >= need and sets % 4 == 0
        assert (parts - 1) * sets < -(-((vocab + 14) // 8) // 256) or parts == 1       # no part for nothing
        assert parts == 1 or rows <= out[2]                    # as many tickets as cut rows
        assert rows * parts < 2 ** 31


def test_every_head_has_a_unit(rules):
    for q in (0, 1, 3, 4, 5, 40, 64):
        for k in (0, 1, 2, 8, 9):
            for each in (1, 4):
                units = [(kind, f) for kind, n in (("q", q), ("k", k), ("v", k)) for f in range(0, n, each)]
                assert rules.rules_units(q, k, k, each) == len(units)


def test_weighing_fits(rules):
    rng, out = random.Random(1), (C.c_int * 2)()
    for _ in range(3000):
        batch, n_kv, held, rows = rng.randint(1, 300), rng.randint(1, 64), int(2 ** rng.uniform(0, 22)), int(2 ** rng.uniform(6, 18))
        assert 1 <= rules.rules_tiles(batch * n_kv, held) <= 32                        # pages of a wave's tiles lie in its lanes, two to a tile
        rules.rules_weigh(batch, n_kv, rows, held, out)
        assert out[1] >= held and out[1] % 256 == 0 and 1 <= out[0] <= max(1, rows // 32)


def test_eviction_fits(rules):
    rng, out = random.Random(2), (C.c_int * 10)()
    for _ in range(3000):
        batch, n_kv, held = rng.randint(1, 300), rng.randint(1, 64), int(2 ** rng.uniform(0, 20))
        keep = rng.randint(1, max(1, held))
        bytes_ = rng.choice([32, 64, 128, 256, 512])
        rules.rules_evict(batch, n_kv, held, keep, rng.randint(0, keep), bytes_, out)
        threads, columns, shares, shift_threads, cached, words, room, plain, plain_room, most = out
        assert 2048 % threads == 0 and 1024 % threads == 0                             # bins are dealt out evenly
        assert bytes_ % columns == 0 and bytes_ // columns >= 16 and shift_threads in (256, 1024) and shift_threads % (bytes_ // columns // 16) == 0
        assert shares >= 0 and (shares == 0 or held - keep > 512)
        assert words * 64 >= held
        for c, r in ((cached, room), (plain, plain_room)):
            assert c % 4 == 0 and c * 4 + words * 8 <= max(r, words * 8)
            assert c >= 4 or r == plain_room
        assert cached >= min(held, 2 ** 15) or held > 2 ** 15
    assert most == 2 ** 20 and rules.rules_evict(1, 1, most, 5, 0, 256, out) is not None and out[4] >= 4
