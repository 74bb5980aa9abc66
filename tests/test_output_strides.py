"""Which strides of an output are refused, without a GPU: every vector needs a place of its own."""
import itertools

import pytest
import torch

from paper_2502_06833_amd import paged
from test_paged_arguments import OnGpu, cache_of


def overlaps(rows, heads, hd, row, head):
    places = [range(r * row + h * head, r * row + h * head + hd) for r in range(rows) for h in range(heads)]
    taken = set()
    for p in places:
        if not taken.isdisjoint(p):
            return True
        taken.update(p)
    return False


def test_strides_are_refused_where_vectors_share_elements_and_nowhere_else():
    flat = torch.zeros(40000, dtype=torch.bfloat16)
    for hd in (32, 64):
        cache = cache_of(shape=(4, 2, 16, hd))
        for rows, heads in ((1, 1), (1, 4), (4, 1), (2, 2), (3, 2), (2, 3), (5, 4), (4, 7)):
            steps = sorted({0, hd // 2, hd - 1, hd, hd + 1, 3 * hd // 2, 2 * hd, 2 * hd + 5, 3 * hd, rows * hd, heads * hd, heads * hd - 1, heads * hd + 3, (rows + 1) * hd, 7 * hd})
            for row, head in itertools.product(steps, steps):
                out = OnGpu(flat.as_strided((rows, heads, hd), (row, head, 1)))
                if overlaps(rows, heads, hd, row, head):
                    with pytest.raises(ValueError):
                        paged._outputs("out", out, cache, rows, heads)
                else:
                    r = paged._outputs("out", out, cache, rows, heads)
                    assert (r.row_stride, r.head_stride) == (row, head)


def test_layouts_of_many_rows():
    of = lambda row, head: OnGpu(torch.empty_strided((1 << 20, 4, 64), (row, head, 1), dtype=torch.bfloat16, device="meta"))  # noqa: E731
    for row, head in ((256, 64), (64, 64 << 20), (64, 70 << 20), (300, 64), (128, 64 + (128 << 20))):
        assert paged._outputs("out", of(row, head), cache_of(), 1 << 20, 4).row_stride == row
    for row, head in ((64, 64), (128, 64), (64, (64 << 20) - 1), (128, 32 + (128 << 10))):
        with pytest.raises(ValueError):
            paged._outputs("out", of(row, head), cache_of(), 1 << 20, 4)
