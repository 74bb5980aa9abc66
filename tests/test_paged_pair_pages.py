"""paged_pair.py's pages: what a window leaves behind goes back to the pool, and nothing that a later row sees does."""
import pytest

import paged_pair


def pool(n_pages, page, window, sinks):
    m = object.__new__(paged_pair.PagedModel)                 # its bookkeeping alone: no weights, no caches, no GPU
    m.page, m.window, m.sinks, m.free, m.pages, m.have = page, window, sinks, list(range(n_pages)), {}, {}
    return m


def seen_later(j, first, window, sinks):
    """Whether a row at position `first` or after sees position j."""
    return not window or j < sinks or j > first - window


@pytest.mark.parametrize("page", [16, 32])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 1), (20, 4), (16, 0), (17, 16), (33, 17), (100, 40)])
@pytest.mark.parametrize("pieces", [[1] * 150, [40, 1, 1, 7, 60, 1, 1, 30], [8] * 20])
def test_pages_are_held_as_long_as_they_are_seen(page, window, sinks, pieces):
    m = pool(40, page, window, sinks)
    first = 0
    for n in pieces:
        m._grow("a", n)
        pages = m.pages["a"]
        assert m.have["a"] == first + n and len(pages) == -(-(first + n) // page)
        for i, p in enumerate(pages):
            positions = range(i * page, min((i + 1) * page, first + n))
            assert (p >= 0) == any(seen_later(j, first, window, sinks) for j in positions), (i, first)
        held = [p for p in pages if p >= 0]
        assert sorted(held + m.free) == list(range(40))      # nobody's or somebody's, never twice
        first += n
    m.drop("a")
    assert sorted(m.free) == list(range(40)) and not m.pages and not m.have


def test_a_pool_that_only_a_window_makes_do_with():
    """240 positions are 15 pages of 16; with a window of 20 and 4 sinks never more than 4 are held."""
    for window, fits in ((20, True), (0, False)):
        m = pool(4, 16, window, 4)
        grow = lambda: [m._grow("a", 1) for _ in range(240)]  # noqa: E731
        if fits:
            grow()
        else:
            with pytest.raises(RuntimeError):
                grow()
