"""A paged cache's append that is refused, at whatever point, leaves every slot as
it was: its pages, those behind its window, and how far it can be rolled back; so
does a compaction (no GPU: the calls fail a host check)."""

import numpy as np
import pytest

from paper_2408_00539_amd.paged import PagedKVCache, PoolExhausted
from tests.test_paged_fork import check, grow

torch = pytest.importorskip("torch")
ROW = torch.zeros(1, 2, 64, dtype=torch.bfloat16)


def _cache(num_pages=40, slots=3, max_pages=20, window=100, sinks=0):
    return PagedKVCache(num_pages, 64, slots, max_pages, 2, 64, device="cpu", window=window,
                        sinks=sinks)


def _state(a):
    return ([list(h) for h in a.held], a.refs.tolist(), a.lens.tolist(), a.table.tolist(),
            list(a._trimmed), sorted(a._free))


def _unchanged(cache, call, error):
    before = _state(cache.alloc)
    with pytest.raises(error):
        call()
    assert _state(cache.alloc) == before
    check(cache.alloc)


@pytest.mark.parametrize("window,sinks", [(100, 0), (64, 70), (None, 0)])
def test_refused_by_the_allocator(window, sinks):
    cache = _cache(window=window, sinks=sinks)
    grow(cache.alloc, 0, 1000)
    grow(cache.alloc, 1, 1280)          # at its capacity
    rows = ROW.expand(2, -1, -1)
    _unchanged(cache, lambda: cache.decode([0, 1], rows, rows, rows), ValueError)
    _unchanged(cache, lambda: cache.decode([0, 0], rows, rows, rows), ValueError)
    _unchanged(cache, lambda: cache.prefill([0, 2], rows, rows, rows, [1, 1281]), ValueError)
    cache.rollback(0, 500)              # nothing behind its window was freed
    assert cache.lens[0] == 500


def test_refused_when_the_pool_is_short():
    cache = _cache(num_pages=24, window=64)
    grow(cache.alloc, 0, 1000)          # 16 pages; trims free 14
    grow(cache.alloc, 1, 64 * 8)        # and 7
    rows = ROW.expand(4, -1, -1)
    _unchanged(cache, lambda: cache.prefill([0, 1], rows, rows, rows, [1, 700]), ValueError)
    _unchanged(cache, lambda: cache.prefill([0, 1, 2], rows, rows, rows, [1, 700, 641]),
               PoolExhausted)
    cache.rollback(0, 100)


@pytest.mark.parametrize("window", [100, None])
def test_refused_arguments(window):
    """Tensors that the attention refuses (here: not on a GPU), with and without a
    shared page to copy first."""
    cache = _cache(window=window)
    grow(cache.alloc, 0, 1000)
    _unchanged(cache, lambda: cache.decode([0], ROW, ROW, ROW), ValueError)
    _unchanged(cache, lambda: cache.prefill([0], ROW, ROW, ROW, [1]), ValueError)
    cache.alloc.fork(0, 1)
    rows = ROW.expand(2, -1, -1)
    _unchanged(cache, lambda: cache.decode([0, 1], rows, rows, rows), ValueError)
    cache.rollback(1, 300)


def test_refused_after_the_copies(monkeypatch):
    """The attention's own checks come after the shared pages' copies."""
    cache = _cache()
    monkeypatch.setattr(cache, "_copy", lambda copies: None)
    grow(cache.alloc, 0, 1000)
    cache.alloc.fork(0, 1)
    _unchanged(cache, lambda: cache.decode([0], ROW, ROW, ROW), ValueError)
    cache.rollback(0, 500)


def test_pages_that_a_refused_call_has_written_stay_freed(monkeypatch):
    """With no other page free, a shared page is copied over one from behind the
    window: what that held is lost, and no rollback leads there."""
    cache = _cache(num_pages=16, slots=2, window=64)
    grow(cache.alloc, 0, 1000)                 # all 16 pages
    cache.alloc.fork(0, 1)
    cache.alloc.rollback(1, 0)
    cache.alloc.fork(0, 1)
    a, written = cache.alloc, []
    # slot 1 keeps only its last page shared
    for i in range(15):
        a._drop(a.held[1][i])
        a.held[1][i], a.table[1, i] = -1, 0
    a._trimmed[1] = (0, 15)
    monkeypatch.setattr(cache, "_copy", lambda copies: written.extend(copies))
    with pytest.raises(ValueError):
        cache.decode([0], ROW, ROW, ROW)
    check(a)
    (old, new, used), = written
    assert used == 1000 % 64 and old == a.held[0][15] == a.held[1][15] and a.refs[old] == 2
    assert all(new not in h for h in a.held) and new in a._free
    at = a._trimmed[0][1]
    assert all(p >= 0 for p in a.held[0][at:]) and a.held[0][:at] == [-1] * at and at > 0
    with pytest.raises(ValueError):
        cache.rollback(0, at * 64 + 10)
    cache.rollback(0, at * 64 + 63 + 1)
    check(a)


def test_trimmed_pages_are_used_last():
    cache = _cache(num_pages=30, window=64)
    a = cache.alloc
    grow(a, 0, 1000)
    free = set(a._free)
    a.trim(0, 64, 0)
    a.reserve(1, 64 * len(free))
    assert set(a.held[1]) == free
    check(a)


def test_a_trimmed_page_serves_the_same_call(monkeypatch):
    """A full pool whose window moves on needs no free page."""
    cache = _cache(num_pages=3, slots=1, window=64)
    monkeypatch.setattr("paper_2408_00539_amd.ops.prefill_paged_window", lambda *a: "o")
    for n in (190, 2, 60, 64, 64):
        assert cache.prefill([0], None, None, None, [n]) == "o"
        check(cache.alloc)
    assert cache.lens[0] == 380 and len([p for p in cache.alloc.held[0] if p >= 0]) <= 3


def test_compaction_that_cannot_copy_moves_nothing():
    cache = _cache()
    grow(cache.alloc, 0, 300)
    grow(cache.alloc, 1, 300)
    cache.release(0)
    _unchanged(cache, cache.compact, ValueError)      # (pools that are not on a GPU)
    assert np.array_equal(cache.alloc.compact()[2], np.arange(5))
