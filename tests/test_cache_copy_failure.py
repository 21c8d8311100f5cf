"""A copy of pages that cannot be made changes nothing in a PagedCache's books: what
was shared stays shared, and a second try does the work.  On the CPU, with a
stand-in for the library's copy."""
import numpy as np
import pytest
import torch

from paper_2606_09508_amd import binding as eb
from paper_2606_09508_amd import decode, prefill

SHAPE = prefill.DecoderShape(hidden=256, n_q_heads=2, n_kv_heads=1, intermediate=256, n_layers=2)


def _books(cache):
    return (cache._table.copy(), cache._length.copy(), cache._refs.copy(), sorted(cache._free))


def _same(a, b):
    return all(np.array_equal(x, y) for x, y in zip(a, b))


@pytest.fixture
def cache(monkeypatch):
    """Sequences of 70, 64 and 10 tokens; the copies fail while `cache.fail`."""
    c = decode.PagedCache(SHAPE, 2, 10, 6, 256, dtype=torch.int8, device="cpu")
    c.fail, c.copied = False, []

    def copy(pages, src, dst):
        if c.fail:
            raise MemoryError("no copy")
        c.copied.append((src.tolist(), dst.tolist()))
    monkeypatch.setattr(eb, "cache_copy", copy)
    c.extend([c.add() for _ in range(3)], [70, 64, 10])
    return c


def test_extend(cache):
    a, _, b = range(3)
    forks = [cache.fork(a), cache.fork(b)]
    before, cache.fail = _books(cache), True
    with pytest.raises(MemoryError):
        cache.extend([a, b, *forks], [1, 130, 2, 0])
    assert _same(before, _books(cache))
    cache.fail = False
    cache.extend([a, b, *forks], [1, 130, 2, 0])
    assert [cache.length(s) for s in (a, b, *forks)] == [71, 140, 72, 10]
    (src, dst), = cache.copied
    # both write on a copy of the page they shared, the other keeps it
    assert src == [int(before[0][a, 1]), int(before[0][b, 0])]
    assert dst == [int(cache._table[a, 1]), int(cache._table[b, 0])]
    assert int(cache._table[forks[0], 1]) == src[0] and int(cache._table[forks[1], 0]) == src[1]
    used = cache._table[cache._table >= 0]
    assert np.array_equal(np.bincount(used, minlength=10), cache._refs)
    assert sorted(cache._free) == np.flatnonzero(cache._refs == 0).tolist()


def test_compact(cache):
    cache.free(0)
    before, cache.fail = _books(cache), True
    with pytest.raises(MemoryError):
        cache.compact()
    assert _same(before, _books(cache))
    cache.fail = False
    assert cache.compact() == 2 and sorted(cache._free) == list(range(2, 10))
