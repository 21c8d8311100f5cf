"""PagedCache's host side on the CPU: which sequence owns which page through
adding, extending, forking, cutting, freeing and compacting, against a plain
list of tokens per sequence.  The copies of pages are made by tensor operations
in the place of the library call."""
import random

import numpy as np
import pytest
import torch

from paper_2606_09508_amd import binding as eb
from paper_2606_09508_amd import decode, prefill

SHAPE = prefill.DecoderShape(hidden=256, n_q_heads=2, n_kv_heads=1, intermediate=256, n_layers=2)


@pytest.fixture(autouse=True)
def copies(monkeypatch):
    def copy(pages, src, dst):
        src, dst = src.tolist(), dst.tolist()
        assert len(set(dst)) == len(dst) and not set(dst) & set(src)
        for t in pages:
            t = t if t.dtype is torch.float32 else t.view(torch.uint8)
            t[:, dst] = t[:, src].clone()
    monkeypatch.setattr(eb, "cache_copy", copy)


def new_cache(n_pages, max_seqs, max_len, page_len=64):
    return decode.PagedCache(SHAPE, 2, n_pages, max_seqs, max_len, page_len, torch.int8, "cpu")


def write(cache, seq, at, value):
    """A token's value into its place, in both layers."""
    page = int(cache._table[seq, at // cache.page_len])
    for i in range(2):
        cache.layer(i).k[page, 0, at % cache.page_len, 0] = value + i


def read(cache, seq):
    table, lengths = cache.table([seq])
    return [int(cache.layer(0).k[int(table[0, p // cache.page_len]), 0, p % cache.page_len, 0])
            for p in range(int(lengths[0]))]


def check(cache, want):
    refs = np.zeros(cache.n_pages, dtype=int)
    for s, tokens in want.items():
        assert cache.length(s) == len(tokens)
        assert read(cache, s) == tokens
        used = cache._table[s][cache._table[s] >= 0]
        assert len(used) == -(-len(tokens) // cache.page_len) and len(set(used)) == len(used)
        refs[used] += 1
        for i, t in ((1, tokens),):      # the other layer moved along
            at = [int(cache.layer(i).k[int(cache._table[s, p // cache.page_len]), 0,
                                       p % cache.page_len, 0]) for p in range(len(t))]
            assert at == [x + 1 for x in t]
    assert (refs == cache._refs).all()
    assert sorted(cache._free) == np.flatnonzero(refs == 0).tolist()


@pytest.mark.parametrize("seed", range(6))
def test_random_histories(seed):
    rng = random.Random(seed)
    cache = new_cache(40, 8, 600)
    want = {}
    for _ in range(150):
        what = rng.choice(["add", "extend", "extend", "extend", "fork", "cut", "free", "compact"])
        if what == "add" and len(want) < 8:
            want[cache.add()] = []
        elif what == "fork" and want and len(want) < 8:
            s = rng.choice(list(want))
            want[cache.fork(s)] = list(want[s])
        elif what == "cut" and want:
            s = rng.choice(list(want))
            n = rng.randrange(len(want[s]) + 1)
            cache.truncate(s, n)
            del want[s][n:]
        elif what == "free" and want and rng.random() < 0.4:
            s = rng.choice(list(want))
            cache.free(s)
            del want[s]
        elif what == "compact":
            moved = cache.compact()
            assert moved >= 0
            live = np.flatnonzero(cache._refs)
            assert live.tolist() == list(range(len(live)))
        elif what == "extend" and want:
            seqs = rng.sample(list(want), rng.randint(1, len(want)))
            counts = [rng.choice([0, 1, 1, 2, 63, 64, 65, 130]) for _ in seqs]
            before = (cache._table.copy(), cache._length.copy(), cache._refs.copy(),
                      sorted(cache._free))
            try:
                cache.extend(seqs, counts)
            except decode.CacheFull:
                after = (cache._table, cache._length, cache._refs, sorted(cache._free))
                assert all(np.array_equal(a, b) for a, b in zip(before, after))
                continue
            for s, c in zip(seqs, counts):
                for _ in range(c):
                    v = rng.randrange(120)
                    write(cache, s, len(want[s]), v)
                    want[s].append(v)
        check(cache, want)


def test_full():
    cache = new_cache(3, 2, 300)
    a, b = cache.add(), cache.add()
    with pytest.raises(decode.CacheFull, match="in use"):
        cache.add()
    with pytest.raises(decode.CacheFull, match="4 pages needed, 3 of 3 free"):
        cache.extend([a, b], [128, 65])
    with pytest.raises(decode.CacheFull, match="exceeds 300"):
        cache.extend([a], [301])
    cache.extend([a, b], [128, 64])
    assert cache.free_pages == 0
    cache.free(a)
    assert cache.free_pages == 2
    cache.extend([b], [128])
    assert cache.length(b) == 192


def test_refusals():
    cache = new_cache(4, 4, 256)
    s = cache.add()
    for call in (lambda: cache.length(3), lambda: cache.fork(1), lambda: cache.free(-1),
                 lambda: cache.table([s, 9])):
        with pytest.raises(ValueError, match="no sequence"):
            call()
    for seqs, counts in (([s, s], [1, 1]), ([s], [-1]), ([s], [1, 2])):
        with pytest.raises(ValueError, match="extend"):
            cache.extend(seqs, counts)
    with pytest.raises(ValueError, match="cut"):
        cache.truncate(s, 1)
    for bad in (dict(n_pages=0), dict(page_len=32), dict(max_seqs=0), dict(max_len=0)):
        args = dict(n_pages=4, max_seqs=2, max_len=100, page_len=64) | bad
        with pytest.raises(ValueError, match="64 or 128"):
            new_cache(**args)
    cache.free(s)
    with pytest.raises(ValueError, match="no sequence"):
        cache.length(s)


def test_two_forks_extended_at_once_share_and_copy():
    cache = new_cache(10, 4, 256)
    a = cache.add()
    cache.extend([a], [70])
    for p in range(70):
        write(cache, a, p, p)
    b, c = cache.fork(a), cache.fork(a)
    assert cache.free_pages == 8
    cache.extend([b, c], [1, 1])          # a keeps the page, b and c get copies of it
    assert cache.free_pages == 6
    for s, v in ((b, 100), (c, 101)):
        write(cache, s, 70, v)
    assert read(cache, a) == list(range(70))
    assert read(cache, b) == list(range(70)) + [100] and read(cache, c)[-1] == 101
    assert len({int(cache._table[s, 0]) for s in (a, b, c)}) == 1
