"""Refusals of ei_cache_attn_shared, on the host before any launch; no GPU is
needed."""
import ctypes
import os

import pytest

from paper_2606_09508_amd import binding as eb

FAKE, ODD = 0x1000, 0x1008       # never dereferenced; ODD is 8-byte aligned only
SHAPE = eb.CacheShape(16, 2, 64, 128, 0)
PAGES = eb.CachePointers(0x1000, 0x1000, 0x1000, 0x1000)
OK, NULL, BAD, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3, -4


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(eb.LIB_PATH):
        pytest.skip("libentropyinfer.so is not built")
    return eb.lib()


def attn(L, q=FAKE, hq=4, T=8, cu=None, n=4, lengths=FAKE, table=FAKE, cols=5, groups=FAKE,
         shared=FAKE, ng=2, shape=SHAPE, pages=PAGES, sc=0.1, o=FAKE, ws=FAKE, nb=1 << 50):
    return L.ei_cache_attn_shared(q, hq, T, cu, n, lengths, table, cols, groups, shared, ng, shape,
                                  pages, sc, o, ws, nb, None)


@pytest.mark.parametrize("shape,status", [
    (eb.CacheShape(-1, 2, 64, 128, 0), BAD), (eb.CacheShape(16, 0, 64, 128, 0), BAD),
    (eb.CacheShape(16, 2, 64, 128, 2), BAD), (eb.CacheShape(16, 2, 96, 128, 0), UNSUPPORTED),
    (eb.CacheShape(16, 2, 64, 64, 0), UNSUPPORTED), (eb.CacheShape(2 ** 30, 4, 64, 128, 0), BAD)])
def test_cache_shapes(L, shape, status):
    assert attn(L, shape=shape) == status
    assert L.ei_cache_attn_shared_workspace_bytes(4, 8, 4, 2, 5, shape) == 0


def test_refusals(L):
    for bad in (dict(T=-1), dict(n=-1), dict(cols=-1), dict(T=7), dict(ng=-1), dict(hq=3),
                dict(hq=0), dict(sc=0.0), dict(sc=float("nan")), dict(sc=float("inf")),
                dict(T=2 ** 30, hq=4, cu=FAKE), dict(cols=2 ** 30), dict(ng=2 ** 31 - 1)):
        assert attn(L, **bad) == BAD, bad
    for bad in (dict(q=None), dict(lengths=None), dict(table=None), dict(groups=None),
                dict(shared=None), dict(o=None), dict(pages=eb.CachePointers(0x1000, 0, 0x1000, 0x1000))):
        assert attn(L, **bad) == NULL, bad
    for bad in (dict(q=ODD), dict(o=ODD), dict(cu=0x1001), dict(groups=0x1002), dict(shared=0x1001),
                dict(lengths=0x1002), dict(table=0x1002), dict(ws=ODD),
                dict(pages=eb.CachePointers(0x1000, 0x1008, 0x1000, 0x1000))):
        assert attn(L, **bad) == UNSUPPORTED, bad
    need = L.ei_cache_attn_shared_workspace_bytes(4, 8, 4, 2, 5, SHAPE)
    assert need > 0
    assert attn(L, nb=need - 1) == WORKSPACE
    assert attn(L, ws=None) == WORKSPACE


def test_nothing_to_do(L):
    none = dict(q=None, lengths=None, table=None, groups=None, shared=None, o=None, ws=None, nb=0)
    assert attn(L, T=0, **none) == OK
    assert attn(L, T=0, n=0, **none) == OK
    assert L.ei_cache_attn_shared_workspace_bytes(4, 0, 4, 2, 5, SHAPE) == 0
    assert L.ei_cache_attn_shared_workspace_bytes(4, 8, 0, 2, 5, SHAPE) == 0
    assert L.ei_cache_attn_shared_workspace_bytes(3, 8, 4, 2, 5, SHAPE) == 0
    assert L.ei_cache_attn_shared_workspace_bytes(4, 8, 4, -2, 5, SHAPE) == 0
