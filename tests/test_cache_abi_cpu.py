"""Refusals of the packed and cache entry points, on the host before any
launch, through the C ABI and through the binding; no GPU is needed."""
import ctypes
import os

import pytest
import torch

from paper_2606_09508_amd import binding as eb

FAKE = ctypes.c_void_p(0x1000)   # never dereferenced
ODD = ctypes.c_void_p(0x1008)    # 8-byte aligned only
SHAPE = eb.CacheShape(16, 2, 64, 128, 0)
PAGES = eb.CachePointers(0x1000, 0x1000, 0x1000, 0x1000)
OK, NULL, BAD, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3, -4


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(eb.LIB_PATH):
        pytest.skip("libentropyinfer.so is not built")
    return eb.lib()


def packed(L, dims=eb.Dims(1, 4, 2, 100, 128), cu=FAKE, n=3, sc=0.1, q=FAKE, o=FAKE):
    return L.ei_packed_prefill_attn(q, FAKE, FAKE, dims, cu, n, sc, 1, o, None)


def test_packed_refusals(L):
    D = eb.Dims
    assert packed(L, D(2, 4, 2, 100, 128)) == BAD
    assert packed(L, D(1, 4, 3, 100, 128)) == BAD
    assert packed(L, D(1, 4, 2, -1, 128)) == BAD
    assert packed(L, D(1, 4, 2, 100, 64)) == UNSUPPORTED
    assert packed(L, n=-1) == BAD
    assert packed(L, n=2 ** 31 - 1) == BAD
    for sc in (0.0, -1.0, float("nan"), float("inf")):
        assert packed(L, sc=sc) == BAD
    assert packed(L, cu=None) == NULL
    assert packed(L, q=None) == NULL
    assert packed(L, o=None) == NULL
    assert packed(L, q=ODD) == UNSUPPORTED
    assert packed(L, cu=ctypes.c_void_p(0x1002)) == UNSUPPORTED
    # nothing to do
    for dims, n in ((D(0, 4, 2, 100, 128), 3), (D(1, 4, 2, 0, 128), 3), (D(1, 4, 2, 100, 128), 0)):
        assert packed(L, dims, cu=None, n=n, q=None, o=None) == OK


def store(L, k=FAKE, T=8, cu=None, n=4, lengths=FAKE, table=FAKE, cols=5, shape=SHAPE, pages=PAGES):
    return L.ei_cache_store(k, FAKE, T, cu, n, lengths, table, cols, shape, pages, None)


def attn(L, q=FAKE, hq=4, T=8, cu=None, n=4, lengths=FAKE, table=FAKE, cols=5, shape=SHAPE,
         pages=PAGES, sc=0.1, ws=FAKE, nb=1 << 40):
    return L.ei_cache_attn(q, hq, T, cu, n, lengths, table, cols, shape, pages, sc, FAKE, ws, nb,
                           None)


def copy(L, shape=SHAPE, layers=2, pages=PAGES, src=FAKE, dst=FAKE, n=3):
    return L.ei_cache_copy(shape, layers, pages, src, dst, n, None)


SHAPES = [(eb.CacheShape(-1, 2, 64, 128, 0), BAD), (eb.CacheShape(16, 0, 64, 128, 0), BAD),
          (eb.CacheShape(16, 2, 64, 128, 2), BAD), (eb.CacheShape(16, 2, 64, 128, -1), BAD),
          (eb.CacheShape(16, 2, 0, 128, 0), UNSUPPORTED),
          (eb.CacheShape(16, 2, 96, 128, 0), UNSUPPORTED),
          (eb.CacheShape(16, 2, 256, 128, 1), UNSUPPORTED),
          (eb.CacheShape(16, 2, 64, 64, 0), UNSUPPORTED), (eb.CacheShape(16, 2, 64, 0, 0), BAD),
          (eb.CacheShape(2 ** 30, 4, 64, 128, 0), BAD)]


@pytest.mark.parametrize("shape,status", SHAPES)
def test_cache_shapes(L, shape, status):
    assert store(L, shape=shape) == status
    assert attn(L, shape=shape) == status
    assert copy(L, shape=shape) == status
    assert L.ei_cache_attn_workspace_bytes(4, 8, 0, 4, 5, shape) == 0


@pytest.mark.parametrize("call", [store, attn])
def test_sequence_refusals(L, call):
    assert call(L, T=-1) == BAD
    assert call(L, n=-1) == BAD
    assert call(L, cols=-1) == BAD
    assert call(L, T=7) == BAD                       # 7 tokens of 4 sequences
    assert call(L, None) == NULL
    assert call(L, lengths=None) == NULL
    assert call(L, table=None) == NULL
    assert call(L, ODD) == UNSUPPORTED
    assert call(L, cu=ctypes.c_void_p(0x1001)) == UNSUPPORTED
    assert call(L, lengths=ctypes.c_void_p(0x1001)) == UNSUPPORTED
    for i, f in enumerate(("k", "v", "k_scale", "v_scale")):
        p = [0x1000] * 4
        p[i] = None
        assert call(L, pages=eb.CachePointers(*p)) == NULL
        p[i] = 0x1008 if i < 2 else 0x1002
        assert call(L, pages=eb.CachePointers(*p)) == UNSUPPORTED
    assert call(L, T=0) == OK
    assert call(L, T=0, n=0) == OK
    # (a cache without pages needs no pointers to them; a store has nothing to do)
    empty = eb.CacheShape(0, 2, 64, 128, 0)
    if call is store:
        assert call(L, shape=empty, pages=eb.CachePointers()) == OK


def test_attn_refusals(L):
    assert attn(L, hq=3) == BAD
    assert attn(L, hq=0) == BAD
    for sc in (0.0, -0.5, float("nan"), float("inf")):
        assert attn(L, sc=sc) == BAD
    assert attn(L, T=2 ** 30, n=2 ** 30) == BAD      # 2^32 query rows
    assert attn(L, cols=2 ** 30) == BAD              # 2^36 tokens a sequence
    need = L.ei_cache_attn_workspace_bytes(4, 8, 0, 4, 100, SHAPE)
    assert need > 0
    assert attn(L, cols=100, ws=None) == WORKSPACE
    assert attn(L, cols=100, nb=need - 1) == WORKSPACE
    assert attn(L, cols=100, ws=ODD) == UNSUPPORTED
    assert L.ei_cache_attn_workspace_bytes(4, 7, 0, 4, 100, SHAPE) == 0
    assert L.ei_cache_attn_workspace_bytes(4, 7, 1, 4, 100, SHAPE) > 0
    assert L.ei_cache_attn_workspace_bytes(3, 8, 0, 4, 100, SHAPE) == 0


def test_copy_refusals(L):
    assert copy(L, layers=-1) == BAD
    assert copy(L, n=-1) == BAD
    assert copy(L, src=None) == NULL
    assert copy(L, dst=None) == NULL
    assert copy(L, src=ctypes.c_void_p(0x1001)) == UNSUPPORTED
    assert copy(L, pages=eb.CachePointers(0x1000, None, 0x1000, 0x1000)) == NULL
    assert copy(L, layers=0) == OK
    assert copy(L, n=0, src=None, dst=None) == OK


def test_binding_refuses_what_is_not_on_a_gpu():
    x = torch.zeros((1, 2, 4, 128), dtype=torch.bfloat16)
    pages = eb.new_cache_pages(4, 2, 64, device="cpu")
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="ROCm device"):
        eb.packed_prefill_attn(x, x, x, i)
    with pytest.raises(ValueError, match="ROCm device"):
        eb.cache_store(x, x, pages, i.view(2, 2), i[:2])
    with pytest.raises(ValueError, match="ROCm device"):
        eb.cache_attn(x, pages, i.view(2, 2), i[:2])
    with pytest.raises(ValueError, match="ROCm device"):
        eb.cache_copy(pages, i, i)
    with pytest.raises(TypeError, match="float8_e4m3fn or int8"):
        eb.new_cache_pages(4, 2, 64, dtype=torch.float16, device="cpu")
    assert eb.new_cache_pages(4, 2, 64, device="cpu", n_layers=3).layer(1).k.shape == (4, 2, 64, 128)
