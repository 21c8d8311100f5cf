"""A prompt of prefill.prefill that fails while it fills a PagedCache gives back
the room that it took, on the CPU: the store is a stand-in for the library's."""
import math

import pytest
import torch

from paper_2606_09508_amd import binding as eb
from paper_2606_09508_amd import decode
from paper_2606_09508_amd import prefill as pf

SHAPE = pf.DecoderShape(hidden=64, n_q_heads=2, n_kv_heads=1, intermediate=48, n_layers=3, vocab=11)
N, B = 70, 2


@pytest.fixture
def stored(monkeypatch):
    """The calls of the store, one of which may be told to fail."""
    calls = []

    def store(k, v, pages, table, lengths, cu=None):
        if calls and calls[0] == "fail":
            raise RuntimeError("no store")
        calls.append((k.shape, lengths.tolist(), table.tolist()))
    monkeypatch.setattr(eb, "cache_store", store)
    return calls


def _setup():
    layers = pf.make_weights(SHAPE, SHAPE.n_layers, 0, torch.device("cpu"))
    cache = decode.PagedCache(SHAPE, SHAPE.n_layers, 8, 4, 200, device="cpu")
    x = torch.randn((B, N, SHAPE.hidden), generator=torch.Generator().manual_seed(1)).bfloat16()
    return layers, cache, x, [cache.add() for _ in range(B)]


def _attention(fail_at=None):
    calls = []

    def attn(q, k, v):
        calls.append(0)
        if len(calls) - 1 == fail_at:
            raise MemoryError("no room")
        return torch.zeros_like(q)
    return attn


def _empty(cache, seqs):
    return all(cache.length(s) == 0 for s in seqs) and cache.free_pages == cache.n_pages


@pytest.mark.parametrize("layer", range(SHAPE.n_layers))
def test_attention_that_fails(layer, stored):
    layers, cache, x, seqs = _setup()
    store = cache.storing(seqs)
    with pytest.raises(MemoryError):
        pf.prefill(x, layers, SHAPE, _attention(layer), store=store)
    assert _empty(cache, seqs)
    # the same sequences take the prompt afterwards, through the same store
    pf.prefill(x, layers, SHAPE, _attention(), store=store)
    assert [cache.length(s) for s in seqs] == [N] * B and cache.free_pages == cache.n_pages - 2 * B


def test_store_that_fails(stored):
    layers, cache, x, seqs = _setup()
    stored.append("fail")
    with pytest.raises(RuntimeError, match="no store"):
        pf.prefill(x, layers, SHAPE, _attention(), store=cache.storing(seqs))
    assert _empty(cache, seqs)


def test_head_that_does_not_fit(stored):
    layers, cache, x, seqs = _setup()
    with pytest.raises(RuntimeError):
        pf.prefill(x, layers, SHAPE, _attention(), torch.zeros((SHAPE.hidden + 1, 5)).bfloat16(),
                   store=cache.storing(seqs))
    assert _empty(cache, seqs)


def test_refusals_cut_nothing(stored):
    """A store that is refused leaves what the sequences hold."""
    layers, cache, x, seqs = _setup()
    store = cache.storing(seqs)
    pf.prefill(x, layers, SHAPE, _attention(), store=store)
    for again in (store, cache.storing(seqs), cache.storing(seqs[:1]), cache.storing([seqs[0]] * B)):
        with pytest.raises(ValueError, match="empty sequences"):
            pf.prefill(x, layers, SHAPE, _attention(), store=again)
    with pytest.raises(RuntimeError):      # fails before it comes to the store
        pf.prefill(x[..., 1:], layers, SHAPE, _attention(), store=store)
    other = [cache.add(), cache.add()]
    with pytest.raises(decode.CacheFull):
        pf.prefill(x.repeat(1, 3, 1), layers, SHAPE, _attention(), store=cache.storing(other))
    assert [cache.length(s) for s in seqs + other] == [N] * B + [0, 0]
    assert cache.free_pages == cache.n_pages - 2 * B


def test_a_store_that_is_a_function(stored):
    """Any callable will do, and the error of a layer comes through."""
    layers, cache, x, seqs = _setup()
    got = []
    with pytest.raises(MemoryError):
        pf.prefill(x, layers, SHAPE, _attention(1), store=lambda i, k, v: got.append(i))
    assert got == [0, 1]
    last, _ = pf.prefill(x, layers, SHAPE, _attention(), store=lambda i, k, v: None)
    assert last.shape == (B, 1, SHAPE.hidden) and math.isfinite(float(last.float().sum()))
