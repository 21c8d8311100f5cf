"""Decoder layers over the paged cache on the GPU.  Prompts against the same
prompts run one by one through the dense attention; steps against the same
layers with their attention computed in float32 by tensor operations from the
cache's pages.  Both sides round to bf16 in the same places, so that the final
hidden states differ by the roundings of two layers: relative RMS 1e-2, the bar
of the prefill's layers."""
import math

import pytest
import torch

from paper_2606_09508_amd import decode, prefill as pf

pytestmark = pytest.mark.gpu

SHAPE = pf.DecoderShape(hidden=512, n_q_heads=8, n_kv_heads=2, head_dim=128, intermediate=1024,
                        n_layers=2, vocab=1000)


def _rel(a, b):
    a, b = a.double(), b.double()
    return float((a - b).norm() / b.norm())


def _setup(dtype=torch.float8_e4m3fn, n_pages=60, max_seqs=8, max_len=1000, page_len=64):
    dev = torch.device("cuda:0")
    layers = pf.make_weights(SHAPE, SHAPE.n_layers, 3, dev)
    g = torch.Generator(device=dev)
    g.manual_seed(5)
    head = (torch.randn((SHAPE.hidden, SHAPE.vocab), generator=g, device=dev)
            / math.sqrt(SHAPE.hidden)).to(torch.bfloat16)
    cache = decode.PagedCache(SHAPE, SHAPE.n_layers, n_pages, max_seqs, max_len, page_len, dtype,
                              dev)
    return layers, head, cache, decode.Decoder(layers, SHAPE, cache, head), g


def _hidden(g, n):
    return torch.randn((1, n, SHAPE.hidden), generator=g, device="cuda").to(torch.bfloat16)


def _values(cache, layer, seq):
    """(k, v) [Hkv, length, 128] of a sequence, as the pages hold them."""
    table, lengths = cache.table([seq])
    n = int(lengths[0])
    at = torch.from_numpy(table[0, :-(-n // cache.page_len)].copy()).long().cuda()
    p = cache.layer(layer)
    return [(c.view(torch.uint8)[at].view(c.dtype).float() * s[at][..., None, None])
            .transpose(0, 1).flatten(1, 2)[:, :n] for c, s in ((p.k, p.k_scale), (p.v, p.v_scale))]


def _reference_step(dec, x, seqs, counts):
    """The step's hidden states after it has run: the pages hold its tokens."""
    cache, shape = dec.cache, dec.shape
    pos = [p for s, c in zip(seqs, counts) for p in range(cache.length(s) - c, cache.length(s))]
    cos, sin = (t[torch.tensor(pos, device="cuda")].contiguous() for t in (dec.cos, dec.sin))
    y = None
    for i, w in enumerate(dec.layers):
        def attn(q, k, v):
            out, at = torch.empty_like(q), 0
            for s, c in zip(seqs, counts):
                kk, vv = _values(cache, i, s)
                kk, vv = (t.repeat_interleave(SHAPE.n_q_heads // SHAPE.n_kv_heads, 0)
                          for t in (kk, vv))
                sc = q[0, :, at:at + c].float() @ kk.transpose(1, 2) / math.sqrt(128)
                last = torch.arange(c, device="cuda")[:, None] + cache.length(s) - c
                sc.masked_fill_(torch.arange(kk.shape[1], device="cuda") > last, -math.inf)
                out[0, :, at:at + c] = (torch.softmax(sc, -1) @ vv).to(q.dtype)
                at += c
            return out
        x, y = pf._layer(x, y, w, shape, attn, cos, sin)
    return pf.finish(x[0], y[0], dec.layers, shape, dec.lm_head)


@pytest.mark.parametrize("dtype", [torch.float8_e4m3fn, torch.int8])
@pytest.mark.parametrize("page_len", [64, 128])
def test_prompts_then_steps(dtype, page_len):
    layers, head, cache, dec, g = _setup(dtype, page_len=page_len)
    lengths = [130, 1, 64, 300]
    x = _hidden(g, sum(lengths))
    seqs = [cache.add() for _ in lengths]
    last, logits = dec.prompts(x, lengths, seqs)
    assert last.shape == (4, SHAPE.hidden) and logits.shape == (4, SHAPE.vocab)
    at = 0
    for i, n in enumerate(lengths):
        one = pf.Attention(SHAPE, 1, n, "dense", pf.SparseConfig(), x.device)
        want, want_logits = pf.prefill(x[:, at:at + n].contiguous(), layers, SHAPE, one, head)
        assert _rel(last[i], want[0, 0]) <= 1e-2 and _rel(logits[i], want_logits[0, 0]) <= 2e-2
        at += n
    for counts in ([1, 1, 1, 1], [1, 1, 1, 1], [3, 1, 70, 2]):
        x = _hidden(g, sum(counts))
        got, got_logits = dec.step(x, seqs, None if max(counts) == 1 else counts)
        want, want_logits = _reference_step(dec, x, seqs, counts)
        assert got.shape == (sum(counts), SHAPE.hidden)
        assert _rel(got, want) <= 1e-2 and _rel(got_logits, want_logits) <= 2e-2
    assert [cache.length(s) for s in seqs] == [135, 4, 136, 304]


def test_sparse_prefill_fills_the_cache():
    """The entropy-guided prompt keeps its keys and values, and a step goes on
    from them."""
    layers, head, cache, dec, g = _setup()
    N = 400
    x = torch.cat([_hidden(g, N), _hidden(g, N)])
    attn = pf.Attention(SHAPE, 2, N, "sparse", pf.SparseConfig(base_budget=256), x.device)
    seqs = [cache.add(), cache.add()]
    with_store = pf.prefill(x, layers, SHAPE, attn, head, store=cache.storing(seqs))
    without = pf.prefill(x, layers, SHAPE, attn, head)
    assert all(torch.equal(a, b) for a, b in zip(with_store, without))
    trace = {}
    cos, sin = pf.rope_tables(N, 128, SHAPE.rope_theta, x.device)
    pf.layer_forward(x, layers[0], SHAPE, attn, cos, sin, trace=trace)
    for b, s in enumerate(seqs):
        k, v = _values(cache, 0, s)
        # e4m3 is off by at most half a step, 2^-4 of the value (and 2^-10 of the page's scale,
        # 2^-10 * 2 * max / 448, where it is subnormal)
        for got, want in ((k, trace["k"][b].float()), (v, trace["v"][b].float())):
            floor = float(want.abs().max()) * 2 / 448 * 2.0 ** -10
            assert bool(((got - want).abs() <= 2.0 ** -4 * want.abs() + floor).all())
    x = _hidden(g, 2)
    got, _ = dec.step(x, seqs)
    want, _ = _reference_step(dec, x, seqs, [1, 1])
    assert _rel(got, want) <= 1e-2


def test_forks_go_their_own_ways():
    """A fork's steps equal those of a sequence of its own with the same
    tokens, bit for bit, and leave the other's as they were, through compaction."""
    layers, head, cache, dec, g = _setup()
    lengths = [100, 100, 30]
    x = _hidden(g, 100)
    a, b, c = (cache.add() for _ in range(3))
    xs = torch.cat([x, x, _hidden(g, 30)], 1)
    dec.prompts(xs, lengths, [a, b, c])
    f = cache.fork(a)
    one, two = _hidden(g, 1), _hidden(g, 1)
    out_f, _ = dec.step(torch.cat([one, two], 1), [f, a])
    out_b, _ = dec.step(torch.cat([one, one], 1), [b, c])    # b: the fork's tokens on its own
    assert torch.equal(out_f[0], out_b[0])
    k_a, k_f, k_b = (_values(cache, 1, s)[0] for s in (a, f, b))
    assert torch.equal(k_f, k_b) and torch.equal(k_a[:, :100], k_f[:, :100])
    assert not torch.equal(k_a[:, 100], k_f[:, 100])
    cache.free(c)
    cache.free(a)
    assert cache.compact() > 0
    assert torch.equal(_values(cache, 1, f)[0], k_f)
    x = _hidden(g, 1)
    again_f, _ = dec.step(torch.cat([x, x], 1), [f, b])
    assert torch.equal(again_f[0], again_f[1])


def test_cut_back_and_go_on():
    """Drafted tokens that are dropped leave no trace but the page's scale."""
    layers, head, cache, dec, g = _setup()
    s, t = cache.add(), cache.add()
    x = _hidden(g, 70)
    dec.prompts(torch.cat([x, x], 1), [70, 70], [s, t])
    dec.step(_hidden(g, 4), [s], [4])
    cache.truncate(s, 70)
    x = _hidden(g, 1)
    got, _ = dec.step(torch.cat([x, x], 1), [s, t])
    assert _rel(got[0], got[1]) <= 2e-2     # (the page of 64 .. may have a larger scale)
    want, _ = _reference_step(dec, torch.cat([x, x], 1), [s, t], [1, 1])
    assert _rel(got, want) <= 1e-2


def test_steps_that_leave_sequences_out():
    """Counts of zero, and a step of no token at all."""
    layers, head, cache, dec, g = _setup()
    s, t = cache.add(), cache.add()
    dec.prompts(_hidden(g, 100), [64, 36], [s, t])
    x = _hidden(g, 3)
    got, _ = dec.step(x, [s, t], [0, 3])
    assert (cache.length(s), cache.length(t)) == (64, 39)
    want, _ = _reference_step(dec, x, [s, t], [0, 3])
    assert _rel(got, want) <= 1e-2
    last, logits = dec.step(x[:, :0], [s, t], [0, 0])
    assert last.shape == (0, SHAPE.hidden) and logits.shape == (0, SHAPE.vocab)
    assert (cache.length(s), cache.length(t)) == (64, 39)


def test_refusals():
    layers, head, cache, dec, g = _setup(n_pages=4)
    s = cache.add()
    with pytest.raises(ValueError, match="is not"):
        dec.step(_hidden(g, 2), [s])
    with pytest.raises(ValueError, match="empty sequences"):
        dec.prompts(_hidden(g, 2), [2, 0], [s, cache.add()])
    with pytest.raises(decode.CacheFull):
        dec.prompts(_hidden(g, 300), [300], [s])
    assert cache.length(s) == 0 and cache.free_pages == 4
    with pytest.raises(RuntimeError):      # another hidden size: the room is given back
        dec.prompts(_hidden(g, 10)[..., :256].contiguous(), [10], [s])
    assert cache.length(s) == 0 and cache.free_pages == 4
    dec.prompts(_hidden(g, 10), [10], [s])
    with pytest.raises(ValueError, match="empty sequences"):
        dec.prompts(_hidden(g, 10), [10], [s])
