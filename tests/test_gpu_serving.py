"""Decoder steps with adapters, shared prefixes and sampling on the GPU, as they
are used together: a prompt, forks of it, steps of them with adapters of their
own, tokens drawn by each one's settings.

The reference runs the same layers with the attention in float32 by tensor
operations from the cache's pages and the adapters by their formula in float64,
each rounded to bf16 where the kernels round, so that hidden states differ by the
roundings of two layers: relative RMS 1e-2, logits 2e-2, as without these.  The
tokens are held to the definition in whole numbers for the logits at hand."""
import math

import pytest
import torch

from paper_2606_09508_amd import binding as eb
from paper_2606_09508_amd import decode, prefill as pf
from test_gpu_sample import reference as drawn

pytestmark = pytest.mark.gpu

SHAPE = pf.DecoderShape(hidden=512, n_q_heads=8, n_kv_heads=2, head_dim=128, intermediate=1024,
                        n_layers=2, vocab=1000)


def _rel(a, b):
    a, b = a.double(), b.double()
    return float((a - b).norm() / b.norm())


def _adapters(n, g, some=False):
    """Corrections about as large as the products; two ranks in the second layer."""
    H, D, I = SHAPE.hidden, SHAPE.head_dim, SHAPE.intermediate
    qh, kh = SHAPE.n_q_heads * D, SHAPE.n_kv_heads * D
    sizes = {"wq": (H, qh), "wk": (H, kh), "wv": (H, kh), "wo": (qh, H), "w_gate": (H, I),
             "w_up": (H, I), "w_down": (I, H)}
    out = []
    for layer in range(SHAPE.n_layers):
        mine = {}
        for j, (name, (a, b)) in enumerate(sizes.items()):
            if some and layer and j % 3 == 1:
                continue
            r = 24 if layer and j % 2 else 16
            mine[name] = eb.Adapters(
                (torch.randn((n, r, a), generator=g, device="cuda") / a ** 0.5).bfloat16(),
                (torch.randn((n, b, r), generator=g, device="cuda") / r ** 0.5).bfloat16(),
                torch.rand((n,), generator=g, device="cuda") if j % 2 else None)
        out.append(mine)
    return out


def _setup(dtype=torch.float8_e4m3fn, page_len=64, n_pages=80, n_adapters=3, share=True, seed=5):
    dev = torch.device("cuda:0")
    layers = pf.make_weights(SHAPE, SHAPE.n_layers, 3, dev)
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    head = (torch.randn((SHAPE.hidden, SHAPE.vocab), generator=g, device=dev)
            / math.sqrt(SHAPE.hidden)).to(torch.bfloat16)
    cache = decode.PagedCache(SHAPE, SHAPE.n_layers, n_pages, 16, 1000, page_len, dtype, dev)
    adapters = _adapters(n_adapters, g, some=True) if n_adapters else None
    dec = decode.Decoder(layers, SHAPE, cache, head, adapters, share)
    dec.shared_least = 1          # (however little it saves)
    return dec, g


def _hidden(g, n):
    return torch.randn((1, n, SHAPE.hidden), generator=g, device="cuda").to(torch.bfloat16)


def _values(cache, layer, seq):
    table, lengths = cache.table([seq])
    n = int(lengths[0])
    at = torch.from_numpy(table[0, :-(-n // cache.page_len)].copy()).long().cuda()
    p = cache.layer(layer)
    return [(c.view(torch.uint8)[at].view(c.dtype).float() * s[at][..., None, None])
            .transpose(0, 1).flatten(1, 2)[:, :n] for c, s in ((p.k, p.k_scale), (p.v, p.v_scale))]


def _formula(mine, adapter, counts):
    """A layer's corrections by the formula, in float64 and rounded once."""
    def correct(h, names, ys):
        out, cu = [], [0]
        for c in counts:
            cu.append(cu[-1] + c)
        for name, y in zip(names, ys):
            z = y.double()
            for s, i in enumerate(adapter):
                if name in mine and i >= 0:
                    a, b, f = mine[name]
                    rows = slice(cu[s], cu[s + 1])
                    d = (h[0, rows].double() @ a[i].double().T) @ b[i].double().T
                    z[0, rows] += d if f is None else d * f[i].double()
            out.append(z.to(y.dtype))
        return out
    return correct


def _reference(dec, x, seqs, counts, adapter):
    """A step's hidden states after it has run: the pages hold its tokens."""
    cache, shape = dec.cache, dec.shape
    pos = [p for s, c in zip(seqs, counts) for p in range(cache.length(s) - c, cache.length(s))]
    cos, sin = (t[torch.tensor(pos, device="cuda")].contiguous() for t in (dec.cos, dec.sin))
    y = None
    for i, w in enumerate(dec.layers):
        def attn(q, k, v):
            out, at = torch.empty_like(q), 0
            for s, c in zip(seqs, counts):
                kk, vv = (t.repeat_interleave(SHAPE.n_q_heads // SHAPE.n_kv_heads, 0)
                          for t in _values(cache, i, s))
                sc = q[0, :, at:at + c].float() @ kk.transpose(1, 2).contiguous() / math.sqrt(128)
                last = torch.arange(c, device="cuda")[:, None] + cache.length(s) - c
                sc.masked_fill_(torch.arange(kk.shape[1], device="cuda") > last, -math.inf)
                out[0, :, at:at + c] = (torch.softmax(sc, -1) @ vv).to(q.dtype)
                at += c
            return out
        x, y = pf._layer(x, y, w, shape, attn, cos, sin,
                         correct=_formula(dec.adapters[i], adapter, counts) if dec.adapters else None)
    return pf.finish(x[0], y[0], dec.layers, shape, dec.lm_head)


def _check_step(dec, x, seqs, counts, adapter):
    got, logits = dec.step(x, seqs, counts, adapter)
    want, want_logits = _reference(dec, x, seqs, counts or [1] * len(seqs),
                                   adapter or [-1] * len(seqs))
    assert got.shape == want.shape and logits.shape == want_logits.shape
    assert _rel(got, want) <= 1e-2 and _rel(logits, want_logits) <= 2e-2
    return logits


def _prompted(dec, g, lengths, adapter=None):
    seqs = [dec.cache.add() for _ in lengths]
    return seqs, *dec.prompts(_hidden(g, sum(lengths)), lengths, seqs, adapter)


@pytest.mark.parametrize("dtype,page_len", [(torch.float8_e4m3fn, 64), (torch.int8, 128)])
def test_forks_adapters_and_draws_together(dtype, page_len):
    dec, g = _setup(dtype, page_len)
    (a, b), _, _ = _prompted(dec, g, [330, 200])
    seqs = [a, b] + [dec.cache.fork(a) for _ in range(3)] + [dec.cache.fork(b)]
    adapter = [0, 2, 0, -1, 2, 1]
    settings = [dict(), dict(temperature=0.7, top_p=0.9), dict(top_k=5),
                dict(temperature=0.0), dict(min_p=0.1, temperature=1.5), dict(top_p=0.5, top_k=40)]
    sampler = decode.Sampler(settings, seed=9)
    embed = _hidden(g, SHAPE.vocab)[0]
    x = _hidden(g, len(seqs))
    us = torch.Generator(device="cuda")
    us.manual_seed(9)
    for _ in range(3):
        logits = _check_step(dec, x, seqs, None, adapter)
        tokens, logs = sampler(logits)
        u = torch.rand((len(seqs),), generator=us, device="cuda").tolist()
        f = lambda v: float(torch.tensor(v, dtype=torch.float32))
        for r, s in enumerate(settings):
            token, log, near = drawn(logits[r].cpu(), u[r], f(s.get("temperature", 1.0)),
                                     s.get("top_k", 0), f(s.get("top_p", 1.0)),
                                     f(s.get("min_p", 0.0)))
            if near > SHAPE.vocab * 2.0 ** -44:
                assert int(tokens[r]) == token
                assert abs(float(logs[r]) - log) <= 2.0 ** -23 * abs(log) + 1e-12
        x = embed[tokens.long()][None]
    # several new tokens of each, not as many
    counts = [3, 1, 1, 20, 2, 5]
    _check_step(dec, _hidden(g, sum(counts)), seqs, counts, adapter)
    # some of them, in another order
    _check_step(dec, _hidden(g, 3), [seqs[4], seqs[1], seqs[0]], None, [1, 0, -1])


def test_long_new_runs_on_a_shared_prefix():
    """Requests behind one prompt: each adds its own part, then single tokens."""
    dec, g = _setup()
    (a,), _, _ = _prompted(dec, g, [256])
    seqs = [a] + [dec.cache.fork(a) for _ in range(5)]
    counts = [40, 64, 1, 17, 100, 33]
    _check_step(dec, _hidden(g, sum(counts)), seqs, counts, [0, 1, 2, -1, 0, 1])
    _check_step(dec, _hidden(g, 6), seqs, None, [0, 1, 2, -1, 0, 1])


def test_prompts_with_adapters():
    dec, g = _setup()
    lengths, adapter = [130, 1, 70], [1, -1, 0]
    x = _hidden(g, sum(lengths))
    seqs = [dec.cache.add() for _ in lengths]
    last, logits = dec.prompts(x, lengths, seqs, adapter)
    at = 0
    for i, n in enumerate(lengths):
        one = pf.Attention(SHAPE, 1, n, "dense", pf.SparseConfig(), x.device)
        cos, sin = pf.rope_tables(n, 128, SHAPE.rope_theta, x.device)
        h, y = x[:, at:at + n].contiguous(), None
        for j, w in enumerate(dec.layers):
            h, y = pf._layer(h, y, w, SHAPE, one, cos, sin,
                             correct=_formula(dec.adapters[j], adapter[i:i + 1], [n]))
        want, want_logits = pf.finish(h[0, -1:], y[0, -1:], dec.layers, SHAPE, dec.lm_head)
        assert _rel(last[i], want[0]) <= 1e-2 and _rel(logits[i], want_logits[0]) <= 2e-2
        at += n


def test_prefill_with_adapters():
    """A batch of prompts, each with its own adapter, through prefill.prefill."""
    dec, g = _setup()
    N = 150
    x = torch.cat([_hidden(g, N) for _ in range(3)])
    attn = pf.Attention(SHAPE, 3, N, "dense", pf.SparseConfig(), x.device)
    last, _ = pf.prefill(x, dec.layers, SHAPE, attn, adapters=dec.adapters, adapter=[2, -1, 0])
    plain, _ = pf.prefill(x, dec.layers, SHAPE, attn)
    assert _rel(last[1], plain[1]) <= 1e-2
    for b, i in ((0, 2), (2, 0)):
        one = pf.Attention(SHAPE, 1, N, "dense", pf.SparseConfig(), x.device)
        cos, sin = pf.rope_tables(N, 128, SHAPE.rope_theta, x.device)
        h, y = x[b:b + 1], None
        for j, w in enumerate(dec.layers):
            h, y = pf._layer(h, y, w, SHAPE, one, cos, sin,
                             correct=_formula(dec.adapters[j], [i], [N]))
        want, _ = pf.finish(h[:, -1:], y[:, -1:], dec.layers, SHAPE)
        assert _rel(last[b], want[0]) <= 1e-2
        assert _rel(plain[b], want[0]) > 0.1


def test_no_adapter_leaves_every_bit():
    dec, g = _setup()
    plain = decode.Decoder(dec.layers, SHAPE, dec.cache, dec.lm_head)
    (a, b), _, _ = _prompted(dec, g, [70, 70])
    x = _hidden(g, 2)
    seqs = [a, b]
    got, _ = dec.step(x, seqs, adapter=[-1, -1])
    for s in seqs:
        dec.cache.truncate(s, 70)
    want, _ = plain.step(x, seqs)
    assert torch.equal(got, want)


def test_generate():
    """The tokens of a generation are those of its steps, drawn one by one; a step
    that fails leaves the sequences as long as they were."""
    dec, g = _setup()
    (a,), _, first = _prompted(dec, g, [200], [1])
    seqs = [a, dec.cache.fork(a), dec.cache.fork(a)]
    again = [dec.cache.fork(a) for _ in range(3)]
    embed = _hidden(g, SHAPE.vocab)[0]
    settings = [dict(temperature=0.8), dict(top_k=20), dict(temperature=0.0)]
    adapter = [1, 0, -1]
    logits = first.expand(3, -1)
    tokens, logs = dec.generate(logits, embed, seqs, 5, decode.Sampler(settings, seed=4), adapter)
    assert tokens.shape == logs.shape == (3, 5) and tokens.dtype == torch.int32
    assert [dec.cache.length(s) for s in seqs] == [205] * 3
    sampler = decode.Sampler(settings, seed=4)
    for i in range(5):
        t, p = sampler(logits)
        assert torch.equal(t, tokens[:, i]) and torch.equal(p, logs[:, i])
        _, logits = dec.step(embed[t.long()][None], again, adapter=adapter)
    none, _ = dec.generate(logits, embed, seqs, 0, sampler, adapter)
    assert none.shape == (3, 0)
    with pytest.raises(ValueError):
        dec.generate(first, embed, seqs, 1, sampler, adapter)
    assert [dec.cache.length(s) for s in seqs] == [205] * 3
