"""What the decoder's host side must not refuse, lose or slow down, on the CPU."""
import numpy as np
import pytest
import torch

from paper_2606_09508_amd import binding as eb
from paper_2606_09508_amd import decode, prefill as pf

SHAPE = pf.DecoderShape(hidden=64, n_q_heads=2, n_kv_heads=1, intermediate=48, n_layers=2)


@pytest.mark.parametrize("n,kernel", [(8192, True), (8193, False)])
def test_more_adapters_than_the_kernel_takes(monkeypatch, n, kernel):
    """The tensor operations stand in, to bf16's rounding of fp32 sums."""
    calls = []
    monkeypatch.setattr(pf, "_kernel_device", lambda dev: dev.type == "cpu")
    monkeypatch.setattr(eb, "adapter_plan", lambda *a: calls.append("plan"))
    monkeypatch.setattr(eb, "adapter_add", lambda *a: calls.append("add"))
    monkeypatch.setattr(eb, "adapter_add_workspace_bytes", lambda *a: 16)
    g = torch.Generator().manual_seed(n)
    t = eb.Adapters((torch.randn((n, 8, 16), generator=g) * 0.1).bfloat16(),
                    (torch.randn((n, 8, 8), generator=g) * 0.1).bfloat16())
    layers = [{"wq": torch.zeros((16, 8), dtype=torch.bfloat16)}]
    assert pf.check_adapters([{"wq": t}], layers) == n
    index = [n - 1, -1, 5]
    own = pf.BatchAdapters([{"wq": t}], n, torch.tensor(index, dtype=torch.int32), 3)
    h = torch.randn((1, 3, 16), generator=g).bfloat16()
    y = torch.randn((1, 3, 8), generator=g).bfloat16()
    got, = own.layer(0)(h, ("wq",), [y.clone()])
    assert calls == (["plan", "add"] if kernel else [])
    if not kernel:
        want = y.double().clone()
        for s, i in enumerate(index):
            if i >= 0:
                want[0, s] += t.b[i].double() @ (t.a[i].double() @ h[0, s].double())
        assert ((got.double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-5).all()


@pytest.mark.parametrize("forks,lone,new", [([8], 8, 1), ([8], 30, 1), ([3, 3], 20, 1), ([2], 1, 1),
                                            ([30, 5], 2, 4), ([2, 6, 4], 0, 1)])
def test_lone_sequences_do_not_thin_the_groups(monkeypatch, forks, lone, new):
    """The tokens for each group that the attention is told of are about the groups' own."""
    monkeypatch.setattr(eb, "cache_copy", lambda pages, src, dst: None)
    cache = decode.PagedCache(SHAPE, 2, 200, 64, 640, 64, torch.int8, "cpu")
    dec = decode.Decoder([], SHAPE, cache, shared_prefixes=True)
    dec.shared_least = 1
    seqs, parents = [], [cache.add() for _ in forks]
    cache.extend(parents, [130] * len(parents))
    families = [[p] + [cache.fork(p) for _ in range(n - 1)] for p, n in zip(parents, forks)]
    others = [cache.add() for _ in range(lone)]
    cache.extend(others, [30] * lone)
    for i in range(max([lone, *forks])):         # one of each in turn
        seqs += [f[i] for f in families if i < len(f)] + others[i:i + 1]
    counts = [new] * len(seqs)
    cache.extend(seqs, counts)
    order, (first, pages) = dec._groups(seqs, counts)
    order = order or list(range(len(seqs)))
    assert sorted(order) == list(range(len(seqs)))
    assert first[0] == 0 and first == sorted(set(first)) and len(pages) == len(first) - 1
    mine = [sorted(seqs[s] for s in order[a:b]) for a, b in zip(first, first[1:])]
    assert sorted(g for g, n in zip(mine, pages) if n) == sorted(sorted(f) for f in families)
    assert all(n == 2 for n in pages[:len(forks)]) and not any(pages[len(forks):])
    assert all(len(g) == 1 for g in mine[len(forks):])
    own = sum(forks) * new / len(forks)
    told = len(seqs) * new / len(pages)
    assert own / 2 <= told <= own * (1 + 1 / len(forks))
    assert np.diff(first).sum() <= len(seqs)


def test_generate_that_fails_leaves_no_unknown_tokens(monkeypatch):
    """The cache ends before the tokens do: whoever called has none of those drawn."""
    monkeypatch.setattr(eb, "cache_copy", lambda pages, src, dst: None)
    cache = decode.PagedCache(SHAPE, 1, 10, 4, 128, 64, torch.int8, "cpu")
    dec = decode.Decoder([], SHAPE, cache, torch.zeros((64, 5)))
    seqs = [cache.add(), cache.add()]
    cache.extend(seqs, [126, 30])

    def step(x, seqs, counts=None, adapter=None):
        cache.extend(seqs, [1] * len(seqs))
        return None, torch.zeros((2, 5))
    monkeypatch.setattr(dec, "step", step)
    embed, drawn = torch.zeros((5, 64)), []

    def sampler(logits):
        drawn.append(1)
        return torch.zeros(2, dtype=torch.int32), torch.zeros(2)
    with pytest.raises(decode.CacheFull):
        dec.generate(torch.zeros((2, 5)), embed, seqs, 4, sampler)
    assert len(drawn) == 3 and [cache.length(s) for s in seqs] == [126, 30]
    tokens, _ = dec.generate(torch.zeros((2, 5)), embed, seqs, 2, sampler)
    assert tokens.shape == (2, 2) and [cache.length(s) for s in seqs] == [128, 32]
