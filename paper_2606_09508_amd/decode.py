"""Generation after the prompt: a paged 8-bit cache of keys and values, batches
of prompts of different lengths, and steps of new tokens over the cache.

``PagedCache`` keeps the pages of all layers and, on the host, which sequence
has which of them: sequences are added, extended, forked (sharing their pages
until one of them writes), cut back, freed, and the pages in use moved
together.  ``Decoder`` runs the decoder layers of ``prefill`` over it:

    cache = PagedCache(shape, n_layers, n_pages=4096, max_seqs=64, max_len=8192)
    dec = Decoder(layers, shape, cache, lm_head)
    seqs = [cache.add() for _ in lengths]
    last, logits = dec.prompts(x, lengths, seqs)      # x [1, sum(lengths), hidden]
    last, logits = dec.step(x_new, seqs)              # x_new [1, len(seqs), hidden]

Sequences that were forked from one prompt share its pages; a ``Decoder`` with
``shared_prefixes`` reads them once for all.  With ``adapters`` (low-rank
corrections of the projections, prefill.check_adapters) each sequence of a call
names its own, and ``Sampler`` draws tokens by each request's settings:

    dec = Decoder(layers, shape, cache, lm_head, adapters, shared_prefixes=True)
    sampler = Sampler([dict(temperature=0.7, top_p=0.9), dict(top_k=40)], device="cuda")
    tokens, logprobs = sampler(logits)
    tokens, logprobs = dec.generate(logits, embed, seqs, 100, sampler, adapter=[0, 3])

A prompt that goes through the entropy-guided attention instead fills the cache
with ``prefill.prefill(x, ..., store=cache.storing(seqs))`` (or of many at once,
their lengths alike).

    python -m paper_2606_09508_amd.decode --steps     # markdown table of step times
    python -m paper_2606_09508_amd.decode --serving   # and of steps of one prompt's forks
"""
from __future__ import annotations

import argparse
import heapq
import math
import sys

import numpy as np
import torch

from . import binding as eb
from . import prefill as pf


class CacheFull(RuntimeError):
    """Not enough free pages (or rows for sequences); nothing was changed."""


class PagedCache:
    """Pages [n_layers, n_pages, Hkv, page_len, D] and their owners.

    Sequences are named by small integers.  All GPU work goes to the current
    stream of the device, so calls belong on one stream."""

    def __init__(self, shape: pf.DecoderShape, n_layers: int, n_pages: int, max_seqs: int,
                 max_len: int, page_len: int = 64, dtype=torch.float8_e4m3fn, device="cuda"):
        if min(n_layers, n_pages, max_seqs, max_len) < 1 or page_len not in (64, 128):
            raise ValueError("a cache has layers, pages of 64 or 128 tokens, sequences and a "
                             "length")
        self.page_len, self.n_pages, self.max_len = page_len, n_pages, max_len
        self.pages = eb.new_cache_pages(n_pages, shape.n_kv_heads, page_len, shape.head_dim,
                                        dtype, device, n_layers)
        self.device = self.pages.k.device
        self._layers = [self.pages.layer(i) for i in range(n_layers)]
        self._table = np.full((max_seqs, -(-max_len // page_len)), -1, dtype=np.int32)
        self._length = np.full(max_seqs, -1, dtype=np.int64)      # -1: not a sequence
        self._refs = np.zeros(n_pages, dtype=np.int64)
        self._free = list(range(n_pages))                         # a heap: lowest first

    # -- what there is ------------------------------------------------------

    def layer(self, i: int) -> eb.CachePages:
        return self._layers[i]

    def length(self, seq: int) -> int:
        return int(self._length[self._known(seq)])

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def table(self, seqs):
        """(page_table, lengths) of these sequences on the host, as wide as the
        longest needs."""
        rows = [self._known(s) for s in seqs]
        cols = max((self._count(self._length[r]) for r in rows), default=0)
        return self._table[rows, :max(cols, 1)], self._length[rows].astype(np.int32)

    def _known(self, seq: int) -> int:
        if not 0 <= seq < len(self._length) or self._length[seq] < 0:
            raise ValueError(f"{seq} is no sequence of this cache")
        return seq

    def _count(self, length) -> int:
        return -(-int(length) // self.page_len)

    # -- sequences ------------------------------------------------------------

    def add(self) -> int:
        """A new, empty sequence."""
        unused = np.flatnonzero(self._length < 0)
        if not len(unused):
            raise CacheFull(f"all {len(self._length)} sequences are in use")
        self._length[unused[0]] = 0
        return int(unused[0])

    def fork(self, seq: int) -> int:
        """A sequence with the same tokens.  It shares the pages; the first of
        the two to write into a page they share gets a copy of it."""
        src, new = self._known(seq), self.add()
        n = self._count(self._length[src])
        self._table[new, :n] = self._table[src, :n]
        self._refs[self._table[src, :n]] += 1
        self._length[new] = self._length[src]
        return new

    def extend(self, seqs, counts) -> None:
        """Room for counts[i] more tokens of seqs[i] (their values come with the
        next store).  Raises CacheFull where the pages do not suffice; whatever it
        raises, it has changed nothing."""
        seqs, counts = list(seqs), [int(c) for c in counts]
        if len(set(seqs)) != len(seqs) or len(counts) != len(seqs) or min(counts, default=0) < 0:
            raise ValueError("extend takes each sequence once, with a count of new tokens")
        plan, refs, need = [], {}, 0
        for s, c in zip(seqs, counts):
            old = self.length(s)
            if old + c > self.max_len:
                raise CacheFull(f"sequence {s} of {old} + {c} tokens exceeds {self.max_len}")
            last = int(self._table[s, old // self.page_len]) if c and old % self.page_len else -1
            left = refs.get(last, int(self._refs[last])) if last >= 0 else 0
            copy = left > 1                       # shared: written on a copy
            if copy:
                refs[last] = left - 1
            new = self._count(old + c) - self._count(old)
            need += new + copy
            plan.append((s, c, last if copy else -1, new))
        if need > len(self._free):
            raise CacheFull(f"{need} pages needed, {len(self._free)} of {self.n_pages} free")
        # the copies first: where they cannot be made, the pages go back
        pages = [heapq.heappop(self._free) for _ in range(need)]
        take, src, dst, found = iter(pages), [], [], []
        for s, c, shared, new in plan:
            if shared >= 0:
                src.append(shared)
                dst.append(next(take))
            found.append([next(take) for _ in range(new)])
        try:
            self._copy(src, dst)
        except BaseException:
            for page in pages:
                heapq.heappush(self._free, page)
            raise
        self._refs[pages] = 1
        own = iter(dst)
        for (s, c, shared, new), fresh in zip(plan, found):
            old = int(self._length[s])
            if shared >= 0:
                self._drop(shared)
                self._table[s, old // self.page_len] = next(own)
            at = self._count(old)
            self._table[s, at:at + new] = fresh
            self._length[s] = old + c

    def truncate(self, seq: int, length: int) -> None:
        """Drops a sequence's tokens from `length` on.  The scales of the page it
        then ends in stay what the dropped tokens made them (NaN, and with it the
        page's other tokens, where those were not finite), and so do the codes
        before them, which were rounded again where a scale grew."""
        old = self.length(seq)
        if not 0 <= length <= old:
            raise ValueError(f"cannot cut {old} tokens to {length}")
        for c in range(self._count(length), self._count(old)):
            self._drop(int(self._table[seq, c]))
            self._table[seq, c] = -1
        self._length[seq] = length

    def free(self, seq: int) -> None:
        self.truncate(seq, 0)
        self._length[seq] = -1

    def compact(self) -> int:
        """Moves the pages in use to the lowest numbers; returns how many moved."""
        used = np.flatnonzero(self._refs > 0)
        n = len(used)
        src, dst = used[used >= n], np.flatnonzero(self._refs[:n] == 0)
        if len(src):
            self._copy(src.tolist(), dst.tolist())
            to = np.arange(self.n_pages, dtype=np.int32)
            to[src] = dst
            self._table = np.where(self._table >= 0, to[self._table], -1).astype(np.int32)
            self._refs[dst] = self._refs[src]
            self._refs[src] = 0
        self._free = list(range(n, self.n_pages))
        return len(src)

    def _drop(self, page: int) -> None:
        self._refs[page] -= 1
        if self._refs[page] == 0:
            heapq.heappush(self._free, page)

    def _copy(self, src, dst) -> None:
        if src:
            both = torch.tensor([src, dst], dtype=torch.int32).to(self.device)
            eb.cache_copy(self.pages, both[0], both[1])

    # -- prompts of the other attentions ------------------------------------------

    def storing(self, seqs):
        """A ``store`` for prefill.prefill: keeps the keys and values of a batch
        of new sequences, all of the prompt's length.  A prompt that fails
        leaves them empty."""
        return _Storing(self, list(seqs))


class _Storing:
    """What PagedCache.storing returns: takes a prompt's layers, in order, and
    gives back the room where the block around them fails."""

    def __init__(self, cache: PagedCache, seqs):
        self.cache, self.seqs = cache, seqs
        self.where, self.took = None, False

    def __call__(self, layer: int, k, v):
        B, _, N, _ = k.shape
        if layer == 0:
            if B != len(self.seqs) or any(self.cache.length(s) for s in self.seqs):
                raise ValueError(f"storing a batch of {B} takes as many empty sequences")
            self.cache.extend(self.seqs, [N] * B)
            self.took = True
            table, lengths = self.cache.table(self.seqs)
            self.where = (torch.from_numpy(np.ascontiguousarray(table)).to(k.device),
                          torch.from_numpy(lengths).to(k.device))
        table, lengths = self.where
        for b in range(B):
            eb.cache_store(k[b:b + 1], v[b:b + 1], self.cache.layer(layer), table[b:b + 1],
                           lengths[b:b + 1])

    def __enter__(self):
        self.took = False
        return self

    def __exit__(self, error, *_):
        if error is not None and self.took:
            for s in self.seqs:
                self.cache.truncate(s, 0)
        self.took = False


def prefix_groups(table, shared):
    """Sequences whose first pages are the same, from their rows of the page table
    [S, columns] and the number of pages of each that all its new tokens see:
    (order, group_seqs, shared_pages), the sequences so ordered that a group's lie
    one behind the other, the groups' first places in that order (and its end),
    and how many pages each group shares.

    In the order of their rows, neighbours share most.  A sequence joins the
    group before it unless leaving the group as it is and beginning another with
    the sequence behind saves more reads of pages than joining, alone or with
    that one, does."""
    n = len(table)
    rows = np.ascontiguousarray(table)
    order = sorted(range(n), key=lambda s: rows[s].tobytes())
    rows, most = rows[order], np.asarray(shared)[order]
    alike = np.zeros(n, dtype=np.int64)      # of pages, with the sequence before
    if n > 1:
        differ = rows[1:] != rows[:-1]
        same = np.where(differ.any(1), differ.argmax(1), rows.shape[1])
        alike[1:] = np.minimum(same, np.minimum(most[1:], most[:-1]))
    alike = alike.tolist() + [0]
    first, pages = [], []
    size, held = 0, 0
    for i in range(n):
        joined = alike[i] if size == 1 else min(held, alike[i])
        saved = (size - 1) * held
        if not i or not joined or saved + alike[i + 1] > max(
                size * joined, (size + 1) * min(joined, alike[i + 1])):
            first.append(i)
            pages.append(0)
            size, held = 1, 0
        else:
            size, held = size + 1, joined
            pages[-1] = held
    return order, first + [n], pages


def _lone_last(order, first, pages, counts):
    """What prefix_groups returned, the sequences that share nothing behind the
    groups: (order, [group_seqs, shared_pages]).  cache_attn_shared takes its tiles by
    the new tokens for each group named, so only so many of the lone ones are
    (each a group) that this stays the groups' own number, and at least half of it.
    (64 forks of 32768 keys beside 64 lone sequences of 1000, 32/8 heads: all named
    212 us a call, none 99, one 99; 3 and 3 forks of 44800 beside 60 of 500: 66, 87, and
    20 named 66.)"""
    parts = list(zip(first, first[1:], pages))
    shared = [order[a:b] for a, b, n in parts if n]
    lone = [order[a] for a, b, n in parts if not n]
    place = [s for g in shared for s in g] + lone
    tokens = sum(counts[s] for g in shared for s in g)
    named = -(-len(shared) * sum(counts[s] for s in lone) // max(tokens, 1))
    sizes = [len(g) for g in shared] + [1] * min(named, len(lone))
    return place, [np.concatenate([[0], np.cumsum(sizes)]).tolist(),
                   [n for n in pages if n] + [0] * (len(sizes) - len(shared))]


class _Batch:
    """What the layers need to know of a packed batch, copied to the device at
    once: the sequences' pages and lengths, their rows, the tokens' positions,
    and their adapters and groups where there are any."""

    def __init__(self, cache: PagedCache, seqs, counts, adapter=None, groups=None):
        table, lengths = cache.table(seqs)
        S, T = len(counts), sum(counts)
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        pos = np.concatenate([np.arange(n - c, n) for n, c in zip(lengths.tolist(), counts)])
        parts = [table.ravel(), lengths, cu, pos]
        if adapter is not None:
            parts.append(adapter)
        if groups is not None:
            parts += groups
        flat = np.concatenate([np.asarray(p, dtype=np.int32) for p in parts])
        at = np.cumsum([len(p) for p in parts])[:-1].tolist()
        table, self.lengths, self.cu, self.positions, *rest = \
            torch.from_numpy(flat).to(cache.device).tensor_split(at)
        self.table = table.view(S, -1)
        self.adapter = None if adapter is None else rest.pop(0)
        self.groups = rest or None       # [first sequences, shared pages]
        self.uniform = T == S * counts[0] and len(set(counts)) == 1


class Decoder:
    """The decoder layers over a cache.  Hidden states in and out are packed,
    [1, tokens, hidden] bf16.

    ``adapters`` (optional) is what prefill.check_adapters takes; prompts, step and
    generate then take ``adapter``, each sequence's number (-1: none).  With
    ``shared_prefixes`` the steps read pages that sequences share once for all of
    them (binding.cache_attn_shared) where that saves enough; its results differ
    by roundings."""

    # cache_attn_shared takes the place of cache_attn from so many keys on (times KV
    # heads) that it does not read again: its plan and join cost 10 to 18 us, which
    # so many keys take (32/8 heads, us of the one and the other: 4 x 4096 shared 29,
    # 30; 16 x 4096 29, 29; 8 x 16384 49, 35; 64 x 4096 84, 36; but 64 x 1024 17, 32)
    shared_least = 5 << 17

    def __init__(self, layers, shape: pf.DecoderShape, cache: PagedCache, lm_head=None,
                 adapters=None, shared_prefixes: bool = False):
        self.layers, self.shape, self.cache, self.lm_head = layers, shape, cache, lm_head
        self.adapters, self.shared_prefixes = adapters, shared_prefixes
        self.n_adapters = 0 if adapters is None else pf.check_adapters(adapters, layers)
        self.scale = 1.0 / math.sqrt(shape.head_dim)
        self.cos, self.sin = pf.rope_tables(cache.max_len, shape.head_dim, shape.rope_theta,
                                            cache.device)

    def prompts(self, x, lengths, seqs, adapter=None):
        """Prompts of empty sequences, one behind the other in x [1, sum(lengths),
        hidden]: (normed hidden state of each one's last token [len(seqs),
        hidden], their logits or None)."""
        lengths = [int(n) for n in lengths]
        if any(self.cache.length(s) for s in seqs) or min(lengths, default=0) < 1:
            raise ValueError("prompts go to empty sequences and have tokens")

        def attend(i, b):
            pages = self.cache.layer(i)

            def attn(q, k, v):
                eb.cache_store(k, v, pages, b.table, b.lengths, b.cu)
                return eb.packed_prefill_attn(q, k, v, b.cu, self.scale)
            return attn
        return self._run(x, seqs, lengths, attend, True, adapter)

    def step(self, x, seqs, counts=None, adapter=None):
        """New tokens of the sequences (counts[i] of seqs[i], one each without),
        packed in x: (normed hidden state of every token [tokens, hidden], their
        logits or None).  Where a layer fails the sequences are cut back to what
        they held."""
        counts = [1] * len(seqs) if counts is None else [int(c) for c in counts]
        ws = {}

        def attend(i, b):
            pages = self.cache.layer(i)
            cu = None if b.uniform else b.cu

            def attn(q, k, v):
                eb.cache_store(k, v, pages, b.table, b.lengths, cu)
                S, cols = b.table.shape
                if not ws:   # (the layers come one after the other: one workspace)
                    if b.groups is None:
                        nb = eb.cache_attn_workspace_bytes(q.shape[1], q.shape[2], cu is not None,
                                                           S, cols, pages)
                    else:
                        nb = eb.cache_attn_shared_workspace_bytes(
                            q.shape[1], q.shape[2], S, b.groups[1].shape[0], cols, pages)
                    ws["ws"] = torch.empty((max(nb, 1),), dtype=torch.uint8, device=q.device)
                if b.groups is None:
                    return eb.cache_attn(q, pages, b.table, b.lengths, cu, self.scale,
                                         workspace=ws["ws"])
                return eb.cache_attn_shared(q, pages, b.table, b.lengths, *b.groups, cu, self.scale,
                                            workspace=ws["ws"])
            return attn
        return self._run(x, seqs, counts, attend, False, adapter, self.shared_prefixes)

    def generate(self, logits, embed, seqs, n: int, sampler, adapter=None):
        """n tokens of each sequence from the logits [len(seqs), vocab] of its last
        token on: each is drawn by the sampler and its row of embed [vocab, hidden]
        put through a step, the last one too, so that the sequences hold them all:
        (tokens int32 [len(seqs), n], their log probabilities).  Where a step fails the
        sequences are cut back to what they held before the first, as truncate does."""
        if self.lm_head is None:
            raise ValueError("generate draws from logits: the decoder has no LM head")
        tokens, logprobs = [], []
        held = {s: self.cache.length(s) for s in seqs}
        try:
            for _ in range(n):
                t, p = sampler(logits)
                # (a row without tokens has -1: it goes on from the first)
                x = embed.index_select(0, t.clamp(min=0))
                _, logits = self.step(x[None], seqs, adapter=adapter)
                tokens.append(t)
                logprobs.append(p)
        except BaseException:
            for s, length in held.items():
                self.cache.truncate(s, length)
            raise
        if not tokens:
            dev = logits.device
            return (torch.empty((len(seqs), 0), dtype=torch.int32, device=dev),
                    torch.empty((len(seqs), 0), device=dev))
        return torch.stack(tokens, 1), torch.stack(logprobs, 1)

    def _run(self, x, seqs, counts, attend, last_only, adapter=None, share=False):
        seqs = list(seqs)
        if x.dim() != 3 or x.shape[0] != 1 or x.shape[1] != sum(counts) or not seqs \
                or len(counts) != len(seqs):
            raise ValueError(f"x {tuple(x.shape)} is not [1, {sum(counts)}, hidden] of "
                             f"{len(counts)} counts for {len(seqs)} sequences")
        if adapter is not None:
            adapter = pf.check_choice(adapter, len(seqs), self.adapters, self.n_adapters)
        held = {s: self.cache.length(s) for s in seqs}
        self.cache.extend(seqs, counts)
        try:
            groups, back = None, None
            if share:
                order, groups = self._groups(seqs, counts)
                if order is not None:        # a group's sequences one behind the other
                    rows = np.split(np.arange(sum(counts)), np.cumsum(counts)[:-1])
                    at = np.concatenate([rows[s] for s in order])
                    at = torch.from_numpy(np.stack([at, np.argsort(at)])).to(x.device)
                    x, back = x.index_select(1, at[0]), at[1]
                    seqs, counts = [seqs[s] for s in order], [counts[s] for s in order]
                    adapter = adapter and [adapter[s] for s in order]
            b = _Batch(self.cache, seqs, counts, adapter, groups)
            own = None if adapter is None else pf.BatchAdapters(
                self.adapters, self.n_adapters, b.adapter, sum(counts),
                None if b.uniform else b.cu)
            cos, sin = (t.index_select(0, b.positions) for t in (self.cos, self.sin))
            y = None
            for i, w in enumerate(self.layers):
                x, y = pf._layer(x, y, w, self.shape, attend(i, b), cos, sin,
                                 correct=None if own is None else own.layer(i))
            x, y = x[0], y[0]
            if back is not None:
                x, y = x.index_select(0, back), y.index_select(0, back)
            if last_only:
                at = (b.cu[1:] - 1).long()
                x, y = x[at], y[at]
            return pf.finish(x, y, self.layers, self.shape, self.lm_head)
        except BaseException:
            # the room is given back; what the layers that ran made of a page's
            # scale and older codes stays, as truncate says
            for s, n in held.items():
                self.cache.truncate(s, n)
            raise

    def _groups(self, seqs, counts):
        """(the order of the sequences, None: as they are; the lists of their groups,
        None: none worth it)."""
        table, lengths = self.cache.table(seqs)
        seen = (lengths - np.asarray(counts)) // self.cache.page_len
        order, first, pages = prefix_groups(table, seen)
        saved = sum((b - a - 1) * n for a, b, n in zip(first, first[1:], pages))
        if saved * self.cache.page_len * self.shape.n_kv_heads < self.shared_least:
            return None, None
        order, groups = _lone_last(order, first, pages, counts)
        return None if order == list(range(len(seqs))) else order, groups


class Sampler:
    """Draws each row's next token by its settings (binding.sample_tokens): a dict
    for each row with any of temperature, top_k, top_p and min_p, or one number of
    rows for plain draws.  The random numbers come from a generator of its own."""

    SETTINGS = {"temperature": (1.0, torch.float32), "top_k": (0, torch.int32),
                "top_p": (1.0, torch.float32), "min_p": (0.0, torch.float32)}

    def __init__(self, requests, device="cuda", seed: int = 0):
        if isinstance(requests, int):
            requests = [{}] * requests
        unknown = {k for r in requests for k in r} - set(self.SETTINGS)
        if unknown:
            raise ValueError(f"no settings of a request: {sorted(unknown)}")
        self.rows = len(requests)
        self.settings = {
            name: torch.tensor([r.get(name, none) for r in requests], dtype=dtype).to(device)
            for name, (none, dtype) in self.SETTINGS.items() if any(name in r for r in requests)}
        self.generator = torch.Generator(device=device)
        self.generator.manual_seed(seed)

    def __call__(self, logits):
        """(tokens int32 [rows], their log probabilities fp32 [rows])."""
        if logits.shape[0] != self.rows:
            raise ValueError(f"logits of {logits.shape[0]} rows for {self.rows} requests")
        if self.rows > 1 and logits.stride(0) < logits.shape[1]:   # (one row, expanded)
            logits = logits.contiguous()
        u = torch.rand((self.rows,), generator=self.generator, device=logits.device)
        return eb.sample_tokens(logits, u, **self.settings)


def step_table(batches, contexts, shape: pf.DecoderShape, n_layers: int, reps: int,
               dtype=torch.float8_e4m3fn, file=sys.stdout):
    """Times of a step of one token per sequence, for batches of sequences that
    hold `context` tokens each (random pages, no prompt is run)."""
    dev = torch.device("cuda:0")
    layers = pf.make_weights(shape, n_layers, 0, dev)
    print(f"Decoder: {n_layers} layers, hidden {shape.hidden}, {shape.n_q_heads}/"
          f"{shape.n_kv_heads} heads of {shape.head_dim}, MLP {shape.intermediate}, random bf16 "
          f"weights; cache of {dtype} pages of 64 tokens; {reps} timed steps.\n", file=file)
    print("| sequences | tokens each | step ms | store + attention ms | cache GB/s in them |",
          file=file)
    print("|---:|---:|---:|---:|---:|", file=file)
    for B in batches:
        for N in contexts:
            per = -(-(N + reps + 8) // 64)
            cache = PagedCache(shape, n_layers, B * per, B, per * 64, dtype=dtype, device=dev)
            for t in cache.pages[:2]:
                for i in range(n_layers):
                    t[i].view(torch.uint8).random_(0, 0x60)
            for t in cache.pages[2:]:
                t.fill_(2.0 ** -7)
            dec = Decoder(layers, shape, cache)
            seqs = [cache.add() for _ in range(B)]
            cache.extend(seqs, [N] * B)
            x = torch.randn((1, B, shape.hidden), device=dev).to(torch.bfloat16)
            for _ in range(3):
                dec.step(x, seqs)
            e = [torch.cuda.Event(enable_timing=True) for _ in range(4)]
            e[0].record()
            for _ in range(reps):
                dec.step(x, seqs)
            e[1].record()
            # the cache's part alone, on the layers in turn
            b = _Batch(cache, seqs, [1] * B)
            q, k = (torch.randn((1, h, B, shape.head_dim), device=dev).to(torch.bfloat16)
                    for h in (shape.n_q_heads, shape.n_kv_heads))
            e[2].record()
            for _ in range(reps):
                for i in range(n_layers):
                    eb.cache_store(k, k, cache.layer(i), b.table, b.lengths)
                    eb.cache_attn(q, cache.layer(i), b.table, b.lengths)
            e[3].record()
            torch.cuda.synchronize()
            full, part = (e[i].elapsed_time(e[i + 1]) / reps for i in (0, 2))
            gbs = n_layers * B * N * shape.n_kv_heads * 2 * shape.head_dim / part / 1e6
            print(f"| {B} | {N} | {full:.2f} | {part:.2f} | {gbs:.0f} |", file=file, flush=True)
            del cache, dec, b
            torch.cuda.empty_cache()


def random_adapters(layers, count: int, rank: int, seed: int = 0):
    """Adapters for all projections of the layers, random bf16, whose corrections
    are about as large as a tenth of the products."""
    dev = layers[0]["wq"].device
    g = torch.Generator(device=dev)
    g.manual_seed(seed)

    def bf16(*shape, scale):
        return (torch.randn(shape, generator=g, device=dev) * scale).to(torch.bfloat16)
    return [{name: eb.Adapters(bf16(count, rank, w[name].shape[0], scale=w[name].shape[0] ** -0.5),
                               bf16(count, w[name].shape[1], rank, scale=0.1 * rank ** -0.5))
             for name in pf.PROJECTIONS} for w in layers]


def serving_table(batches, contexts, shape: pf.DecoderShape, n_layers: int, reps: int,
                  dtype=torch.float8_e4m3fn, own: int = 200, count: int = 8, rank: int = 16,
                  file=sys.stdout):
    """Times of a step of one token per sequence, for forks of one sequence of
    `context` tokens (random pages) that hold `own` more each: plain, with the
    shared pages read once, with adapters too, and with the draw of the next tokens
    (top-p) behind it."""
    dev = torch.device("cuda:0")
    layers = pf.make_weights(shape, n_layers, 0, dev)
    adapters = random_adapters(layers, count, rank)
    g = torch.Generator(device=dev)
    g.manual_seed(1)
    head = (torch.randn((shape.hidden, shape.vocab), generator=g, device=dev)
            / math.sqrt(shape.hidden)).to(torch.bfloat16)
    print(f"Decoder: {n_layers} layers, hidden {shape.hidden}, {shape.n_q_heads}/"
          f"{shape.n_kv_heads} heads of {shape.head_dim}, MLP {shape.intermediate}, vocabulary "
          f"{shape.vocab}, random bf16 weights; forks of one sequence with {own} tokens of their "
          f"own, {count} adapters of rank {rank} on all projections; cache of {dtype} pages of 64 "
          f"tokens; {reps} timed steps, ms.\n", file=file)
    print("| forks | shared tokens | step | shared prefix | + adapters | + draw (top-p) |", file=file)
    print("|---:|---:|---:|---:|---:|---:|", file=file)
    for B in batches:
        for N in contexts:
            per = -(-(own + 4 * (reps + 4)) // 64) + 1
            cache = PagedCache(shape, n_layers, -(-N // 64) + B * per, B, N + per * 64, dtype=dtype,
                               device=dev)
            for t in cache.pages[:2]:
                for i in range(n_layers):
                    t[i].view(torch.uint8).random_(0, 0x60)
            for t in cache.pages[2:]:
                t.fill_(2.0 ** -7)
            seqs = [cache.add()]
            cache.extend(seqs, [N])
            seqs += [cache.fork(seqs[0]) for _ in range(B - 1)]
            cache.extend(seqs, [own] * B)
            x = torch.randn((1, B, shape.hidden), device=dev).to(torch.bfloat16)
            sampler = Sampler([dict(temperature=0.8, top_p=0.95)] * B, dev)
            adapter = [i % (count + 1) - 1 for i in range(B)]
            times = []
            for share, which, draw in ((False, None, False), (True, None, False),
                                       (True, adapter, False), (True, adapter, True)):
                dec = Decoder(layers, shape, cache, head, adapters, share)
                e = [torch.cuda.Event(enable_timing=True) for _ in range(2)]
                for i in range(reps + 3):
                    if i == 3:
                        e[0].record()
                    _, logits = dec.step(x, seqs, adapter=which)
                    if draw:
                        sampler(logits)
                e[1].record()
                torch.cuda.synchronize()
                times.append(e[0].elapsed_time(e[1]) / reps)
            print(f"| {B} | {N} | " + " | ".join(f"{t:.2f}" for t in times) + " |", file=file,
                  flush=True)
            del cache, dec
            torch.cuda.empty_cache()


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", action="store_true", help="time steps of one token per sequence")
    ap.add_argument("--serving", action="store_true",
                    help="time steps of forks of one sequence, with adapters and draws")
    ap.add_argument("--layers", type=int, default=pf.LLAMA3_8B.n_layers)
    ap.add_argument("--reps", type=int, default=20)
    ap.add_argument("--batches", default="1,16,64")
    ap.add_argument("--contexts", default="1024,8192,32768")
    ap.add_argument("--int8", action="store_true", help="pages in int8 (e4m3 without)")
    args = ap.parse_args()
    if not (args.steps or args.serving):
        ap.print_help()
        return
    if not torch.cuda.is_available():
        print("a ROCm GPU is needed", file=sys.stderr)
        sys.exit(1)
    for wanted, table in ((args.steps, step_table), (args.serving, serving_table)):
        if wanted:
            table([int(n) for n in args.batches.split(",")],
                  [int(n) for n in args.contexts.split(",")], pf.LLAMA3_8B, args.layers, args.reps,
                  torch.int8 if args.int8 else torch.float8_e4m3fn)


if __name__ == "__main__":
    main()
