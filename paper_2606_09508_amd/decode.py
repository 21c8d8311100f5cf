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

A prompt that goes through the entropy-guided attention instead fills the cache
with ``prefill.prefill(x, ..., store=cache.storing(seqs))`` (or of many at once,
their lengths alike).

    python -m paper_2606_09508_amd.decode --steps     # markdown table of step times
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


class _Batch:
    """What the layers need to know of a packed batch, copied to the device at
    once: the sequences' pages and lengths, their rows, the tokens' positions."""

    def __init__(self, cache: PagedCache, seqs, counts):
        table, lengths = cache.table(seqs)
        S, T = len(counts), sum(counts)
        cu = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        pos = np.concatenate([np.arange(n - c, n) for n, c in zip(lengths.tolist(), counts)])
        flat = np.concatenate([table.ravel(), lengths, cu, pos.astype(np.int32)])
        dev = torch.from_numpy(flat).to(cache.device)
        a, b = table.size, table.size + S
        self.table, self.lengths = dev[:a].view(S, -1), dev[a:b]
        self.cu = dev[b:b + S + 1]
        self.positions = dev[b + S + 1:]
        self.uniform = T == S * counts[0] and len(set(counts)) == 1


class Decoder:
    """The decoder layers over a cache.  Hidden states in and out are packed,
    [1, tokens, hidden] bf16."""

    def __init__(self, layers, shape: pf.DecoderShape, cache: PagedCache, lm_head=None):
        self.layers, self.shape, self.cache, self.lm_head = layers, shape, cache, lm_head
        self.scale = 1.0 / math.sqrt(shape.head_dim)
        self.cos, self.sin = pf.rope_tables(cache.max_len, shape.head_dim, shape.rope_theta,
                                            cache.device)

    def prompts(self, x, lengths, seqs):
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
        return self._run(x, seqs, lengths, attend, last_only=True)

    def step(self, x, seqs, counts=None):
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
                if not ws:   # (the layers come one after the other: one workspace)
                    nb = eb.cache_attn_workspace_bytes(q.shape[1], q.shape[2], cu is not None,
                                                       b.lengths.shape[0], b.table.shape[1], pages)
                    ws["ws"] = torch.empty((max(nb, 1),), dtype=torch.uint8, device=q.device)
                return eb.cache_attn(q, pages, b.table, b.lengths, cu, self.scale,
                                     workspace=ws["ws"])
            return attn
        return self._run(x, seqs, counts, attend, last_only=False)

    def _run(self, x, seqs, counts, attend, last_only):
        seqs = list(seqs)
        if x.dim() != 3 or x.shape[0] != 1 or x.shape[1] != sum(counts) or not seqs \
                or len(counts) != len(seqs):
            raise ValueError(f"x {tuple(x.shape)} is not [1, {sum(counts)}, hidden] of "
                             f"{len(counts)} counts for {len(seqs)} sequences")
        held = [self.cache.length(s) for s in seqs]
        self.cache.extend(seqs, counts)
        try:
            b = _Batch(self.cache, seqs, counts)
            cos, sin = (t.index_select(0, b.positions) for t in (self.cos, self.sin))
            y = None
            for i, w in enumerate(self.layers):
                x, y = pf._layer(x, y, w, self.shape, attend(i, b), cos, sin)
            x, y = x[0], y[0]
            if last_only:
                at = (b.cu[1:] - 1).long()
                x, y = x[at], y[at]
            return pf.finish(x, y, self.layers, self.shape, self.lm_head)
        except BaseException:
            # the room is given back; what the layers that ran made of a page's
            # scale and older codes stays, as truncate says
            for s, n in zip(seqs, held):
                self.cache.truncate(s, n)
            raise


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


def main():
    ap = argparse.ArgumentParser(description=__doc__.split("\n\n")[0])
    ap.add_argument("--steps", action="store_true", help="time steps of one token per sequence")
    ap.add_argument("--layers", type=int, default=pf.LLAMA3_8B.n_layers)
    ap.add_argument("--reps", type=int, default=20)
    ap.add_argument("--batches", default="1,16,64")
    ap.add_argument("--contexts", default="1024,8192,32768")
    ap.add_argument("--int8", action="store_true", help="pages in int8 (e4m3 without)")
    args = ap.parse_args()
    if not args.steps:
        ap.print_help()
        return
    if not torch.cuda.is_available():
        print("a ROCm GPU is needed", file=sys.stderr)
        sys.exit(1)
    step_table([int(n) for n in args.batches.split(",")],
               [int(n) for n in args.contexts.split(",")], pf.LLAMA3_8B, args.layers, args.reps,
               torch.int8 if args.int8 else torch.float8_e4m3fn)


if __name__ == "__main__":
    main()
