"""The operators between a batch of prompts and the tokens generated after
them: what each computes in plain tensor operations, and the cases they are
measured on.

    packed  attention over several prompts of different lengths that lie one
            behind the other in one tensor
    store   new keys and values into the pages of a cache that holds 8 bits
            per element, with a scale for each page and KV head
    attend  attention of each sequence's newest tokens over such a cache
    copy    pages of every layer's cache copied to other pages

Token tensors are [1, heads, tokens, 128] in bf16, sequence s being the tokens
cu[s] .. cu[s + 1] - 1.  A page is [KV heads, page_len, 128] in e4m3 or int8
and stands for code * scale.  ``lengths`` counts a sequence's tokens in the
cache, its newest ones included.  A scale is the least power of two (2^-126 at
least) with which the page's largest element stays inside +-448 (e4m3) or
+-127 (int8); it never falls while a page fills up.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
QMAX = {"e4m3": 448.0, "int8": 127.0}
DTYPE = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


# --------------------------------------------------------------------------
# The cases
# --------------------------------------------------------------------------

def _text(lengths):
    return ",".join(str(n) for n in lengths)


def _ints(text):
    return [int(n) for n in text.split(",")]


def _packed(name, q_heads, kv_heads, lengths, causal=True):
    return dict(name=name, kind="packed", q_heads=q_heads, kv_heads=kv_heads,
                lengths=_text(lengths), causal=causal)


def _cache(name, kind, kv_heads, held, new, page_len=64, form="e4m3", q_heads=0):
    """held: tokens of each sequence before the new ones; new: how many come."""
    return dict(name=name, kind=kind, q_heads=q_heads, kv_heads=kv_heads, held=_text(held),
                new=_text(new), page_len=page_len, form=form)


def _copy(name, layers, kv_heads, page_len, pages, moves, form="e4m3"):
    return dict(name=name, kind="copy", layers=layers, kv_heads=kv_heads, page_len=page_len,
                pages=pages, moves=moves, form=form)


def listed():
    return [
        # three short questions to a small model: the call's own latency
        _packed("packed-4h-short", 4, 1, [100, 28, 7]),
        # what a server of an 8B model has waiting: prompts of all lengths
        _packed("packed-32h-ragged", 32, 8, [1531, 517, 2047, 64, 1000, 1, 900, 2100]),
        # long documents beside chats, 64k tokens in all
        _packed("packed-32h-64k", 32, 8, [24576, 16384, 8191, 5000, 4096, 3999, 2047, 777, 300, 166]),
        # a batch of long prompts into the cache, right after their prefill
        _cache("store-8h-32k", "store", 8, [0, 0, 0, 0], [16384, 8191, 5000, 3193]),
        # one generated token of each of 64 sequences, anywhere in its page
        _cache("store-8h-64x1", "store", 8, [37 * i + 64 * (i % 3) for i in range(64)], [1] * 64),
        # the next pieces of prompts that come in pieces, continuing inside a page
        _cache("store-4h-pieces-int8", "store", 4, [1000, 64, 0, 4095, 517, 130],
               [512, 512, 333, 512, 1, 700], 128, "int8"),
        # one user of a small model
        _cache("attend-4h-1x1000", "attend", 1, [999], [1], q_heads=4),
        # a decoding batch of an 8B model, lengths as they come
        _cache("attend-32h-32x4k", "attend", 8, [131 + 253 * i for i in range(32)], [1] * 32,
               q_heads=32),
        # four drafted tokens a sequence, 70B heads, int8 pages
        _cache("attend-64h-6x16k-int8", "attend", 8, [16384, 9000, 12345, 16000, 8191, 14000],
               [4] * 6, 128, "int8", q_heads=64),
        # long documents being answered, one short question among them
        _cache("attend-32h-8x128k", "attend", 8,
               [131071, 120000, 98303, 131070, 65535, 110000, 131071, 999], [1] * 8, q_heads=32),
        # the last, half-filled pages of 16 sequences that fork, all layers
        _copy("copy-32l-fork", 32, 8, 64, 256, 16),
        # closing the holes that finished sequences left
        _copy("copy-32l-compact-int8", 32, 8, 128, 400, 150, "int8"),
    ]


def _log_int(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    n = math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))
    return max(lo, min(hi, int(n)))


HEADS = [(4, 1), (8, 2), (16, 16), (28, 4), (32, 8), (32, 8), (64, 8)]


def draw(rng):
    kind = rng.choice(["packed", "packed", "store", "store", "attend", "attend", "attend", "copy"])
    hq, hkv = rng.choice(HEADS)
    page_len, form = rng.choice([64, 64, 128]), rng.choice(["e4m3", "e4m3", "int8"])
    if kind == "packed":
        top = _log_int(rng, 16, 16384 if hq <= 32 else 8192)     # the longest prompt
        seqs = _log_int(rng, 1, max(1, min(100, 65536 * 32 // max(hq, 32) // top)))
        c = _packed("", hq, hkv, [_log_int(rng, max(1, top // 50), top) for _ in range(seqs)],
                    rng.random() < 0.85)
    elif kind == "store":
        if rng.random() < 0.4:      # a decoding step
            seqs = _log_int(rng, 1, 256)
            new = [rng.choice([1, 1, 1, 2, 5]) for _ in range(seqs)]
            held = [_log_int(rng, 1, 3000) for _ in range(seqs)]
        else:
            seqs = _log_int(rng, 1, 16)
            new = [_log_int(rng, 1, 32768 // seqs) for _ in range(seqs)]
            held = [rng.choice([0, 0, _log_int(rng, 1, 3000)]) for _ in range(seqs)]
        c = _cache("", "store", hkv, held, new, page_len, form)
    elif kind == "attend":
        # tokens in the batch: up to what the largest listed case holds
        seqs = _log_int(rng, 1, 200)
        top = _log_int(rng, 16, max(16, min(131072, 780000 * 8 // max(hkv, 8) // seqs)))
        n = rng.choice([1, 1, 1, 1, 2, 4, 7])
        new = [n] * seqs if rng.random() < 0.7 else [rng.choice([0, 1, n]) for _ in range(seqs)]
        new[0] = max(new[0], 1)
        c = _cache("", "attend", hkv, [_log_int(rng, max(1, top // 20), top) for _ in range(seqs)],
                   new, page_len, form, hq)
    else:
        layers = rng.choice([1, 2, 16, 32])
        most = 150 * 32 * 1024 // (layers * hkv * page_len)
        moves = _log_int(rng, 1, max(1, min(most, 2000)))
        c = _copy("", layers, hkv, page_len, 2 * moves + rng.randrange(0, 100), moves, form)
    del c["name"]
    return c


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------

def _device():
    return torch.device("cuda:0")


def _generator(seed):
    g = torch.Generator(device=_device())
    g.manual_seed(int(seed))
    return g


def _offsets(lengths):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return at


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device=_device())


def _tokens(g, heads, tokens, spread):
    """bf16 [1, heads, tokens, 128] whose channels differ in size, as keys do."""
    x = torch.randn((1, heads, tokens, D), generator=g, device=_device())
    if spread:
        x *= torch.exp(spread * torch.randn((heads, 1, D), generator=g, device=_device()))
    return x.to(torch.bfloat16)


def _codes(g, shape, form):
    """Codes as a filled page holds them: the largest of a page near the end
    of the range."""
    out = torch.empty(shape, dtype=DTYPE[form], device=_device())
    flat = out.view(-1, D)
    piece = 1 << 22
    for r in range(0, flat.shape[0], piece):
        x = torch.randn(flat[r:r + piece].shape, generator=g, device=_device())
        x = (x * (QMAX[form] / 5.0)).clamp_(-QMAX[form], QMAX[form])
        flat[r:r + piece] = x.to(DTYPE[form]) if form == "e4m3" else x.round_().to(torch.int8)
    return out


def _scales(g, shape, form):
    e = torch.randint(0, 3, shape, generator=g, device=_device()) - 1
    return torch.exp2(e.float()) * 2.0 ** round(math.log2(5.0 / QMAX[form]))


def prepare(case, seed):
    st, g, kind = dict(case), _generator(seed), case["kind"]
    if kind == "packed":
        lengths = _ints(case["lengths"])
        st["offsets"] = _offsets(lengths)
        T = st["offsets"][-1]
        st.update(cu=_i32(st["offsets"]), q=_tokens(g, case["q_heads"], T, 0.0),
                  k=_tokens(g, case["kv_heads"], T, 0.5), v=_tokens(g, case["kv_heads"], T, 0.0))
        st["out"] = torch.empty_like(st["q"])
        return st
    P, form, hkv = case["page_len"], case["form"], case["kv_heads"]
    if kind == "copy":
        shape = (case["layers"], case["pages"], hkv, P, D)
        at = torch.randperm(case["pages"], generator=g, device=_device()).to(torch.int32)
        st.update(src=at[:case["moves"]].contiguous(),
                  dst=at[case["moves"]:2 * case["moves"]].contiguous())
    else:
        held, new = _ints(case["held"]), _ints(case["new"])
        lengths = [a + b for a, b in zip(held, new)]
        counts = [-(-n // P) for n in lengths]
        # the sequences' pages lie anywhere in a pool that has a few more
        pool = sum(counts) + 3
        at = torch.randperm(pool, generator=g, device=_device()).to(torch.int32)
        cols = torch.arange(max(counts), device=_device())
        first, n = _i32(_offsets(counts)[:-1])[:, None], _i32(counts)[:, None]
        table = torch.where(cols < n, at[(first + cols).clamp_(max=pool - 1).long()], -1)
        st.update(table=table.to(torch.int32).contiguous(), lengths=_i32(lengths),
                  longest=max(lengths), most_new=max(new), offsets=_offsets(new))
        st["cu"] = None if len(set(new)) == 1 else _i32(st["offsets"])
        T, shape = st["offsets"][-1], (pool, hkv, P, D)
        if kind == "store":
            st.update(k=_tokens(g, hkv, T, 0.5), v=_tokens(g, hkv, T, 0.0))
        else:
            st["q"] = _tokens(g, case["q_heads"], T, 0.0) * 0.5
    st["pages"] = tuple([_codes(g, shape, form) for _ in range(2)]
                        + [_scales(g, shape[:-2], form) for _ in range(2)])
    return st


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------

def run(st):
    kind = st["kind"]
    if own:
        from paper_2606_09508_amd import binding as eb
        if kind == "packed":
            return eb.packed_prefill_attn(st["q"], st["k"], st["v"], st["cu"],
                                          causal=st["causal"], out=st["out"])
        pages = eb.CachePages(*st["pages"])
        if kind == "attend":
            return eb.cache_attn(st["q"], pages, st["table"], st["lengths"], st["cu"])
        if kind == "store":
            eb.cache_store(st["k"], st["v"], pages, st["table"], st["lengths"], st["cu"])
        else:
            eb.cache_copy(pages, st["src"], st["dst"])
        return st["pages"]
    if kind == "packed":
        return _plain_packed(st)
    if kind == "attend":
        return _plain_attend(st)
    return _plain_store(st) if kind == "store" else _plain_copy(st)


def _softmax_of(s, seen, v):
    """softmax(s over the keys that are seen) v; a row that sees none is zero."""
    s = s.masked_fill_(~seen, -math.inf)
    p = torch.exp_(s - s.amax(-1, keepdim=True).clamp_(min=torch.finfo(s.dtype).min))
    total = p.sum(-1, keepdim=True)
    return (p.flatten(1, -2) @ v).view(*p.shape[:-1], D) / torch.where(total > 0, total, 1.0)


def _plain_packed(st):
    """Blocks of query rows against the keys from the first one's sequence on
    (all rows at once would need tokens x tokens scores per head)."""
    q, k, v = (st[n][0].float() for n in "qkv")
    hq, T, _ = q.shape
    hkv = k.shape[0]
    token = torch.arange(T, device=q.device)
    seq = torch.searchsorted(st["cu"][1:].contiguous(), token, right=True, out_int32=True)
    first, end = st["cu"][seq], st["cu"][seq + 1]
    out = torch.empty_like(q)
    rows = 1024
    for r0 in range(0, T, rows):
        r1 = min(T, r0 + rows)
        j0 = max(a for a in st["offsets"] if a <= r0)
        j1 = r1 if st["causal"] else min(a for a in st["offsets"] if a >= r1)
        s = q[:, r0:r1].reshape(hkv, -1, D) @ k[:, j0:j1].transpose(1, 2)
        s = s.mul_(1.0 / math.sqrt(D)).view(hkv, hq // hkv, r1 - r0, j1 - j0)
        last = token[r0:r1, None] if st["causal"] else end[r0:r1, None] - 1
        seen = (token[j0:j1] >= first[r0:r1, None]) & (token[j0:j1] <= last)
        out[:, r0:r1] = _softmax_of(s, seen, v[:, j0:j1]).reshape(hq, -1, D)
    return out[None].to(torch.bfloat16)


def _token_places(st, P):
    """Sequence, page, row in the page of every new token."""
    T, S = st["offsets"][-1], st["lengths"].numel()
    cu = _i32(st["offsets"])
    token = torch.arange(T, device=cu.device, dtype=torch.int32)
    seq = torch.searchsorted(cu[1:].contiguous(), token, right=True)
    pos = st["lengths"][seq] - cu[seq + 1] + token
    return seq, st["table"][seq, pos // P].long(), pos % P


def _plain_attend(st):
    kc, vc, ks, vs = st["pages"]
    P, hkv = kc.shape[2], kc.shape[1]
    table = st["table"].clamp(min=0).long()
    S, cols = table.shape

    def values(codes, scale):
        x = codes.view(torch.uint8)[table].view(codes.dtype).float() * scale[table][..., None, None]
        return x.transpose(1, 2).reshape(S, hkv, cols * P, D)

    # the queries of each sequence in a row of their own, padded to the most
    T, n = st["offsets"][-1], st["most_new"]
    cu = _i32(st["offsets"])
    have = (cu[1:] - cu[:-1])[:, None]
    i = torch.arange(n, device=cu.device)
    at = (cu[:-1, None] + i).clamp_(max=T - 1).long()
    pos = st["lengths"][:, None] - have + i
    hq = st["q"].shape[1]
    q = st["q"][0].float()[:, at].view(hkv, hq // hkv, S, n, D).permute(2, 0, 1, 3, 4)
    s = q.reshape(S * hkv, -1, D) @ values(kc, ks).view(S * hkv, -1, D).transpose(1, 2)
    s = s.mul_(1.0 / math.sqrt(D)).view(S, hkv, hq // hkv, n, cols * P)
    seen = (torch.arange(cols * P, device=cu.device) <= pos[..., None])[:, None, None]
    o = _softmax_of(s.view(S * hkv, hq // hkv, n, cols * P),
                    seen.expand(S, hkv, 1, n, cols * P).reshape(S * hkv, 1, n, cols * P),
                    values(vc, vs).view(S * hkv, -1, D))
    o = o.view(S, hq, n, D).transpose(1, 2)
    out = o[i < have].transpose(0, 1)        # [hq, T, D], the padding left out
    return out[None].to(torch.bfloat16)


def _round_to(x, form):
    return x.to(torch.float8_e4m3fn) if form == "e4m3" else torch.round(x).to(torch.int8)


def _plain_store(st):
    P, form = st["page_len"], st["form"]
    seq, page, row = _token_places(st, P)
    new = _i32(st["offsets"])
    have = new[1:] - new[:-1]
    begin = st["lengths"] - have
    # each sequence's first touched page, with the rows it held before
    # (a sequence without new tokens keeps its page)
    column = (begin // P).clamp(max=st["table"].shape[1] - 1)
    part = st["table"].gather(1, column[:, None].long())[:, 0].clamp(min=0).long()
    old = torch.where(have > 0, begin % P, 0)
    continued = old > 0
    for codes, scale, x in zip(st["pages"][:2], st["pages"][2:], (st["k"], st["v"])):
        x = x[0].float().transpose(0, 1)                                  # [T, hkv, D]
        top = torch.zeros_like(scale).index_reduce_(0, page, x.abs().amax(-1), "amax")
        m, e = torch.frexp(top.double() / QMAX[form])
        e = torch.where(m == 0.5, e - 1, e).clamp(min=-126)
        e = torch.where(top == 0, -126, e)
        fresh = torch.exp2(e.double()).float()
        kept = torch.zeros_like(scale).index_put_(
            (part,), torch.where(continued[:, None], scale[part], 0.0), accumulate=True)
        now = torch.maximum(fresh, kept)
        # rows held before, at the new scale
        was = codes.view(torch.uint8)[part]
        again = _round_to(was.view(codes.dtype).float()
                          * (scale[part] / now[part])[..., None, None], form).view(torch.uint8)
        mine = torch.arange(P, device=page.device) < old[:, None]
        keep = torch.where(mine[:, None, :, None], again, was)
        codes.view(torch.uint8)[part[continued]] = keep[continued]
        codes.view(torch.uint8)[page, :, row] = _round_to(x / now[page][..., None], form).view(
            torch.uint8)
        scale[page] = now[page]
    return st["pages"]


def _plain_copy(st):
    src, dst = st["src"].long(), st["dst"].long()
    for t in st["pages"]:
        t = t if t.dtype == torch.float32 else t.view(torch.uint8)
        t[:, dst] = t[:, src]
    return st["pages"]


# --------------------------------------------------------------------------
# What a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    kind, hkv = case["kind"], case["kv_heads"]
    if kind == "packed":
        lengths, hq = _ints(case["lengths"]), case["q_heads"]
        pairs = sum(n * (n + 1) / 2 if case["causal"] else n * n for n in lengths)
        return {"bytes": 2 * D * sum(lengths) * 2 * (hq + hkv), "flops": 4 * D * hq * pairs}
    P = case["page_len"]
    if kind == "copy":
        return {"bytes": 2 * case["layers"] * case["moves"] * hkv * (2 * P * D + 8), "flops": 0}
    held, new = _ints(case["held"]), _ints(case["new"])
    if kind == "store":
        pages = sum(-(-(a + b) // P) - a // P for a, b in zip(held, new) if b)
        return {"bytes": hkv * (sum(new) * 2 * D * (2 + 1) + 8 * pages), "flops": 0}
    lengths = [a + b for a, b in zip(held, new) if b]
    pairs = sum(b * a + b * (b + 1) / 2 for a, b in zip(held, new))
    return {"bytes": hkv * sum(2 * D * n + 8 * -(-n // P) for n in lengths)
            + 2 * 2 * D * case["q_heads"] * sum(new),
            "flops": 4 * D * case["q_heads"] * pairs}


# --------------------------------------------------------------------------
# The definitions in 64 bits, one sequence at a time
# --------------------------------------------------------------------------

def _attention64(q, k, v, first):
    """q [hq, n, D] over k, v [hkv, L, D]; query i sees the keys up to first + i."""
    hq, n, _ = q.shape
    L = k.shape[1]
    out = torch.zeros((hq, n, D), dtype=torch.float64, device=q.device)
    step = max(1, (1 << 27) // max(L, 1))
    for h in range(hq):
        kh, vh = (t[h // (hq // t.shape[0])].double() for t in (k, v))
        for i in range(0, n, step):
            x = (q[h, i:i + step].double() @ kh.T) / math.sqrt(D)
            if first is not None:
                last = first + torch.arange(i, i + x.shape[0], device=x.device)
                x[torch.arange(L, device=x.device) > last[:, None]] = -math.inf
            out[h, i:i + step] = torch.softmax(x, -1) @ vh
    return out


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "copy":
        return None
    cu = st["offsets"]
    if kind == "packed":
        out = torch.empty(st["q"].shape, dtype=torch.float64, device=_device())
        for a, b in zip(cu, cu[1:]):
            out[0, :, a:b] = _attention64(*(st[n][0, :, a:b] for n in "qkv"),
                                          0 if case["causal"] else None)
        return out
    P, form = case["page_len"], case["form"]
    kc, vc, ks, vs = st["pages"]
    lengths = st["lengths"].tolist()
    if kind == "attend":
        out = torch.empty(st["q"].shape, dtype=torch.float64, device=_device())
        for s, L in enumerate(lengths):
            n = cu[s + 1] - cu[s]
            if n == 0:
                continue
            at = st["table"][s, :-(-L // P)].long()
            k, v = ((c.view(torch.uint8)[at].view(c.dtype).float().double()
                     * f[at].double()[..., None, None]).transpose(0, 1).flatten(1, 2)[:, :L]
                    for c, f in ((kc, ks), (vc, vs)))
            out[0, :, cu[s]:cu[s + 1]] = _attention64(st["q"][0, :, cu[s]:cu[s + 1]], k, v, L - n)
        return out
    values, scales = [], []
    for codes, scale, x in ((kc, ks, st["k"]), (vc, vs, st["v"])):
        values.append(codes.float().double())
        scales.append(scale.double())
        for s, L in enumerate(lengths):
            n = cu[s + 1] - cu[s]
            p = L - n
            while p < L:
                page, r = int(st["table"][s, p // P]), p % P
                take = min(P - r, L - p)
                t = cu[s] + p - (L - n)
                rows = x[0, :, t:t + take].double()                      # [hkv, take, D]
                top = rows.abs().amax((1, 2)) / QMAX[form]
                least = torch.exp2(torch.ceil(torch.log2(top)).clamp(min=-126.0))
                if r:
                    least = torch.maximum(least, scales[-1][page])
                    values[-1][page, :, :r] *= (scales[-1][page] / least)[:, None, None]
                values[-1][page, :, r:r + take] = rows / least[:, None, None]
                scales[-1][page] = least
                p += take
    # (a page's int8 codes are whole numbers)
    return [*(values if form == "e4m3" else (None, None)), *scales]
