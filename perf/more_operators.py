"""The operators of a step of many continuations: what each computes in plain
tensor operations, and the cases they are measured on.

    shared    attention of the newest tokens of sequences that share the first
              pages of their cache, in groups
    sample    the next token of each row of logits: temperature, top-k, top-p,
              min-p, and a given random number
    adapters  low-rank corrections, of a request's own choice, added to the
              projections that all requests share

shared.  q is [1, heads, tokens, 128] in bf16, sequence s being the tokens
cu[s] .. cu[s + 1] - 1; pages, page table and lengths are those of the paged
8-bit cache.  Group g is the sequences groups[g] .. groups[g + 1] - 1, whose
rows of the page table begin with the same shared[g] pages.

sample.  w_i = exp((x_i - max x) / T), NaN counting as -inf.  Kept are: the k
largest (equal ones by the lowest index); of them the shortest run in the same
order whose weight is at least p of theirs; of them those with w_i >= min_p.
The token is the first kept one at which the weights, summed by index, pass u
times their total.  T = 0 takes the largest.  A row with nothing above -inf
gives -1 and -inf.  Returned with it is the logarithm of its share.

adapters.  y[t] += scale[a] (x[t] A_a^T) B_a^T with a the adapter of the token's
sequence (below zero: none), A_a [rank, in], B_a [out, rank].
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

def _text(values):
    return ",".join(str(n) for n in values)


def _ints(text):
    return [int(n) for n in text.split(",")]


def _shared(name, q_heads, kv_heads, sizes, prefixes, own_tokens, new, page_len=64, form="e4m3"):
    """sizes, prefixes: sequences of each group and their common tokens;
    own_tokens: each sequence's further ones; new: how many of those are new."""
    return dict(name=name, kind="shared", q_heads=q_heads, kv_heads=kv_heads, sizes=_text(sizes),
                prefixes=_text(prefixes), own_tokens=_text(own_tokens), new=_text(new),
                page_len=page_len, form=form)


def _sample(name, rows, vocab, settings, dtype="bf16", allowed=1.0):
    """settings: "temperature", "top-p", "top-k", "min-p" (all rows alike) or
    "mixed" (each row its own); allowed: the share of tokens not masked out."""
    return dict(name=name, kind="sample", rows=rows, vocab=vocab, settings=settings, dtype=dtype,
                allowed=allowed)


QKV, LAYER = "qkv", "layer"


def _adapters(name, hidden, kv_width, mlp, rank, adapters, new, calls, spread=1):
    """new: tokens of each sequence; one sequence in ``spread`` + 1 and more goes
    without an adapter (0: none does)."""
    return dict(name=name, kind="adapters", hidden=hidden, kv_width=kv_width, mlp=mlp, rank=rank,
                adapters=adapters, new=_text(new), calls=calls, spread=spread)


def listed():
    return [
        # two answers to one short question, a small model: the call's latency
        _shared("shared-4h-2x1000", 4, 1, [2], [960], [40, 25], [1, 1]),
        # sixteen samples of an answer to an 8k prompt, an 8B model
        _shared("shared-32h-16x8k", 32, 8, [16], [8192], [37 + 29 * i for i in range(16)], [1] * 16),
        # sixty-four samples over one long document
        _shared("shared-32h-64x32k", 32, 8, [64], [32768], [100 + 13 * i for i in range(64)],
                [1] * 64),
        # requests behind the system prompts of four tenants, one of them with none,
        # four drafted tokens each, 70B heads, int8 pages
        _shared("shared-64h-4tenants-int8", 64, 8, [9, 5, 1, 17], [4096, 12288, 0, 2048],
                [131 + 61 * (i * 7 % 32) for i in range(32)], [4] * 32, 128, "int8"),
        # one user's next token
        _sample("sample-1x128256-top-p", 1, 128256, "top-p"),
        # a decoding batch, every request with settings of its own
        _sample("sample-64x128256-mixed", 64, 128256, "mixed"),
        # a large batch at a temperature, nothing cut off
        _sample("sample-256x128256", 256, 128256, "temperature"),
        # answers held to a grammar: most tokens masked out, in one row all
        _sample("sample-12x32001-fp32-masked", 12, 32001, "mixed", "fp32", 0.01),
        # one request with an adapter of a small model, one token
        _adapters("adapters-1x1-qkv", 1024, 256, 2048, 8, 4, [1], QKV, 0),
        # a decoding batch over 24 adapters, all projections of an 8B layer
        _adapters("adapters-64x1-layer", 4096, 1024, 14336, 16, 24, [1] * 64, LAYER, 7),
        # pieces of prompts beside single tokens, larger ranks
        _adapters("adapters-pieces-layer", 4096, 1024, 14336, 64, 6,
                  [512, 1, 333, 1, 1, 700, 128, 1], LAYER, 7),
        # prompts of 16k tokens in all
        _adapters("adapters-16k-qkv", 4096, 1024, 14336, 16, 4, [8192, 4000, 1531, 517, 2047, 97],
                  QKV, 5),
    ]


def _log_int(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    n = math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))
    return max(lo, min(hi, int(n)))


HEADS = [(4, 1), (8, 2), (16, 16), (28, 4), (32, 8), (32, 8), (64, 8)]
WIDTHS = [(512, 128, 1024), (1024, 256, 2048), (2048, 512, 8192), (4096, 1024, 14336),
          (4096, 1024, 14336)]


def _draw_once(rng, kind):
    if kind == "shared":
        hq, hkv = rng.choice(HEADS)
        page_len, form = rng.choice([64, 64, 128]), rng.choice(["e4m3", "e4m3", "int8"])
        sizes = [_log_int(rng, 1, 64) for _ in range(_log_int(rng, 1, 6))]
        prefixes = [rng.choice([0, 1, 1, 1, 1]) * page_len
                    * _log_int(rng, 1, 32768 // page_len) for _ in sizes]
        n = rng.choice([1, 1, 1, 1, 2, 4])
        S, most = sum(sizes), _log_int(rng, 8, 3000)
        new = [n] * S if rng.random() < 0.7 else [rng.choice([0, 1, n]) for _ in range(S)]
        new[0] = max(new[0], 1)
        return _shared("", hq, hkv, sizes, prefixes,
                       [max(b, _log_int(rng, 1, most)) for b in new], new, page_len, form)
    if kind == "sample":
        vocab = rng.choice([128256, 128256, _log_int(rng, 100, 200000)])
        rows = _log_int(rng, 1, 256)
        return _sample("", rows, vocab,
                       rng.choice(["temperature", "top-p", "top-k", "min-p", "mixed", "mixed"]),
                       rng.choice(["bf16", "bf16", "fp32"]), rng.choice([1.0, 1.0, 0.3, 0.01]))
    hidden, kv_width, mlp = rng.choice(WIDTHS)
    rank, adapters = rng.choice([8, 16, 16, 32, 64]), _log_int(rng, 1, 40)
    if rng.random() < 0.5:      # a decoding step
        new = [rng.choice([1, 1, 1, 1, 2, 5])] * _log_int(rng, 1, 200)
    else:
        new = [_log_int(rng, 1, 4000) for _ in range(_log_int(rng, 1, 8))]
    return _adapters("", hidden, kv_width, mlp, rank, adapters, new, rng.choice([QKV, LAYER]),
                     rng.choice([0, 1, 7]))


def _cost(case):
    w = work(case)
    return max(w["bytes"], w["flops"] / 250)


def draw(rng):
    """One more case, of no more work than the largest listed one of its kind."""
    kind = rng.choice(["shared", "shared", "sample", "sample", "adapters", "adapters"])
    most = max(_cost(c) for c in listed() if c["kind"] == kind)
    case = _draw_once(rng, kind)
    while _cost(case) > most:
        case = _draw_once(rng, kind)
    del case["name"]
    return case


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


def _normal(g, shape, scale=1.0):
    return (torch.randn(shape, generator=g, device=_device()) * scale).to(torch.bfloat16)


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


def _prepare_shared(case, st, g):
    P, form, hkv = case["page_len"], case["form"], case["kv_heads"]
    sizes, prefixes = _ints(case["sizes"]), _ints(case["prefixes"])
    mine, new = _ints(case["own_tokens"]), _ints(case["new"])
    group = [i for i, n in enumerate(sizes) for _ in range(n)]
    lengths = [prefixes[i] + n for i, n in zip(group, mine)]
    first, at, rows = {}, 0, []
    for i, n in enumerate(prefixes):
        first[i], at = at, at + n // P
    cols = max(-(-n // P) for n in lengths)
    for i, n in zip(group, mine):
        c = -(-n // P)
        row = list(range(first[i], first[i] + prefixes[i] // P)) + list(range(at, at + c))
        at += c
        rows.append(row + [-1] * (cols - len(row)))
    pool = at + 3
    shuffle = torch.randperm(pool, generator=g, device=_device()).to(torch.int32)
    table = torch.tensor(rows, dtype=torch.int64, device=_device())
    st["table"] = torch.where(table < 0, -1, shuffle[table.clamp(min=0)]).contiguous()
    st.update(lengths=_i32(lengths), groups=_i32(_offsets(sizes)),
              shared=_i32([n // P for n in prefixes]), offsets=_offsets(new),
              most_new=max(new), most_shared=max(prefixes) // P, most_size=max(sizes),
              most_own=max(-(-n // P) for n in mine), group=_i32(group))
    tokens = [sum(n for n, i in zip(new, group) if i == j) for j in range(len(sizes))]
    st.update(group_tokens=_i32(_offsets(tokens)), most_tokens=max(tokens))
    st["cu"] = None if len(set(new)) == 1 else _i32(st["offsets"])
    st["q"] = _normal(g, (1, case["q_heads"], sum(new), D), 0.5)
    shape = (pool, hkv, P, D)
    st["pages"] = tuple([_codes(g, shape, form) for _ in range(2)]
                        + [_scales(g, shape[:-2], form) for _ in range(2)])


SETTINGS = {  # temperature, top-k, top-p, min-p
    "temperature": [(0.8, 0, 1.0, 0.0)], "top-p": [(0.7, 0, 0.95, 0.0)],
    "top-k": [(1.0, 50, 1.0, 0.0)], "min-p": [(1.2, 0, 1.0, 0.05)],
    "mixed": [(0.8, 0, 1.0, 0.0), (0.7, 0, 0.95, 0.0), (0.0, 0, 1.0, 0.0), (1.0, 50, 1.0, 0.0),
              (1.5, 0, 1.0, 0.02), (0.6, 40, 0.9, 0.0), (1.0, 1000, 0.99, 0.001),
              (1.0, 0, 0.5, 0.0), (1.3, 0, 0.9, 0.1), (0.9, 1, 1.0, 0.0)],
}


def _prepare_sample(case, st, g):
    rows, vocab, dev = case["rows"], case["vocab"], _device()
    # a broad bulk, and a few dozen tokens that may follow
    x = torch.randn((rows, vocab), generator=g, device=dev) * 2.2
    likely = torch.randint(0, vocab, (rows, min(60, vocab)), generator=g, device=dev)
    x.scatter_add_(1, likely, torch.rand(likely.shape, generator=g, device=dev) * 12.0)
    if case["allowed"] < 1:
        x[torch.rand(x.shape, generator=g, device=dev) >= case["allowed"]] = -math.inf
        x[rows // 2] = -math.inf
    s = SETTINGS[case["settings"]]
    s = [s[i % len(s)] for i in range(rows)]
    f = torch.tensor([[a, c, d] for a, _, c, d in s], dtype=torch.float32, device=dev)
    st.update(logits=x.to(torch.bfloat16) if case["dtype"] == "bf16" else x,
              temperature=f[:, 0].contiguous(), top_p=f[:, 1].contiguous(),
              min_p=f[:, 2].contiguous(), top_k=_i32([b for _, b, _, _ in s]))
    # (multiples of 2^-24 inside (0, 1))
    u = torch.randint(1, 1 << 24, (rows,), generator=g, device=dev)
    st["u"] = u.float() * 2.0 ** -24


def _calls(case):
    """(width of x, widths of the y) of each call."""
    h, kv, mlp = case["hidden"], case["kv_width"], case["mlp"]
    calls = [(h, (h, kv, kv))]
    return calls if case["calls"] == QKV else calls + [(h, (h,)), (h, (mlp, mlp)), (mlp, (h,))]


def _index(case):
    """The adapter of each sequence."""
    n, spread = case["adapters"], case["spread"]
    return [-1 if spread and i % (spread + 1) == spread else (i * 5 + i // 3) % n
            for i in range(len(_ints(case["new"])))]


def _prepare_adapters(case, st, g):
    new, n, r = _ints(case["new"]), case["adapters"], case["rank"]
    T = sum(new)
    index = _index(case)
    st.update(index=_i32(index), offsets=_offsets(new), tokens=T,
              token_adapter=_i32([a for a, c in zip(index, new) for _ in range(c)]))
    st["cu"] = None if len(set(new)) == 1 else _i32(st["offsets"])
    st["sets"] = []
    for width, outs in _calls(case):
        st["sets"].append(dict(
            x=_normal(g, (T, width)), y=[_normal(g, (T, m)) for m in outs],
            a=[_normal(g, (n, r, width), 1.0 / math.sqrt(width)) for _ in outs],
            b=[_normal(g, (n, m, r), 0.3 / math.sqrt(r)) for m in outs],
            scale=torch.rand((n,), generator=g, device=_device()) * 2.0))


def prepare(case, seed):
    st, g = dict(case), _generator(seed)
    {"shared": _prepare_shared, "sample": _prepare_sample,
     "adapters": _prepare_adapters}[case["kind"]](case, st, g)
    return st


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------

def run(st):
    kind = st["kind"]
    if own:
        from paper_2606_09508_amd import binding as eb
        if kind == "shared":
            return eb.cache_attn_shared(st["q"], eb.CachePages(*st["pages"]), st["table"],
                                        st["lengths"], st["groups"], st["shared"], st["cu"])
        if kind == "sample":
            return eb.sample_tokens(st["logits"], st["u"], st["temperature"], st["top_k"],
                                    st["top_p"], st["min_p"])
        plan = eb.adapter_plan(st["index"], st["adapters"], st["tokens"], st["cu"])
        for c in st["sets"]:
            eb.adapter_add(c["x"], c["y"], [eb.Adapters(a, b, c["scale"])
                                            for a, b in zip(c["a"], c["b"])], plan)
        return [c["y"] for c in st["sets"]]
    if kind == "shared":
        return _plain_shared(st)
    return _plain_sample(st) if kind == "sample" else _plain_adapters(st)


def _scores(q, k, seen):
    s = (q @ k.transpose(1, 2)).mul_(1.0 / math.sqrt(D))
    return s.masked_fill_(~seen, -math.inf)


def _plain_shared(st):
    """Each group's tokens against its common keys, each sequence's against its
    own, the two softmaxes joined."""
    kc, vc, ks, vs = st["pages"]
    P, hkv, hq, T = kc.shape[2], kc.shape[1], st["q"].shape[1], st["offsets"][-1]
    G, dev = hq // hkv, kc.device
    cu = _i32(st["offsets"])
    group, S = st["group"].long(), st["lengths"].numel()

    def values(codes, scale, table):
        x = codes.view(torch.uint8)[table].view(codes.dtype).float() * scale[table][..., None, None]
        return x.transpose(1, 2).reshape(table.shape[0] * hkv, -1, D)

    def side(first, have, most, table, keys_seen):
        """Maxima, sums and sums of values of the tokens first[b] + i, i <
        have[b], over the keys of row b of the table, back in the tokens' order."""
        B, L = table.shape[0], table.shape[1] * P
        i = torch.arange(most, device=dev)
        at = (first[:, None] + i).clamp_(max=T - 1).long()
        q = st["q"][0].float()[:, at].view(hkv, G, B, most, D).permute(2, 0, 1, 3, 4)
        seen = torch.arange(L, device=dev) < keys_seen[:, None, None, :, None]
        seen = seen.expand(B, hkv, G, most, L).reshape(B * hkv, G * most, L)
        s = _scores(q.reshape(B * hkv, G * most, D), values(kc, ks, table), seen)
        m = s.amax(-1, keepdim=True)
        p = torch.exp_(s - m.clamp(min=-3e38))
        parts = (m, p.sum(-1, keepdim=True), p @ values(vc, vs, table))
        mine = i < have[:, None]
        return [x.view(B, hkv, G, most, -1).permute(0, 3, 1, 2, 4)[mine] for x in parts]

    new = cu[1:] - cu[:-1]
    # (a table without columns would leave the maxima undefined)
    cols = torch.arange(max(st["most_shared"], 1), device=dev)
    leaders = st["table"][st["groups"][:-1].long()]
    reach = cols.clamp(max=leaders.shape[1] - 1).expand(len(leaders), -1)
    gt = st["group_tokens"]
    common = st["shared"][:, None] * P
    m1, l1, o1 = side(gt[:-1], gt[1:] - gt[:-1], st["most_tokens"],
                      leaders.gather(1, reach).clamp(min=0).long(),
                      common.expand(-1, st["most_tokens"]))
    at = st["shared"][group][:, None] + torch.arange(st["most_own"], device=dev)
    mine = st["table"].gather(1, at.clamp(max=st["table"].shape[1] - 1).long()).clamp(min=0).long()
    pos = st["lengths"][:, None] - new[:, None] + torch.arange(st["most_new"], device=dev)
    m2, l2, o2 = side(cu[:-1], new, st["most_new"], mine, pos + 1 - common[group])
    m = torch.maximum(m1, m2)
    a, b = torch.exp(m1 - m), torch.exp(m2 - m)
    o = (o1 * a + o2 * b) / (l1 * a + l2 * b)
    return o.view(T, hq, D).transpose(0, 1)[None].to(torch.bfloat16)


def _plain_sample(st):
    x = st["logits"].double()
    x = torch.where(x.isnan(), -math.inf, x)
    V = x.shape[1]
    t, p, least = (st[n].double()[:, None] for n in ("temperature", "top_p", "min_p"))
    k = st["top_k"][:, None]
    k = torch.where((k <= 0) | (t == 0), V, k)
    k = torch.where(t == 0, 1, k)
    t = torch.where(t == 0, 1.0, t)
    x, order = torch.sort(x, dim=1, descending=True, stable=True)
    w = torch.exp((x - x[:, :1]) / t)
    w = torch.where(x == x[:, :1], 1.0, w)
    w = torch.where(x == -math.inf, 0.0, w)
    w = torch.where(torch.arange(V, device=x.device) < k, w, 0.0)
    total = w.cumsum(1)
    before = total - w
    w = torch.where((before < p * total[:, -1:]) | (p >= 1), w, 0.0)
    w = torch.where(w >= least.clamp(max=1.0), w, 0.0)
    w = torch.zeros_like(w).scatter_(1, order, w)     # by index
    total = w.cumsum(1)
    passed = total > st["u"].double()[:, None] * total[:, -1:]
    token = passed.int().argmax(1)
    share = w.gather(1, token[:, None])[:, 0] / total[:, -1]
    some = total[:, -1] > 0
    return (torch.where(some, token, -1).to(torch.int32),
            torch.where(some, torch.log(share), -math.inf).float())


def _plain_adapters(st):
    """Every token times every adapter, the others' results set to zero."""
    a = st["token_adapter"]
    n = st["adapters"]
    mine = a[:, None] == torch.arange(n, device=a.device)
    for c in st["sets"]:
        x = c["x"].float()
        factor = torch.where(mine, c["scale"], 0.0)[:, :, None]
        for y, A, B in zip(c["y"], c["a"], c["b"]):
            r = A.shape[1]
            v = (x @ A.float().view(n * r, -1).T).view(-1, n, r) * factor
            d = v.view(-1, n * r) @ B.float().transpose(1, 2).reshape(n * r, -1)
            y.copy_((y.float() + d).to(torch.bfloat16))
    return [c["y"] for c in st["sets"]]


# --------------------------------------------------------------------------
# What a pass cannot do without
# --------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    if kind == "sample":
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": case["rows"] * (case["vocab"] * size + 28),
                "flops": 2 * case["rows"] * case["vocab"]}
    new = _ints(case["new"])
    if kind == "adapters":
        index, r = _index(case), case["rank"]
        used = len({a for a, n in zip(index, new) if a >= 0 and n})
        tokens = sum(n for a, n in zip(index, new) if a >= 0)
        b = f = 0
        for width, outs in _calls(case):
            each = len(outs) * width + sum(outs)
            b += 2 * used * r * each + 2 * tokens * (width + 2 * sum(outs))
            f += 2 * tokens * r * each
        return {"bytes": b, "flops": f}
    P, hkv, hq = case["page_len"], case["kv_heads"], case["q_heads"]
    sizes, prefixes, mine = (_ints(case[n]) for n in ("sizes", "prefixes", "own_tokens"))
    group = [i for i, n in enumerate(sizes) for _ in range(n)]
    live = {i for i, b in zip(group, new) if b}
    keys = sum(prefixes[i] for i in live) + sum(a for a, b in zip(mine, new) if b)
    pages = sum(prefixes[i] // P for i in live) + sum(-(-a // P) for a, b in zip(mine, new) if b)
    pairs = sum(b * (prefixes[i] + a - b) + b * (b + 1) / 2 for i, a, b in zip(group, mine, new))
    return {"bytes": hkv * (2 * D * keys + 8 * pages) + 2 * 2 * D * hq * sum(new),
            "flops": 4 * D * hq * pairs}


# --------------------------------------------------------------------------
# The definitions in 64 bits, one sequence, row or token's adapter at a time
# --------------------------------------------------------------------------

def _exact_shared(case, st):
    P, cu = case["page_len"], st["offsets"]
    kc, vc, ks, vs = st["pages"]
    hq, hkv = case["q_heads"], case["kv_heads"]
    out = torch.empty(st["q"].shape, dtype=torch.float64, device=_device())
    for s, L in enumerate(st["lengths"].tolist()):
        n = cu[s + 1] - cu[s]
        if n == 0:
            continue
        at = st["table"][s, :-(-L // P)].long()
        k, v = ((c.view(torch.uint8)[at].view(c.dtype).float().double()
                 * f[at].double()[..., None, None]).transpose(0, 1).flatten(1, 2)[:, :L]
                for c, f in ((kc, ks), (vc, vs)))
        q = st["q"][0, :, cu[s]:cu[s + 1]].double().view(hkv, -1, D)
        x = (torch.bmm(q, k.transpose(1, 2).contiguous()) / math.sqrt(D)).view(hkv, -1, n, L)
        last = L - n + torch.arange(n, device=x.device)
        x[..., torch.arange(L, device=x.device) > last[:, None]] = -math.inf
        out[0, :, cu[s]:cu[s + 1]] = torch.bmm(torch.softmax(x, -1).view(hkv, -1, L),
                                               v.contiguous()).view(hq, n, D)
    return out


def _exact_sample(case, st):
    logs = torch.empty(case["rows"], dtype=torch.float64)
    settings = [st[n].double().tolist() for n in ("u", "temperature", "top_k", "top_p", "min_p")]
    x = st["logits"].double().cpu()
    for r, (u, t, k, p, least) in enumerate(zip(*settings)):
        there = torch.nonzero(x[r] > -math.inf)[:, 0]
        if not there.numel():
            logs[r] = -math.inf
            continue
        if t == 0:
            logs[r] = 0.0
            continue
        y = x[r, there]
        by = torch.argsort(-y, stable=True)
        y, there = y[by], there[by]
        share = torch.softmax(y / t, 0)
        if k > 0:
            share, there = share[:int(k)], there[:int(k)]
        if p < 1:
            sums = torch.cumsum(share, 0)
            n = int((sums < p * sums[-1]).sum()) + 1
            share, there = share[:n], there[:n]
        keep = share >= least * share[0]
        share, there = share[keep], there[keep]
        share = share[torch.argsort(there)]
        sums = torch.cumsum(share, 0)
        logs[r] = torch.log(share[int((sums <= u * sums[-1]).sum())] / sums[-1])
    return None, logs


def _exact_adapters(case, st):
    out = []
    for c in st["sets"]:
        ys = [y.double() for y in c["y"]]
        for s, a in enumerate(_index(case)):
            if a < 0:
                continue
            rows = slice(st["offsets"][s], st["offsets"][s + 1])
            for y, A, B in zip(ys, c["a"], c["b"]):
                v = c["x"][rows].double() @ A[a].double().T
                y[rows] += float(c["scale"][a]) * (v @ B[a].double().T)
        out.append(ys)
    return out


def exact(case, seed):
    return {"shared": _exact_shared, "sample": _exact_sample,
            "adapters": _exact_adapters}[case["kind"]](case, prepare(case, seed))
