"""The attention over the cache in float64, and how far fp32 sums and
probabilities of 16 bits may be from it (for tests/test_*cache_precision*.py)."""
import math

import torch

D = 128
E4M3, INT8 = torch.float8_e4m3fn, torch.int8
QMAX = {E4M3: 448.0, INT8: 127.0}
HALF = 2.0 ** -8   # half a bf16 step, relative


def case(held, new, hq, hkv, P, dtype, seed, spare):
    """Pages, table, lengths, offsets and queries on the CPU.  Rows 2i and 2i + 1
    of V cancel, so that an output is far smaller than its terms and the
    probabilities' own errors show."""
    g = torch.Generator().manual_seed(seed)
    lengths = [a + b for a, b in zip(held, new)]
    cols = max(-(-n // P) for n in lengths) + spare
    n_pages = sum(-(-n // P) for n in lengths) + 1
    at = torch.randperm(n_pages, generator=g).tolist()
    table = torch.full((len(lengths), cols), -1, dtype=torch.int32)
    for s, n in enumerate(lengths):
        for c in range(-(-n // P)):
            table[s, c] = at.pop()
    x = (torch.randn((2, n_pages, hkv, P, D), generator=g) * (QMAX[dtype] / 4)).clamp(
        -QMAX[dtype], QMAX[dtype])
    x[1, :, :, 1::2] = -x[1, :, :, ::2]
    codes = x.to(E4M3) if dtype is E4M3 else x.round().to(INT8)
    scale = torch.exp2(torch.randint(-9, -6, (2, n_pages, hkv), generator=g).float())
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    q = (torch.randn((1, hq, cu[-1], D), generator=g) * 0.05).to(torch.bfloat16)
    return dict(k=codes[0].clone(), v=codes[1].clone(), ks=scale[0].clone(), vs=scale[1].clone(),
                table=table, lengths=lengths, cu=cu, q=q)


def sequence(c, s):
    """(queries [hkv, G, n, D], K, V [hkv, L, D] in float64, V's scales [hkv, L],
    which keys each query sees [n, L]) of a sequence."""
    P, hkv, n, L = c["k"].shape[2], c["k"].shape[1], c["cu"][s + 1] - c["cu"][s], c["lengths"][s]
    p = torch.arange(L)
    page, row = c["table"][s][p // P].long(), p % P
    k, v = (t.float().double()[page, :, row].transpose(0, 1) for t in (c["k"], c["v"]))
    ks, vs = (t.double()[page].transpose(0, 1) for t in (c["ks"], c["vs"]))
    q = c["q"][0, :, c["cu"][s]:c["cu"][s + 1]].double()
    return (q.view(hkv, -1, n, D), k * ks[..., None], v * vs[..., None], vs,
            p <= (L - n + torch.arange(n))[:, None])


def reference(c):
    """(output in float64, how far a result may be off), [1, hq, T, D].

    With w the weights and a = w |v|, an output r is off by
      HALF |r|          its own rounding,
      2^-16 a           a weight as the sum of two bf16 numbers: the first is
                        within 2^-8 of it, the second within 2^-8 of the rest,
      2 * 130 e mag a   fp32 scores, sums of 128 products of magnitudes `mag`
                        in all, and the same in the sum the weights are
                        divided by; e = 2^-23, as matrix cores may truncate,
      (3 L + 32) e a    sums over L keys (the weights', and each of the two
                        products') and single roundings: the exponential, the
                        scales, the joining of parts, the quotient."""
    out = torch.zeros(c["q"].shape, dtype=torch.float64)
    off = torch.zeros_like(out)
    for s in range(len(c["lengths"])):
        q, k, v, _, seen = sequence(c, s)
        hkv, L = k.shape[:2]
        if q.shape[2] == 0:
            continue
        x = (q.flatten(1, 2) @ k.transpose(1, 2)).view(*q.shape[:3], L) / math.sqrt(D)
        mag = (q.flatten(1, 2).abs() @ k.abs().transpose(1, 2)).amax() / math.sqrt(D)
        w = torch.softmax(x.masked_fill(~seen, -math.inf), -1).flatten(1, 2)
        r, a = w @ v, w @ v.abs()
        e = 2.0 ** -23
        bound = 1.01 * (HALF * r.abs() + (2.0 ** -16 + (260 * mag + 3 * L + 32) * e) * a)
        at = slice(c["cu"][s], c["cu"][s + 1])
        out[0, :, at], off[0, :, at] = (t.view(*q.shape).flatten(0, 1) for t in (r, bound))
    return out, off


def emulate(c, numbers):
    """The output with the weights times V's scale as the sum of `numbers` bf16
    numbers, all else in float64."""
    out = torch.zeros(c["q"].shape, dtype=torch.float64)
    for s in range(len(c["lengths"])):
        q, k, v, vs, seen = sequence(c, s)
        if q.shape[2] == 0:
            continue
        x = (q.flatten(1, 2) @ k.transpose(1, 2)).view(*q.shape[:3], -1) / math.sqrt(D)
        x = x.masked_fill(~seen, -math.inf)
        p = torch.exp(x - x.amax(-1, keepdim=True)).flatten(1, 2)
        weight = p * vs[:, None]
        got = torch.zeros_like(weight)
        for _ in range(numbers):
            got += (weight - got).to(torch.bfloat16).double()
        o = (got / vs[:, None]) @ v / p.sum(-1, keepdim=True)
        at = slice(c["cu"][s], c["cu"][s + 1])
        out[0, :, at] = o.view(*q.shape).flatten(0, 1)
    return out.to(torch.bfloat16)


# held, new tokens; query heads, KV heads: one row tile of 16 rows, of 32, two of 32
CASES = [([0, 1, 5, 30, 62, 63], [1] * 6, 4, 1), ([9, 40, 17, 3], [1] * 4, 8, 4),
         ([20, 2, 50], [1, 3, 4], 16, 2), ([33, 7], [7, 9], 16, 2)]
