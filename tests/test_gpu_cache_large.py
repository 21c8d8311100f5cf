"""Cache attention in launches that fill the chip, whose keys are dealt out in
longer and shorter runs: against float64, and with values that tell which keys
came in.  cache_share_model names the path each launch takes."""
import math

import pytest
import torch

from cache_share_model import LARGE, large
from paper_2606_09508_amd import binding as eb

pytestmark = pytest.mark.gpu

D = 128
HALF = 2.0 ** -8   # half a bf16 step, relative
E4M3, INT8 = torch.float8_e4m3fn, torch.int8


def _setup(plan, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    S, P = len(plan.new), plan.page_len
    counts = [-(-n // P) for n in plan.lengths]
    n_pages = sum(counts) + 2
    at = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((S, plan.cols), -1, dtype=torch.int32, device="cuda")
    first = 0
    for s, c in enumerate(counts):
        table[s, :c] = at[first:first + c]
        first += c
    top = 448.0 if dtype is E4M3 else 127.0
    codes = []
    for _ in range(2):
        x = torch.randn((n_pages, plan.hkv, P, D), generator=g, device="cuda")
        x = x.mul_(top / 4).clamp_(-top, top)
        codes.append(x.to(E4M3) if dtype is E4M3 else x.round_().to(INT8))
    e = [torch.randint(-9, -6, (n_pages, plan.hkv), generator=g, device="cuda") for _ in range(2)]
    cu = [0]
    for n in plan.new:
        cu.append(cu[-1] + n)
    q = torch.randn((1, plan.hq, cu[-1], D), generator=g, device="cuda").to(torch.bfloat16)
    return eb.CachePages(*codes, *(torch.exp2(x.float()) for x in e)), table, cu, q


def _attend(plan, q, pages, table, cu):
    lengths = torch.tensor(plan.lengths, dtype=torch.int32, device="cuda")
    offsets = None if len(set(plan.new)) == 1 else torch.tensor(cu, dtype=torch.int32, device="cuda")
    return eb.cache_attn(q, pages, table, lengths, offsets)


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("name", LARGE)
def test_against_float64(name, dtype):
    """An output r with a = (its weights) |v| is off by HALF |r|, its rounding, and of
    a by 2^-16, the weights' 16 bits; 2 * 130 e mag, fp32 scores of magnitudes
    `mag`, also in the weights' sum; and e for each sum's additions one after the
    other: 32 a step of a wave's run for the weights and for each of the two
    products, one a part that is joined, one a wave of a workgroup.  e = 2^-23, as
    matrix cores may truncate; 1.01 for the products of these."""
    _, plan = large(name)
    plan.check()
    pages, table, cu, q = _setup(plan, dtype, 5)
    q = (q * 0.3).to(torch.bfloat16)
    got = _attend(plan, q, pages, table, cu)[0].double()
    adds = 3 * 32 * plan.most_steps + 2 * plan.most_parts + 40
    some = range(len(plan.new)) if len(plan.new) <= 60 else range(0, len(plan.new), 13)
    for s in some:
        n, L, P = plan.new[s], plan.lengths[s], plan.page_len
        if n == 0:
            continue
        at = table[s, :-(-L // P)].long()
        for h in range(plan.hkv):
            k, v = ((c.view(torch.uint8)[at, h].view(c.dtype).float().double()
                     * f[at, h].double()[:, None, None]).flatten(0, 1)[:L]
                    for c, f in ((pages.k, pages.k_scale), (pages.v, pages.v_scale)))
            G = plan.hq // plan.hkv
            heads = slice(h * G, (h + 1) * G)
            x = q[0, heads, cu[s]:cu[s + 1]].double().reshape(-1, D)
            c = 1.0 / math.sqrt(D)
            score = (x @ k.T.contiguous() * c).view(G, n, L)
            mag = float((x.abs() @ k.abs().T.contiguous()).max()) * c
            last = L - n + torch.arange(n, device="cuda")
            score.masked_fill_(torch.arange(L, device="cuda") > last[:, None], -math.inf)
            w = torch.softmax(score, -1).flatten(0, 1)
            r, a = w @ v, w @ v.abs()
            off = 1.01 * (HALF * r.abs() + (2.0 ** -16 + (260 * mag + adds) * 2.0 ** -23) * a)
            err = (got[heads, cu[s]:cu[s + 1]].reshape(-1, D) - r).abs()
            assert bool((err <= off).all()), (s, h, float((err / off).max()))


@pytest.mark.parametrize("name", LARGE)
def test_every_key_counts_once(name):
    """Weights all alike, and the keys of a step of 32 in a dim that only steps 128
    further on share: an output is the share of its dim's keys among those seen.
    Leaving out a step or taking it twice moves an element by an eleventh of
    itself at least (40001 tokens); it may be off by its rounding, 2^-8, and those
    of the sums."""
    _, plan = large(name)
    plan.check()
    pages, table, cu, q = _setup(plan, E4M3, 6)
    q.zero_()
    P = plan.page_len
    v = torch.zeros(pages.v.shape, device="cuda")
    pages.v_scale.fill_(0.5)
    dims = []
    for s, L in enumerate(plan.lengths):
        p = torch.arange(-(-L // P) * P, device="cuda")
        dim = p // 32 % D
        dims.append(dim[:L])
        v[table[s, p // P].long(), :, p % P, dim] = 2.0
    pages.v.copy_(v.to(E4M3))
    got = _attend(plan, q, pages, table, cu)[0].double()
    for s, L in enumerate(plan.lengths):
        for i in range(plan.new[s]):
            sees = L - plan.new[s] + i + 1
            share = torch.bincount(dims[s][:sees], minlength=D).double() / sees
            err = (got[:, cu[s] + i] - share).abs()
            assert bool((err <= (2.0 ** -8 + 1e-3) * share).all()), (s, i)
