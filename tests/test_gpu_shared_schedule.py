"""Shared-prefix attention with more work than the least run of each worker: runs
of several steps that cross items, items that are whole runs, and divisions that
leave a rest, against float64 on the GPU."""
import math

import pytest
import torch

from paper_2606_09508_amd import binding as eb

pytestmark = pytest.mark.gpu

D, P = 128, 64


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _offsets(n):
    cu = [0]
    for x in n:
        cu.append(cu[-1] + x)
    return cu


def _call(sizes, prefixes, mine, hq, hkv, seed):
    """Groups (sizes, shared pages) of sequences of one new token with `mine` tokens of
    their own: the arguments of the call, and each group's sequences."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    group = [i for i, n in enumerate(sizes) for _ in range(n)]
    S, at = len(group), 0
    common = []
    for n in prefixes:
        common.append(list(range(at, at + n)))
        at += n
    rows = []
    for i, m in zip(group, mine):
        n = -(-m // P)
        rows.append(common[i] + list(range(at, at + n)))
        at += n
    cols = max(map(len, rows))
    order = torch.randperm(at, generator=g, device="cuda").to(torch.int32)
    table = _i32([r + [0] * (cols - len(r)) for r in rows])
    table = order[table.long()].contiguous()
    codes = torch.empty((2, at, hkv, P, D), dtype=torch.float8_e4m3fn, device="cuda")
    for side in codes:
        x = torch.randn(side.shape, generator=g, device="cuda")
        side.copy_((x * 112).clamp_(-448, 448).to(torch.float8_e4m3fn))
    scales = torch.exp2(torch.randint(-9, -5, (2, at, hkv), generator=g, device="cuda").float())
    pages = eb.CachePages(codes[0], codes[1], scales[0], scales[1])
    lengths = _i32([prefixes[i] * P + m for i, m in zip(group, mine)])
    q = (torch.randn((1, hq, S, D), generator=g, device="cuda") * 0.5).to(torch.bfloat16)
    return q, pages, table, lengths, _i32(_offsets(sizes)), _i32(prefixes)


def _check(got, q, pages, table, lengths, group_seqs, shared):
    """A score is off by 128 roundings of its products' sum (in base 2 by 1.5 times
    that, as is the exponential by ln 2 times that), a probability by that, by one
    of exp2's last places and by fp16's half step; sums by 2^-23 a key; all of it once
    in the sums of values, once in the sum of weights."""
    hq, hkv = q.shape[1], pages.k.shape[1]
    assert torch.isfinite(got).all()
    for s, L in enumerate(lengths.tolist()):
        at = table[s, :-(-L // P)].long()
        k, v = ((c.view(torch.uint8)[at].view(c.dtype).double() * f[at].double()[..., None, None])
                .transpose(0, 1).flatten(1, 2)[:, :L].contiguous()
                for c, f in ((pages.k, pages.k_scale), (pages.v, pages.v_scale)))
        x = q[0, :, s].double().view(hkv, -1, D)
        kt = k.transpose(1, 2).contiguous()
        p = torch.softmax(x @ kt / math.sqrt(D), -1)
        steep = float((x.abs() @ kt.abs()).max()) / math.sqrt(D)
        want, size = (p @ v).view(hq, D), (p @ v.abs()).view(hq, D)
        rel = 2 * (128 * 2.0 ** -23 * steep + 2.0 ** -22 + L * 2.0 ** -23) + 2.0 ** -11
        off = rel * size + L * 2.0 ** -32 * size.max()
        assert ((got[0, :, s].double() - want).abs() <= off + 2.0 ** -8 * (want.abs() + off)).all(), s


# wide tiles: 16 items of 64 steps, four to a run; of 64.5 steps, which do not divide; of
# 63; 8 items of 64 rows, two steps to a run, and a rest; groups of unequal lengths;
# equal ones of different tiles
@pytest.mark.parametrize("sizes,prefixes,hq,hkv", [
    ([64], [128], 32, 8), ([64], [129], 32, 8), ([64], [126], 32, 8),
    ([12], [128], 32, 8), ([12], [131], 32, 8), ([10], [257], 32, 8),
    ([40, 24], [150, 77], 32, 8), ([33, 40, 33], [96, 64, 64], 32, 8), ([20, 50], [128, 128], 32, 8),
    ([90], [512], 8, 2), ([90], [515], 8, 2),
    # few rows: more steps than the least run of 2048 waves
    ([2, 3], [700, 900], 32, 8), ([3], [1200], 32, 8), ([2, 1, 2], [500, 0, 650], 64, 8),
])
def test_runs_of_many_steps(sizes, prefixes, hq, hkv):
    S = sum(sizes)
    args = _call(sizes, prefixes, [3 + 37 * i % 150 for i in range(S)], hq, hkv, S)
    got = eb.cache_attn_shared(*args)
    _check(got, *args)
    assert torch.equal(got, eb.cache_attn_shared(*args))


def test_long_keys_of_each_sequence():
    """More steps of the sequences' own keys than the waves' least runs."""
    args = _call([36], [128], [2500 + 41 * i for i in range(36)], 32, 8, 5)
    _check(eb.cache_attn_shared(*args), *args)
