"""Attention of sequences that share their first pages, against the attention of
each sequence by itself on the CPU in float64."""
import math

import pytest
import torch

from paper_2606_09508_amd import binding as eb

pytestmark = pytest.mark.gpu

D = 128
E4M3, INT8 = torch.float8_e4m3fn, torch.int8
QMAX = {E4M3: 448.0, INT8: 127.0}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32)


def _offsets(n):
    cu = [0]
    for x in n:
        cu.append(cu[-1] + x)
    return cu


class Batch:
    """Groups (sizes, shared pages) of sequences with `mine` further tokens each, the
    last `new` of them new."""

    def __init__(self, sizes, prefixes, mine, new, hq, hkv, P, dtype, seed=0, spare=1):
        g = _gen(seed)
        self.hq, self.hkv, self.P, self.dtype = hq, hkv, P, dtype
        group = [i for i, n in enumerate(sizes) for _ in range(n)]
        self.lengths = [prefixes[i] * P + m for i, m in zip(group, mine)]
        self.new, self.cu = new, _offsets(new)
        self.group_seqs, self.shared = _offsets(sizes), list(prefixes)
        pool = sum(prefixes) + sum(-(-m // P) for m in mine) + 3
        at = torch.randperm(pool, generator=g).tolist()
        common = [[at.pop() for _ in range(n)] for n in prefixes]
        cols = max(-(-n // P) for n in self.lengths) + spare
        self.table = []
        for i, m in zip(group, mine):
            row = common[i] + [at.pop() for _ in range(-(-m // P))]
            self.table.append(row + [-1] * (cols - len(row)))
        x = torch.randn((2, pool, hkv, P, D), generator=g) * (QMAX[dtype] / 4)
        x = x.clamp(-QMAX[dtype], QMAX[dtype])
        self.codes = x.to(E4M3) if dtype is E4M3 else x.round().to(INT8)
        self.scales = torch.exp2(torch.randint(-9, -5, (2, pool, hkv), generator=g).float())
        self.q = (torch.randn((1, hq, self.cu[-1], D), generator=g) * 0.5).to(torch.bfloat16)

    def run(self, packed=True, **more):
        pages = eb.CachePages(self.codes[0].clone().cuda(), self.codes[1].clone().cuda(),
                              self.scales[0].clone().cuda(), self.scales[1].clone().cuda())
        return eb.cache_attn_shared(
            self.q.cuda(), pages, _i32(self.table).cuda(), _i32(self.lengths).cuda(),
            _i32(self.group_seqs).cuda(), _i32(self.shared).cuda(),
            _i32(self.cu).cuda() if packed else None, **more)

    def reference(self):
        """(result, softmax times |v|, the largest |q||k| sum of a score, keys)."""
        out = torch.zeros(self.q.shape[1:], dtype=torch.float64)
        size, steep, most = out.clone(), 0.0, 0
        G, P = self.hq // self.hkv, self.P
        for s, L in enumerate(self.lengths):
            n = self.cu[s + 1] - self.cu[s]
            L = max(L, 0)
            k, v, here = [], [], []
            for c in range(min(-(-L // P), len(self.table[s]))):
                page = self.table[s][c]
                rows = min(P, L - c * P)
                ok = 0 <= page < self.codes.shape[1]
                page = page if ok else 0
                for to, side in ((k, 0), (v, 1)):
                    to.append(self.codes[side, page, :, :rows].float().double()
                              * self.scales[side, page].double()[:, None, None])
                here += [ok] * rows
            if n == 0 or not here:
                continue
            k, v, here = torch.cat(k, 1), torch.cat(v, 1), torch.tensor(here)
            pos = self.lengths[s] - n + torch.arange(n)
            seen = here & (torch.arange(len(here)) <= pos[:, None])
            k, v = k[:, here], v[:, here]
            seen = seen[:, here]
            most = max(most, int(here.sum()))
            for h in range(self.hq):
                q = self.q[0, h, self.cu[s]:self.cu[s + 1]].double()
                if not k.shape[1]:
                    continue
                x = q @ k[h // G].T / math.sqrt(D)
                steep = max(steep, float((q.abs() @ k[h // G].nan_to_num().abs().T).max())
                            / math.sqrt(D))
                x = x.masked_fill(~seen, -math.inf)
                p = torch.softmax(x, -1).nan_to_num() if seen.any() else torch.zeros_like(x)
                p = torch.where(seen.any(1, keepdim=True), p, 0.0)
                out[h, self.cu[s]:self.cu[s + 1]] = p @ v[h // G]
                size[h, self.cu[s]:self.cu[s + 1]] = p @ v[h // G].abs()
        return out[None], size[None], steep, most

    def check(self, got=None, packed=True):
        """A score is off by 128 roundings of its products' sum (in base 2 by 1.5 times
        that, as is the exponential by ln 2 times that), a probability by that, by one
        of exp2's last places and by fp16's half step; sums by 2^-23 a key; all of
        it once in the sums of values, once in the sum of weights."""
        got = (self.run(packed) if got is None else got).cpu().double()
        want, size, steep, most = self.reference()
        rel = 2 * (128 * 2.0 ** -23 * steep + 2.0 ** -22 + most * 2.0 ** -23) + 2.0 ** -11
        off = rel * size + most * 2.0 ** -32 * size.max()
        assert torch.isfinite(got).all()
        assert ((got - want).abs() <= off + 2.0 ** -8 * (want.abs() + off)).all()
        return got


HEADS = [(4, 1), (8, 2), (7, 1), (8, 8), (16, 2)]


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("P", [64, 128])
@pytest.mark.parametrize("hq,hkv", HEADS)
@pytest.mark.parametrize("sizes,prefixes,mine,new", [
    ([2], [1], [1, 1], [1, 1]),
    ([3], [5], [30, 1, 65], [1, 1, 1]),
    ([9, 1, 4], [3, 0, 7], [17 * i % 140 + 5 for i in range(14)], [1 + i % 5 for i in range(14)]),
    ([20], [4], [10 + i for i in range(20)], [1] * 20),
    ([40, 3], [9, 2], [1 + 5 * i for i in range(43)], [1] * 43),
    ([2, 2], [3, 2], [90, 100, 40, 40], [33, 0, 7, 31]),
])
def test_against_each_by_itself(sizes, prefixes, mine, new, hq, hkv, P, dtype):
    Batch(sizes, prefixes, mine, new, hq, hkv, P, dtype, seed=P + hq).check()


@pytest.mark.parametrize("hq,hkv", [(4, 1), (16, 2)])
def test_the_same_number_of_tokens_each(hq, hkv):
    for new in (1, 3, 8):
        b = Batch([12], [6], [8 + i for i in range(12)], [new] * 12, hq, hkv, 64, E4M3, seed=new)
        assert torch.equal(b.check(packed=False), b.check(packed=True))


@pytest.mark.parametrize("pages", [1, 2, 3, 100, 257])
def test_lengths_of_the_shared_part(pages):
    """From a half-filled step to more steps than there are workers."""
    Batch([30], [pages], [3] * 30, [1] * 30, 4, 1, 64, E4M3, seed=pages).check()
    Batch([3], [pages], [70] * 3, [1] * 3, 4, 1, 64, E4M3, seed=pages).check()


@pytest.mark.parametrize("groups,size", [(1, 257), (256, 1), (257, 1), (300, 4), (255, 1), (2, 128)])
def test_many_sequences_and_groups(groups, size):
    """More than a thread each of the smaller plan has, and as many."""
    S = groups * size
    b = Batch([size] * groups, [1 + g % 2 for g in range(groups)], [1 + i % 70 for i in range(S)],
              [1] * S, 2, 1, 64, E4M3, seed=groups)
    b.check()
    b.group_seqs, b.shared = b.group_seqs[:groups // 2 + 1], b.shared[:groups // 2]
    b.check()


def test_many_rows_of_one_sequence():
    """A group of one: its new tokens read what lies before them once."""
    Batch([1, 1], [20, 0], [300, 64], [257, 64], 8, 2, 64, E4M3, seed=3).check()


@pytest.mark.parametrize("size", [2, 30])
def test_shared_pages_that_new_tokens_lie_in(size):
    """All sequences have the same pages; the new tokens are somewhere in them."""
    b = Batch([size], [4], [1] * size, [1] * size, 4, 1, 64, E4M3, seed=size)
    for s in range(size):
        b.lengths[s] = 40 + (37 * s) % 200
    b.shared = [5]
    b.table = [list(b.table[0]) for _ in range(size)]
    b.check()
    b.lengths[1] = 0
    b.check()
    b.lengths[0] = -3
    b.check()


@pytest.mark.parametrize("size", [2, 30])
def test_numbers_that_make_no_sense(size):
    """Shares below zero or past the table, sequences of no group, empty groups."""
    b = Batch([size], [3], [20] * size, [1] * size, 4, 1, 64, E4M3, seed=size, spare=0)
    for shared in ([-5], [2 ** 31 - 1], [-2 ** 31]):
        b.shared = shared if shared[0] < 0 else [3]
        b.check()
    b.group_seqs, b.shared = [0], []
    b.check()
    b.group_seqs, b.shared = [1, 1, size - 1, size - 1], [3, 3, 3]
    b.check()
    b.group_seqs, b.shared = [-7, size + 9], [3]
    b.check()


@pytest.mark.parametrize("groups", [[0, 30, 0, 30, 0, 30], [30, 0], [20, 10, 25, 5],
                                    [2 ** 31 - 1, -2 ** 31, 30]])
def test_groups_that_do_not_ascend_touch_nothing_outside(groups):
    b = Batch([30], [3], [20] * 30, [1] * 30, 4, 1, 64, E4M3, seed=1)
    b.group_seqs, b.shared = groups, [3] * (len(groups) - 1)
    out = torch.full((3 * 4 * 30 * D,), 7.0, dtype=torch.bfloat16, device="cuda")
    n = 4 * 30 * D
    b.run(out=out[n:2 * n].view(1, 4, 30, D))
    assert (out[:n] == 7).all() and (out[2 * n:] == 7).all()


@pytest.mark.parametrize("cu", [[0, 9, 3, 12], [12, 0, 12, 0], [-5, 100, 7, 2 ** 31 - 1]])
def test_offsets_that_do_not_ascend_touch_nothing_outside(cu):
    for groups, shared in (([0, 3], [2]), ([0], [])):
        b = Batch([3], [2], [40] * 3, [4] * 3, 16, 1, 64, E4M3, seed=1)
        b.cu, b.group_seqs, b.shared = cu, groups, shared
        n = 16 * 12 * D
        out = torch.full((3 * n,), 7.0, dtype=torch.bfloat16, device="cuda")
        b.run(out=out[n:2 * n].view(1, 16, 12, D))
        assert (out[:n] == 7).all() and (out[2 * n:] == 7).all()


def test_rows_of_no_sequence_are_left():
    b = Batch([20], [2], [40] * 20, [1] * 20, 4, 1, 64, E4M3, seed=4)
    whole = b.check()
    b.q = torch.cat([b.q[:, :, :3] * 0 + float("nan"), b.q, b.q[:, :, :2] * float("inf")], 2)
    b.cu = [3 + i for i in range(21)]
    out = torch.full(b.q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    got = b.run(out=out).cpu().double()
    assert (got[:, :, :3] == 7).all() and (got[:, :, 23:] == 7).all()
    assert torch.equal(got[:, :, 3:23], whole)


@pytest.mark.parametrize("size", [3, 30])
def test_pages_that_are_none(size):
    b = Batch([size], [6], [100] * size, [1] * size, 4, 1, 64, E4M3, seed=size)
    for c, page in ((0, -1), (3, 10 ** 6), (7, -2 ** 31)):
        for s in range(size):
            if c < 6 or s % 2:
                b.table[s][c] = page
    b.check()
    for s in range(size):
        b.table[s] = [-1] * len(b.table[s])
    assert (b.run() == 0).all()


@pytest.mark.parametrize("size", [3, 30])
def test_what_is_not_finite(size):
    """Rows behind a sequence's end and pages of others hold NaN; a page of NaN makes
    NaN of those who see it."""
    b = Batch([size, 2], [5, 3], [30] * (size + 2), [1] * (size + 2), 4, 1, 64, E4M3, seed=size)
    raw = b.codes.view(torch.uint8)
    clean = b.check()
    last = [b.table[s][(n - 1) // 64] for s, n in enumerate(b.lengths)]
    for page in last:
        raw[:, page, :, 30:] = 0x7f
    assert torch.equal(b.run().cpu().double(), clean)
    b.scales[1, last[1]] = float("nan")       # a page of sequence 1 alone
    got = b.run().cpu().double()
    assert got[:, :, 1].isnan().all()
    keep = [i for i in range(size + 2) if i != 1]
    assert torch.equal(got[:, :, keep], clean[:, :, keep])
    b.scales[0, b.table[0][2]] = float("nan")        # a page of the first group
    got = b.run().cpu().double()
    assert got[:, :, :size].isnan().all()
    assert torch.equal(got[:, :, size:], clean[:, :, size:])


@pytest.mark.parametrize("size", [3, 30])
@pytest.mark.parametrize("scales", [
    [0.0, 0.0, 2.0 ** -7, 0.0, 0.0], [2.0 ** -60, 2.0 ** 50, 2.0 ** -7, 2.0 ** 3, 2.0 ** -40],
    [0.3, 1.7, 3e-5, 0.01, 1000.0], [-0.5, 0.25, -3.0, 0.1, 0.7], [2.0 ** -80] * 5, [2.0 ** 55] * 5])
def test_scales_of_the_values(size, scales):
    b = Batch([size], [5], [40] * size, [1] * size, 4, 1, 64, E4M3, seed=size)
    for c, f in enumerate(scales):
        b.scales[1, b.table[0][c]] = f
    for s in range(size):
        b.scales[1, b.table[s][5]] = scales[2]
    got = b.run().cpu().double()
    want, size_, steep, most = b.reference()
    rel = 2 * (128 * 2.0 ** -23 * steep + 2.0 ** -22 + most * 2.0 ** -23) + 2.0 ** -11
    off = rel * size_ + most * 2.0 ** -32 * size_.amax(-1, keepdim=True)
    assert ((got - want).abs() <= off + 2.0 ** -8 * (want.abs() + off)).all()


@pytest.mark.parametrize("size", [3, 30])
@pytest.mark.parametrize("where", ["first", "last"])
def test_one_key_far_above_the_others(size, where):
    """A running maximum that jumps, in the shared part or behind it."""
    b = Batch([size], [9], [40] * size, [1] * size, 4, 1, 64, E4M3, seed=size)
    page = b.table[0][0 if where == "first" else 8]
    b.codes[0, page, 0, 17] = (b.q[0, 0, 0].float() * 400).clamp(-448, 448).to(E4M3)
    b.scales[0, page] = 0.5
    b.check()
    b.q *= 8
    b.check()


def test_against_cache_attn():
    b = Batch([5, 25], [10, 4], [30 + i for i in range(30)], [1] * 30, 8, 2, 64, E4M3, seed=6)
    pages = eb.CachePages(b.codes[0].cuda(), b.codes[1].cuda(), b.scales[0].cuda(),
                          b.scales[1].cuda())
    b.check(eb.cache_attn(b.q.cuda(), pages, _i32(b.table).cuda(), _i32(b.lengths).cuda()))
    b.check()


def test_streams_graphs_and_one_workspace():
    b = Batch([5, 25], [10, 4], [30 + i for i in range(30)], [1] * 30, 8, 2, 64, E4M3, seed=7)
    pages = eb.CachePages(b.codes[0].cuda(), b.codes[1].cuda(), b.scales[0].cuda(),
                          b.scales[1].cuda())
    q, table, lengths = b.q.cuda(), _i32(b.table).cuda(), _i32(b.lengths).cuda()
    groups, shared = _i32(b.group_seqs).cuda(), _i32(b.shared).cuda()
    ws = torch.empty(eb.cache_attn_shared_workspace_bytes(8, 30, 30, 2, table.shape[1], pages),
                     dtype=torch.uint8, device="cuda").fill_(0xff)

    def call(out=None, workspace=ws):
        return eb.cache_attn_shared(q, pages, table, lengths, groups, shared, out=out,
                                    workspace=workspace)

    want = call(workspace=None)
    assert torch.equal(call(), want) and torch.equal(call(), want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = call(workspace=None)
    side.synchronize()
    assert torch.equal(other, want)
    out = torch.empty_like(q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(out)
    for i in range(4):
        lengths.sub_(i)
        shared.copy_(_i32([10, 4] if i % 2 == 0 else [3, 0]))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, call(workspace=None))


def test_binding_refusals():
    b = Batch([2], [1], [5, 5], [1, 1], 4, 1, 64, E4M3)
    with pytest.raises(ValueError, match="offsets for"):
        b.shared = [1, 1]
        b.run()
    b.shared = [1]
    with pytest.raises(eb.EIError, match="WORKSPACE"):
        b.run(workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError, match="does not match q"):
        b.run(out=torch.empty((1, 4, 3, D), dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError, match="does not match the pages"):
        b.q = b.q[..., :64].contiguous()
        b.run()
