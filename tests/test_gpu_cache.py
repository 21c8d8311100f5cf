"""The paged 8-bit cache: storing, attention over it, copies of its pages,
against plain implementations on the CPU in float64, a page or a sequence at a
time."""
import math

import pytest
import torch

from paper_2606_09508_amd import binding as eb

pytestmark = pytest.mark.gpu

D = 128
HALF = 2.0 ** -8   # half a bf16 step, relative
E4M3, INT8 = torch.float8_e4m3fn, torch.int8
QMAX = {E4M3: 448.0, INT8: 127.0}


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _rand(shape, seed, scale=1.0):
    return (torch.randn(shape, generator=_gen(seed)) * scale).to(torch.bfloat16)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32)


def _offsets(lengths):
    cu = [0]
    for n in lengths:
        cu.append(cu[-1] + n)
    return cu


def _table(lengths, P, n_pages, seed=0, spare=1):
    """Pages anywhere in the pool, none twice; -1 behind a sequence's own."""
    at = torch.randperm(n_pages, generator=_gen(seed)).tolist()
    cols = max(-(-max(n, 0) // P) for n in lengths) + spare
    rows = []
    for n in lengths:
        c = -(-max(n, 0) // P)
        rows.append([at.pop() for _ in range(c)] + [-1] * (cols - c))
    return rows


def _bytes(t):
    return t.view(torch.uint8)


def _pages(n_pages, hkv, P, dtype, seed):
    """Filled pages on the CPU, codes and scales as a store leaves them."""
    x = torch.randn((2, n_pages, hkv, P, D), generator=_gen(seed)) * (QMAX[dtype] / 4)
    x = x.clamp(-QMAX[dtype], QMAX[dtype])
    codes = x.to(E4M3) if dtype is E4M3 else x.round().to(INT8)
    scale = torch.exp2(torch.randint(-9, -5, (2, n_pages, hkv), generator=_gen(seed + 1)).float())
    return eb.CachePages(codes[0].clone(), codes[1].clone(), scale[0].clone(), scale[1].clone())


def _cuda(pages):
    return eb.CachePages(*(t.cuda() for t in pages))


# --------------------------------------------------------------------------
# Store
# --------------------------------------------------------------------------

def _round(x, dtype):
    return x.float().to(E4M3) if dtype is E4M3 else torch.round(x).to(INT8)


def store_reference(pages, k, v, table, lengths, cu):
    """The definition, a page at a time, in float64 (every value before the
    rounding to a code is exact there)."""
    for codes, scale, x in ((pages.k, pages.k_scale, k), (pages.v, pages.v_scale, v)):
        dtype, P = codes.dtype, codes.shape[2]
        for s in range(len(lengths)):
            n = cu[s + 1] - cu[s]
            begin = lengths[s] - n
            p = max(begin, 0)
            while p < lengths[s]:
                r, take = p % P, min(P - p % P, lengths[s] - p)
                c, at = p // P, cu[s] + p - begin
                p += take
                page = table[s][c] if c < len(table[s]) else -1
                if not 0 <= page < codes.shape[0]:
                    continue
                for h in range(codes.shape[1]):
                    rows = x[0, h, at:at + take].double()
                    old = float(scale[page, h]) if r else 0.0
                    top = float(rows.abs().max())
                    if not math.isfinite(top) or math.isnan(old):
                        scale[page, h] = math.nan
                        _bytes(codes)[page, h, r:r + take] = 0
                        continue
                    e = -126
                    while math.ldexp(QMAX[dtype], e) < top:
                        e += 1
                    new = max(old, math.ldexp(1.0, e))
                    if r and new != old:
                        was = codes[page, h, :r].double() if dtype is INT8 else \
                            codes[page, h, :r].float().double()
                        _bytes(codes)[page, h, :r] = _bytes(_round(was * (old / new), dtype))
                    _bytes(codes)[page, h, r:r + take] = _bytes(_round(rows / new, dtype))
                    scale[page, h] = new


def same_pages(got, want):
    for name, a, b in zip(want._fields, got, want):
        a = a.cpu()
        if a.dtype is E4M3:      # (-0 and 0 are one value)
            a, b = a.float(), b.float()
        assert torch.equal(a.isnan(), b.isnan()), name
        assert torch.equal(a.nan_to_num() if a.is_floating_point() else a,
                           b.nan_to_num() if b.is_floating_point() else b), name


def run_store(held, new, hkv, P, dtype, packed=True, scale=1.0, seed=0, edit=None):
    lengths = [a + b for a, b in zip(held, new)]
    cu = _offsets(new)
    n_pages = sum(-(-max(n, 0) // P) for n in lengths) + 2
    table = _table(lengths, P, n_pages, seed)
    pages = _pages(n_pages, hkv, P, dtype, seed + 10)
    k, v = _rand((1, hkv, cu[-1], D), seed + 1, scale), _rand((1, hkv, cu[-1], D), seed + 2, scale)
    if edit:
        edit(pages, k, v, table)
    dev = _cuda(pages)
    eb.cache_store(k.cuda(), v.cuda(), dev, _i32(table).cuda(), _i32(lengths).cuda(),
                   _i32(cu).cuda() if packed else None)
    store_reference(pages, k, v, table, lengths, cu)
    same_pages(dev, pages)
    return dev, pages


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("P", [64, 128])
@pytest.mark.parametrize("held,new", [
    ([0], [1]), ([0, 0, 0], [63, 64, 65]), ([5, 63, 64, 127], [1, 1, 1, 1]),
    ([100, 0, 37, 200, 1], [0, 129, 300, 0, 2]), ([1, 1], [127, 126]),
    (list(range(0, 140, 7)), [1, 2] * 10), ([0] * 3, [0, 0, 1]),
])
def test_store(held, new, P, dtype):
    run_store(held, new, 2, P, dtype)


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("each", [1, 2, 64, 65, 100])
def test_store_equal_counts_without_offsets(each, dtype):
    run_store([0, 63, 64, 10, 200], [each] * 5, 3, 64, dtype, packed=False)


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("scale", [1e-38, 1e-20, 2.0 ** -9, 30.0, 1e30])
def test_store_rescales_what_the_page_holds(scale, dtype):
    """New rows far smaller and far larger than the rows the page has."""
    run_store([7, 40, 0], [9, 10, 11], 2, 64, dtype, scale=scale)


@pytest.mark.parametrize("dtype", [E4M3, INT8])
def test_store_scale_at_its_borders(dtype):
    """Largest elements at the end of the code range and a bf16 step past it,
    zero rows, and the largest and smallest numbers there are."""
    q = QMAX[dtype]
    for i, top in enumerate([q, q * (1 + 2.0 ** -7), q * (1 - 2.0 ** -8), 1.0, 2.0, 0.0,
                             3.3895313892515355e38, 2.0 ** -126, 2.0 ** -133, 1.5 * 2.0 ** -120]):
        def edit(pages, k, v, table):
            t = torch.tensor(top).to(torch.bfloat16)
            for x in (k, v):
                x.clamp_(-1, 1).mul_(t * 0.999)
                x[0, :, 3, 5] = -t
        run_store([0, 9], [20, 7], 1, 64, dtype, seed=i, edit=edit)


@pytest.mark.parametrize("dtype", [E4M3, INT8])
def test_store_of_non_finite_elements(dtype):
    """They make their page and head NaN, and only those; a page that was NaN
    stays so until its row 0 is stored again."""
    def edit(pages, k, v, table):
        k[0, 1, 70, 3] = math.inf
        v[0, 0, 2, 127] = math.nan
        pages.k_scale[table[1][0], 0] = math.nan
    dev, _ = run_store([0, 10], [130, 20], 2, 64, dtype, edit=edit)
    assert int(dev.k_scale.isnan().sum()) == 2 and int(dev.v_scale.isnan().sum()) == 1


def test_store_to_places_that_are_none():
    """Pages outside the pool, columns past the table and negative positions
    are left out, the other tokens stored."""
    hkv, P = 2, 64
    pages = _pages(6, hkv, P, E4M3, 3)
    table = [[0, 99, 1], [-1, 2, 3], [4, 5, -7]]
    lengths, new = [190, 300, 3], [190, 300, 5]      # 300 > 3 columns; begin = -2
    cu = _offsets(new)
    k, v = _rand((1, hkv, cu[-1], D), 4), _rand((1, hkv, cu[-1], D), 5)
    dev = _cuda(pages)
    eb.cache_store(k.cuda(), v.cuda(), dev, _i32(table).cuda(), _i32(lengths).cuda(),
                   _i32(cu).cuda())
    store_reference(pages, k, v, table, lengths, cu)
    same_pages(dev, pages)


@pytest.mark.parametrize("lead", [1, 70, 1000])
def test_store_behind_rows_of_no_sequence(lead):
    """The offsets begin at `lead`: the rows before are nobody's, also where the
    first sequence begins pages into its table."""
    hkv, P = 2, 64
    pages = _pages(40, hkv, P, E4M3, 3)
    lengths, new = [1200, 30, 129], [10, 30, 129]
    table = _table(lengths, P, 40)
    cu = [lead + c for c in _offsets(new)]
    k, v = _rand((1, hkv, cu[-1] + 5, D), 4), _rand((1, hkv, cu[-1] + 5, D), 5)
    dev = _cuda(pages)
    eb.cache_store(k.cuda(), v.cuda(), dev, _i32(table).cuda(), _i32(lengths).cuda(),
                   _i32(cu).cuda())
    store_reference(pages, k, v, table, lengths, cu)
    same_pages(dev, pages)


def test_token_by_token_is_close_to_all_at_once():
    """Every roundings' sum stays below one step of the final scale: exact for
    e4m3 values of the normal range, under a step for int8."""
    P, hkv, n = 64, 1, 64
    k = _rand((1, hkv, n, D), 7) * torch.logspace(-2, 2, n).to(torch.bfloat16)[:, None]
    for dtype in (E4M3, INT8):
        table, one = _i32([[1]]).cuda(), _cuda(_pages(2, hkv, P, dtype, 8))
        all_ = _cuda(_pages(2, hkv, P, dtype, 8))
        for i in range(n):
            x = k[:, :, i:i + 1].contiguous().cuda()
            eb.cache_store(x, x, one, table, _i32([i + 1]).cuda())
        eb.cache_store(k.cuda(), k.cuda(), all_, table, _i32([n]).cuda())
        assert torch.equal(one.k_scale[1], all_.k_scale[1])
        a, b = (t.k[1].float().cpu() for t in (one, all_))
        if dtype is INT8:   # each within one step of x / scale, the last within half
            assert float((a - b).abs().max()) <= 1.5
        else:               # half a step of 2^-9, once more for each of up to two subnormal roundings
            assert bool(((a - b).abs() <= 2.0 ** -9).all())
            assert torch.equal(a[b.abs() > 2.0 ** -6], b[b.abs() > 2.0 ** -6])


# --------------------------------------------------------------------------
# Attention
# --------------------------------------------------------------------------

def values(codes, scale):
    return codes.float().double() * scale.double()[..., None, None]


def attn_reference(q, pages, table, lengths, cu):
    """Output in float64 and how far a result may be off (as for the packed
    prompts: one rounding of the output, one of each probability, and the
    errors of fp32 sums of 128 products)."""
    kf, vf = values(pages.k, pages.k_scale), values(pages.v, pages.v_scale)
    P, hkv, hq = kf.shape[2], kf.shape[1], q.shape[1]
    o, off = torch.zeros(q.shape, dtype=torch.float64), torch.zeros(q.shape, dtype=torch.float64)
    c = 1.0 / math.sqrt(D)
    for s in range(len(lengths)):
        n = cu[s + 1] - cu[s]
        L = max(min(lengths[s], len(table[s]) * P), 0)
        ok = [p for p in range(L) if 0 <= table[s][p // P] < kf.shape[0]]
        for i in range(n):
            at = [p for p in ok if p <= lengths[s] - n + i]
            if not at:
                continue
            pg, rw = torch.tensor([table[s][p // P] for p in at]), torch.tensor(at) % P
            kk, vv = kf[pg, :, rw].transpose(0, 1), vf[pg, :, rw].transpose(0, 1)
            qq = q[0, :, cu[s] + i].double().view(hkv, hq // hkv, D)
            w = torch.softmax(qq @ kk.transpose(1, 2) * c, -1)
            mag = (qq.abs() @ kk.abs().transpose(1, 2)).amax() * c
            r, a = w @ vv, w @ vv.abs()
            o[0, :, cu[s] + i] = r.view(hq, D)
            off[0, :, cu[s] + i] = (1.01 * (HALF * r.abs() + (HALF + 2 * 130 * 2.0 ** -24 * mag
                                                             + 1e-5) * a)).view(hq, D)
    return o, off


def run_attn(held, new, hq, hkv, P, dtype, packed=True, seed=0, spare=1, edit=None):
    lengths = [a + b for a, b in zip(held, new)]
    cu = _offsets(new)
    n_pages = sum(-(-max(n, 0) // P) for n in lengths) + 2
    table = _table(lengths, P, n_pages, seed, spare)
    pages = _pages(n_pages, hkv, P, dtype, seed + 10)
    q = _rand((1, hq, cu[-1], D), seed + 1, 0.3)
    if edit:
        edit(pages, table, lengths)
    got = eb.cache_attn(q.cuda(), _cuda(pages), _i32(table).cuda(), _i32(lengths).cuda(),
                        _i32(cu).cuda() if packed else None).cpu()
    ref, off = attn_reference(q, pages, table, lengths, cu)
    err = (got.double() - ref).abs()
    assert bool((err <= off).all()), float((err - off).max())
    return got


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("P", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (7, 1), (4, 4), (20, 1), (6, 2)])
def test_attn_lengths(hq, hkv, P, dtype):
    run_attn([0, 30, 31, 32, 62, 63, 64, 127, 128, 500], [1] * 10, hq, hkv, P, dtype, packed=False)


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("new", [[2] * 4, [4, 0, 1, 9], [1, 40, 0, 0], [17, 3, 16, 5]])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (16, 2), (5, 5)])
def test_attn_several_new_tokens(new, hq, hkv, dtype):
    """Queries that see different numbers of keys, over more than one tile of
    rows."""
    run_attn([0, 100, 63, 250], new, hq, hkv, 64, dtype)


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("n", [3000, 5001])
def test_attn_long_sequence_in_parts(n, dtype):
    run_attn([n, 3], [1, 1], 8, 2, 64, dtype)


def test_attn_many_sequences():
    run_attn([(37 * i) % 200 for i in range(150)], [1] * 150, 8, 2, 64, E4M3)
    run_attn([(37 * i) % 200 for i in range(150)], [i % 3 for i in range(150)], 8, 2, 64, INT8)


def test_attn_wide_table():
    """A table far wider than the sequences are long."""
    run_attn([100, 40, 300], [1, 1, 1], 8, 2, 64, E4M3, spare=500)


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (16, 2), (24, 1)])
@pytest.mark.parametrize("held,new", [
    ([30] * 5, [1, 0, 3, 0, 2]),                       # items alike: a workgroup each
    ([0, 0, 1500, 0, 3], [1, 0, 2, 5, 0]),             # one far longer than the others
    ([7, 2500, 64, 0, 0, 900], [0, 1, 9, 0, 0, 1]),
    ([5] * 70 + [1100], [i % 2 for i in range(70)] + [3]),
    ([2000] + [1] * 130, [1] + [0] * 129 + [4]),       # the last of many without tokens
])
def test_attn_wide_table_of_ragged_sequences(held, new, hq, hkv, dtype):
    """The launches that find their share of the work on the device."""
    run_attn(held, new, hq, hkv, 64, dtype, spare=40)


def test_calls_of_no_tokens_and_of_no_sequences():
    pages, no = _cuda(_pages(4, 2, 64, E4M3, 1)), torch.empty((1, 2, 0, D), dtype=torch.bfloat16)
    before = [t.clone() for t in pages]
    for rows in (0, 3):
        table, lengths = torch.zeros((rows, 40), dtype=torch.int32), _i32([64] * rows)
        for cu in (None, torch.zeros(rows + 1, dtype=torch.int32).cuda()):
            eb.cache_store(no.cuda(), no.cuda(), pages, table.cuda(), lengths.cuda(), cu)
            got = eb.cache_attn(no.cuda(), pages, table.cuda(), lengths.cuda(), cu)
            assert got.shape == no.shape
        q = torch.ones((1, 2, rows, D), dtype=torch.bfloat16).cuda()
        assert eb.cache_attn(q[:, :, :0].contiguous(), pages, table[:, :0].contiguous().cuda(),
                             lengths.cuda()).numel() == 0
    none = torch.empty(0, dtype=torch.int32).cuda()
    eb.cache_copy(pages, none, none)
    assert all(torch.equal(_bytes(a), _bytes(b)) for a, b in zip(pages, before))


@pytest.mark.parametrize("spare", [1, 100])
def test_attn_far_before_the_first_position(spare):
    """More new tokens than the sequence holds, on pages and on none: the rows
    before position 0 see nothing."""
    def edit(pages, table, lengths):
        lengths[0], table[1][0] = 70, -1
        lengths[1] = 3
    got = run_attn([0, 0, 5], [400, 300, 2], 4, 2, 64, E4M3, edit=edit, spare=spare)
    assert bool((got[0, :, :330] == 0).all()) and bool((got[0, :, 400:700] == 0).all())
    assert bool((got[0, :, 330:400] != 0).any(-1).all())


@pytest.mark.parametrize("dtype", [E4M3, INT8])
def test_attn_rows_without_keys(dtype):
    """Length zero, and queries before the first position."""
    def edit(pages, table, lengths):
        lengths[0], lengths[1] = 0, 2      # 1 and 5 queries
        lengths[2] = -4
    wide = run_attn([3, 10, 8], [1, 5, 2], 4, 2, 64, dtype, edit=edit, spare=100)
    got = run_attn([3, 10, 8], [1, 5, 2], 4, 2, 64, dtype, edit=edit)
    assert bool((wide[0, :, [0, 1, 2, 3, 6, 7]] == 0).all())
    assert bool((got[0, :, [0, 1, 2, 3, 6, 7]] == 0).all())
    assert bool((got[0, :, 4:6] != 0).any())


def test_attn_pages_that_are_none():
    """Keys on pages outside the pool, and behind the table, are not seen."""
    def edit(pages, table, lengths):
        table[0][1], table[0][3] = -1, 10 ** 6
        table[1][0] = -5
        lengths[2] = 5000
    run_attn([400, 60, 100], [1, 1, 1], 8, 2, 64, E4M3, edit=edit)


@pytest.mark.parametrize("P", [64, 128])
def test_attn_does_not_read_behind_the_end(P):
    """NaN codes behind a sequence's last row, and NaN pages of others."""
    def edit(pages, table, lengths):
        for s, L in enumerate(lengths):
            if L % P:
                for t in (pages.k, pages.v):
                    _bytes(t)[table[s][L // P], :, L % P:] = 0x7f
        used = {p for row in table for p in row}
        for p in range(pages.k.shape[0]):
            if p not in used:
                pages.k_scale[p] = pages.v_scale[p] = math.nan
    run_attn([0, 5, 64, 77, 300], [1, 2, 1, 3, 1], 8, 2, P, E4M3, edit=edit)


@pytest.mark.parametrize("dtype", [E4M3, INT8])
def test_attn_nan_page_reaches_only_who_sees_it(dtype):
    """The page of the newest tokens is NaN: queries before it are not."""
    P = 64
    lengths, cu = [70], [0, 10]                       # queries at 60 .. 69
    pages = _pages(3, 2, P, dtype, 1)
    q = _rand((1, 4, 10, D), 2)
    table = [[0, 1]]
    want = eb.cache_attn(q.cuda(), _cuda(pages), _i32(table).cuda(), _i32(lengths).cuda(),
                         _i32(cu).cuda())
    pages.k_scale[1] = pages.v_scale[1] = math.nan
    got = eb.cache_attn(q.cuda(), _cuda(pages), _i32(table).cuda(), _i32(lengths).cuda(),
                        _i32(cu).cuda())
    assert torch.equal(got[:, :, :4], want[:, :, :4])
    assert bool(got[:, :, 4:].isnan().all())


def test_attn_scores_of_any_size():
    """Scores that rise by hundreds from page to page, and huge negative ones."""
    for sign in (1.0, -1.0):
        def edit(pages, table, lengths):
            pages.k_scale.mul_(sign * 50.0)
        run_attn([700, 90], [1, 3], 4, 1, 64, E4M3, edit=edit)


def test_attn_without_a_single_page():
    """A table without columns, and a pool without pages: zero rows."""
    q = _rand((1, 4, 2, D), 2).cuda()
    lengths = _i32([20, 30]).cuda()
    some, none = (eb.new_cache_pages(n, 2, 64) for n in (3, 0))
    table = torch.zeros((2, 0), dtype=torch.int32, device="cuda")
    assert bool((eb.cache_attn(q, some, table, lengths) == 0).all())
    for cols in (2, 100):
        table = torch.zeros((2, cols), dtype=torch.int32, device="cuda")
        assert bool((eb.cache_attn(q, none, table, lengths) == 0).all())
        eb.cache_store(q[:, :2].contiguous(), q[:, :2].contiguous(), none, table, lengths)


@pytest.mark.parametrize("n", [30, 2500])
def test_attn_non_finite_queries_stay_alone(n):
    """A query that is NaN or infinite makes its own row so, and no other, also
    of those that share its tile."""
    def run(q):
        pages = _cuda(_pages(-(-n // 64) + 1, 2, 64, E4M3, 1))
        table = torch.arange(-(-n // 64), dtype=torch.int32, device="cuda")[None]
        return eb.cache_attn(q.cuda(), pages, table.contiguous(), _i32([n]).cuda(),
                             _i32([0, 3]).cuda())
    q = _rand((1, 8, 3, D), 4)
    want = run(q)
    q[0, 2, 1, 7] = math.nan
    q[0, 5, 0, 100] = math.inf
    got = run(q)
    bad = torch.zeros((1, 8, 3), dtype=torch.bool, device="cuda")
    bad[0, 2, 1] = bad[0, 5, 0] = True
    assert torch.equal(got[~bad], want[~bad])
    assert bool(got[bad].isnan().all())


@pytest.mark.parametrize("cols", [3, 40])
def test_attn_thousands_of_sequences(cols):
    """More items than waves, in the launches of short and of long tables."""
    S, hkv = 2100, 8
    lengths = [1 + (13 * i) % 150 for i in range(S)]
    pages = _pages(400, hkv, 64, E4M3, 1)
    table = torch.randint(0, 400, (S, cols), generator=_gen(2)).to(torch.int32)
    q = _rand((1, 16, S, D), 3)
    got = eb.cache_attn(q.cuda(), _cuda(pages), table.cuda(), _i32(lengths).cuda()).cpu()
    some = list(range(0, S, 97)) + [S - 1]
    ref, off = attn_reference(q[:, :, some], pages, table[some].tolist(),
                              [lengths[i] for i in some], list(range(len(some) + 1)))
    assert bool(((got[:, :, some].double() - ref).abs() <= off).all())
    assert bool((got != 0).any(-1).all())


def test_attn_leaves_rows_of_no_sequence():
    pages = _cuda(_pages(4, 2, 64, E4M3, 1))
    q = _rand((1, 4, 12, D), 2).cuda()
    out = torch.full_like(q, 3.0)
    eb.cache_attn(q, pages, _i32([[0], [1]]).cuda(), _i32([20, 30]).cuda(),
                  _i32([2, 3, 5]).cuda(), out=out)
    assert bool((out[:, :, :2] == 3.0).all()) and bool((out[:, :, 5:] == 3.0).all())
    assert bool((out[:, :, 2:5] != 3.0).any(-1).all())


@pytest.mark.parametrize("lead", [1, 70, 1000])
@pytest.mark.parametrize("spare", [1, 60])
def test_attn_behind_rows_of_no_sequence(lead, spare):
    lengths, new = [400, 30, 129], [10, 1, 3]
    table = _table(lengths, 64, 12, spare=spare)
    pages, cu = _pages(12, 2, 64, E4M3, 1), [lead + c for c in _offsets(new)]
    q = _rand((1, 8, cu[-1] + 5, D), 2)
    out = torch.full_like(q, 3.0).cuda()
    eb.cache_attn(q.cuda(), _cuda(pages), _i32(table).cuda(), _i32(lengths).cuda(),
                  _i32(cu).cuda(), out=out)
    got = out.cpu()
    assert bool((got[:, :, :lead] == 3.0).all()) and bool((got[:, :, cu[-1]:] == 3.0).all())
    ref, off = attn_reference(q, pages, table, lengths, cu)
    err = (got.double() - ref).abs()[:, :, lead:cu[-1]]
    assert bool((err <= off[:, :, lead:cu[-1]]).all())


@pytest.mark.parametrize("cu", [[0, 500, 10, 600], [600, 300, 200, 0], [-5, 100, 9000, 350],
                                [700, 800, 900, 1000]])
@pytest.mark.parametrize("spare", [1, 60])
def test_offsets_that_are_no_ascending_list(cu, spare):
    """Nothing outside the tensors and the sequences' own pages is touched."""
    T, lengths = 600, [650, 610, 30]
    table = _table(lengths, 64, 24, spare=spare)
    mine = sorted(p for row in table for p in row if p >= 0)
    pages, q = _cuda(_pages(24, 2, 64, E4M3, 1)), _rand((1, 8, T, D), 2).cuda()
    before = [t.clone() for t in pages]
    room = torch.full((3 * q.numel(),), 3.0, dtype=torch.bfloat16, device="cuda")
    out = room[q.numel():2 * q.numel()].view(q.shape)
    args = _i32(table).cuda(), _i32(lengths).cuda(), _i32(cu).cuda()
    eb.cache_attn(q, pages, *args, out=out)
    assert bool((room[:q.numel()] == 3.0).all()) and bool((room[2 * q.numel():] == 3.0).all())
    kv = q[:, :2].contiguous()
    eb.cache_store(kv, kv, pages, *args)
    others = [p for p in range(24) if p not in mine]
    assert all(torch.equal(_bytes(a)[others], _bytes(b)[others]) for a, b in zip(pages, before))


def test_on_a_device_that_is_not_the_current_one(monkeypatch):
    """Each entry point calls itself with its tensors' device made current."""
    pages, table, lengths = _cuda(_pages(8, 2, 64, E4M3, 1)), _i32([[0, 1], [2, 3]]).cuda(), \
        _i32([70, 128]).cuda()
    q, kv, cu = _rand((1, 4, 2, D), 2).cuda(), _rand((1, 2, 2, D), 3).cuda(), _i32([0, 1, 2]).cuda()
    one = _i32([4]).cuda()

    def run():
        eb.cache_store(kv, kv, pages, table, lengths)
        eb.cache_copy(pages, one - 4, one)
        return (eb.cache_attn(q, pages, table, lengths, cu),
                eb.packed_prefill_attn(q, kv, kv, cu), *(t.clone() for t in pages))
    want, asked = run(), []

    def elsewhere_first():
        asked.append(len(asked) % 2)
        return 1 - asked[-1]       # device 1, then (inside) device 0
    monkeypatch.setattr(eb, "_current_device", elsewhere_first)
    got = run()
    assert len(asked) == 8
    assert all(torch.equal(_bytes(a), _bytes(b)) for a, b in zip(got, want))


def test_attn_is_the_same_every_time():
    pages = _cuda(_pages(200, 8, 64, E4M3, 1))
    table = torch.randperm(200, generator=_gen(1)).to(torch.int32).view(2, 100).cuda()
    q, lengths = _rand((1, 32, 2, D), 3).cuda(), _i32([6400, 5000]).cuda()
    first = eb.cache_attn(q, pages, table, lengths)
    for _ in range(20):
        assert torch.equal(eb.cache_attn(q, pages, table, lengths), first)


def test_cache_past_32_bits():
    """Pages more than 2^32 bytes into the pool."""
    hkv, P, n_pages = 8, 128, 40000                    # 5.2 GB each of K and V
    pages = eb.new_cache_pages(n_pages, hkv, P)
    L = 300
    k, v = _rand((1, hkv, L, D), 1), _rand((1, hkv, L, D), 2)
    table = [[39999, 3, 33333]]
    eb.cache_store(k.cuda(), v.cuda(), pages, _i32(table).cuda(), _i32([L]).cuda())
    host = eb.new_cache_pages(3, hkv, P, device="cpu")
    store_reference(host, k, v, [[0, 1, 2]], [L], [0, L])
    at = torch.tensor(table[0], device="cuda")
    same_pages(eb.CachePages(*(_bytes(t)[at].view(t.dtype) if t.dtype is E4M3 else t[at]
                               for t in pages)), host)
    q = _rand((1, 32, 1, D), 3)
    got = eb.cache_attn(q.cuda(), pages, _i32(table).cuda(), _i32([L]).cuda()).cpu()
    ref, off = attn_reference(q, host, [[0, 1, 2]], [L], [0, 1])
    assert bool(((got.double() - ref).abs() <= off).all())
    eb.cache_copy(pages, _i32([39999, 33333]).cuda(), _i32([39000, 7]).cuda())
    assert torch.equal(_bytes(pages.k)[39000], _bytes(pages.k)[39999])
    assert torch.equal(_bytes(pages.v)[7], _bytes(pages.v)[33333])


# --------------------------------------------------------------------------
# Copy
# --------------------------------------------------------------------------

@pytest.mark.parametrize("hkv,P,layers", [(1, 64, None), (3, 64, 2), (8, 128, 4), (5, 128, 1)])
@pytest.mark.parametrize("dtype", [E4M3, INT8])
def test_copy(hkv, P, layers, dtype):
    n = 20
    one = [_pages(n, hkv, P, dtype, 100 * i) for i in range(layers or 1)]
    host = eb.CachePages(*(torch.stack([_bytes(t) if t.dtype is E4M3 else t for t in ts]).view(
        ts[0].dtype) for ts in zip(*one))) if layers else one[0]
    dev = _cuda(host)
    at = torch.randperm(n, generator=_gen(3)).tolist()
    src, dst = at[:7] + [-1, 3, n, at[0]], at[7:14] + [at[14], -2, at[15], at[16]]
    eb.cache_copy(dev, _i32(src).cuda(), _i32(dst).cuda())
    for a, b in zip(src, dst):
        if 0 <= a < n and 0 <= b < n:
            for t in host:
                t = t if t.dtype is torch.float32 else _bytes(t)
                if layers:
                    t[:, b] = t[:, a]
                else:
                    t[b] = t[a]
    for a, b in zip(dev, host):
        assert torch.equal(_bytes(a).cpu(), _bytes(b))


# --------------------------------------------------------------------------
# Together
# --------------------------------------------------------------------------

@pytest.mark.parametrize("spare", [1, 40])
@pytest.mark.parametrize("dtype", [E4M3, INT8])
def test_a_decoding_loop_captured(dtype, spare):
    """Prompts stored, then steps of one token each as a captured graph, the
    lengths kept on the device; every step against the same calls run eagerly
    and against float64."""
    S, hq, hkv, P = 3, 8, 2, 64
    prompts, steps = [60, 1, 130], 8
    total = [n + steps for n in prompts]
    n_pages = sum(-(-n // P) for n in total)
    table = _table(total, P, n_pages, 5, spare)
    dtab = _i32(table).cuda()
    k, v = _rand((1, hkv, sum(prompts), D), 1), _rand((1, hkv, sum(prompts), D), 2)
    cu = _i32(_offsets(prompts)).cuda()

    def fresh():
        pages = eb.new_cache_pages(n_pages, hkv, P, dtype=dtype)
        eb.cache_store(k.cuda(), v.cuda(), pages, dtab, _i32(prompts).cuda(), cu)
        return pages

    new = [[_rand((1, h, S, D), 50 + 3 * i + j) for j, h in enumerate((hq, hkv, hkv))]
           for i in range(steps)]
    eager, graphed = fresh(), fresh()
    q, kk, vv = (x.cuda() for x in new[0])
    lengths = _i32(prompts).cuda()
    out = torch.zeros_like(q)

    def step(pages):
        lengths.add_(1)
        eb.cache_store(kk, vv, pages, dtab, lengths)
        eb.cache_attn(q, pages, dtab, lengths, out=out)

    scratch = fresh()
    step(scratch)          # (warm-up outside the capture)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(graphed)
    lengths.copy_(_i32(prompts))
    for i in range(steps):
        for t, x in zip((q, kk, vv), new[i]):
            t.copy_(x)
        graph.replay()
        got = out.clone()
        lengths.sub_(1)
        step(eager)
        torch.cuda.synchronize()
        assert torch.equal(got, out), i
        for a, b in zip(graphed, eager):
            assert torch.equal(_bytes(a), _bytes(b)), i
        ref, off = attn_reference(new[i][0], eb.CachePages(*(t.cpu() for t in eager)), table,
                                  [n + i + 1 for n in prompts], list(range(S + 1)))
        assert bool(((got.cpu().double() - ref).abs() <= off).all()), i


def test_two_streams_with_workspaces_of_their_own():
    pages = _cuda(_pages(200, 8, 64, E4M3, 1))
    table = torch.randperm(200, generator=_gen(1)).to(torch.int32).view(2, 100).cuda()
    qs = [_rand((1, 32, 2, D), 3 + i).cuda() for i in range(2)]
    lengths = _i32([6400, 5000]).cuda()
    want = [eb.cache_attn(q, pages, table, lengths) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for st, q in zip(streams, qs):
            with torch.cuda.stream(st):
                got.append(eb.cache_attn(q, pages, table, lengths))
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
