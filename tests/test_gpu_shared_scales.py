"""Shared-prefix attention over pages whose values are zero or tiny: the cache's
store gives a page without values the scale 2^-126, and what a key weighs must
not depend on the scale of its value."""
import pytest
import torch

from paper_2606_09508_amd import binding as eb
from test_gpu_serving import _check_step, _hidden, _setup
from test_gpu_shared import E4M3, INT8, Batch, _i32

pytestmark = pytest.mark.gpu

TINY = 2.0 ** -126       # of a page of zeros, as ei_cache_store writes it
# sequences of a group of 4 heads: 16 rows and few, tiles of 64 rows, of 128
SIZES = [3, 12, 30]


def _check(b):
    """As Batch.check, with the error beside a row's own largest products, and that of
    a page's factor of the sum of weights: a power of 2 whose exponent, 2^8 at most, is
    rounded twice to 24 bits, 2 * 2^-17 ln 2."""
    got = b.run().cpu().double()
    want, size, steep, most = b.reference()
    rel = 2 * (128 * 2.0 ** -23 * steep + 2.0 ** -22 + most * 2.0 ** -23 + 2.0 ** -16) + 2.0 ** -11
    off = rel * size + most * 2.0 ** -32 * size.amax(-1, keepdim=True)
    assert torch.isfinite(got).all()
    assert ((got - want).abs() <= off + 2.0 ** -8 * (want.abs() + off)).all()
    return got


@pytest.mark.parametrize("dtype,P", [(E4M3, 64), (E4M3, 128), (INT8, 64), (INT8, 128)])
@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("empty", [[0], [6], [0, 1], [2, 3], [0, 2, 4, 6], [0, 1, 2, 3, 4, 5],
                                   list(range(7))])
@pytest.mark.parametrize("scale", [TINY, 0.0, 2.0 ** -130])
def test_pages_without_values(dtype, P, size, empty, scale):
    b = Batch([size], [7], [40] * size, [1] * size, 4, 1, P, dtype, seed=size)
    for c in empty:
        b.codes.view(torch.uint8)[1, b.table[0][c]] = 0
        b.scales[1, b.table[0][c]] = scale
    _check(b)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("below", [8, 15, 30, 60])
@pytest.mark.parametrize("scale", [2.0 ** -7, 1.0, 2.0 ** 20])
@pytest.mark.parametrize("where", [0, 60])
def test_many_keys_without_values_below_one_with(size, below, scale, where):
    """4000 keys on pages of zeros, each `below` binary places under the keys of the
    one page that has values: at 8 they weigh 15 times what those do."""
    b = Batch([size], [64], [1] * size, [1] * size, 4, 1, 64, E4M3, seed=size)
    b.q *= 2.0 ** -8
    b.q[..., 0] = 16.0
    b.scales[0] = 1.0
    page = b.table[0][where]
    raw = b.codes.view(torch.uint8)
    raw[1, b.table[0][:64]] = 0
    b.scales[1, b.table[0][:64]] = TINY
    b.codes[:, page] = (torch.randn(b.codes[0, page].shape, generator=torch.Generator()
                                    .manual_seed(size)) * 100).to(E4M3)[None]
    b.scales[1, page] = scale
    # a score is 16 k_0 / sqrt(128) log2(e) in binary places: 2.04 k_0
    b.codes[0, :, :, :, 0] = 0.0
    b.codes[0, page, :, :, 0] = float(round(below / 2.04))
    for s in range(size):
        b.codes.view(torch.uint8)[1, b.table[s][64]] = 0
        b.scales[1, b.table[s][64]] = TINY
    _check(b)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("scales", [[2.0 ** -110] * 5, [2.0 ** -118] * 5, [1.0, 0.0, 2.0 ** -40, 1.0, 0.0],
                                    [2.0 ** -100, 2.0 ** -7, 2.0 ** -118, 1.0, 2.0 ** -70],
                                    [2.0 ** 60, 2.0 ** -126, 2.0 ** 60, 2.0 ** -60, 2.0 ** 0],
                                    [0.0, 0.0, 2.0 ** -40, 0.0, 0.0]])
def test_far_scales(size, scales):
    b = Batch([size], [5], [40] * size, [1] * size, 4, 1, 64, E4M3, seed=size)
    for c, f in enumerate(scales):
        b.scales[1, b.table[0][c]] = f
    for s in range(size):
        b.scales[1, b.table[s][5]] = scales[2]
    _check(b)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("dtype,P", [(E4M3, 64), (INT8, 128)])
def test_pages_that_the_store_wrote(size, dtype, P):
    """Zeros stored over a page, between others and at the beginning, in one KV head:
    as cache_attn, of which either side is off by the output's rounding."""
    g = torch.Generator(device="cuda").manual_seed(size)
    n, hkv = 6 * P, 2
    pages = eb.new_cache_pages(6 + size, hkv, P, 128, dtype)
    k = torch.randn((1, hkv, n, 128), generator=g, device="cuda").to(torch.bfloat16)
    v = torch.randn((1, hkv, n, 128), generator=g, device="cuda").to(torch.bfloat16)
    v[:, 0, :P] = 0
    v[:, 0, 3 * P:5 * P] = 0
    eb.cache_store(k, v, pages, _i32([list(range(6))]).cuda(), _i32([n]).cuda())
    assert (pages.v_scale[0, 0] == TINY).all()
    table = _i32([list(range(6)) + [6 + s] for s in range(size)]).cuda()
    lengths = _i32([n + 1] * size).cuda()
    own = torch.randn((2, 1, hkv, size, 128), generator=g, device="cuda").to(torch.bfloat16)
    eb.cache_store(own[0], own[1], pages, table, lengths)
    q = torch.randn((1, 8, size, 128), generator=g, device="cuda").to(torch.bfloat16)
    want = eb.cache_attn(q, pages, table, lengths).double()
    got = eb.cache_attn_shared(q, pages, table, lengths, _i32([0, size]).cuda(),
                               _i32([6]).cuda()).double()
    # (either is rounded once; weights of 11 bits move a row by 2^-11 of its |v|, 0.1)
    assert ((got - want).abs() <= 2.0 ** -7 * want.abs() + 2.0 ** -11 * 0.5).all()
    assert got.abs().max() > 0.05


@pytest.mark.parametrize("forks", [9, 15])
def test_a_step_behind_hidden_states_of_zeros(forks):
    """A prompt that begins with padding, and holds some: its keys and values are 0."""
    dec, g = _setup(n_adapters=0)
    dec.layers[1]["wv"][:, :128] = 0         # (and a head of values without any)
    x = _hidden(g, 330)
    x[:, :100] = 0
    x[:, 190:260] = 0
    a = dec.cache.add()
    dec.prompts(x, [330], [a])
    seqs = [a] + [dec.cache.fork(a) for _ in range(forks - 1)]
    assert (dec.cache.pages.v_scale[0] == TINY).any() and (dec.cache.pages.v_scale[1] == TINY).any()
    for _ in range(2):
        _check_step(dec, _hidden(g, len(seqs)), seqs, None, None)


@pytest.mark.parametrize("size", SIZES)
@pytest.mark.parametrize("below", [8, 16, 20, 24])
@pytest.mark.parametrize("first", [0, 1])
def test_dims_that_only_light_keys_have(size, below, first):
    """Keys far below the others are all that some dims have: an fp16 number that is not
    normal still counts."""
    b = Batch([size], [2], [1] * size, [1] * size, 4, 1, 64, E4M3, seed=size)
    b.q *= 2.0 ** -8
    b.q[..., 0] = 16.0
    b.scales[0], b.scales[1] = 1.0, 2.0 ** -7
    heavy, light = b.table[0][first], b.table[0][1 - first]
    for page in range(b.codes.shape[1]):
        b.codes[0, page, :, :, 0] = 0.0
    b.codes[0, heavy, :, :, 0] = float(round(below / 2.04))
    b.codes.view(torch.uint8)[1, heavy, :, :, 64:] = 0
    b.codes[1, light, :, :, 64:] = 448.0
    for s in range(size):
        b.codes.view(torch.uint8)[1, b.table[s][2], :, :, 64:] = 0
    got = _check(b)
    assert (got[..., 64:] > 0).all()
