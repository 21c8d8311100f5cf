"""What a query of packed prompts does not see never reaches it, whatever it
holds: its own sequence's later keys and values, those of the sequences before
and behind it, and the places past a sequence's end in its last key block.  In
both kernels: tiles of 128 rows, and tiles of 32 whose keys the waves share."""
import math

import pytest
import torch

from paper_2606_09508_amd import binding as eb

pytestmark = pytest.mark.gpu

D, G = 128, 2
# query heads that make a launch of these sequences one of 128-row tiles (more
# than 128 of them in all) or of 32-row ones
HEADS = {"tiles": 64, "split": 4}
BAD = [math.inf, -math.inf, math.nan]


def _rand(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _tensors(heads, T):
    return tuple(_rand((1, h, T, D), i).cuda() for i, h in enumerate((heads, heads // G, heads // G)))


def _run(q, k, v, cu, causal=True):
    return eb.packed_prefill_attn(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"),
                                  causal=causal)


def _same(got, want):
    """Equal bits, NaN and infinities in the same places."""
    nan = want.isnan()
    assert torch.equal(got.isnan(), nan)
    assert torch.equal(got.masked_fill(nan, 0.0), want.masked_fill(nan, 0.0))


@pytest.mark.parametrize("kernel", HEADS)
@pytest.mark.parametrize("n", [150, 257, 321, 64 * 5])
@pytest.mark.parametrize("bad", BAD)
def test_later_values_of_the_sequence(kernel, n, bad):
    """Row j of V is not finite in a few dims: queries before j keep their bits
    in every dim, those from j on in the other dims, and in these dims they are
    what the value is (each of its weights is positive)."""
    cu = [0, n, n + 130]
    q, k, v = _tensors(HEADS[kernel], cu[-1])
    want = _run(q, k, v, cu)
    for j in (1, 31, 32, 63, 64, 100, n // 2 + 1, n - 2, n - 1):
        x, y = v.clone(), want.clone()
        for dim in (0, 7, 37, 127):
            x[:, :, j, dim] = bad
            y[:, :, j:n, dim] = bad
        _same(_run(q, k, x, cu), y)


@pytest.mark.parametrize("kernel", HEADS)
def test_several_values_of_all_kinds(kernel):
    """A query's dim is NaN from where it sees one, or infinities of both signs."""
    n = 300
    q, k, v = _tensors(HEADS[kernel], n)
    want = _run(q, k, v, [0, n])
    x, y = v.clone(), want.clone()
    for j, dim, bad in ((70, 5, math.inf), (90, 5, -math.inf), (91, 6, -math.inf), (120, 6, math.nan),
                        (130, 100, math.inf), (131, 100, math.inf), (299, 101, math.nan)):
        x[:, :, j, dim] = bad
        y[:, :, j:, dim] += bad
    _same(_run(q, k, x, [0, n]), y)


@pytest.mark.parametrize("kernel", HEADS)
@pytest.mark.parametrize("n", [65, 150, 300])
def test_last_value_over_all_keys(kernel, n):
    """Over all keys every query sees the last value: infinite, not NaN, also
    where the last key block has places past it."""
    cu = [0, n, n + 150]
    q, k, v = _tensors(HEADS[kernel], cu[-1])
    want = _run(q, k, v, cu, causal=False)
    x, y = v.clone(), want.clone()
    x[:, :, n - 1, 3] = math.inf
    y[:, :, :n, 3] = math.inf
    _same(_run(q, k, x, cu, causal=False), y)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kernel", HEADS)
@pytest.mark.parametrize("lengths", [(150, 140, 170), (129, 300, 131), (200, 64, 330)])
def test_sequences_before_and_behind(lengths, kernel, causal):
    """The other sequences' keys and values are NaN and infinite."""
    cu = [0, lengths[0], sum(lengths[:2]), sum(lengths)]
    q, k, v = _tensors(HEADS[kernel], cu[-1])
    want = _run(q, k, v, cu, causal)
    for s in range(3):
        for bad_k, bad_v in ((math.nan, math.inf), (math.inf, math.nan), (-math.inf, -math.inf)):
            x, y = torch.full_like(k, bad_k), torch.full_like(v, bad_v)
            x[:, :, cu[s]:cu[s + 1]] = k[:, :, cu[s]:cu[s + 1]]
            y[:, :, cu[s]:cu[s + 1]] = v[:, :, cu[s]:cu[s + 1]]
            got = _run(q, x, y, cu, causal)
            assert torch.equal(got[:, :, cu[s]:cu[s + 1]], want[:, :, cu[s]:cu[s + 1]])


@pytest.mark.parametrize("kernel", HEADS)
@pytest.mark.parametrize("bad", BAD)
def test_later_keys_of_the_sequence(kernel, bad):
    """Queries before a key that is not finite stay finite and as they were, but
    for the roundings of another running maximum: each of their probabilities
    is rounded to bf16 once more (2^-8 of it) and the output too."""
    n = 300
    q, k, v = _tensors(HEADS[kernel], n)
    want = _run(q, k, v, [0, n])
    # the sum of a query's weights times |v|, head by head
    c = 1.0 / math.sqrt(D)
    x = (q[0].double() @ k[0].double().repeat_interleave(G, 0).transpose(1, 2)) * c
    i = torch.arange(n, device="cuda")
    w = torch.softmax(x.masked_fill(i > i[:, None], -math.inf), -1)
    a = w @ v[0].double().repeat_interleave(G, 0).abs()
    off = 1.01 * 2 * (2.0 ** -8 * want[0].double().abs() + (2.0 ** -8 + 1e-4) * a)
    for j in (1, 33, 100, n - 1):
        y = k.clone()
        y[:, :, j] = bad
        got = _run(q, y, v, [0, n])
        err = (got[0].double() - want[0].double()).abs()[:, :j]
        assert bool((err <= off[:, :j]).all())
