"""Attention over packed sequences against each sequence's dense attention in
float64 on the CPU."""
import math

import pytest
import torch

from paper_2606_09508_amd import binding as eb

pytestmark = pytest.mark.gpu

D = 128
HALF = 2.0 ** -8   # half a bf16 step, relative


def _rand(shape, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(torch.bfloat16)


def reference(q, k, v, causal):
    """One sequence, q [Hq, n, D], k and v [Hkv, n, D]: the output in float64
    and how far a result may be off.  The output is rounded once (HALF of
    itself).  Each probability is rounded to bf16 (HALF of it, so HALF of
    w @ |v| in all) and carries the errors of its fp32 score: a sum of 128
    products is off by at most 128 * 2^-24 of the sum of their magnitudes,
    and as much moves the probability and the sum they are divided by."""
    G = q.shape[0] // k.shape[0]
    q, k, v = q.double(), k.double().repeat_interleave(G, 0), v.double().repeat_interleave(G, 0)
    c = 1.0 / math.sqrt(D)
    x = (q @ k.transpose(1, 2)) * c
    mag = (q.abs() @ k.abs().transpose(1, 2)).amax((1, 2), keepdim=True) * c
    if causal:
        n = q.shape[1]
        x = x.masked_fill(torch.arange(n) > torch.arange(n)[:, None], -math.inf)
    w = torch.softmax(x, -1)
    o = w @ v
    off = 1.01 * (HALF * o.abs() + (HALF + 2 * 130 * 2.0 ** -24 * mag + 1e-5) * (w @ v.abs()))
    return o, off


def check(got, q, k, v, cu, causal):
    for a, b in zip(cu, cu[1:]):
        if b <= a:
            continue
        o, off = reference(q[0, :, a:b], k[0, :, a:b], v[0, :, a:b], causal)
        err = (got[0, :, a:b].double() - o).abs()
        assert bool((err <= off).all()), (a, b, float((err / off).max()))


def offsets(lengths, start=0):
    cu = [start]
    for n in lengths:
        cu.append(cu[-1] + n)
    return cu


LENGTHS = [
    [1],
    [0, 5, 0, 0, 1],
    [127, 128, 129],
    [64, 65, 63, 1, 2],
    [700, 1, 300, 33],
    [3, 0, 1, 2] * 20,                       # more sequences than a wave has lanes
    [i % 37 for i in range(200)] + [600],
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hkv", [(4, 1), (6, 2), (3, 3), (16, 8)])
@pytest.mark.parametrize("lengths", LENGTHS, ids=lambda l: f"{len(l)}x{max(l)}")
def test_packed_matches_each_sequence(lengths, hq, hkv, causal):
    cu = offsets(lengths)
    T = cu[-1]
    q, k, v = _rand((1, hq, T, D), 1), _rand((1, hkv, T, D), 2), _rand((1, hkv, T, D), 3)
    got = eb.packed_prefill_attn(q.cuda(), k.cuda(), v.cuda(),
                                 torch.tensor(cu, dtype=torch.int32, device="cuda"),
                                 causal=causal).cpu()
    check(got, q, k, v, cu, causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("hq,hkv,lengths", [
    (4, 1, [2048]), (8, 2, [400, 129, 40, 500]), (4, 4, [1000, 1, 1500]), (2, 1, [130] * 20),
    (3, 1, [600, 0, 0, 700, 33])])
def test_packed_small_launches(hq, hkv, lengths, causal):
    """Launches of few tiles, whose keys are shared out over the waves."""
    cu = offsets(lengths)
    T = cu[-1]
    q, k, v = _rand((1, hq, T, D), 7), _rand((1, hkv, T, D), 8), _rand((1, hkv, T, D), 9)
    got = eb.packed_prefill_attn(q.cuda(), k.cuda(), v.cuda(),
                                 torch.tensor(cu, dtype=torch.int32, device="cuda"),
                                 causal=causal).cpu()
    check(got, q, k, v, cu, causal)


def test_packed_thousands_of_sequences():
    lengths = [(7 * i) % 11 for i in range(4500)]
    cu = offsets(lengths)
    T = cu[-1]
    q, k, v = _rand((1, 4, T, D), 1), _rand((1, 2, T, D), 2), _rand((1, 2, T, D), 3)
    got = eb.packed_prefill_attn(q.cuda(), k.cuda(), v.cuda(),
                                 torch.tensor(cu, dtype=torch.int32, device="cuda")).cpu()
    check(got, q, k, v, cu, True)


@pytest.mark.parametrize("hq,hkv,n", [(32, 8, 700), (28, 4, 2000), (40, 40, 300)])
def test_packed_larger_launches(hq, hkv, n):
    """Launches of several rounds, whose tiles are dealt out over the chip."""
    cu = offsets([n, n // 3, 1, n // 2 + 1, 130])
    T = cu[-1]
    q, k, v = _rand((1, hq, T, D), 4), _rand((1, hkv, T, D), 5), _rand((1, hkv, T, D), 6)
    got = eb.packed_prefill_attn(q.cuda(), k.cuda(), v.cuda(),
                                 torch.tensor(cu, dtype=torch.int32, device="cuda")).cpu()
    check(got, q, k, v, cu, True)


@pytest.mark.parametrize("lead", [17, 1000])
def test_rows_outside_every_sequence_are_left(lead):
    cu = offsets([40, 0, 200], start=lead)
    T = cu[-1] + 150
    q, k, v = (_rand((1, 4, T, D), i).cuda() for i in range(3))
    out = torch.full_like(q, 7.0)
    eb.packed_prefill_attn(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"), out=out)
    assert bool((out[:, :, :lead] == 7.0).all()) and bool((out[:, :, cu[-1]:] == 7.0).all())
    check(out.cpu(), q.cpu(), k.cpu(), v.cpu(), cu, True)


def test_values_behind_a_sequence_do_not_reach_it():
    """The next sequence's NaN and infinite keys and values, and a query's
    later ones."""
    cu = offsets([100, 60])
    q, k, v = (_rand((1, 4, 160, D), 10 + i) for i in range(3))
    bad_k, bad_v = k.clone(), v.clone()
    bad_k[:, :, 100:] = math.nan
    bad_v[:, :, 100:] = math.inf
    dev = torch.tensor(cu, dtype=torch.int32, device="cuda")
    good = eb.packed_prefill_attn(q.cuda(), k.cuda(), v.cuda(), dev)
    got = eb.packed_prefill_attn(q.cuda(), bad_k.cuda(), bad_v.cuda(), dev)
    assert torch.equal(got[:, :, :100], good[:, :, :100])
    assert bool(got[:, :, 100:].isnan().all())


def test_offsets_that_leave_the_tensor_are_clamped():
    """Lists that descend or point outside: those sequences are empty or end
    with the tensor, and the others are as they were."""
    q, k, v = (_rand((1, 4, 300, D), 20 + i).cuda() for i in range(3))
    out = torch.zeros_like(q)
    cu = [-50, 100, 90, 90, 2 ** 31 - 1, 5]      # [0, 100), -, -, [90, 300), -
    eb.packed_prefill_attn(q, k, v, torch.tensor(cu[:2], dtype=torch.int32, device="cuda"),
                           out=out)
    check(out.cpu(), q.cpu(), k.cpu(), v.cpu(), [0, 100], True)
    eb.packed_prefill_attn(q, k, v, torch.tensor(cu[3:], dtype=torch.int32, device="cuda"),
                           out=out)
    check(out.cpu(), q.cpu(), k.cpu(), v.cpu(), [90, 300], True)


def test_packed_offsets_past_32_bits():
    """More than 2^32 bytes and 2^31 elements of queries: the last sequences
    against a launch of their own."""
    T, hq, hkv = 300000, 64, 8
    lengths = [100] * 2999 + [37, 63]
    cu = offsets(lengths)
    q = torch.zeros((1, hq, T, D), dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros((1, hkv, T, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    small = [_rand((1, h, 200, D), i).cuda() for i, h in enumerate((hq, hkv, hkv))]
    for t, x in zip((q, k, v), small):
        t[:, :, -200:] = x
    got = eb.packed_prefill_attn(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"))
    check(got[:, :, -200:].cpu(), *(x.cpu() for x in small), [0, 100, 137, 200], True)


def test_packed_graph_replays_with_other_lengths():
    """A captured call reads the offsets of the replay."""
    q, k, v = (_rand((1, h, 640, D), 30 + h).cuda() for h in (8, 2, 2))
    cu = torch.tensor(offsets([300, 300, 40]), dtype=torch.int32, device="cuda")
    out = torch.zeros_like(q)
    eb.packed_prefill_attn(q, k, v, cu, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eb.packed_prefill_attn(q, k, v, cu, out=out)
    for lengths in ([300, 300, 40], [1, 2, 3], [0, 600, 40], [640, 0, 0]):
        cu.copy_(torch.tensor(offsets(lengths), dtype=torch.int32))
        out.fill_(5.0)
        graph.replay()
        want = torch.full_like(out, 5.0)
        eb.packed_prefill_attn(q, k, v, cu, out=want)
        torch.cuda.synchronize()
        assert torch.equal(out, want), lengths
