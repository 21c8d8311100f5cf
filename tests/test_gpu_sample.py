"""Sampling on the GPU against its definition on the CPU: weights in multiples of
2^-44 as Python's whole numbers, one token after the other."""
import math

import pytest
import torch

from paper_2606_09508_amd import binding as eb

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
INF, NAN = math.inf, math.nan


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _i32(x):
    return torch.tensor(x, dtype=torch.int32)


def reference(x, u, t=1.0, k=0, p=1.0, least=0.0):
    """(token, log of its share, distance of u * total to the next sum, of the total)."""
    x = [float(v) for v in x.double()]
    there = [i for i, v in enumerate(x) if v > -INF]
    if not there:
        return -1, -INF, 1.0
    there.sort(key=lambda i: (-x[i], i))
    top = x[there[0]]
    if not t > 0:
        return there[0], 0.0, 1.0
    real = [1.0 if x[i] == top else 0.0 if top == INF else math.exp(max((x[i] - top) / t, -700.0))
            for i in there]
    w = [int(math.floor(r * 2.0 ** 44 + 0.5)) for r in real]
    n = len(there)
    if k > 0:
        n = min(n, k)
    if p < 1:
        want, run, m = p * sum(w[:n]), 0, 0
        while m < n and (run < want or m == 0):
            run += w[m]
            m += 1
        n = m
    keep = [(there[j], w[j], real[j]) for j in range(n)
            if not least > 0 or real[j] >= min(least, 1.0)]
    keep.sort()
    total = sum(v for _, v, _ in keep)
    u = min(u, 1 - 2.0 ** -24) if u > 0 else 0.0
    run, near = 0, 1.0
    token = None
    for i, v, r in keep:
        run += v
        near = min(near, abs(run - u * total) / total)
        if token is None and run > math.floor(u * total):
            token, share = i, r / (total * 2.0 ** -44)
    return token, math.log(share), near


def check(x, u, t=None, k=None, p=None, least=None, view=None):
    rows = x.shape[0]
    dev = [None if v is None else torch.tensor(v, dtype=torch.int32 if n == "k" else F32).cuda()
           for n, v in (("t", t), ("k", k), ("p", p), ("m", least))]
    xs = x.cuda() if view is None else view(x)
    tokens, logs = eb.sample_tokens(xs, torch.tensor(u, dtype=F32).cuda(), *dev)
    tokens, logs = tokens.tolist(), logs.tolist()
    f = lambda v: float(torch.tensor(v, dtype=F32))
    for r in range(rows):
        token, log, near = reference(
            x[r], f(u[r]), 1.0 if t is None else f(t[r]), 0 if k is None else k[r],
            1.0 if p is None else f(p[r]), 0.0 if least is None else f(least[r]))
        # (a weight of 2^44 steps may be a step off where exp rounds otherwise: a sum
        # of n of them passes another u only within n 2^-44 of it)
        if near > x.shape[1] * 2.0 ** -44:
            assert tokens[r] == token, (r, tokens[r], token)
        if token >= 0 and tokens[r] == token:
            # its log in 64 bits, rounded to 32
            assert abs(logs[r] - log) <= 2.0 ** -24 * abs(log) + 1e-12 * max(1, abs(log)), r
        elif token < 0:
            assert logs[r] == -INF
    return tokens


def logits(rows, vocab, seed, dtype=BF16, scale=2.2, likely=20):
    g = _gen(seed)
    x = torch.randn((rows, vocab), generator=g) * scale
    at = torch.randint(0, vocab, (rows, min(likely, vocab)), generator=g)
    return x.scatter_add_(1, at, torch.rand(at.shape, generator=g) * 10).to(dtype)


def us(rows, seed):
    return torch.rand((rows,), generator=_gen(seed + 1000)).tolist()


VOCABS = [1, 2, 63, 64, 65, 1000, 1023, 4099, 32001]


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", VOCABS)
def test_temperature(vocab, dtype):
    x = logits(5, vocab, vocab, dtype)
    check(x, us(5, vocab), [1.0, 0.3, 2.5, 0.0, 1e-3])
    check(x, us(5, vocab + 1))


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", VOCABS)
def test_top_k(vocab, dtype):
    x = logits(8, vocab, vocab, dtype)
    check(x, us(8, vocab), [1.0, 0.7, 2.0, 1.0, 5.0, 1.0, 1.0, 1.0],
          [1, 2, 7, 40, 200, vocab - 1, vocab, 0])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", VOCABS)
def test_top_p(vocab, dtype):
    x = logits(9, vocab, vocab, dtype)
    check(x, us(9, vocab), [1.0, 0.7, 2.0, 1.0, 9.0, 1.0, 1.0, 1.0, 1.0], None,
          [0.9, 0.95, 0.5, 1e-6, 0.99, 1.0, 0.0, 0.9999, -1.0])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("vocab", VOCABS)
def test_min_p_and_all_together(vocab, dtype):
    x = logits(6, vocab, vocab, dtype)
    check(x, us(6, vocab), None, None, None, [0.0, 0.05, 0.5, 1.0, 2.0, 1e-4])
    check(x, us(6, vocab + 5), [1.0, 0.8, 1.5, 0.0, 3.0, 1.0], [50, 20, 3, 5, 1000, 0],
          [0.9, 0.5, 0.99, 0.9, 0.8, 0.7], [0.01, 0.1, 0.0, 0.2, 0.3, 0.02])


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("scale", [1e-3, 0.05, 1.0, 20.0, 1e4])
def test_flat_and_steep_rows(scale, dtype):
    """From nearly all tokens kept to next to none, cuts anywhere."""
    x = logits(10, 6007, 31, F32, scale, 1).to(dtype)
    x[8:, 1500:] = torch.finfo(dtype).min
    x[9, 50:] = -1e30
    u = us(10, 31)
    p = [0.9, 0.999, 0.1, 0.5, 0.9999, 0.3, 0.95, 1.0, 0.9, 0.97]
    k = [0, 0, 5000, 1500, 0, 30, 4097, 2999, 900, 1499]
    for t in (1.0, 0.2, 6.0):
        check(x, u, [t] * 10, None, p)
        check(x, u, [t] * 10, k)
        check(x, u, [t] * 10, k, p)
        check(x, u, [t] * 10, k, p, [1e-3] * 10)
        check(x, u, [t] * 10, None, None, [1e-3] * 10)


def test_signaling_nan_is_no_token():
    x = logits(1, 500, 2, F32)
    x[0, 7] = 1e5
    raw = x.clone().view(torch.int32)
    raw[0, 7], raw[0, 100] = 0x7f800001, -0x7fffff
    y = raw.view(F32)
    assert y[0, 7].isnan() and y[0, 100].isnan()
    x[0, 7] = x[0, 100] = -INF
    for t, k in ((1.0, 0), (0.0, 0), (1.0, 10)):
        a = eb.sample_tokens(y.cuda(), torch.tensor([0.4]).cuda(), torch.tensor([t]).cuda(),
                             _i32([k]).cuda())
        assert a[0].tolist() == check(x, [0.4], [t], [k])


@pytest.mark.parametrize("vocab", [3, 130, 5000])
def test_equal_logits(vocab):
    """Ties: by the lowest index, whatever cuts between them."""
    x = torch.zeros((7, vocab)).to(BF16)
    tokens = check(x, [0.5, 0.999, 0.0, 0.99, 0.5, 0.7, 0.3], [1.0] * 5 + [0.0, INF],
                   [0, 2, 0, vocab // 2, 0, 0, 0], [1.0, 1.0, 0.5, 0.5, 1.0, 1.0, 1.0],
                   [0.0, 0.0, 0.0, 0.0, 1.0, 0.0, 0.0])
    assert tokens[1] == 1 and tokens[5] == 0
    assert tokens[0] == vocab // 2 and tokens[2] == 0
    g = _gen(vocab)
    x = torch.randint(-3, 3, (12, vocab), generator=g).to(BF16)
    check(x, us(12, vocab), None, [1 + i * vocab // 12 for i in range(12)],
          [0.3 + 0.06 * i for i in range(12)])
    # 0 and -0 are one value
    x = torch.zeros((2, vocab)).to(BF16)
    x[:, 0] = -0.0
    assert check(x, [0.0, 0.0], [0.0, 1.0], [0, 1])[0] == 0


def test_what_is_not_finite():
    x = logits(9, 700, 3, F32)
    x[0] = -INF
    x[1] = NAN
    x[2, 5:] = -INF
    x[3, ::3] = NAN
    x[4, [17, 400, 401]] = INF
    x[5] = INF
    x[6, 1:] = -INF
    x[7, 600:] = torch.finfo(F32).min
    x[8] = torch.finfo(F32).min
    for dtype in (F32, BF16):
        y = x.to(dtype)
        tokens = check(y, us(9, 4))
        assert tokens[0] == tokens[1] == -1 and tokens[4] in (17, 400, 401) and tokens[6] == 0
        check(y, us(9, 5), [0.7] * 9, [30] * 9, [0.9] * 9, [0.01] * 9)
        check(y, us(9, 6), [0.0] * 9)
        check(y, us(9, 7), [INF] * 9, [0] * 9, [0.5] * 9)
        check(y, us(9, 8), [1e-40] * 9, [0] * 9, [0.99] * 9)


def test_settings_that_are_none():
    x = logits(8, 300, 9)
    u = us(8, 9)
    plain = check(x, u)
    assert check(x, u, [1.0] * 8, [0, -5, 300, 1000, 2 ** 31 - 1, -2 ** 31, 0, 0],
                 [1.0, 2.0, NAN, INF, 1.0, 1.0, 1.0, 1.0],
                 [0.0, -1.0, NAN, -INF, 0.0, 0.0, 0.0, 0.0]) == plain
    greedy = check(x, u, [0.0, -1.0, NAN, -INF, 0.0, 0.0, -0.0, 0.0])
    assert greedy == x.float().argmax(1).tolist()
    assert check(x, [NAN, -1.0, -INF, 0.0] * 2) == check(x, [0.0] * 8)
    assert check(x, [1.0, 2.0, INF, 1 - 2.0 ** -24] * 2) == check(x, [1 - 2.0 ** -24] * 8)


def test_every_number_gives_its_token():
    """Weights 1, 1/2, 1/4, ... of 16 tokens, u over all of [0, 1): as often as they
    weigh, exactly."""
    n = 4096
    x = (-torch.arange(16) * math.log(2.0))[None].expand(n, 16).contiguous()
    u = ((torch.arange(n) + 0.5) / n).float()
    tokens, logs = eb.sample_tokens(x.cuda(), u.cuda())
    w = 0.5 ** torch.arange(16).double()
    for i, c in enumerate(torch.bincount(tokens.cpu().long(), minlength=16).tolist()):
        assert abs(c - n * float(w[i] / w.sum())) <= 1.0
    want = torch.log(w / w.sum())[tokens.cpu().long()]
    # (ln 2 in fp32 is off by 2^-25 of itself, times 15 of them)
    assert ((logs.cpu().double() - want).abs() <= 2.0 ** -24 * want.abs() + 16 * 2.0 ** -25).all()


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_rows_that_lie_apart(dtype):
    x = logits(4, 1001, 11, dtype)

    def wide(y):
        z = torch.full((4, 1203), 50.0, dtype=dtype)
        z[:, 101:1102] = y
        return z.cuda()[:, 101:1102]

    def last(y):
        z = torch.full((4, 3, 1001), 50.0, dtype=dtype)
        z[:, -1] = y
        return z.cuda()[:, -1]

    for view in (wide, last):
        check(x, us(4, 12), [1.0, 0.5, 0.0, 2.0], [0, 10, 0, 0], [1.0, 1.0, 1.0, 0.9], view=view)


@pytest.mark.parametrize("rows,vocab", [(1, 128256), (2, 200003), (40, 50257), (300, 1500),
                                        (3, 524288)])
def test_large(rows, vocab):
    """Against the definition in vectors of 64 bits (rows at a time)."""
    x = logits(rows, vocab, rows, BF16, 2.2, 60)
    t = [(1.0, 0.7, 1.4)[r % 3] for r in range(rows)]
    p = [(1.0, 0.95, 0.9, 0.6)[r % 4] for r in range(rows)]
    k = [(0, 0, 500, 50, 3)[r % 5] for r in range(rows)]
    u = us(rows, rows)
    f = lambda v, d=F32: torch.tensor(v, dtype=d).cuda()
    tokens, logs = eb.sample_tokens(x.cuda(), f(u), f(t), f(k, torch.int32), f(p))
    again, _ = eb.sample_tokens(x.cuda(), f(u), f(t), f(k, torch.int32), f(p))
    assert torch.equal(tokens, again)
    for r in range(rows):
        y, by = torch.sort(x[r].double(), descending=True, stable=True)
        w = torch.floor(torch.exp((y - y[0]) / float(f(t)[r])) * 2.0 ** 44 + 0.5).long()
        if k[r]:
            w[k[r]:] = 0
        before = w.cumsum(0) - w
        if p[r] < 1:
            w = torch.where(before.double() < float(f(p)[r]) * float(w.sum()), w, 0)
        v = torch.zeros_like(w).scatter_(0, by, w)
        sums = v.cumsum(0)
        want = float(f(u)[r]) * float(sums[-1])
        near = (sums.double() - want).abs().min() / float(sums[-1])
        token = int((sums > want).int().argmax())
        if float(near) > vocab * 2.0 ** -44:
            assert int(tokens[r]) == token, r
            log = math.log(float(v[token]) / float(sums[-1]))
            # (the reference's own weight is a multiple of 2^-44)
            tol = 2.0 ** -24 * abs(log) + 2.0 ** 0 / float(v[token])
            assert abs(float(logs[r]) - log) <= tol + 1e-12


def test_given_outputs_streams_and_graphs():
    x = logits(6, 5003, 21).cuda()
    t = torch.tensor([1.0, 0.7, 0.0, 1.0, 1.3, 1.0]).cuda()
    k = torch.tensor([0, 40, 0, 0, 0, 5], dtype=torch.int32).cuda()
    p = torch.tensor([1.0, 0.9, 1.0, 0.8, 1.0, 1.0]).cuda()
    u = torch.rand((6,), generator=_gen(22)).cuda()
    out = torch.full((6,), -7, dtype=torch.int32, device="cuda")
    logs = torch.zeros(6, device="cuda")
    ws = torch.empty(max(eb.sample_workspace_bytes(6, 5003), 1), dtype=torch.uint8, device="cuda")
    want = [v.clone() for v in eb.sample_tokens(x, u, t, k, p)]
    got = eb.sample_tokens(x, u, t, k, p, out=out, logprobs=logs, workspace=ws)
    assert got[0] is out and got[1] is logs
    assert torch.equal(out, want[0]) and torch.equal(logs, want[1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = eb.sample_tokens(x, u, t, k, p)
    side.synchronize()
    assert torch.equal(other[0], want[0]) and torch.equal(other[1], want[1])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        eb.sample_tokens(x, u, t, k, p, out=out, logprobs=logs, workspace=ws)
    for i in range(3):
        u.copy_(torch.rand((6,), generator=_gen(30 + i)))
        graph.replay()
        torch.cuda.synchronize()
        now = eb.sample_tokens(x, u, t, k, p)
        assert torch.equal(out, now[0]) and torch.equal(logs, now[1])


def test_binding_refusals():
    x, u = logits(3, 50, 1).cuda(), torch.zeros(3).cuda()
    with pytest.raises(ValueError, match="one behind the other"):
        eb.sample_tokens(x.t(), torch.zeros(50).cuda())
    with pytest.raises(ValueError, match="one behind the other"):
        eb.sample_tokens(x[:1].expand(3, 50), u)
    with pytest.raises(ValueError, match="3 rows"):
        eb.sample_tokens(x, u[:2])
    with pytest.raises(TypeError, match="top_k must be"):
        eb.sample_tokens(x, u, None, u)
    with pytest.raises(ValueError, match="contiguous"):
        eb.sample_tokens(x[0], u)
    with pytest.raises(TypeError, match="u must be"):
        eb.sample_tokens(x, None)
    with pytest.raises(ValueError, match="ROCm device"):
        eb.sample_tokens(x, u.cpu())
    assert eb.sample_tokens(x[:0], u[:0])[0].shape == (0,)
    assert eb.sample_tokens(x[:, :0], u)[0].tolist() == [-1, -1, -1]


def _in_many_rows(x, u, t, k, p, m):
    """The same rows many times over: as many as get a workgroup each."""
    n = -(-200 // x.shape[0])
    got = eb.sample_tokens(x.cuda().repeat(n, 1), *(torch.tensor(v, dtype=d).cuda().repeat(n)
                           for v, d in ((u, F32), (t, F32), (k, torch.int32), (p, F32), (m, F32))))
    got = [v.view(n, -1) for v in got]
    assert all(torch.equal(v, v[:1].expand_as(v)) for v in got)
    return [v[0] for v in got]


def _rows_of_all_kinds(vocab):
    g = _gen(vocab)
    x = logits(12, vocab, vocab, F32)
    x[1] *= 1e-3                                   # near 0, flat
    x[2] = -x[2].abs() - 30                        # all below 0
    x[3] = -INF
    x[4, ::2] = NAN
    x[5, [7, vocab // 2, vocab - 1]] = INF
    x[6] = torch.randint(-3, 4, (vocab,), generator=g)            # ties over the whole row
    x[7] = -INF
    x[7, vocab - 1] = -3.0                         # one token, the last
    x[8] = torch.rand((vocab,), generator=g) * 2.0 ** -40         # all nearer to 0 than 2^-30
    x[8, ::3] *= -1
    x[8, vocab // 3] = 8.0                         # (and far below the largest)
    x[9, : vocab // 2] = torch.finfo(BF16).min
    x[10] *= 1e30
    x[11] = 0.0
    return x.to(BF16)


@pytest.mark.parametrize("vocab", [65536, 65537, 73728, 128256, 524288])
def test_a_row_is_the_same_in_one_workgroup_and_in_several(vocab):
    """Sums of weights are whole numbers: every bit is the same, however a row is
    divided, in any company."""
    x = _rows_of_all_kinds(vocab)
    n = x.shape[0]
    settings = [([1.0] * n, [0] * n, [1.0] * n, [0.0] * n),
                ([0.7] * n, [0] * n, [0.9] * n, [0.0] * n),
                ([1.0] * n, [vocab // 3] * n, [1.0] * n, [0.0] * n),
                ([1.3] * n, [1000 + i for i in range(n)], [0.5 + 0.04 * i for i in range(n)], [1e-3] * n),
                ([0.0] * n, [0] * n, [1.0] * n, [0.0] * n),
                ([INF, 1.0, 0.0, 2.0] * 3, [0, 1, 0, 50] * 3, [0.9, 1.0, 1.0, 0.3] * 3,
                 [0.0, 0.0, 0.0, 0.2] * 3)]
    for i, (t, k, p, m) in enumerate(settings):
        u = us(n, vocab + i)
        want = _in_many_rows(x, u, t, k, p, m)
        got = eb.sample_tokens(x.cuda(), *(torch.tensor(v, dtype=d).cuda() for v, d in
                               ((u, F32), (t, F32), (k, torch.int32), (p, F32), (m, F32))))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), i
        for r in (0, 6, 9):
            one = eb.sample_tokens(x[r:r + 1].cuda(), *(torch.tensor(v[r:r + 1], dtype=d).cuda()
                                   for v, d in ((u, F32), (t, F32), (k, torch.int32), (p, F32),
                                                (m, F32))))
            assert torch.equal(one[0], want[0][r:r + 1]) and torch.equal(one[1], want[1][r:r + 1])


def test_rows_in_several_workgroups_against_the_definition():
    x = _rows_of_all_kinds(73729)
    n = x.shape[0]
    check(x, us(n, 1), [1.0] * n, [0] * n, [0.9] * n)
    check(x, us(n, 2), [0.8] * n, [700] * n, [0.95] * n, [1e-3] * n)
    check(x, us(n, 3))


def test_two_calls_at_once_with_a_workspace_each():
    x, u = logits(4, 80000, 5).cuda(), torch.tensor(us(4, 5), dtype=F32).cuda()
    p = torch.full((4,), 0.8).cuda()
    want = eb.sample_tokens(x, u, top_p=p)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ws = [torch.empty(eb.sample_workspace_bytes(4, 80000), dtype=torch.uint8, device="cuda")
          for _ in range(2)]
    assert ws[0].numel() > 0
    for _ in range(5):
        here = eb.sample_tokens(x, u, top_p=p, workspace=ws[0])
        with torch.cuda.stream(side):
            there = eb.sample_tokens(x, u, top_p=p, workspace=ws[1])
        torch.cuda.synchronize()
        for got in (here, there):
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with pytest.raises(eb.EIError):
        eb.sample_tokens(x, u, workspace=ws[0][:-256])


def test_captured_rows_in_several_workgroups():
    """A graph of such a call, replayed with other settings and numbers between eager
    calls; its workspace is its own."""
    x = logits(5, 80000, 8).cuda()
    u, p, k = torch.zeros(5).cuda(), torch.ones(5).cuda(), torch.zeros(5, dtype=torch.int32).cuda()
    t = torch.ones(5).cuda()
    for _ in range(2):
        eb.sample_tokens(x, u, t, k, p)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out, logs = eb.sample_tokens(x, u, t, k, p)
    for i in range(4):
        u.copy_(torch.tensor(us(5, i), dtype=F32))
        p.fill_((1.0, 0.9, 0.5, 0.99)[i])
        k.fill_((0, 100, 0, 20000)[i])
        t.copy_(torch.tensor([1.0, 0.0, 0.5, 3.0, 1.0]))
        x[i] = -INF if i == 3 else x[i]
        want = eb.sample_tokens(x, u, t, k, p)
        graph.replay()
        again = eb.sample_tokens(x, u, t, k, p)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(logs, want[1])
        assert torch.equal(again[0], want[0])
