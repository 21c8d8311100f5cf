"""Sampling of long fp32 rows against the definition: rows of many blocks, more
tokens in a bin than the list holds, cuts in the farthest bin."""
import math

import pytest
import torch

from paper_2606_09508_amd import binding as eb
from test_gpu_sample import F32, _gen, logits, us

pytestmark = pytest.mark.gpu


def _check(x, u, t, k, p):
    """The definition in vectors of 64 bits, rows at a time.  (A weight of 2^44 steps may
    be a step off where exp rounds otherwise: a sum of n of them passes another u, or
    another share of top-p, only within n 2^-44 of it.)"""
    vocab = x.shape[1]
    f = lambda v, d=F32: torch.tensor(v, dtype=d).cuda()
    tokens, logs = eb.sample_tokens(x.cuda(), f(u), f(t), f(k, torch.int32), f(p))
    again, _ = eb.sample_tokens(x.cuda(), f(u), f(t), f(k, torch.int32), f(p))
    assert torch.equal(tokens, again)
    compared = 0
    for r in range(len(u)):
        y, by = torch.sort(x[r].double(), descending=True, stable=True)
        w = torch.floor(torch.exp((y - y[0]) / float(f(t)[r])) * 2.0 ** 44 + 0.5)
        w = torch.where(y > -math.inf, w, 0).long()
        if k[r]:
            w[k[r]:] = 0
        near = 1.0
        if p[r] < 1:
            total = float(w.sum())
            before = (w.cumsum(0) - w).double()
            want = float(f(p)[r]) * total
            near = float((before - want).abs().min()) / total
            w = torch.where(before < want, w, 0)
        v = torch.zeros_like(w).scatter_(0, by, w)
        sums = v.cumsum(0)
        want = float(f(u)[r]) * float(sums[-1])
        near = min(near, float((sums.double() - want).abs().min()) / float(sums[-1]))
        token = int((sums > want).int().argmax())
        if near > vocab * 2.0 ** -44:
            compared += 1
            assert int(tokens[r]) == token, r
            log = math.log(float(v[token]) / float(sums[-1]))
            # (the reference's own weights are multiples of 2^-44, each off by a half, and
            # the sum's error is at most a half for each token of 2^44 at least)
            tol = 2.0 ** -24 * abs(log) + 1.0 / float(v[token]) + vocab * 2.0 ** -45
            assert abs(float(logs[r]) - log) <= tol + 1e-12
    assert compared >= len(u) // 2


CUTS = [(0, 1.0), (50, 1.0), (0, 0.95), (500, 0.9), (0, 0.6), (20000, 1.0), (100000, 0.9999),
        (100000, 1.0), (0, 0.9999), (60000, 0.5)]


@pytest.mark.parametrize("rows,vocab", [(1, 128256), (20, 128256), (2, 200003), (40, 50257),
                                        (300, 1500), (10, 524288)])
def test_long_rows(rows, vocab):
    cuts = [CUTS[r % len(CUTS)] for r in range(rows)]
    _check(logits(rows, vocab, rows, F32, 2.2, 60), us(rows, rows),
           [(1.0, 0.7, 1.4)[r % 3] for r in range(rows)], [c[0] for c in cuts], [c[1] for c in cuts])


@pytest.mark.parametrize("vocab", [128256, 524288])
def test_rows_that_crowd_the_bins(vocab):
    """Nearly equal logits (a bin holds more than the list), and a few far above all."""
    x = torch.randn((len(CUTS), vocab), generator=_gen(vocab)) * 0.01
    _check(x, us(len(CUTS), 1), [1.0] * len(CUTS), [c[0] for c in CUTS], [c[1] for c in CUTS])
    x[:, ::30011] += 15.0
    _check(x, us(len(CUTS), 2), [1.0] * len(CUTS), [c[0] for c in CUTS], [c[1] for c in CUTS])
    x[:, 1::2] = -math.inf
    _check(x, us(len(CUTS), 3), [1.0] * len(CUTS), [c[0] for c in CUTS], [c[1] for c in CUTS])
