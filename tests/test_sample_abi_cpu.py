"""Refusals of ei_sample_tokens, on the host before any launch, through the C ABI
and through the binding; no GPU is needed."""
import os

import pytest
import torch

from paper_2606_09508_amd import binding as eb

FAKE = 0x1000       # never dereferenced
OK, NULL, BAD, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3, -4
NAMES = ("u", "temperature", "top_k", "top_p", "min_p", "tokens", "logprobs")


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(eb.LIB_PATH):
        pytest.skip("libentropyinfer.so is not built")
    return eb.lib()


def sample(L, logits=FAKE, fmt=0, rows=3, vocab=1000, stride=1000, ws=FAKE, nb=1 << 40, **ptr):
    return L.ei_sample_tokens(logits, fmt, rows, vocab, stride, *(ptr.get(n, FAKE) for n in NAMES),
                              ws, nb, None)


def test_refusals(L):
    for bad in (dict(fmt=2), dict(fmt=-1), dict(rows=-1), dict(vocab=-1), dict(stride=999),
                dict(rows=2 ** 31 - 1, stride=2 ** 62)):
        assert sample(L, **bad) == BAD, bad
    assert sample(L, vocab=2 ** 19 + 1, stride=2 ** 20) == UNSUPPORTED
    for bad in (dict(logits=None), dict(u=None), dict(tokens=None)):
        assert sample(L, **bad) == NULL, bad
    assert sample(L, logits=0x1001) == UNSUPPORTED
    assert sample(L, logits=0x1002, fmt=1) == UNSUPPORTED
    for n in NAMES:
        assert sample(L, **{n: 0x1002}) == UNSUPPORTED, n


def test_workspace(L):
    for fmt in (0, 1):
        need = L.ei_sample_workspace_bytes(3, 1000, fmt)
        if need:
            assert sample(L, fmt=fmt, ws=None) == WORKSPACE
            assert sample(L, fmt=fmt, nb=need - 1) == WORKSPACE
            assert sample(L, fmt=fmt, ws=0x1008) == UNSUPPORTED
    for bad in ((-1, 1000, 0), (3, -1, 0), (3, 1000, 2), (3, 2 ** 19 + 1, 0)):
        assert L.ei_sample_workspace_bytes(*bad) == 0


def test_no_rows(L):
    assert sample(L, None, rows=0, u=None, tokens=None, ws=None, nb=0) == OK


def test_binding_refuses_tensors_of_the_host():
    x, u = torch.zeros((2, 8)), torch.zeros(2)
    with pytest.raises(ValueError, match="ROCm device"):
        eb.sample_tokens(x, u)
    with pytest.raises(TypeError, match="bfloat16 or float32"):
        eb.sample_tokens(x.half(), u)
    with pytest.raises(TypeError, match="torch.Tensor"):
        eb.sample_tokens(None, u)
