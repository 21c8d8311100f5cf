"""Refusals of the adapters' entry points, on the host before any launch, through
the C ABI and through the binding; no GPU is needed."""
import ctypes
import os

import pytest
import torch

from paper_2606_09508_amd import binding as eb

FAKE, ODD = 0x1000, 0x1008       # never dereferenced; ODD is 8-byte aligned only
OK, NULL, BAD, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3, -4
BATCH = eb.AdapterBatch(40, 8, 6)
MANY = 1 << 40


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(eb.LIB_PATH):
        pytest.skip("libentropyinfer.so is not built")
    return eb.lib()


def plan(L, index=FAKE, cu=None, batch=BATCH, data=FAKE, nb=MANY):
    return L.ei_adapter_plan(index, cu, batch, data, nb, None)


def add(L, x=FAKE, n_in=64, rank=16, outs=(64, 32), n=None, batch=BATCH, data=FAKE, data_nb=MANY,
        ws=FAKE, ws_nb=MANY, a=FAKE, b=FAKE, scale=FAKE, y=FAKE, null=False):
    t = (eb.AdapterTarget * max(len(outs), 1))(*[eb.AdapterTarget(a, b, scale, y, o) for o in outs])
    return L.ei_adapter_add(x, n_in, rank, None if null else t, len(outs) if n is None else n, batch,
                            data, data_nb, ws, ws_nb, None)


@pytest.mark.parametrize("batch,status", [
    (eb.AdapterBatch(-1, 8, 6), BAD), (eb.AdapterBatch(40, -1, 6), BAD),
    (eb.AdapterBatch(40, 8, -1), BAD), (eb.AdapterBatch(40, 8, 8193), UNSUPPORTED)])
def test_batches(L, batch, status):
    assert plan(L, batch=batch) == status
    assert add(L, batch=batch) == status
    assert L.ei_adapter_plan_bytes(batch) == 0
    assert L.ei_adapter_add_workspace_bytes(batch, 64, 16, 2) == 0


def test_plan_refusals(L):
    need = L.ei_adapter_plan_bytes(BATCH)
    assert need > 0
    assert plan(L, batch=eb.AdapterBatch(41, 8, 6)) == BAD
    assert plan(L, index=None) == NULL
    assert plan(L, index=0x1002) == UNSUPPORTED
    assert plan(L, cu=0x1001) == UNSUPPORTED
    assert plan(L, data=None) == WORKSPACE
    assert plan(L, nb=need - 1) == WORKSPACE
    assert plan(L, data=ODD) == UNSUPPORTED


@pytest.mark.parametrize("batch", [eb.AdapterBatch(0, 8, 6), eb.AdapterBatch(40, 0, 6),
                                   eb.AdapterBatch(40, 8, 0)])
def test_nothing_to_do(L, batch):
    assert L.ei_adapter_plan_bytes(batch) == 0
    assert plan(L, None, None, batch, None, 0) == OK
    assert add(L, None, batch=batch, data=None, data_nb=0, ws=None, ws_nb=0, a=None, y=None) == OK


def test_add_refusals(L):
    need = L.ei_adapter_add_workspace_bytes(BATCH, 64, 16, 2)
    assert need >= 40 * 32 * 4
    for bad in (dict(n_in=0), dict(n_in=-8), dict(rank=0), dict(n=-1), dict(outs=(64, 0)),
                dict(outs=(-8,))):
        assert add(L, **bad) == BAD, bad
    for bad in (dict(n_in=60), dict(rank=12), dict(rank=136), dict(outs=(8,) * 5),
                dict(outs=(64, 36)), dict(x=ODD), dict(a=ODD), dict(b=ODD), dict(y=ODD),
                dict(scale=0x1002), dict(data=ODD), dict(ws=ODD)):
        assert add(L, **bad) == UNSUPPORTED, bad
    for bad in (dict(x=None), dict(a=None), dict(b=None), dict(y=None), dict(null=True)):
        assert add(L, **bad) == NULL, bad
    for bad in (dict(data=None), dict(data_nb=L.ei_adapter_plan_bytes(BATCH) - 1), dict(ws=None),
                dict(ws_nb=need - 1)):
        assert add(L, **bad) == WORKSPACE, bad
    assert add(L, outs=(), x=None, null=True) == OK


def test_sizes_of_many_tokens(L):
    # (no overflow: the bytes grow with the tokens)
    big = eb.AdapterBatch(2 ** 31 - 1, 2 ** 31 - 1, 8192)
    assert L.ei_adapter_plan_bytes(big) > 4 * (2 ** 31 - 1)
    assert L.ei_adapter_add_workspace_bytes(big, 8, 128, 4) >= 4 * 512 * (2 ** 31 - 1)


def test_binding_refuses_tensors_of_the_host():
    i = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="ROCm device"):
        eb.adapter_plan(i, 3, 4)
    plan_ = eb.AdapterPlan(torch.zeros(64, dtype=torch.uint8), eb.AdapterBatch(4, 4, 3))
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="ROCm device"):
        eb.adapter_add(x, [x], [eb.Adapters(x[None], x[None])], plan_)
    with pytest.raises(TypeError, match="torch.Tensor"):
        eb.adapter_add(None, [x], [], plan_)
