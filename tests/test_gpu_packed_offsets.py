"""Offsets of packed prompts that point outside the tensors, and lists that do not
ascend: the first are clamped, the second touch nothing outside the tensors."""
import pytest
import torch

from paper_2606_09508_amd import binding as eb

pytestmark = pytest.mark.gpu

D, HKV = 128, 2


def _rand(shape, seed):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16)


def _roomy(t, fill):
    """(t's values, and where they lie in a tensor three times as large)."""
    room = torch.full((3 * t.numel(),), fill, dtype=t.dtype, device="cuda")
    room[t.numel():2 * t.numel()] = t.flatten().cuda()
    return room, room[t.numel():2 * t.numel()].view(t.shape)


def _tensors(heads, T):
    """q, k and v with NaN around them, so that a row read outside shows."""
    return [_roomy(_rand((1, h, T, D), i), float("nan"))[1] for i, h in enumerate((heads, HKV, HKV))]


@pytest.mark.parametrize("heads", [4, 64])     # 32-row tiles, 128-row tiles
def test_offsets_outside_are_clamped(heads):
    T, cu = 300, [-50, -3, 100, 100, 250, 2 ** 31 - 1]
    q, k, v = _tensors(heads, T)
    room, out = _roomy(torch.zeros((1, heads, T, D), dtype=torch.bfloat16), 3.0)
    want = torch.zeros_like(out)
    for offsets, o in ((cu, out), ([0, 0, 100, 100, 250, T], want)):
        eb.packed_prefill_attn(q, k, v, torch.tensor(offsets, dtype=torch.int32, device="cuda"),
                               out=o)
    n = out.numel()
    assert torch.equal(out, want) and not bool(out.isnan().any())
    assert bool((room[:n] == 3.0).all()) and bool((room[2 * n:] == 3.0).all())


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("heads", [4, 64])
@pytest.mark.parametrize("cu", [[0, 1000, 10, 20], [-50, 100, 90, 90, 2 ** 31 - 1, 5],
                                [1000, 600, 300, 0], [0, 1000] * 20, [900, -1, 2000, 10, 990],
                                [2 ** 31 - 1, -2 ** 31] * 70, [1000, 0] + [500] * 200])
def test_lists_that_do_not_ascend(cu, heads, causal):
    """A row holds what was there or the attention over rows of the tensors:
    finite, as those are; and nothing around the output is written."""
    T = 1000
    q, k, v = _tensors(heads, T)
    room, out = _roomy(torch.full((1, heads, T, D), 7.0, dtype=torch.bfloat16), 3.0)
    eb.packed_prefill_attn(q, k, v, torch.tensor(cu, dtype=torch.int32, device="cuda"),
                           causal=causal, out=out)
    n = out.numel()
    assert bool(out.isfinite().all())
    assert bool((room[:n] == 3.0).all()) and bool((room[2 * n:] == 3.0).all())
