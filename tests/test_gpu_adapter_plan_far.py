"""The adapters' plan for as many tokens as 31 bits count."""
import pytest
import torch

from paper_2606_09508_amd import binding as eb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cu,index", [([0, 2 ** 31 - 1], [0]), ([0, 700, 2 ** 31 - 2], [1, 1])])
def test_the_most_tokens(cu, index):
    T, n = 2 ** 31 - 1, len(index)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()
    plan = eb.adapter_plan(i32(index), 2, T, i32(cu))
    whole = plan.data
    assert whole.numel() > 4 * T
    held = cu[-1]
    tiles = int(whole[:4].view(torch.int32))
    assert tiles == -(-held // 64)
    at = whole.numel() - 4 * T           # of the list, the plan's last part
    for i in (0, 2 ** 20, 2 ** 30 + 7, held - 2 ** 20):
        part = whole[at + 4 * i:at + 4 * (i + 2 ** 20)].view(torch.int32)
        assert torch.equal(part, torch.arange(i, i + 2 ** 20, dtype=torch.int32, device="cuda"))
    for t in (0, tiles // 2, tiles - 1):
        adapter, begin, count, _ = whole[64 + 16 * t:80 + 16 * t].view(torch.int32).tolist()
        assert (adapter, begin, count) == (index[0], 64 * t, min(64, held - 64 * t))
    del plan, whole
    torch.cuda.empty_cache()
