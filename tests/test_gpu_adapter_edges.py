"""Low-rank adapters at the end of fp32's range, against the formula."""
import math

import pytest
import torch

from paper_2606_09508_amd import binding as eb
from test_gpu_adapters import BF16, reference, run

pytestmark = pytest.mark.gpu

FMAX = 2.0 ** 128 - 2.0 ** 104


@pytest.mark.parametrize("tokens", [3, 800])
@pytest.mark.parametrize("rank", [8, 40])
def test_an_inner_product_past_the_largest_bf16(tokens, rank):
    """scale (x A^T) is a finite fp32 number that bf16 would round to infinity."""
    scales = [FMAX, -FMAX, 2.0 ** 128 - 2.0 ** 119, 2.0 ** 128 - 2.0 ** 119 - 2.0 ** 105,
              2.0 ** 128 - 2.0 ** 120, 2.0 ** 127, 1.0]
    n = len(scales)
    x = torch.zeros((tokens, 16), dtype=BF16)
    x[:, 3] = 1.0
    a = torch.zeros((n, rank, 16), dtype=BF16)
    a[:, 5, 3] = 1.0
    b = torch.zeros((n, 64, rank), dtype=BF16)
    b[:, :, 5] = torch.tensor([2.0 ** -(100 + i % 20) * (-1) ** i for i in range(64)])
    ads = [eb.Adapters(a, b, torch.tensor(scales, dtype=torch.float32))]
    new = [tokens] * n
    xs, ys = x.repeat(n, 1), [torch.ones((tokens * n, 64), dtype=BF16)]
    got, = run(xs, ys, ads, list(range(n)), new)
    cu = [i * tokens for i in range(n + 1)]
    (want,), _ = reference(xs, ys, ads, list(range(n)), cu)
    # V enters with 16 bits, y is rounded once
    assert ((got.double() - want).abs() <= (2.0 ** -16 + 2.0 ** -8) * want.abs()).all()


@pytest.mark.parametrize("tokens", [3, 800])
def test_an_infinite_entry_of_b_is_no_finite_output(tokens):
    """It makes its output infinite or NaN for the tokens of its adapter, no other one."""
    g = torch.Generator().manual_seed(tokens)
    x = torch.randn((2 * tokens, 64), generator=g).to(BF16)
    ads = [eb.Adapters(torch.randn((2, 8, 64), generator=g).to(BF16),
                       torch.randn((2, 128, 8), generator=g).to(BF16))]
    ys = [torch.randn((2 * tokens, 128), generator=g).to(BF16)]
    clean, = run(x, ys, ads, [0, 1], [tokens] * 2)
    ads[0].b[1, 70, 3] = math.inf
    got, = run(x, ys, ads, [0, 1], [tokens] * 2)
    assert not torch.isfinite(got[tokens:, 70]).any()
    got[tokens:, 70] = clean[tokens:, 70]
    assert torch.equal(got, clean)


@pytest.mark.parametrize("T,counts", [
    # of adapters 0, 1, 2: the places behind the second one pass 2^31, or 2^32
    (65536, [100, 2 ** 31 - 64, 0]), (65536, [100, 2 ** 31 - 64, 2 ** 31 + 300]),
    (65535, [2 ** 31, 40, 2 ** 31 - 16]), (40000, [2 ** 31 - 1, 2 ** 31 - 1, 500])])
def test_offsets_that_count_past_32_bits_touch_nothing_outside(T, counts):
    """Sequences that name the tokens again and again (and go back between)."""
    index, cu = [], [0]
    for a in reversed(range(3)):
        left = counts[a]
        while left:
            n = min(left, T)
            index += [a, -1]
            cu += [n, 0]
            left -= n
    g = torch.Generator().manual_seed(T)
    x = torch.randn((T, 64), generator=g).to(BF16).cuda()
    y = torch.randn((T + 256, 64), generator=g).to(BF16)
    ad = eb.Adapters(torch.randn((3, 8, 64), generator=g).to(BF16).cuda(),
                     torch.randn((3, 64, 8), generator=g).to(BF16).cuda())
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()
    plan = eb.adapter_plan(i32(index), 3, T, i32(cu))
    need = eb.adapter_add_workspace_bytes(plan, 64, 8, 1)
    ws = torch.full((need + 65536,), 0x5a, dtype=torch.uint8, device="cuda")
    # tiles of the plan: their adapter, first place and tokens, behind 64 bytes
    n = int(plan.data[:4].view(torch.int32))
    tiles = plan.data[64:64 + 16 * n].view(torch.int32).view(n, 4).cpu()
    some = tiles[tiles[:, 2] > 0]
    assert (some[:, 1] >= 0).all() and (some[:, 1] + some[:, 2] <= T).all()
    assert ((some[:, 0] >= 0) & (some[:, 0] < 3)).all()
    dev = y.cuda()
    eb.adapter_add(x, [dev[128:128 + T]], [ad], plan, ws)
    got = dev.cpu()
    assert torch.equal(got[:128], y[:128]) and torch.equal(got[128 + T:], y[128 + T:])
    assert (ws[need:] == 0x5a).all()
