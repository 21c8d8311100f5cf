"""Shared-prefix attention of sequences whose length is below zero: they hold nothing."""
import pytest

from test_gpu_shared import E4M3, Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("groups,size", [(1, 3), (1, 30), (260, 2)])
@pytest.mark.parametrize("length", [-1, -2 ** 31, -2 ** 31 + 1])
def test_a_length_below_zero_is_none(groups, size, length):
    S = groups * size
    b = Batch([size] * groups, [2] * groups, [20] * S, [2] * S, 4, 1, 64, E4M3, seed=size)
    b.check()
    for s in (1, S - 1):
        b.lengths[s] = length
    got = b.check()
    for s in (1, S - 1):
        assert (got[:, :, 2 * s:2 * s + 2] == 0).all()
