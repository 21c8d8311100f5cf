"""That the bound on the cache attention's results tells 16 significant bits of
its probabilities from the 8 of a single bf16 number: both emulated on the CPU."""
import pytest
import torch

from cache_precision import CASES, E4M3, INT8, case, emulate, reference


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("held,new,hq,hkv", CASES)
def test_the_bound_holds_for_two_numbers_and_not_for_one(held, new, hq, hkv, dtype):
    c = case(held, new, hq, hkv, 64, dtype, 3, 1)
    want, off = reference(c)
    over = [((emulate(c, n).double() - want).abs() > off).float().mean() for n in (1, 2)]
    assert float(over[1]) == 0.0
    assert float(over[0]) > 0.02     # of all elements
