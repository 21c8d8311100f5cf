"""Attention over the cache keeps 16 significant bits of its probabilities, in the
launches of short tables and in those whose keys are dealt out."""
import pytest
import torch

from cache_precision import CASES, E4M3, INT8, case, reference
from paper_2606_09508_amd import binding as eb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("P,spare", [(64, 1), (64, 60), (128, 1), (128, 30)])
@pytest.mark.parametrize("held,new,hq,hkv", CASES)
def test_probabilities(held, new, hq, hkv, P, spare, dtype):
    for seed in (3, 4):
        c = case(held, new, hq, hkv, P, dtype, seed, spare)
        pages = eb.CachePages(*(c[n].cuda() for n in ("k", "v", "ks", "vs")))
        i32 = [torch.tensor(c[n], dtype=torch.int32).cuda() for n in ("lengths", "cu")]
        got = eb.cache_attn(c["q"].cuda(), pages, c["table"].cuda(), *i32).cpu()
        want, off = reference(c)
        err = (got.double() - want).abs()
        assert bool((err <= off).all()), float((err / off).max())
