"""Attention over the cache keeps 16 significant bits of its probabilities, in the
launches of short tables and in those whose keys are dealt out."""
import pytest
import torch

from cache_precision import CASES, E4M3, INT8, case, reference
from paper_2606_09508_amd import binding as eb

pytestmark = pytest.mark.gpu


def check(c):
    pages = eb.CachePages(*(c[n].cuda() for n in ("k", "v", "ks", "vs")))
    i32 = [torch.tensor(c[n], dtype=torch.int32).cuda() for n in ("lengths", "cu")]
    got = eb.cache_attn(c["q"].cuda(), pages, c["table"].cuda(), *i32).cpu()
    want, off = reference(c)
    err = (got.double() - want).abs()
    assert bool((err <= off).all()), float((err / off).max())


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("P,spare", [(64, 1), (64, 60), (128, 1), (128, 30)])
@pytest.mark.parametrize("held,new,hq,hkv", CASES)
def test_probabilities(held, new, hq, hkv, P, spare, dtype):
    for seed in (3, 4):
        check(case(held, new, hq, hkv, P, dtype, seed, spare))


@pytest.mark.parametrize("dtype", [E4M3, INT8])
@pytest.mark.parametrize("spare", [1, 60])
@pytest.mark.parametrize("exponent", [-90, 64])
def test_the_range_of_the_values_scales(exponent, spare, dtype):
    """At both ends of the scales that the header names, also where the scores
    rise so slowly that the running maximum stays 2^16 and more behind."""
    for rising in (False, True):
        c = case([300, 700, 64], [1, 2, 1], 8, 2, 64, dtype, 3, spare)
        c["vs"] = torch.exp2(torch.full_like(c["vs"], float(exponent)))
        if rising:
            c["ks"].fill_(1.0)
            c["q"][..., 0] = 1.0
            c["k"].copy_((c["k"].float() * 2.0 ** -6).to(c["k"].dtype))
            for s, n in enumerate(c["lengths"]):
                p = torch.arange(n)
                x = torch.clamp(p * (2.0 if dtype is E4M3 else 0.5), max=120.0).round()
                c["k"][c["table"][s][p // 64].long(), :, p % 64, 0] = x.to(dtype)[:, None].expand(-1, 2)
        check(c)
