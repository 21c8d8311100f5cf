"""The dealing-out of a long table's keys over the waves of a launch, on the host:
nothing left out or taken twice, whatever the lengths; and that the launches of
the GPU's test take the paths they are named for."""
import random

import pytest

from cache_share_model import LARGE, Plan, large


@pytest.mark.parametrize("seed", range(40))
def test_every_step_once(seed):
    rng = random.Random(seed)
    for _ in range(5):
        S = rng.choice([1, 2, 5, 17, 70])
        top = rng.choice([40, 700, 9000, 40000 // S + 100])
        lengths = [rng.choice([0, 1, top, rng.randint(0, top)]) for _ in range(S)]
        one = rng.choice([1, 1, 4, 7])
        new = [one] * S if rng.random() < 0.6 else [rng.choice([0, 1, one]) for _ in range(S)]
        hkv = rng.choice([1, 2, 8])
        if sum(new):
            Plan(lengths, new, hkv * rng.choice([1, 4, 8]), hkv, 64,
                 max(33, -(-top // 64) + rng.choice([0, 50]))).check()


@pytest.mark.parametrize("name", LARGE)
def test_what_the_large_launches_are_there_for(name):
    want, plan = large(name)
    plan.check()
    assert want <= plan.features, plan.features
