"""Decoder steps of forks beside sequences that share nothing, in any order."""
import pytest

from test_gpu_serving import _check_step, _hidden, _prompted, _setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("new", [1, 3])
@pytest.mark.parametrize("forks", [2, 8])
def test_forks_beside_lone_sequences(forks, new):
    dec, g = _setup()
    (a,), _, _ = _prompted(dec, g, [330])
    lone, _, _ = _prompted(dec, g, [40, 65, 3, 200, 64])
    family = [a] + [dec.cache.fork(a) for _ in range(forks - 1)]
    seqs = [s for pair in zip(lone, family) for s in pair] + family[len(lone):] + lone[len(family):]
    counts = [1 + (i + new) % new for i in range(len(seqs))]
    order, groups = dec._groups(seqs, [0] * len(seqs))
    assert order is not None and sum(n > 0 for n in groups[1]) == 1 and len(groups[1]) < len(lone)
    adapter = [i % 4 - 1 for i in range(len(seqs))]
    for _ in range(2):
        _check_step(dec, _hidden(g, sum(counts)), seqs, counts, adapter)
