"""GPU tests of attention with shaped scores and of its weight sums over batches of few
pairs whose lengths lie far apart: a long pair then has more shares than the others."""
import numpy as np
import pytest

from test_gpu_shaped import KINDS, Case, check_weights, gpu  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu

# name: (requests' lengths, kv heads); never more pairs than compute units.
BATCHES = {
    "last": ([300] * 31 + [30000], 2),
    "first": ([25000, 16, 0, 700], 8),
    "behind_64_requests": ([40] * 100 + [0, 20000] + [5] * 60, 1),
    "among_empty_ones": ([0] * 70 + [12000], 3),
    "every_other": ([2500, 1] * 20, 4),
    "two_lengths": ([9000] + [700] * 12, 16),
    "one_token_each": ([1] * 200, 1),
}


@pytest.mark.parametrize("group", [2, 8])
@pytest.mark.parametrize("name", BATCHES)
@pytest.mark.parametrize("kind", KINDS)
def test_attention(kind, name, group):
    lens, hkv = BATCHES[name]
    c = Case(kind, lens, hkv, group, seed=60, extra_cols=2)
    first = c.check()
    c.check(None, 8.0, None, *c.ranges("document"))
    again = c.attend()  # counts are zero after every call, and results the same
    assert all(np.array_equal(a, b) for a, b in zip(first, again))


@pytest.mark.parametrize("name", BATCHES)
@pytest.mark.parametrize("kind", KINDS)
def test_weights(kind, name):
    lens, hkv = BATCHES[name]
    c = Case(kind, lens, hkv, 2, seed=61)
    check_weights(c)
    check_weights(c, None, None, *c.ranges("window"), in_place=True)
