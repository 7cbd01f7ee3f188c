"""The plain implementations that the packed cache's and eviction's tests hold the
kernels to, checked against their definitions by hand (no GPU)."""
import numpy as np
import pytest

import shaped_ref as R


def _group(x):
    """x in the first 32 dims, zeros elsewhere."""
    row = np.zeros((1, R.D))
    row[0, :len(x)] = x
    code, byte = R.quantise(row)
    return code[0, :len(x)], byte[0], R.values(code, byte)[0, :len(x)]


@pytest.mark.parametrize("top,e", [(6.0, 0), (6.96875, 0), (7.0, 1), (8.0, 1), (13.875, 1),
                                   (14.0, 2), (3.5, 0), (3.484375, -1), (1.0, -2), (0.5, -3),
                                   (2.0 ** -130, -125), (3e38, 125)])
def test_exponent_is_the_smallest_under_which_the_top_is_below_seven(top, e):
    _, byte, _ = _group([top])
    assert byte[0] == e + 127 and np.all(byte[1:] == 0)


def test_numbers_round_to_the_nearest_and_ties_to_the_even_code():
    x = [6, 0.25, 0.375, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.5, -0.75, -2.5, 0.1, -0.3]
    _, byte, v = _group(x)
    assert byte[0] == 127
    assert v.tolist() == [6, 0, 0.5, 1, 1, 2, 2, 4, 4, 6, -1, -2, 0, -0.5]


def test_values_above_the_largest_number_are_cut():
    _, byte, v = _group([3.3e38, 1.0])
    assert byte[0] == 252 and v[0] == 6 * 2.0 ** 125


@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_a_group_with_an_infinity_or_nan_reads_as_nan(bad):
    row = np.ones((1, R.D))
    row[0, 40] = bad
    code, byte = R.quantise(row)
    v = R.values(code, byte)[0]
    assert byte[0].tolist() == [125, 255, 125, 125]
    assert np.isnan(v[32:64]).all() and np.all(v[:32] == 1) and np.all(v[64:] == 1)


def test_pack_and_unpack_are_inverse_and_fill_every_byte_once():
    rng = np.random.default_rng(0)
    x = [R.bf16(rng.standard_normal((3, 2, R.BS, R.D))) for _ in range(2)]
    (kc, kb), (vc, vb) = R.quantise(x[0]), R.quantise(x[1])
    k, v = R.unpack(R.pack(kc, kb, vc, vb))
    assert np.array_equal(k, R.values(kc, kb)) and np.array_equal(v, R.values(vc, vb))
    pk, pv, ke, ve = R._places()
    at = np.concatenate([pk[:, ::2].ravel(), pv[:, ::2].ravel(), ke.ravel(), ve.ravel()])
    assert sorted(at.tolist()) == list(range(R.RECORD))


def test_rounding_is_off_by_at_most_half_a_step():
    rng = np.random.default_rng(1)
    x = R.bf16(rng.standard_normal((400, R.D)) * 2.0 ** rng.integers(-20, 20, (400, 1)))
    code, byte = R.quantise(x)
    y = R.values(code, byte)
    unit = np.repeat(2.0 ** (byte.astype(float) - 127), 32, axis=-1)
    m = np.abs(x) / unit  # below 7; steps of 0.5 up to 2, 1 up to 4, 2 above
    step = np.where(m <= 2, 0.5, np.where(m <= 4, 1.0, 2.0))
    assert np.all(np.abs(x - y) <= step / 2 * unit)


def test_kept_tokens_by_hand():
    nan = np.nan
    assert R.kept_tokens(np.array([3., 1, 3, 2, 9]), 5, 3, 0).tolist() == [0, 2, 4]
    assert R.kept_tokens(np.array([3., 1, 3, 2, 9]), 5, 2, 0).tolist() == [0, 4]
    assert R.kept_tokens(np.array([3., 1, 3, 2, 0]), 5, 2, 1).tolist() == [0, 4]
    assert R.kept_tokens(np.array([3., 1, 3, 2, 0]), 5, 2, 7).tolist() == [3, 4]
    assert R.kept_tokens(np.array([0., nan, np.inf, 2]), 4, 1, 0).tolist() == [1]
    assert R.kept_tokens(np.array([0., 0, -1, -0.]), 4, 2, 0).tolist() == [0, 1]
    assert R.kept_tokens(np.array([1., 2]), 2, 0, 5).tolist() == []
