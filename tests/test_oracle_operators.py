"""Pins of the oracle of scored attention, rotary positions and token log probabilities (CPU only)."""
import math

import numpy as np
import pytest

import oracle


def _rows(seed, n, delta, hq=4, hkv=2, d=8):
    rng = np.random.default_rng(seed)
    return rng.standard_normal((delta, hq, d)), rng.standard_normal((n + delta, hkv, d)), rng.standard_normal((n + delta, hkv, d))


def test_without_changes_it_is_delta_attention():
    q, k, v = _rows(1, 7, 5)
    want = oracle.delta_attend(q, k[:7], v[:7], k[7:], v[7:], 0.3)
    got = oracle.scored_attend(q, k, v, 7, 0.3)
    assert np.allclose(got[0], want[0], atol=1e-13) and np.allclose(got[1], want[1], atol=1e-13)


def test_a_wide_cap_changes_nothing_and_a_narrow_one_makes_weights_equal():
    q, k, v = _rows(2, 9, 3)
    plain = oracle.scored_attend(q, k, v, 9, 0.5)[0]
    assert np.allclose(oracle.scored_attend(q, k, v, 9, 0.5, cap=1e6)[0], plain, atol=1e-9)
    even = oracle.scored_attend(q, k, v, 9, 0.5, cap=1e-9)[0]
    for i in range(3):
        assert np.allclose(even[i, 0], v[:10 + i, 0].mean(axis=0), atol=1e-7)


def test_ranges_by_hand():
    q, k, v = _rows(3, 6, 4, hq=2, hkv=1)
    assert np.allclose(oracle.scored_attend(q, k, v, 6, 0.5, window=1)[0], v[6:, [0, 0]])  # only itself
    seen = oracle.scored_attend(q, k, v, 6, 0.5, prefix=10)[0]  # everything, whatever the row's position
    s = 0.5 * (q[0, 1] @ k[:, 0].T)
    w = np.exp(s) / np.exp(s).sum()
    assert np.allclose(seen[0, 1], w @ v[:, 0])
    out, lse, _, _ = oracle.scored_attend(q, k, v, 6, 0.5, first=[0, 7, 99, 9])
    assert np.allclose(out[1], v[7, 0]) and np.allclose(out[3], v[9, 0])
    assert (out[2] == 0).all() and (lse[2] == -np.inf).all()


def test_a_slope_is_a_weight_by_distance():
    q, k, v = _rows(4, 5, 1, hq=2, hkv=1)
    k[:] = 0
    out, lse, _, _ = oracle.scored_attend(q, k, v, 5, 1.0, slopes=[0.5, 2.0])
    for h, slope in enumerate((0.5, 2.0)):
        w = np.exp(-slope * np.arange(5, -1, -1))
        assert np.allclose(out[0, h], (w / w.sum()) @ v[:, 0]) and np.isclose(lse[0, h], math.log(w.sum()))


@pytest.mark.parametrize("pairs", [False, True])
def test_products_of_turned_rows_depend_on_the_distance_alone(pairs):
    rng = np.random.default_rng(5)
    x, y = rng.standard_normal((1, 1, 16)), rng.standard_normal((1, 1, 16))
    f = 100.0 ** (-np.arange(6) / 6)
    dots = [(oracle.rotate(x, [a], f, 12, pairs)[0] * oracle.rotate(y, [a - 9], f, 12, pairs)[0]).sum() for a in (9, 500, 123456)]
    assert np.allclose(dots, dots[0], atol=1e-6)
    back = oracle.rotate(oracle.rotate(x, [77], f, 12, pairs)[0], [-77], f, 12, pairs)[0]
    assert np.allclose(back, x, atol=1e-12)


def test_halves_are_pairs_in_another_order_and_the_rest_stays():
    rng = np.random.default_rng(6)
    x = rng.standard_normal((3, 2, 10))
    f = [1.0, 0.25, 0.01]
    halves = oracle.rotate(x, [0, 3, 50], f, 6, False)[0]
    order = [0, 3, 1, 4, 2, 5, 6, 7, 8, 9]
    pairs = oracle.rotate(x[..., order], [0, 3, 50], f, 6, True)[0]
    assert np.allclose(halves[..., order], pairs)
    assert np.array_equal(halves[0], x[0]) and np.array_equal(halves[..., 6:], x[..., 6:])
    quarter = oracle.rotate(np.eye(2)[None, :1], [1], [math.pi / 2], 2, False, amplitude=3.0)[0]
    assert np.allclose(quarter[0, 0], [0, 3], atol=1e-6)


def test_norm_by_hand():
    x = np.array([[[3.0, 4.0]]])
    assert np.allclose(oracle.rotate(x, [0], [1.0], 2, False, eps=0.0, weight=[1.0, 2.0])[0], [[[3 / math.sqrt(12.5), 8 / math.sqrt(12.5)]]])


def test_logprobs_by_hand():
    x = np.log(np.array([[0.5, 0.25, 0.125, 0.125]]))
    lp, rank, ent, ids, tlp = oracle.token_logprobs(x, [3], n_top=3)
    assert np.isclose(lp[0], math.log(0.125)) and rank[0] == 2 and np.isclose(ent[0], 1.75 * math.log(2))
    assert ids[0].tolist() == [0, 1, 2] and np.allclose(tlp[0], np.log([0.5, 0.25, 0.125]))
    hot = oracle.token_logprobs(x, [0], scale=1e3)
    assert np.isclose(hot[0][0], 0) and np.isclose(hot[2][0], 0)


def test_logprobs_of_masked_and_broken_rows():
    inf, nan = np.inf, np.nan
    x = np.array([[0.0, -inf, 0.0], [-inf, -inf, -inf], [1.0, nan, 2.0], [inf, 0.0, inf]])
    lp, rank, ent, ids, _ = oracle.token_logprobs(x, [1, 0, 2, 5], n_top=2)
    assert lp[0] == -inf and rank[0] == 2 and np.isclose(ent[0], math.log(2)) and ids[0].tolist() == [0, 2]
    assert np.isnan(lp[1]) and np.isnan(ent[1]) and ids[1].tolist() == [0, 1]
    assert np.isnan(lp[2]) and rank[2] == 1 and ids[2].tolist() == [1, 2]
    assert lp[3] == -inf and rank[3] == 3 and ids[3].tolist() == [0, 2]
