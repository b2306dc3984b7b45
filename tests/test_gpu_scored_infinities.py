"""dk_scored_attend where visible keys or values are infinite.

A visible key whose product with a query is -infinity has the capped score -cap, like any other: the row's other keys and its
log-sum-exp are those of the definition.  An infinity of V that a row sees makes the row infinite at that depth, however small
its weight is and however the keys were cut.  Bounds as in test_gpu_scored: those of the same batch with finite keys, since the
score of an infinite product is off by the cap's own rounding alone."""
import numpy as np
import pytest
import torch

import oracle
from paper_2605_26289_amd import binding as dk
from test_gpu_scored import Batch, _bounds, _dev

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def _reload(b):
    """The pool's cells as the host copies are now."""
    for s, n, k, v in zip(b.slots, b.hist, b.k, b.v):
        b.pool.trim(s, 0)
        if n:
            b.pool.append([s], [0, n], _dev(k[:n], b.dtype), _dev(v[:n], b.dtype))


def _near(got, want, tol):
    with np.errstate(invalid="ignore"):
        return (got == want) | (np.isnan(got) & np.isnan(want)) | (np.isfinite(want) & (np.abs(got - want) <= tol))


KEYS = {  # first and last position (from the end of the cached tokens where negative) whose keys are infinite
    "all": (0, None), "early": (0, -40), "one": (-3, -2), "late": (-40, None),
}


@pytest.mark.parametrize("staged", [False, True], ids=["appended", "staged"])
@pytest.mark.parametrize("which", list(KEYS))
@pytest.mark.parametrize("hist,delta,window", [([200], [2], 0), ([200], [2], 1), ([3000], [1], 0), ([3000, 90], [4, 1], 700), ([150, 400], [70, 40], 0),
                                               ([150, 400], [70, 40], 5), ([3000], [90], 0)],
                         ids=["few", "itself", "long", "few_window", "many", "many_window", "many_long"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_visible_products_of_minus_infinity_are_capped(dtype, d, hist, delta, window, which, staged):
    cap, scale = 2.0, 0.2
    b = Batch(30, 4, 2, d, dtype, hist=hist, delta=delta)
    b.q[:, :, 0] = -1.0
    finite = [k.copy() for k in b.k]
    for n, k in zip(hist, b.k):
        first, last = KEYS[which]
        k[first if first >= 0 else n + first:None if last is None else n + last, :, 0] = INF
    _reload(b)
    out, lse = b.run(dk.Scores(cap=cap, window=window), staged, scale)
    for i, n in enumerate(hist):
        r = slice(int(b.cu[i]), int(b.cu[i + 1]))
        want = oracle.scored_attend(b.q[r], b.k[i], b.v[i], n, scale, cap, window=window)
        size = oracle.scored_attend(b.q[r], finite[i], b.v[i], n, scale, cap, window=window)[3]
        tol, ltol = _bounds((want[0], want[1], want[2], size), dtype, n + delta[i], d, cap, 0.0)
        assert np.isfinite(want[1]).all()
        assert (np.abs(out[r] - want[0]) <= tol).all(), (i, np.argwhere(~(np.abs(out[r] - want[0]) <= tol))[:4], out[r].ravel()[:4])
        assert (np.abs(lse[r] - want[1]) <= ltol).all(), (i, lse[r].ravel()[:4], want[1].ravel()[:4])


@pytest.mark.parametrize("value", [INF, -INF, NAN, "both"], ids=["inf", "-inf", "nan", "both"])
@pytest.mark.parametrize("n,delta", [(60, 2), (3000, 1), (3000, 9), (3000, 90)], ids=["whole", "inside", "merge", "many"])
@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_visible_infinities_of_v_whose_weight_vanishes(dtype, d, n, delta, value):
    """The first token's V, thousands of units of score below the last one's: in one piece of the keys and in many."""
    slopes = [4.0, 3.0, 5.0, 4.0]
    b = Batch(31, 4, 2, d, dtype, hist=[n], delta=[delta])
    clean = b.v[0].copy()
    b.v[0][0, 0, 5] = INF if value == "both" else value
    if value == "both":
        b.v[0][n // 2, 0, 5] = -INF  # (in another piece, where there are several)
    _reload(b)
    out, lse = b.run(dk.Scores(slopes=torch.tensor(slopes, device="cuda")), False, 0.2)
    want = oracle.scored_attend(b.q, b.k[0], clean, n, 0.2, slopes=np.float32(slopes))
    tol, ltol = _bounds(want, dtype, n + delta, d, 0.0, max(slopes) * (n + delta))
    expected = want[0].copy()
    expected[:, :2, 5] = NAN if value == "both" else value
    ok = _near(out, expected, tol)
    assert ok.all(), (np.argwhere(~ok)[:4], out[~ok][:4], expected[~ok][:4])
    assert (np.abs(lse - want[1]) <= ltol).all()
