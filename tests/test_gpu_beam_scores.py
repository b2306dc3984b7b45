"""dk_beam_select where the beams' cumulative scores are far from zero, as those of long continuations are: results, and that a call takes
no longer for it.  Rows and tokens are compared always: the inputs' best continuations are checked to be apart."""
import numpy as np
import pytest
import torch

from test_gpu_beam import SUM_TOL
from paper_2605_26289_amd import binding as dk
from paper_2605_26289_amd import workloads as wl

pytestmark = pytest.mark.gpu

ROWS, VOCAB = 8, 128256


def logits_of(seed, dtype, rows=ROWS, vocab=VOCAB, spread=2.5):
    x = (np.random.default_rng(seed).standard_normal((rows, vocab), dtype=np.float32) * np.float32(spread))
    return torch.from_numpy(x).to(torch.bfloat16).float().numpy() if dtype == "bf16" else x


def best(x, scores, cu, n, scale=1.0):
    """The n best of every group, from all scores in 64 bits: by score, row, logit, token."""
    groups = len(cu) - 1
    rows, tokens, out = np.zeros((groups, n), np.int64), np.zeros((groups, n), np.int64), np.zeros((groups, n))
    for g in range(groups):
        y = scale * x[cu[g]:cu[g + 1]].astype(np.float64)
        top = y.max(1, keepdims=True)
        s = scores[cu[g]:cu[g + 1], None].astype(np.float64) + (y - top) - np.log(np.exp(y - top).sum(1, keepdims=True))
        some = np.argpartition(-s, 4 * n, axis=None)[:4 * n] if s.size > 4 * n else np.arange(s.size)
        r, t = np.unravel_index(some, s.shape)
        order = np.lexsort((t, -y[r, t], r, -s[r, t]))[:n]
        rows[g], tokens[g], out[g] = r[order] + cu[g], t[order], s[r, t][order]
    return rows, tokens, out


class Call:
    def __init__(self, x, cu, n, dtype, scale=1.0):
        rows, vocab = x.shape
        assert vocab % 8 == 0
        kind = torch.bfloat16 if dtype == "bf16" else torch.float32
        code = dk.BF16 if dtype == "bf16" else dk.F32
        self.logits = torch.from_numpy(x).to("cuda", kind)
        self.scores = torch.empty(rows, dtype=torch.float32, device="cuda")
        self.out = [torch.empty((len(cu) - 1, n), dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
        ws = torch.empty(dk.beam_workspace_bytes(rows, vocab, code, n), dtype=torch.uint8, device="cuda")
        cu_dev = torch.tensor(cu, dtype=torch.int32, device="cuda")
        self.run = lambda: dk.beam_select(len(cu) - 1, rows, cu_dev, self.logits, code, vocab, vocab, self.scores, n, *self.out, ws, scale=scale)

    def __call__(self, scores):
        self.scores.copy_(torch.from_numpy(scores))
        for o in self.out:
            o.fill_(-7)
        self.run()
        torch.cuda.synchronize()
        return [o.cpu().numpy() for o in self.out]

    def shortest_us(self, scores, times=15):
        self.scores.copy_(torch.from_numpy(scores))
        took = []
        for _ in range(times):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            self.run()
            b.record()
            b.synchronize()
            took.append(a.elapsed_time(b) * 1e3)
        return min(took)


def check(got, want, n):
    s = want[2]
    gaps = s[:, :-1] - s[:, 1:]
    assert ((gaps == 0) | (gaps > 2 * SUM_TOL)).all(), "inputs with continuations that are too close to tell apart"
    assert np.array_equal(got[0], want[0][:, :n]) and np.array_equal(got[1], want[1][:, :n])
    assert (np.abs(got[2] - s[:, :n]) <= SUM_TOL + 2.0 ** -24 * (np.abs(s[:, :n]) + 1)).all()


def spread_scores(seed, rows, offset):
    return (np.random.default_rng(seed).standard_normal(rows) * 2 + offset).astype(np.float32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [16, 64])
@pytest.mark.parametrize("offset", [-20.0, -300.0, -700.0, -40000.0, 5000.0])
def test_far_scores(dtype, n, offset):
    x, scores = logits_of(1, dtype), spread_scores(2, ROWS, offset)
    check(Call(x, [0, ROWS], n, dtype)(scores), best(x, scores, [0, ROWS], n + 1), n)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_scores_that_differ_by_much(dtype):
    """Rows hundreds apart, one group near zero and one far from it, a row that takes no part."""
    x = logits_of(3, dtype, 12, 40000)
    scores = spread_scores(4, 12, -3.0)
    scores[:4] += np.float32([-300, -700, 0, -4])
    scores[6:] += np.float32([-900, -901, -1500, -900.5, -903, -2000])
    scores[8] = -np.inf
    want = best(np.delete(x, 8, 0), np.delete(scores, 8), [0, 6, 11], 41)
    want[0][want[0] >= 8] += 1
    check(Call(x, [0, 6, 12], 40, dtype)(scores), want, 40)


@pytest.mark.parametrize("n", [16, 64])
def test_far_scores_take_no_longer(n):
    """The same logits behind scores near -20 and far below: the bound that continuations have to reach is as tight.

    (With a bound of as many bits of the score itself, a call on these took many times as long.)"""
    x = logits_of(1, "bf16")
    call = Call(x, [0, ROWS], n, "bf16")
    near, far = spread_scores(2, ROWS, -20.0), [spread_scores(2, ROWS, o) for o in (-300.0, -700.0, -5000.0)]
    call.shortest_us(near)
    us = call.shortest_us(near)
    for scores in far:
        took = call.shortest_us(scores)
        print(f"n {n}: {us:.1f} us near zero, {took:.1f} us at {scores.mean():.0f}", flush=True)
        assert took <= 2 * us


@pytest.mark.parametrize("scale", [0.700066, 0.695115, 0.70306, 0.709371])
def test_the_scale_is_rounded_once(scale):
    """A row whose sum shows little but how scale log2(e) was rounded.

    Every chunk of 4096 (256 lanes of 2 x 8) holds one 0 among the first wavefront's logits and 3072 of -8 among those of the other three: sums
    within a wavefront are whole numbers, S = 1 + 3072 w with w = 2^(-8 c), and c is all that is rounded in -8 c.  In steps of 2^-24: of w
    two (the exponential's last place) and 8 scale times the error of c, each by the share W = 3072 w / S; of the three sums of
    wavefronts one each, by the partial sum's size.  The chunks' sums are added in fp64.  (With scale and log2(e) rounded before their
    product ln S was 9.6 steps off and more, by arithmetic.)"""
    vocab = 32 * 4096
    x = np.full((32, 2, 256, 8), -8.0, np.float32)
    x[:, :, :64] = -np.inf
    x[:, 0, 0, 0] = 0.0
    x = x.reshape(1, vocab)
    exact = scale * 1.4426950408889634
    w = 3072 * np.exp(-8 * scale)
    steps = w / (1 + w) * (2 + 2.0 ** 24 * abs(float(np.float32(exact)) / exact - 1) * 8 * scale) + (3 + 2 * w) / (1 + w)
    ln_s = np.log(32 * (1 + w))
    score = np.float32(ln_s + 1 / 64)
    got = Call(x, [0, 1], 1, "bf16", scale)(np.float32([score]))
    assert got[0][0, 0] == 0 and got[1][0, 0] == 0
    assert abs(float(got[2][0, 0]) - (float(score) - ln_s)) <= 2.0 ** -24 * (steps + 0.1)  # (the result is 1/64: its own rounding is 2^-31)


def check_every_way(x, scores, cu, n, dtype, scale):
    """What holds however close scores are: every continuation is one, none twice, its score is right, those of a row are in the row's exact
    order (their differences have no part in the row's sum), rows are in order within the roundings, and nothing better is left out."""
    got = Call(x, cu, n, dtype, scale)(scores)
    for g in range(len(cu) - 1):
        rows = slice(cu[g], cu[g + 1])
        y = scale * x[rows].astype(np.float64)
        top = y.max(1, keepdims=True)
        with np.errstate(invalid="ignore"):
            s = scores[rows, None].astype(np.float64) + (y - top) - np.log(np.exp(y - top).sum(1, keepdims=True))
        s[~np.isfinite(scores[rows])] = -np.inf
        r, t, out = got[0][g] - cu[g], got[1][g], got[2][g]
        count = min(n, int(np.isfinite(s).sum()))
        assert (got[0][g][count:] == -1).all() and (t[count:] == -1).all() and np.isneginf(out[count:]).all()
        r, t, out = r[:count], t[:count], out[:count]
        assert (r >= 0).all() and (r < s.shape[0]).all() and (t >= 0).all() and (t < s.shape[1]).all()
        assert len(set(zip(r.tolist(), t.tolist()))) == count
        mine = s[r, t]
        assert (np.abs(out - mine) <= SUM_TOL + 2.0 ** -24 * (np.abs(mine) + 1)).all()
        assert (mine[:-1] - mine[1:] >= -2 * SUM_TOL).all()
        taken = np.zeros(s.shape, bool)
        taken[r, t] = True
        assert not (~taken & (s > mine[-1] + 2 * SUM_TOL)).any()
        for row in set(r.tolist()):
            of = t[r == row]
            order = np.lexsort((np.arange(s.shape[1]), -x[cu[g] + row].astype(np.float64)))[:len(of)]
            assert np.array_equal(of, order)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab", [504, 6552, 20000])
@pytest.mark.parametrize("lead,offset", [(None, -20.0), (18.0, -20.0), (None, -800.0), (18.0, -800.0), (0.0, -800.0)])
def test_first_steps_and_rows_that_lead(dtype, vocab, lead, offset):
    x, scores = logits_of(31, dtype, 60, vocab), spread_scores(32, 60, offset)
    if lead is None:
        scores[[i for i in range(60) if i not in (5, 28)]] = -np.inf
    else:
        scores[[5, 28]] += np.float32(lead)
    for n in (1, 8, 32, 64):
        check_every_way(x, scores, [0, 28, 60], n, dtype, 0.69)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [0.0, -700.0])
def test_more_lanes_reach_the_first_bound_than_there_is_room_for(dtype, offset):
    x = logits_of(33, dtype, 40, 60000)
    scores = (-20.0 - np.linspace(0, 1, 40)).astype(np.float32)
    scores[[7, 21]] = -14.5, -13.8
    for n in (5, 63, 64):
        check_every_way(x, scores + np.float32(offset), [0, 40], n, dtype, 1.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("offset", [-20.0, -700.0])
def test_masks_of_the_lowest_value_that_leave_fewer_than_n(dtype, offset):
    """Three tokens a row are allowed, the others hold the type's lowest value: continuations all the same, equal ones by the thousand."""
    lowest = float(torch.finfo(torch.bfloat16).min) if dtype == "bf16" else -3e38
    x = np.full((6, 9000), lowest, np.float32)
    x[:, [5, 700, 8999]] = logits_of(34, dtype, 6, 8)[:, :3]
    scores = spread_scores(35, 6, offset)
    for n in (12, 40):
        check_every_way(x, scores, [0, 4, 6], n, dtype, 1.0)
