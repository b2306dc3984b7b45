"""dk_scored_attend against the fp64 oracle, element by element, with bounds made of the roundings a correct kernel makes.

Of an output o = sum p v (A = sum p |v| the same over |v|, p the exact weights):
  store      half a step of the type: 2^-8 |o| (bf16), 2^-24 |o| (fp32)
  weights    bf16 pools may round each weight once to bf16 before the product with V: 2^-8 A
  scores     D + 8 roundings of 2^-24 of at most S = |scale| sum |q k|; the cap's tanh 2^-21 of the cap; the bias two roundings
             of slope * distance; a factor 1 +- 2 x that on every weight, numerator and denominator: 4 ds A
  sums       n + 32 additions of 2^-24, twice
The log-sum-exp is off by ds + (n + 32) 2^-24 and its own rounding."""
import numpy as np
import pytest
import torch

import oracle
from paper_2605_26289_amd import DevicePool
from paper_2605_26289_amd import binding as dk
from paper_2605_26289_amd import workloads as wl

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def _dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to("cuda", torch.bfloat16 if dtype == "bf16" else torch.float32)


def _bounds(ref, dtype, n_keys, d, cap, slope_reach):
    o, lse, mag, size = ref
    eps = 2.0 ** -24
    ds = (d + 8) * eps * size + 2.0 ** -21 * cap + 4 * eps * slope_reach
    adds = (n_keys + 32) * eps
    weights = 2.0 ** -8 if dtype == "bf16" else 0.0
    tol = (2.0 ** -8 if dtype == "bf16" else eps) * np.abs(o) + mag * (weights + 4 * ds[..., None] + 2 * adds) * 1.01 + 1e-30
    finite = np.where(np.isfinite(lse), lse, 0.0)
    return tol, ds + adds + 4 * eps * (np.abs(finite) + 1)


class Batch:
    """Sessions of a pool with the host copy of what they hold."""

    def __init__(self, seed, hq, hkv, d, dtype, hist, delta, granule=0, share=0, spoil=False):
        self.rng = np.random.default_rng(seed)
        self.shape, self.dtype, self.hist, self.delta = (hq, hkv, d), dtype, hist, delta
        self.pool = DevicePool(len(hist), sum(hist) + sum(delta) + 600 * (len(hist) + 2) + share, hq, hkv, d, dtype, granule_cells=granule)
        self.slots = [self.pool.acquire() for _ in hist]
        self.cu = np.concatenate([[0], np.cumsum(delta)]).astype(np.int32)
        draw = lambda n, h: wl.normal(self.rng, (n, h, d), dtype)  # noqa: E731
        self.q = wl.normal(self.rng, (sum(delta), hq, d), dtype) * np.float32(2)
        self.k, self.v = [], []
        pk, pv = draw(share, hkv), draw(share, hkv)
        for b, s in enumerate(self.slots):
            if share and b:
                self.pool.alias(self.slots[0], s, share)
            elif share:
                self.pool.append([s], [0, share], _dev(pk, dtype), _dev(pv, dtype))
        for b, (n, new) in enumerate(zip(hist, delta)):
            k, v = draw(n + new, hkv), draw(n + new, hkv)
            if n:
                self.pool.append([self.slots[b]], [0, n], _dev(k[:n], dtype), _dev(v[:n], dtype))
            self.k.append(np.concatenate([pk, k]))
            self.v.append(np.concatenate([pv, v]))
        self.share = share

    def new(self, rows):
        x = [r[self.share + n:] for r, n in zip(rows, self.hist)]
        return _dev(np.concatenate(x), self.dtype)

    def run(self, scores, staged, scale, lse=True):
        kn, vn = self.new(self.k), self.new(self.v)
        if not staged:
            self.pool.append(self.slots, self.cu, kn, vn)
        q = _dev(self.q, self.dtype)
        out = torch.full_like(q, NAN)
        l = torch.full(q.shape[:2], NAN, dtype=torch.float32, device="cuda") if lse else None
        self.pool.scored_attend(self.slots, self.cu, q, scale, scores, kn if staged else None, vn if staged else None, out=out, lse=l)
        torch.cuda.synchronize()
        return out.float().cpu().numpy(), l.cpu().numpy() if lse else None

    def check(self, staged=False, scale=None, cap=0.0, slopes=None, window=0, prefix=None, first=None):
        hq, hkv, d = self.shape
        scale = d ** -0.5 if scale is None else scale
        sl = None if slopes is None else torch.tensor(slopes, dtype=torch.float32, device="cuda")
        out, lse = self.run(dk.Scores(cap=cap, slopes=sl, window=window, prefix=prefix, first=first), staged, scale)
        for b, (n, new) in enumerate(zip(self.hist, self.delta)):
            r = slice(int(self.cu[b]), int(self.cu[b + 1]))
            ref = oracle.scored_attend(self.q[r], self.k[b], self.v[b], self.share + n, scale, cap,
                                       None if slopes is None else np.float32(slopes), window, 0 if prefix is None else prefix[b],
                                       None if first is None else first[r])
            reach = 0.0 if slopes is None else max(slopes) * (self.share + n + new)
            tol, ltol = _bounds(ref, self.dtype, self.share + n + new, d, cap, reach)
            got, want = out[r], ref[0]
            bad = ~(np.abs(got - want) <= tol)
            assert not bad.any(), (b, np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4], tol[bad][:4])
            empty = np.isneginf(ref[1])
            assert np.array_equal(np.isneginf(lse[r]), empty) and (got[empty] == 0).all()
            lbad = ~empty & ~(np.abs(lse[r] - np.where(empty, 0, ref[1])) <= ltol)
            assert not lbad.any(), (b, np.argwhere(lbad)[:4].tolist(), lse[r][lbad][:4], ref[1][lbad][:4])
        return out


SHAPES = [(8, 2, 128, "bf16"), (8, 2, 64, "bf16"), (6, 2, 128, "bf16"), (7, 1, 64, "bf16"), (4, 4, 128, "bf16"), (4, 1, 64, "f32"),
          (6, 2, 128, "f32")]
SLOPES = [0.5, 0.25, 2.0, 0.0, 0.01, 1.0, 0.125, 0.03]
MASKS = {
    "none": {}, "cap": dict(cap=5.0), "slopes": dict(slopes=True), "window": dict(window=33),
    "prefix": dict(prefix=True), "first": dict(first=True),
    "all": dict(cap=20.0, slopes=True, window=70, prefix=True, first=True),
}


def _masks(batch, spec):
    """The masks of a kind for a batch: prefixes of every sort, documents, rows that see nothing."""
    m = dict(spec)
    rng = np.random.default_rng(77)
    if m.get("slopes"):
        m["slopes"] = (SLOPES * 2)[:batch.shape[0]]
    if m.get("prefix"):
        m["prefix"] = [[0, batch.share + n + new, batch.share + n + 1, 10 ** 9, n // 2][b % 5] for b, (n, new) in enumerate(zip(batch.hist, batch.delta))]
    if m.get("first"):
        f = []
        for n, new in zip(batch.hist, batch.delta):
            p = batch.share + n + np.arange(new)
            starts = np.sort(rng.integers(0, batch.share + n + new, size=4))
            mine = np.array([max([0] + [s for s in starts if s <= x]) for x in p])
            mine[rng.random(new) < 0.15] = 2 ** 40  # padding
            f += mine.tolist()
        m["first"] = f
    return m


@pytest.mark.parametrize("staged", [False, True], ids=["appended", "staged"])
@pytest.mark.parametrize("kind", list(MASKS))
@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_batches_of_all_lengths(hq, hkv, d, dtype, kind, staged):
    b = Batch(3, hq, hkv, d, dtype, hist=[0, 1, 130, 63, 400, 17], delta=[3, 1, 70, 0, 1, 9], granule=48)
    b.check(staged, **_masks(b, MASKS[kind]))


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 128, "bf16"), (6, 2, 64, "bf16"), (8, 2, 128, "f32")])
@pytest.mark.parametrize("kind", ["cap", "all"])
def test_long_turns_through_an_alias(hq, hkv, d, dtype, kind):
    b = Batch(4, hq, hkv, d, dtype, hist=[200, 5, 77], delta=[150, 90, 40], granule=32, share=301)
    b.check(False, **_masks(b, MASKS[kind]))


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 128, "bf16"), (8, 2, 64, "bf16"), (4, 1, 64, "f32")])
@pytest.mark.parametrize("masks", [dict(cap=30.0), dict(cap=30.0, window=500), dict(slopes=SLOPES[:4])], ids=["cap", "window", "slopes"])
def test_single_tokens_over_long_caches(hq, hkv, d, dtype, masks):
    if "slopes" in masks:
        masks = dict(slopes=SLOPES[:hq])
    b = Batch(5, hq, hkv, d, dtype, hist=[5000, 12, 2047], delta=[1, 1, 2])
    b.check(False, **masks)


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_any_finite_scale(scale, dtype):
    b = Batch(6, 4, 2, 64, dtype, hist=[90, 300], delta=[5, 40])
    b.check(False, scale=scale, cap=10.0)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_windows_of_one_and_of_everything(dtype, d):
    b = Batch(7, 4, 2, d, dtype, hist=[40, 700], delta=[8, 100])
    out = b.check(False, window=1)
    for i, (n, new) in enumerate(zip(b.hist, b.delta)):
        r = slice(int(b.cu[i]), int(b.cu[i + 1]))
        own = np.repeat(b.v[i][n:], 2, axis=1)  # only itself: its V
        # The weight is 2^d, where d, the score less itself, may keep what rounding the score took off (a fused multiply-add does):
        # (2^d v) (1 / 2^d) takes three roundings of 2^-24, far below half a step of bf16, where V comes back to the bit.
        assert np.array_equal(out[r], own) if dtype == "bf16" else (np.abs(out[r] - own) <= 3.01 * 2.0 ** -24 * np.abs(own)).all()
    b = Batch(7, 4, 2, d, dtype, hist=[40, 700], delta=[8, 100])
    b.check(True, window=2 ** 31 - 1)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("delta", [[2, 1], [30, 60]], ids=["few", "many"])
@pytest.mark.parametrize("value", [NAN, INF, -INF], ids=["nan", "inf", "-inf"])
def test_what_hidden_positions_hold_does_not_matter(dtype, d, delta, value):
    """Spoiled K and V outside of what the rows see, at tile-internal places: the results are those of clean rows, to the bit."""
    clean, spoilt = [Batch(8, 4, 2, d, dtype, hist=[100, 333], delta=delta) for _ in range(2)]
    first = []
    for i, (n, new) in enumerate(zip(spoilt.hist, delta)):
        lo = n - 19
        first += [lo] * new
        for x in (spoilt.k[i], spoilt.v[i]):
            x[:lo] = value
        spoilt.pool.trim(spoilt.slots[i], 0)
        spoilt.pool.append([spoilt.slots[i]], [0, n], _dev(spoilt.k[i][:n], dtype), _dev(spoilt.v[i][:n], dtype))
    scores = dict(cap=7.0, first=first)
    got, want = (b.run(dk.Scores(**scores), True, 0.2) for b in (spoilt, clean))
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("n,delta", [(150, 70), (600, 2)])
def test_infinities_that_some_rows_see(dtype, d, n, delta):
    """One infinity and one NaN of V: rows that see them say so at that depth, the others and the other depths are as without."""
    b = Batch(9, 4, 2, d, dtype, hist=[n], delta=[delta])
    clean = b.v[0].copy()
    at_inf, at_nan = n - 3, n + delta - 1  # the last new token's V is seen by itself alone
    b.v[0][at_inf, 0, 5] = INF
    b.v[0][at_nan, 1, 9] = NAN
    b.pool.trim(b.slots[0], 0)
    b.pool.append([b.slots[0]], [0, n], _dev(b.k[0][:n], dtype), _dev(b.v[0][:n], dtype))
    first = [n - 10 if i % 2 else n - 2 for i in range(delta)]
    out, _ = b.run(dk.Scores(cap=9.0, first=first), True, 0.2)
    ref = oracle.scored_attend(b.q, b.k[0], clean, n, 0.2, 9.0, first=first)
    tol, _ = _bounds(ref, dtype, n + delta, d, 9.0, 0.0)
    for i in range(delta):
        want = ref[0][i].copy()
        for h in range(4):
            if h < 2 and first[i] <= at_inf:
                want[h, 5] = INF
            if h >= 2 and i == delta - 1:
                want[h, 9] = NAN
        with np.errstate(invalid="ignore"):
            ok = (out[i] == want) | (np.isnan(out[i]) & np.isnan(want)) | (np.isfinite(want) & (np.abs(out[i] - want) <= tol[i]))
        assert ok.all(), (i, np.argwhere(~ok)[:4], out[i][~ok][:4], want[~ok][:4])


@pytest.mark.parametrize("staged", [False, True], ids=["appended", "staged"])
@pytest.mark.parametrize("kind", list(MASKS))
@pytest.mark.parametrize("most", [4, 9], ids=["one_block", "two_blocks"])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 2, 64), (14, 2, 128)])
def test_batches_of_few_rows(hq, hkv, d, most, kind, staged):
    b = Batch(13, hq, hkv, d, "bf16", hist=[0, 1, 130, 63, 1400, 17], delta=[3, 1, most, 0, 1, 4], granule=48, share=70)
    b.check(staged, **_masks(b, MASKS[kind]))


# 66 thousand cells of 4 KiB, read past the caches; in the last batch by a launch of their own beside a prefill chunk's
@pytest.mark.parametrize("hist,delta,masks", [([33000, 33000], [1, 9], dict(cap=5.0)), ([33000, 33000], [40, 3], dict(window=32990)),
                                              ([33000, 40, 33000], [5, 90, 3], dict(cap=5.0))], ids=["few", "two_blocks", "chunk"])
def test_batches_that_no_cache_holds(hist, delta, masks):
    Batch(12, 8, 8, 128, "bf16", hist=hist, delta=delta).check(**masks)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("kind", ["cap", "all", "first"])
def test_many_rows_in_fp32(d, kind):
    b = Batch(18, 16, 4, d, "f32", hist=[60, 200], delta=[330, 320])  # 328 items of 32 rows
    b.check(True, **_masks(b, MASKS[kind]))


# beside a prefill chunk, short entries are in its launch; more row tiles than run at a time are cut once more
def test_short_entries_beside_chunks():
    Batch(14, 32, 1, 64, "bf16", hist=[300, 5, 2000, 0, 900], delta=[40, 1, 2, 270, 1]).check(cap=20.0, window=700)
    Batch(15, 8, 8, 128, "bf16", hist=[500, 700, 900, 600], delta=[700, 900, 1, 800]).check(cap=20.0)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 2, 64), (3, 3, 128)])
def test_few_rows_over_long_caches_are_merged_again_and_again(hq, hkv, d):
    """Split rows, some without a visible key, merged by the last workgroup of their splits: every call, with others in between."""
    b = Batch(16, hq, hkv, d, "bf16", hist=[5000, 900, 3], delta=[2, 1, 1])
    first = [0, 2 ** 40, 600, 0]
    want = b.check(cap=20.0, first=first)
    s = dk.Scores(cap=20.0, first=first)
    q, ones = _dev(b.q, "bf16"), [slice(0, 2), slice(2, 3), slice(3, 4)]
    for i in range(6):
        for j, r in enumerate(ones):  # alone each is cut more finely: as exact, not the same bits
            got = b.pool.scored_attend([b.slots[j]], [0, r.stop - r.start], q[r], d ** -0.5, dk.Scores(cap=20.0, first=first[r]))
            assert np.allclose(got.float().cpu().numpy(), want[r], rtol=2.0 ** -6, atol=2.0 ** -6)
        again = b.pool.scored_attend(b.slots, b.cu, q, d ** -0.5, s)
        assert np.array_equal(again.float().cpu().numpy(), want), i


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
def test_infinities_in_a_long_cache(dtype, d):
    """One infinity and one NaN of V in different pieces of a long cache that a single token sees."""
    n = 3000
    b = Batch(17, 4, 2, d, dtype, hist=[n], delta=[1])
    clean = b.v[0].copy()
    b.v[0][200, 0, 5], b.v[0][2500, 1, 9] = -INF, NAN
    b.pool.trim(b.slots[0], 0)
    b.pool.append([b.slots[0]], [0, n], _dev(b.k[0][:n], dtype), _dev(b.v[0][:n], dtype))
    out, _ = b.run(dk.Scores(cap=9.0), False, 0.2)
    ref = oracle.scored_attend(b.q, b.k[0], clean, n, 0.2, 9.0)
    tol, _ = _bounds(ref, dtype, n + 1, d, 9.0, 0.0)
    want = ref[0].copy()
    want[:, :2, 5], want[:, 2:, 9] = -INF, NAN
    with np.errstate(invalid="ignore"):
        ok = (out == want) | (np.isnan(out) & np.isnan(want)) | (np.isfinite(want) & (np.abs(out - want) <= tol))
    assert ok.all(), (np.argwhere(~ok)[:4], out[~ok][:4], want[~ok][:4])


def test_without_changes_it_agrees_with_delta_attend():
    b = Batch(10, 8, 2, 128, "bf16", hist=[500, 30], delta=[40, 3])
    got, lse = b.run(dk.Scores(), False, 0.1)
    q, l = _dev(b.q, "bf16"), torch.empty((43, 8), dtype=torch.float32, device="cuda")
    want = b.pool.attend(b.slots, b.cu, q, 0.1, lse=l).float().cpu().numpy()
    # each rounds its weights and its result once: twice two half steps, and the weights' sums are near the result's size
    assert np.allclose(got, want, rtol=2.0 ** -6, atol=2.0 ** -6) and np.allclose(lse, l.cpu().numpy(), atol=1e-4)


def test_the_same_call_twice_gives_the_same_bits_and_needs_no_lse():
    b = Batch(11, 8, 2, 128, "bf16", hist=[3000, 700, 64], delta=[1, 33, 5])
    s = dk.Scores(cap=25.0, window=900)
    one = b.run(s, False, 0.1)
    q = _dev(b.q, "bf16")
    for _ in range(3):
        again = b.pool.scored_attend(b.slots, b.cu, q, 0.1, s)
        assert np.array_equal(again.float().cpu().numpy(), one[0])


def test_cells_past_four_gigabytes():
    hq, hkv, d = 8, 4, 128
    cells = 5 * 2 ** 20  # 1.25 GiB of K a head: head 3's rows start past 2^32 bytes
    pool = DevicePool(2, cells, hq, hkv, d, "bf16", granule_cells=4096)
    filler, slot = pool.acquire(), pool.acquire()
    dk.kv_reserve(pool.handle, [filler], [0, cells - 8192])
    rng = np.random.default_rng(12)
    n, new = 3000, 5
    k, v = (wl.normal(rng, (n + new, hkv, d), "bf16") for _ in range(2))
    q = wl.normal(rng, (new, hq, d), "bf16")
    pool.append([slot], [0, n + new], _dev(k, "bf16"), _dev(v, "bf16"))
    assert dk.seq_cells(pool.handle, slot).min() > 4 * 2 ** 20
    out = pool.scored_attend([slot], [0, new], _dev(q, "bf16"), 0.1, dk.Scores(cap=30.0)).float().cpu().numpy()
    ref = oracle.scored_attend(q, k, v, n, 0.1, 30.0)
    tol, _ = _bounds(ref, "bf16", n + new, d, 30.0, 0.0)
    assert (np.abs(out - ref[0]) <= tol).all()


def test_captured_and_replayed_beside_other_work():
    b = Batch(13, 8, 2, 128, "bf16", hist=[1500, 40], delta=[1, 3])
    s = dk.Scores(cap=25.0)
    want, _ = b.run(s, False, 0.1)
    q = _dev(b.q, "bf16")
    out = torch.zeros_like(q)
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        b.pool.scored_attend(b.slots, b.cu, q, 0.1, s, out=out)
    for i in range(4):
        out.zero_()
        other = b.pool.scored_attend(b.slots, b.cu, q, 0.1, dk.Scores(window=7 + i))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(out.float().cpu().numpy(), want) and not torch.equal(out, other)


def test_two_graphs_share_a_workspace():
    b = Batch(19, 8, 2, 128, "bf16", hist=[4000, 2500], delta=[1, 12])
    calls = [(0, slice(0, 1), dk.Scores(cap=25.0)), (1, slice(1, 13), dk.Scores(window=2000))]
    kn, vn = b.new(b.k), b.new(b.v)
    b.pool.append(b.slots, b.cu, kn, vn)
    q = _dev(b.q, "bf16")
    graphs, outs, want = [], [], []
    for j, r, s in calls:  # (eager once: the workspace is as large as it gets)
        want.append(b.pool.scored_attend([b.slots[j]], [0, r.stop - r.start], q[r].clone(), 0.1, s))
    torch.cuda.synchronize()
    for j, r, s in calls:
        rows = q[r].clone()
        outs.append(torch.zeros_like(rows))
        graphs.append((torch.cuda.CUDAGraph(), rows))
        with torch.cuda.graph(graphs[-1][0], stream=torch.cuda.Stream()):
            b.pool.scored_attend([b.slots[j]], [0, r.stop - r.start], rows, 0.1, s, out=outs[-1])
    for order in ((0, 1), (1, 0), (0, 0, 1), (1, 1, 0)):
        for o in outs:
            o.zero_()
        for g in order:
            graphs[g][0].replay()
        eager = b.pool.scored_attend([b.slots[0]], [0, 1], q[:1].clone(), 0.1, calls[0][2])
        torch.cuda.synchronize()
        for got, ref in zip(outs + [eager], want + [want[0]]):  # merged by a launch or inside: the same sums in another order
            assert torch.allclose(got.float(), ref.float(), rtol=2.0 ** -7, atol=1e-6), order


def test_a_call_that_needs_an_upload_is_not_captured():
    hist = [20] * 100
    b = Batch(14, 4, 1, 64, "bf16", hist=hist, delta=[1] * 100)
    s = dk.Scores(cap=25.0)
    want, _ = b.run(s, False, 0.1)  # (the workspace is large enough from here on)
    q = _dev(b.q, "bf16")
    graph = torch.cuda.CUDAGraph()
    with pytest.raises(dk.DeltaKVError, match="UNSUPPORTED"):
        with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
            b.pool.scored_attend(b.slots, b.cu, q, 0.1, s)
    torch.cuda.synchronize()
    assert np.array_equal(b.pool.scored_attend(b.slots, b.cu, q, 0.1, s).float().cpu().numpy(), want)
