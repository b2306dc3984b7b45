"""dk_shared_attend against the fp64 oracle, element by element, with bounds made of the roundings a correct kernel makes.

Of an output o = sum p v (A = sum p |v|, p the exact weights):
  store      half a step of the type: 2^-8 |o| (bf16), 2^-24 |o| (fp32)
  weights    bf16 pools round each weight once to bf16 before the product with V: 2^-8 A
  scores     D + 8 roundings of 2^-24 of at most S = |scale| sum |q k|, a factor 1 +- 2 x that on every weight, numerator and denominator: 4 ds A
  sums       n + 32 additions of 2^-24, twice
  pieces     a row's pieces are scaled and added, some 40 of them: 2^-24 each way, 64 roundings
The log-sum-exp is off by ds + (n + 96) 2^-24 and its own rounding."""
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


def bounds(ref, dtype, n_keys, d):
    o, lse, mag, size = ref
    eps = 2.0 ** -24
    ds = (d + 8) * eps * size
    adds = (n_keys + 96) * eps
    weights = 2.0 ** -8 if dtype == "bf16" else 0.0
    tol = (2.0 ** -8 if dtype == "bf16" else eps) * np.abs(o) + mag * (weights + 4 * ds[..., None] + 2 * adds) * 1.01 + 1e-30
    return tol, ds + adds + 4 * eps * (np.abs(lse) + 1)


class Tree:
    """Sequences of a pool with the host copy of what they hold: `spec` lists (parent index or None, positions taken over, own tokens)."""

    def __init__(self, seed, hq, hkv, d, dtype, spec, granule=0, spare=0):
        self.rng = np.random.default_rng(seed)
        self.shape, self.dtype = (hq, hkv, d), dtype
        self.pool = DevicePool(len(spec) + spare, sum(own for _, _, own in spec) + 6000 + 600 * (len(spec) + spare), hq, hkv, d, dtype,
                               granule_cells=granule)
        self.slots, self.k, self.v = [], [], []
        for parent, taken, own in spec:
            self.slots.append(self.pool.acquire())
            self.k.append(np.zeros((0, hkv, d), np.float32) if parent is None else self.k[parent][:taken])
            self.v.append(np.zeros((0, hkv, d), np.float32) if parent is None else self.v[parent][:taken])
            if parent is not None:
                self.pool.alias(self.slots[parent], self.slots[-1], taken)
            self.grow(len(self.slots) - 1, own)

    def draw(self, n, heads):
        return wl.normal(self.rng, (n, heads, self.shape[2]), self.dtype)

    def grow(self, i, n, k=None, v=None):
        if n == 0:
            return
        k, v = (self.draw(n, self.shape[1]), self.draw(n, self.shape[1])) if k is None else (k, v)
        self.pool.append([self.slots[i]], [0, n], _dev(k, self.dtype), _dev(v, self.dtype))
        self.k[i], self.v[i] = np.concatenate([self.k[i], k]), np.concatenate([self.v[i], v])

    def batch(self, which, delta, staged, spoil=None):
        """Inputs of a call: entry b continues sequence which[b] by delta[b] tokens."""
        hq, hkv, d = self.shape
        self.cu = np.concatenate([[0], np.cumsum(delta)]).astype(np.int32)
        n = int(self.cu[-1])
        self.q = wl.normal(self.rng, (n, hq, d), self.dtype) * np.float32(2)
        self.kn, self.vn = self.draw(n, hkv), self.draw(n, hkv)
        if spoil is not None:
            spoil(self.kn, self.vn)
        self.which, self.delta, self.staged = which, delta, staged
        self.n_past = [len(self.k[i]) for i in which]
        self.call_slots = [self.slots[i] for i in which]
        if not staged:
            self.pool.append(self.call_slots, self.cu, _dev(self.kn, self.dtype), _dev(self.vn, self.dtype))
            for b, i in enumerate(which):
                r = slice(int(self.cu[b]), int(self.cu[b + 1]))
                self.k[i], self.v[i] = np.concatenate([self.k[i], self.kn[r]]), np.concatenate([self.v[i], self.vn[r]])

    def run(self, scale, lse=True, stream=None):
        new = (_dev(self.kn, self.dtype), _dev(self.vn, self.dtype)) if self.staged else (None, None)
        q = _dev(self.q, self.dtype)
        out = torch.full_like(q, NAN)
        sums = torch.full(q.shape[:2], NAN, dtype=torch.float32, device="cuda") if lse else None
        self.pool.shared_attend(self.call_slots, self.cu, q, scale, *new, out=out, lse=sums)
        torch.cuda.synchronize()
        return out.float().cpu().numpy(), sums.cpu().numpy() if lse else None

    def check(self, out, lse, scale, entries=None, rows=None):
        d = self.shape[2]
        for b in range(len(self.which)) if entries is None else entries:
            r = slice(int(self.cu[b]), int(self.cu[b + 1]))
            if r.start == r.stop:
                continue
            keys = np.concatenate([self.k[self.which[b]][:self.n_past[b]], self.kn[r]])
            values = np.concatenate([self.v[self.which[b]][:self.n_past[b]], self.vn[r]])
            ref = oracle.scored_attend(self.q[r], keys, values, self.n_past[b], scale)
            tol, ltol = bounds(ref, self.dtype, len(keys), d)
            bad = ~(np.abs(out[r] - ref[0]) <= tol)
            assert not bad.any(), (b, np.argwhere(bad)[:4].tolist(), out[r][bad][:4], ref[0][bad][:4], tol[bad][:4])
            if lse is not None:
                lbad = ~(np.abs(lse[r] - ref[1]) <= ltol)
                assert not lbad.any(), (b, np.argwhere(lbad)[:4].tolist(), lse[r][lbad][:4], ref[1][lbad][:4])

    def run_and_check(self, which, delta, staged, scale=None, **kw):
        scale = self.shape[2] ** -0.5 if scale is None else scale
        self.batch(which, delta, staged)
        out, lse = self.run(scale, **kw)
        self.check(out, lse, scale)
        return out, lse


SHAPES = [(8, 2, 128, "bf16"), (8, 2, 64, "bf16"), (6, 2, 128, "bf16"), (7, 1, 64, "bf16"), (4, 4, 128, "bf16"), (16, 1, 128, "bf16"),
          (4, 1, 64, "f32"), (6, 2, 128, "f32")]
# two prompts, a longer one behind the first, sequences behind each, one that shares nothing, one that is empty
FOREST = [(None, 0, 333), (None, 0, 150), (0, 333, 200)] + [(0, 333, x) for x in (0, 1, 40, 130)] + [(1, 150, x) for x in (7, 300)] + \
         [(2, 533, x) for x in (0, 3, 64, 65, 90)] + [(None, 0, 77), (None, 0, 0), (2, 400, 20)]


@pytest.mark.parametrize("staged", [False, True], ids=["appended", "staged"])
@pytest.mark.parametrize("hq,hkv,d,dtype", SHAPES)
def test_forests_of_prefixes(hq, hkv, d, dtype, staged):
    t = Tree(3, hq, hkv, d, dtype, FOREST, granule=48)
    which = [13, 4, 9, 16, 3, 7, 15, 5, 12, 8, 10, 14, 6, 11]
    delta = [1, 9, 3, 2, 1, 70, 5, 0, 1, 1, 20, 33, 2, 1]
    t.run_and_check(which, delta, staged)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 128, "bf16"), (8, 2, 64, "bf16"), (6, 2, 128, "bf16"), (8, 2, 128, "f32")])
@pytest.mark.parametrize("members,prefix,delta", [(5, 3000, 1), (40, 700, 1), (33, 1500, 2), (12, 2500, 9), (3, 640, 100)])
def test_one_prefix_of_many(hq, hkv, d, dtype, members, prefix, delta):
    t = Tree(4, hq, hkv, d, dtype, [(None, 0, prefix)] + [(0, prefix, 5 * i) for i in range(members)], granule=64)
    t.run_and_check(list(range(1, members + 1)), [delta] * members, False)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64)])
def test_the_donor_is_of_the_batch(dtype, d):
    t = Tree(5, 4, 2, d, dtype, [(None, 0, 900), (0, 900, 0), (0, 500, 30), (0, 0, 12)], granule=32)
    t.run_and_check([0, 1, 2, 3], [2, 3, 1, 4], False)
    t.run_and_check([3, 2, 1, 0], [1, 1, 1, 1], True)


@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_any_finite_scale(scale, dtype):
    t = Tree(6, 4, 2, 64, dtype, [(None, 0, 400), (0, 400, 10), (0, 400, 0), (0, 400, 200)])
    t.run_and_check([1, 2, 3], [2, 1, 40], False, scale=scale)


@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 128, "bf16"), (14, 2, 64, "bf16"), (4, 1, 64, "f32")])
def test_single_tokens_long_caches_and_turns_in_one_batch(hq, hkv, d, dtype):
    t = Tree(7, hq, hkv, d, dtype, [(None, 0, 6000), (None, 0, 4500)] + [(0, 6000, 10), (0, 6000, 2000), (0, 5999, 0), (1, 1, 3)])
    t.run_and_check([1, 2, 3, 4, 5], [1, 1, 200, 130, 1], False)


def test_one_token_of_one_sequence_and_none_of_any():
    for dtype in ("bf16", "f32"):
        t = Tree(8, 4, 2, 128, dtype, [(None, 0, 0), (None, 0, 1)])
        t.run_and_check([0], [1], True)
        t.run_and_check([1], [1], False)
        t.run_and_check([0, 1], [1, 2], True)
        empty = torch.empty((0, 4, 128), dtype=t.pool.torch_dtype, device="cuda")
        t.pool.shared_attend(t.slots, [0, 0, 0], empty, 1.0)
        t.pool.shared_attend([], [0], empty, 1.0)


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128)])
@pytest.mark.parametrize("delta", [[2, 3, 1], [40, 20, 60]], ids=["few", "many"])
@pytest.mark.parametrize("value", [NAN, INF, -INF], ids=["nan", "inf", "-inf"])
def test_what_later_tokens_hold_does_not_matter(dtype, d, delta, value):
    """The last new token of every sequence is spoiled.  The rows before it: log-sum-exps, which V has no part in, as without, to the bit;
    sums that met 0 * infinity are made anew, their weights rounded against the row's final maximum and not a running one and added in
    another order, so they are held to the same bounds against the oracle as clean rows are, not to the clean rows' bits."""
    got = []
    for spoiled in (False, True):
        t = Tree(9, 4, 2, d, dtype, [(None, 0, 200), (0, 200, 5), (0, 200, 30), (0, 200, 0)], granule=16)
        cu = np.concatenate([[0], np.cumsum(delta)])
        def spoil(k, v):
            if spoiled:
                k[cu[1:] - 1] = value
                v[cu[1:] - 1] = value
        t.batch([1, 2, 3], delta, True, spoil)
        got.append(t.run(0.1))
    for b in range(3):
        if delta[b] == 1:
            continue
        r = slice(int(cu[b]), int(cu[b + 1]) - 1)
        assert np.array_equal(got[0][1][r], got[1][1][r])
        keys, values = (np.concatenate([x[b + 1], y[r]]) for x, y in ((t.k, t.kn), (t.v, t.vn)))
        ref = oracle.scored_attend(t.q[r], keys, values, len(t.k[b + 1]), 0.1)
        tol, _ = bounds(ref, dtype, len(keys), d)
        for out, _ in got:
            assert (np.abs(out[r] - ref[0]) <= tol).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64)])
@pytest.mark.parametrize("members", [3, 20])
def test_infinities_of_a_shared_prefix(dtype, d, members):
    """V of the prefix holds an infinity and a NaN: every row says so at that depth, the other depths are as without."""
    rng = np.random.default_rng(10)
    k, v = wl.normal(rng, (700, 2, d), dtype), wl.normal(rng, (700, 2, d), dtype)
    bad = v.copy()
    bad[300, 0, 5], bad[650, 1, 9], bad[10, 1, 33], bad[690, 1, 33] = INF, NAN, INF, -INF
    t = Tree(11, 8, 2, d, dtype, [(None, 0, 0)], spare=members)
    t.grow(0, 700, k, bad)
    for i in range(members):
        t.slots.append(t.pool.acquire())
        t.pool.alias(t.slots[0], t.slots[-1], 700)
        t.k.append(k)
        t.v.append(v)
        t.grow(i + 1, 3 * i)
    t.batch(list(range(1, members + 1)), [2] * members, False)
    out = t.run(0.2)[0]
    assert np.isposinf(out[:, :4, 5]).all() and np.isnan(out[:, 4:, [9, 33]]).all()
    # the other depths are those of the clean values
    for b in range(members):
        r = slice(2 * b, 2 * b + 2)
        keys, values = t.k[b + 1], t.v[b + 1]  # (the new tokens among them)
        ref = oracle.scored_attend(t.q[r], keys, values, t.n_past[b], 0.2)
        tol, _ = bounds(ref, dtype, len(keys), d)
        fine = np.abs(out[r] - ref[0]) <= tol
        fine[:, :4, 5] = fine[:, 4:, [9, 33]] = True
        assert fine.all(), (b, np.argwhere(~fine)[:4])


@pytest.mark.parametrize("members", [4, 90], ids=["in the arguments", "carried"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_captured_and_replayed(members, dtype):
    """Two graphs that share a workspace, replayed several times beside eager work: every replay is the eager result."""
    t = Tree(12, 4, 2, 64, dtype, [(None, 0, 1000)] + [(0, 1000, i % 7) for i in range(members)])
    need = 0
    calls = []
    for lo in (0, members // 2):
        which = list(range(1 + lo, members + 1))
        t.batch(which, [1] * len(which), True)
        calls.append((t.call_slots, t.cu, _dev(t.q, dtype), _dev(t.kn, dtype), _dev(t.vn, dtype)))
        need = max(need, dk.shared_workspace_bytes(t.pool.handle, t.call_slots, t.cu, True))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    outs = [torch.full_like(c[2], NAN) for c in calls]
    want = []
    for c, out in zip(calls, outs):
        dk.shared_attend(t.pool.handle, c[0], c[1], c[2], out, 0.125, c[3], c[4], workspace=ws)
        torch.cuda.synchronize()
        want.append(out.clone())
    graphs = []
    for c, out in zip(calls, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            dk.shared_attend(t.pool.handle, c[0], c[1], c[2], out, 0.125, c[3], c[4], workspace=ws)
        graphs.append(g)
    for turn in range(4):
        for i in (0, 1, 0) if turn % 2 else (1, 0):
            outs[i].fill_(NAN)
            graphs[i].replay()
            if turn == 2:
                torch.cuda.synchronize()
            c = calls[1 - i]
            eager = torch.empty_like(c[2])
            dk.shared_attend(t.pool.handle, c[0], c[1], c[2], eager, 0.125, c[3], c[4], workspace=ws)
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want[i]) and torch.equal(eager, want[1 - i])


def test_another_stream_and_its_own_results_again():
    t = Tree(13, 8, 2, 128, "bf16", [(None, 0, 2000)] + [(0, 2000, 9 * i) for i in range(6)])
    t.batch(list(range(1, 7)), [3] * 6, False)
    first, lse = t.run(0.09)
    s = torch.cuda.Stream()
    q = _dev(t.q, "bf16")
    outs = [torch.empty_like(q) for _ in range(3)]
    s.wait_stream(torch.cuda.current_stream())
    for out in outs:
        dk.shared_attend(t.pool.handle, t.call_slots, t.cu, q, out, 0.09, workspace=t.pool.workspace, stream=s)
    s.synchronize()
    for out in outs:
        assert np.array_equal(out.float().cpu().numpy(), first)
    t.check(first, lse, 0.09)


def test_what_was_planned():
    t = Tree(14, 8, 2, 128, "bf16", [(None, 0, 2000)] + [(0, 2000, 10) for i in range(20)])
    t.run_and_check(list(range(1, 21)), [1] * 20, False, lse=False)
    plan = dk.last_plan(t.pool.handle)
    assert plan["route"] == "shared" and plan["merges"] == 20 and plan["row_items"] > 0 and plan["stream_items"] >= 20
