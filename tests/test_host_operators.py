"""Refusals and host-side parts of scored attention, rotary positions and token log probabilities (no GPU).

Nothing here launches: every call is turned down before it would, or has no rows."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2605_26289_amd import binding as dk

FLT_MAX = float(np.finfo(np.float32).max)


def _pool(n_slots=4, arena_cells=4096, granule=16, hq=8, hkv=2, d=64, dtype=dk.BF16):
    return dk.pool_create(dk.PoolDesc(n_slots, 0, arena_cells, granule, hq, hkv, d, dtype, 256 * 10, 256 * 20, 256 * 30, 1 << 20))


def _i32(*values):
    return np.asarray(values, dtype=np.int32).tobytes()


def _attend(pool, scores, slots=(0,), cu=(0, 2), q=1 << 40, k=None, v=None, scale=1.0, out=2 << 40, ws=1 << 16, ws_bytes=1 << 20):
    return dk.lib().dk_scored_attend(pool, len(slots), _i32(*slots), _i32(*cu), q, k, v, scale, scores.address if scores else None,
                                     out, None, ws, ws_bytes, None)


@pytest.fixture
def pool():
    p = _pool()
    dk.seq_acquire(p)
    dk.kv_reserve(p, [0], [0, 10])
    yield p
    dk.pool_destroy(p)


@pytest.mark.parametrize("scores", [dict(cap=-1.0), dict(cap=float("nan")), dict(cap=float("inf")), dict(window=-1), dict(prefix=[-1]),
                                    dict(first=[0, -5])])
def test_scored_attend_refuses_bad_scores(pool, scores):
    s = dk.Scores(**scores)
    assert _attend(pool, s) == -1
    out = C.c_int64()
    assert dk.lib().dk_scored_workspace_bytes(pool, 1, _i32(0), _i32(0, 2), 0, s.address, C.byref(out)) == -1


@pytest.mark.parametrize("cap", [1e-4, 1025.0, FLT_MAX])
def test_scored_attend_refuses_caps_it_would_be_inexact_for(pool, cap):
    assert _attend(pool, dk.Scores(cap=cap)) == -6


def test_scored_attend_refuses_bad_calls(pool):
    s = dk.Scores(cap=30.0)
    assert _attend(pool, None) == -1
    assert _attend(None, s) == -1
    assert _attend(pool, s, scale=float("nan")) == -1 and _attend(pool, s, scale=float("inf")) == -1
    assert _attend(pool, s, k=4096) == -1  # K without V
    assert _attend(pool, s, cu=(0, 11)) == -1  # more new tokens than the slot has
    assert _attend(pool, s, cu=(1, 2)) == -1 and _attend(pool, s, cu=(0, -1)) == -1
    assert _attend(pool, s, slots=(1,)) == -4 and _attend(pool, s, slots=(0, 0), cu=(0, 1, 2)) == -5
    assert _attend(pool, s, q=None) == -1 and _attend(pool, s, out=None) == -1
    assert _attend(pool, s, q=4100) == -6 and _attend(pool, s, out=8200) == -6 and _attend(pool, s, k=4104, v=4096) == -6
    assert _attend(pool, s, ws=None) == -7 and _attend(pool, s, ws=(1 << 16) + 8) == -7
    need = dk.scored_workspace_bytes(pool, [0], [0, 2], False, s)
    assert need > 0 and _attend(pool, s, ws_bytes=need - 1) == -7
    assert dk.seq_len(pool, 0) == 10
    assert _attend(pool, s, cu=(0, 0), q=None, out=None, ws=None) == 0  # no rows


def test_scored_attend_refuses_an_output_over_its_inputs(pool):
    s, row = dk.Scores(cap=30.0), 8 * 64 * 2
    assert _attend(pool, s, out=1 << 40) == -1 and _attend(pool, s, out=(1 << 40) + 2 * row - 16) == -1
    new = dict(k=4 << 40, v=5 << 40)
    for at in new.values():
        assert _attend(pool, s, out=at, **new) == -1 and _attend(pool, s, out=at - 2 * row + 16, **new) == -1
    assert _attend(pool, s, out=(1 << 40) + 2 * row, ws=None) == -7  # next to them is fine


def test_scored_attend_without_staging_memory_refuses_what_needs_an_upload(pool):
    first = np.zeros(1500, dtype=np.int64)  # 6000 bytes of descriptors
    dk.kv_reserve(pool, [0], [0, 1500])
    s = dk.Scores(first=first)
    need = dk.scored_workspace_bytes(pool, [0], [0, 1500], False, s)
    assert _attend(pool, s, cu=(0, 1500), ws_bytes=need) == -7


def test_the_binding_checks_what_the_library_cannot_see(pool):
    class Rows:  # of a shape, never launched
        shape = (2, 8, 64)

        def data_ptr(self):
            return 4096

    for bad in (dict(prefix=[1, 2]), dict(first=[0]), dict(first=[0, 0, 0])):
        with pytest.raises(dk.DeltaKVError, match="INVALID"):
            dk.scored_attend(pool, [0], [0, 2], Rows(), Rows(), 1.0, dk.Scores(**bad))
        with pytest.raises(dk.DeltaKVError, match="INVALID"):
            dk.scored_workspace_bytes(pool, [0], [0, 2], False, dk.Scores(**bad))


class _Rotary:
    def __init__(self, **kw):
        base = dict(rotary_dim=64, pairs=0, inv_freq=256, amplitude=1.0, norm=0, eps=0.0, q_weight=None, k_weight=None)
        base.update(kw)
        self.desc = dk.RotaryDesc(*[base[f[0]] for f in dk.RotaryDesc._fields_])
        self.address = C.addressof(self.desc)


BAD_ROTARY = [(dict(rotary_dim=63), -1), (dict(rotary_dim=66), -1), (dict(rotary_dim=-2), -1), (dict(inv_freq=None), -1),
              (dict(amplitude=float("nan")), -1), (dict(amplitude=float("inf")), -1), (dict(norm=1, eps=-1.0), -1),
              (dict(norm=1, eps=float("nan")), -1), (dict(norm=1, q_weight=264), -6), (dict(norm=1, k_weight=258), -6)]


def _append(pool, rotary, slots=(0,), cu=(0, 2), q=1 << 40, qs=512, k=2 << 40, ks=128, v=3 << 40, vs=128, out=4 << 40):
    return dk.lib().dk_rotate_append(pool, len(slots), _i32(*slots), _i32(*cu), rotary.address if rotary else None, q, qs, k, ks,
                                     v, vs, out, None)


@pytest.mark.parametrize("bad,status", BAD_ROTARY)
def test_rotations_that_are_none(pool, bad, status):
    r = _Rotary(**bad)
    assert _append(pool, r) == status and dk.seq_len(pool, 0) == 10
    assert dk.lib().dk_rotate_rows(dk.BF16, 64, 2, 256, r.address, 8, 1 << 40, 512, 2 << 40, 0, None, 0, None, None) == status


def test_rotate_append_refuses_bad_calls(pool):
    r = _Rotary()
    assert _append(pool, None) == -1 and _append(None, r) == -1
    assert _append(pool, r, slots=(2,)) == -4 and _append(pool, r, slots=(0, 0), cu=(0, 1, 2)) == -5
    assert _append(pool, r, cu=(1, 2)) == -1
    for missing in ("q", "k", "v", "out"):
        assert _append(pool, r, **{missing: None}) == -1
    assert _append(pool, r, qs=511) == -1 and _append(pool, r, ks=120) == -1 and _append(pool, r, vs=127) == -1  # strides below a token
    assert _append(pool, r, qs=516) == -6 and _append(pool, r, ks=130) == -6  # strides not whole 16 bytes
    assert _append(pool, r, q=(1 << 40) + 8) == -6 and _append(pool, r, out=(4 << 40) + 4) == -6
    assert _append(pool, r, out=(1 << 40) + 512) == -1  # half over Q
    assert _append(pool, r, out=1 << 40, qs=768) == -1  # over a strided Q
    assert _append(pool, r, out=2 << 40) == -1 and _append(pool, r, out=(3 << 40) + 16) == -1  # over K, over V
    assert _append(pool, r, cu=(0, 1 << 20)) == -3  # no cells
    assert dk.seq_len(pool, 0) == 10
    assert _append(pool, r, cu=(0, 0), q=None, k=None, v=None, out=None) == 0


def test_rotate_append_in_pieces_of_cells_needs_staging_memory():
    """A token each of more sessions than the kernel arguments hold runs: nothing is appended."""
    p, rotary = _pool(n_slots=400, arena_cells=16384, granule=4), _Rotary()
    slots = [dk.seq_acquire(p) for _ in range(320)]
    held = dk.pool_stats(p)
    assert _append(p, rotary, slots=slots, cu=range(321)) == -7  # 320 runs of one token
    assert dk.pool_stats(p) == held and all(dk.seq_len(p, s) == 0 for s in slots)
    dk.pool_destroy(p)


def test_rotate_rows_refuses_bad_calls():
    rotary = _Rotary()

    def rows(dtype=dk.BF16, d=64, n=2, pos=256, hq=2, q=1 << 20, qs=128, qo=2 << 20, hk=1, k=3 << 20, ks=64, ko=4 << 20):
        return dk.lib().dk_rotate_rows(dtype, d, n, pos, rotary.address, hq, q, qs, qo, hk, k, ks, ko, None)

    assert rows(dtype=7) == -6 and rows(d=96) == -6 and rows(n=-1) == -1 and rows(hq=-1) == -1 and rows(pos=None) == -1
    assert rows(q=None) == -1 and rows(ko=None) == -1 and rows(qs=120) == -1 and rows(qs=132) == -6 and rows(k=(3 << 20) + 2) == -6
    assert rows(qo=(1 << 20) + 16) == -1 and rows(qo=3 << 20) == -1 and rows(ko=2 << 20) == -1 and rows(ko=1 << 20) == -1
    assert rows(qo=1 << 20, qs=256) == -1 and rows(n=1 << 31) == -6
    assert rows(n=0, pos=None, q=None) == 0 and rows(hq=0, hk=0, q=None, k=None) == 0


def test_the_binding_takes_rows_whose_tokens_are_contiguous():
    import torch
    rotary = dk.Rotary(0)
    x = torch.zeros((4, 2, 128))
    for bad in (x[:, :, ::2], x.transpose(0, 1), x[0]):
        with pytest.raises(dk.DeltaKVError, match="INVALID"):
            dk.rotate_rows(torch.zeros(4, dtype=torch.int64), bad, None, rotary, torch.zeros_like(x), None)
    with pytest.raises(dk.DeltaKVError, match="INVALID"):
        dk.Rotary(64, torch.zeros(31))
    with pytest.raises(dk.DeltaKVError, match="INVALID"):
        dk.Rotary(64, torch.zeros(32, dtype=torch.float64))


def test_frequencies():
    r, base = 64, 10000.0
    plain = base ** (-np.arange(r // 2) / (r // 2))
    got, amp = dk.rotary_freqs(r, base)
    assert np.array_equal(got, plain.astype(np.float32)) and amp == 1.0
    assert np.allclose(dk.rotary_freqs(r, base, dk.ROTARY_LINEAR, [4, 0, 0, 0])[0], plain / 4, rtol=1e-7)
    wide = dk.rotary_freqs(r, base, dk.ROTARY_BASE, [4, 0, 0, 0])[0]
    assert wide[0] == 1.0 and np.isclose(wide[-1], plain[-1] / 4, rtol=1e-6)  # the slowest pair is stretched by the factor
    # bands: a wavelength below 8192 / 4 stays, one above 8192 / 1 is stretched by 8, in between both by share
    bands = dk.rotary_freqs(128, 500000.0, dk.ROTARY_BANDS, [8, 1, 4, 8192])[0].astype(np.float64)
    f = 500000.0 ** (-np.arange(64) / 64)
    for got_f, was in zip(bands, f):
        wave = 2 * math.pi / was
        share = 1.0 if wave < 2048 else 0.0 if wave > 8192 else (8192 / wave - 1) / 3
        assert np.isclose(got_f, share * was + (1 - share) * was / 8, rtol=1e-6)
    assert (bands[:20] == f[:20].astype(np.float32)).all() and np.allclose(bands[-5:], f[-5:] / 8, rtol=1e-6)
    # ramp over the pairs between those that turn 32 times and once within 4096
    ramp, amp = dk.rotary_freqs(128, 10000.0, dk.ROTARY_RAMP, [16, 1, 32, 4096])
    f = 10000.0 ** (-np.arange(64) / 64)
    lo, hi = math.floor(64 * math.log(4096 / (32 * 2 * math.pi)) / math.log(10000)), math.ceil(64 * math.log(4096 / (2 * math.pi)) / math.log(10000))
    assert (lo, hi) == (20, 46)
    share = 1 - np.clip((np.arange(64) - lo) / (hi - lo), 0, 1)
    assert np.allclose(ramp, share * f + (1 - share) * f / 16, rtol=1e-6) and np.isclose(amp, 0.1 * math.log(16) + 1)
    assert len(dk.rotary_freqs(0, base)[0]) == 0


@pytest.mark.parametrize("args,status", [
    ((63, 10000.0), -1), ((-2, 10000.0), -1), ((64, 0.0), -1), ((64, float("inf")), -1), ((64, 10000.0, 9), -6), ((64, 10000.0, 1), -1),
    ((64, 10000.0, 1, [0, 0, 0, 0]), -1), ((2, 10000.0, 2, [4, 0, 0, 0]), -1), ((64, 10000.0, 3, [8, 4, 1, 8192]), -1),
    ((64, 10000.0, 3, [8, 4, 4, 8192]), -1), ((64, 10000.0, 4, [8, 0, 32, 8192]), -1), ((64, 10000.0, 4, [8, 1, 32, 0]), -1),
    ((64, 1.0, 4, [8, 1, 32, 8192]), -1)])
def test_frequencies_that_are_none(args, status):
    with pytest.raises(dk.DeltaKVError) as e:
        dk.rotary_freqs(*args)
    assert e.value.status == status


def test_token_logprobs_refuses_bad_calls():
    def call(rows=3, logits=4096, dtype=dk.BF16, vocab=1000, stride=1000, scale=1.0, tokens=512, lp=1024, rank=None, ent=None, n_top=0,
             ids=None, tlp=None, ws=1 << 16, ws_bytes=1 << 24):
        return dk.lib().dk_token_logprobs(rows, logits, dtype, vocab, stride, scale, tokens, lp, rank, ent, n_top, ids, tlp, ws, ws_bytes, None)

    assert call(rows=-1) == -1 and call(vocab=0) == -1 and call(vocab=1 << 31, stride=1 << 31) == -1 and call(stride=992) == -1
    assert call(dtype=5) == -6 and call(logits=4104) == -6 and call(stride=1004) == -6 and call(logits=None) == -1
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert call(scale=scale) == -1
    assert call(scale=1e-7) == -6 and call(scale=2e6) == -6
    assert call(rows=1 << 24, vocab=8, stride=8) == -6 and call(vocab=2 ** 24 + 1, stride=2 ** 31) == -6
    assert call(rows=1 << 23, vocab=4096, stride=4096) == -6
    assert call(tokens=None) == -1 and call(tokens=None, lp=None, rank=2048) == -1
    assert call(n_top=-1) == -1 and call(n_top=33, ids=2048) == -6 and call(n_top=5) == -1 and call(ids=2048) == -1 and call(tlp=2048) == -1
    assert call(vocab=4, stride=8, n_top=5, ids=2048) == -1  # more alternatives than tokens
    assert call(ws=None) == -7 and call(ws=(1 << 16) + 16) == -7
    need = dk.logprobs_workspace_bytes(3, 1000, dk.BF16, 20)
    assert call(n_top=20, ids=2048, ws_bytes=need - 1) == -7
    assert call(rows=0, logits=None, ws=None) == 0
    with pytest.raises(dk.DeltaKVError, match="UNSUPPORTED"):
        dk.logprobs_workspace_bytes(1, 1000, dk.BF16, 33)
