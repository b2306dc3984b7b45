"""Refusals and host-side parts of shared attention, reordering and beam selection (no GPU).

Nothing here launches: every call is turned down before it would, has no rows, or needs no copy."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

from paper_2605_26289_amd import binding as dk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FLT_MAX = float(np.finfo(np.float32).max)


def _pool(n_slots=6, arena_cells=4096, granule=16, hq=8, hkv=2, d=64, dtype=dk.BF16):
    return dk.pool_create(dk.PoolDesc(n_slots, 0, arena_cells, granule, hq, hkv, d, dtype, 256 * 10, 256 * 20, 256 * 30, 1 << 20))


def _i32(*values):
    return np.asarray(values, dtype=np.int32).tobytes()


def _attend(pool, slots=(0,), cu=(0, 2), q=1 << 40, k=None, v=None, scale=1.0, out=2 << 40, lse=None, ws=1 << 16, ws_bytes=1 << 20):
    return dk.lib().dk_shared_attend(pool, len(slots), _i32(*slots), _i32(*cu), q, k, v, scale, out, lse, ws, ws_bytes, None)


@pytest.fixture
def pool():
    p = _pool()
    dk.seq_acquire(p)
    dk.kv_reserve(p, [0], [0, 10])
    yield p
    dk.pool_destroy(p)


def test_shared_attend_refuses_bad_calls(pool):
    assert _attend(None) == -1
    assert _attend(pool, scale=float("nan")) == -1 and _attend(pool, scale=float("inf")) == -1
    assert _attend(pool, k=4096) == -1  # K without V
    assert _attend(pool, cu=(0, 11)) == -1  # more new tokens than the slot has
    assert _attend(pool, cu=(1, 2)) == -1 and _attend(pool, cu=(0, -1)) == -1
    assert _attend(pool, slots=(1,)) == -4 and _attend(pool, slots=(0, 0), cu=(0, 1, 2)) == -5
    assert _attend(pool, q=None) == -1 and _attend(pool, out=None) == -1
    assert _attend(pool, q=4100) == -6 and _attend(pool, out=8200) == -6 and _attend(pool, k=4104, v=4096) == -6
    assert _attend(pool, ws=None) == -7 and _attend(pool, ws=(1 << 16) + 8) == -7
    need = dk.shared_workspace_bytes(pool, [0], [0, 2], False)
    assert need > 0 and _attend(pool, ws_bytes=need - 1) == -7
    assert dk.seq_len(pool, 0) == 10
    assert _attend(pool, cu=(0, 0), q=None, out=None, ws=None) == 0  # no rows
    assert dk.lib().dk_shared_attend(pool, 0, None, None, None, None, None, 1.0, None, None, None, 0, None) == 0


def test_shared_attend_refuses_outputs_over_inputs_or_one_another(pool):
    row = 8 * 64 * 2
    assert _attend(pool, out=1 << 40) == -1 and _attend(pool, out=(1 << 40) + 2 * row - 16) == -1
    new = dict(k=4 << 40, v=5 << 40)
    for at in new.values():
        assert _attend(pool, out=at, **new) == -1 and _attend(pool, lse=at + 16, **new) == -1
    assert _attend(pool, lse=(2 << 40) + 16) == -1 and _attend(pool, lse=1 << 40) == -1
    assert _attend(pool, out=(1 << 40) + 2 * row, lse=(1 << 40) + 4 * row, ws=None) == -7  # next to them is fine


def test_shared_workspace_query(pool):
    out = C.c_int64()
    call = dk.lib().dk_shared_workspace_bytes
    assert call(None, 1, _i32(0), _i32(0, 2), 0, C.byref(out)) == -1 and call(pool, 1, _i32(0), _i32(0, 2), 0, None) == -1
    assert call(pool, 1, _i32(0), _i32(0, 2), 2, C.byref(out)) == -1 and call(pool, 1, _i32(3), _i32(0, 2), 0, C.byref(out)) == -4
    with pytest.raises(dk.DeltaKVError):
        dk.shared_workspace_bytes(pool, [0], [0], False)


def test_too_many_heads_or_rows_are_refused():
    p = _pool(hq=1 << 16, hkv=1 << 16, d=64)
    dk.seq_acquire(p)
    dk.kv_reserve(p, [0], [0, 4])
    assert _attend(p, ws_bytes=1 << 40) == -6  # a staged row would be found by more than 24 bits
    dk.pool_destroy(p)
    p = _pool(hq=1 << 12, hkv=1, d=64)
    dk.seq_acquire(p)
    dk.kv_reserve(p, [0], [0, 200])
    assert _attend(p, cu=(0, 128), ws_bytes=1 << 40) == -6  # 2^31 / 4096^2 tokens
    dk.pool_destroy(p)


def test_reorder_refuses_bad_calls(pool):
    call = dk.lib().dk_seq_reorder
    for _ in range(3):
        dk.seq_acquire(pool)
    assert call(None, 1, _i32(0), _i32(0), None) == -1
    assert call(pool, -1, _i32(0), _i32(0), None) == -1 and call(pool, 1, None, _i32(0), None) == -1 and call(pool, 1, _i32(0), None, None) == -1
    assert call(pool, 2, _i32(0, 5), _i32(0, 0), None) == -4 and call(pool, 2, _i32(0, 0), _i32(0, 0), None) == -5
    assert call(pool, 2, _i32(0, 1), _i32(0, 2), None) == -1 and call(pool, 2, _i32(0, 1), _i32(-1, 0), None) == -1
    assert call(pool, 0, None, None, None) == 0
    with pytest.raises(dk.DeltaKVError):
        dk.seq_reorder(pool, [0, 1], [0])
    assert dk.seq_len(pool, 0) == 10 and dk.seq_len(pool, 1) == 0


def test_reorders_that_need_no_copy(pool):
    """Permutations hand the chains over, cells and all; states of whole granules are aliased."""
    a, b, c = 0, dk.seq_acquire(pool), dk.seq_acquire(pool)
    dk.kv_reserve(pool, [b], [0, 32])
    before = {s: dk.seq_cells(pool, s).tolist() for s in (a, b, c)}
    dk.seq_reorder(pool, [a, b, c], [1, 2, 0], stream=1)
    assert dk.seq_cells(pool, a).tolist() == before[b] and dk.seq_cells(pool, b).tolist() == before[c] and dk.seq_cells(pool, c).tolist() == before[a]
    held = dk.pool_stats(pool)[0]
    dk.seq_reorder(pool, [a, b, c], [0, 0, 2], stream=1)  # 32 tokens are two granules
    assert dk.seq_cells(pool, b).tolist() == before[b] and dk.pool_stats(pool)[0] == held
    cells = [dk.kv_reserve(pool, [s], [0, 5]).tolist() for s in (a, b)]
    assert not set(cells[0]) & set(cells[1])
    dk.seq_reorder(pool, [a, b, c], [0, 1, 2], stream=1)
    assert dk.seq_cells(pool, a).tolist() == before[b] + cells[0]


def test_reorder_without_room_for_its_copies():
    p = _pool(arena_cells=32)
    a, b, c = (dk.seq_acquire(p) for _ in range(3))
    dk.kv_reserve(p, [a], [0, 5])
    dk.kv_reserve(p, [b], [0, 5])
    with pytest.raises(dk.DeltaKVError) as e:
        dk.seq_reorder(p, [a, b, c], [0, 1, 0], stream=1)
    assert e.value.name == "NO_CELLS" and [dk.seq_len(p, s) for s in (a, b, c)] == [5, 5, 0]
    dk.pool_destroy(p)


@pytest.mark.parametrize("sanitizer", [None, "address,undefined"])
def test_reorders_against_a_model(tmp_path, sanitizer):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path / "reorder_check")
    flags = [f"-fsanitize={sanitizer}"] if sanitizer else []
    cmd = [cxx, "-std=c++17", "-O1", "-g", "-pthread", *flags, os.path.join(ROOT, "tests", "reorder_check.cpp"),
           os.path.join(ROOT, "paper_2605_26289_amd", "csrc", "pool.cpp"), "-o", exe]
    built = subprocess.run(cmd, capture_output=True, text=True)
    if built.returncode != 0 and sanitizer and "cannot find" in built.stderr.lower():
        pytest.skip("sanitizer runtime not installed")
    assert built.returncode == 0, built.stderr[-3000:]
    run = subprocess.run([exe, "200"], capture_output=True, text=True, timeout=300)
    if run.returncode != 0 and sanitizer and "runtime does not come first" in run.stderr:
        pytest.skip("another preloaded library keeps the sanitizer runtime from loading first")
    assert run.returncode == 0 and run.stdout.startswith("ok"), (run.stdout[-3000:], run.stderr[-2000:])


def _select(groups=1, rows=4, cu=1 << 40, logits=2 << 40, dtype=dk.BF16, vocab=1000, stride=1000, scale=1.0, scores=3 << 40, n=8, row=4 << 40,
            token=5 << 40, score=6 << 40, ws=1 << 16, ws_bytes=1 << 30):
    return dk.lib().dk_beam_select(groups, rows, cu, logits, dtype, vocab, stride, scale, scores, n, row, token, score, ws, ws_bytes, None)


def test_beam_select_refuses_bad_calls():
    assert _select(groups=-1) == -1 and _select(rows=-1) == -1 and _select(vocab=0) == -1 and _select(stride=999) == -1 and _select(n=0) == -1
    assert _select(n=65) == -6 and _select(dtype=2) == -6 and _select(vocab=(1 << 20) + 1, stride=(1 << 20) + 8) == -6
    assert _select(rows=1 << 24) == -6 and _select(rows=1 << 20, vocab=1 << 15, stride=1 << 15) == -6 and _select(groups=1 << 24) == -6
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        assert _select(scale=scale) == -1
    assert _select(scale=2.0 ** -21) == -6 and _select(scale=2.0 ** 21) == -6
    for name in ("cu", "logits", "scores", "row", "token", "score"):
        assert _select(**{name: None}) == -1
    assert _select(logits=(2 << 40) + 8) == -6 and _select(stride=1001) == -6
    assert _select(ws=None) == -7 and _select(ws=(1 << 16) + 16) == -7
    need = dk.beam_workspace_bytes(4, 1000, dk.BF16, 8)
    assert _select(ws_bytes=need - 1) == -7
    assert _select(groups=0) == 0
    out = C.c_int64()
    assert dk.lib().dk_beam_workspace_bytes(4, 1000, dk.BF16, 8, None) == -1 and dk.lib().dk_beam_workspace_bytes(4, 1000, 7, 8, C.byref(out)) == -6
