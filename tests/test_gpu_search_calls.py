"""Calls of dk_shared_attend, dk_seq_reorder and dk_beam_select beyond their results at ordinary sizes: where descriptors travel, cells and
logits beyond 2^31 bytes, captures, other streams, and what the probes of a pool say."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_beam import NAN, SUM_TOL, select
from test_gpu_reorder import Beams
from test_gpu_shared import Tree, bounds
from paper_2605_26289_amd import DevicePool
from paper_2605_26289_amd import binding as dk
from paper_2605_26289_amd import workloads as wl

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("members,what", [(50, "both kernels' in their arguments"), (140, "the merge's in its arguments"), (260, "all in the workspace")])
def test_descriptors_travel_all_ways(members, what, dtype):
    t = Tree(21, 4, 2, 64, dtype, [(None, 0, 700)] + [(0, 700, i % 5) for i in range(members)], granule=16)
    t.run_and_check(list(range(1, members + 1)), [1 + i % 2 for i in range(members)], False)
    assert dk.last_plan(t.pool.handle)["merges"] == members


@pytest.mark.parametrize("n", [64, 65, 1100, 4600])
def test_many_sequences_behind_one_prompt(n):
    """One token each: every work item and every merged row is found among that many."""
    hq, hkv, d, prompt = 2, 1, 64, 150
    pool = DevicePool(n + 1, 16 * (n + 20), hq, hkv, d, "bf16", granule_cells=16)
    root, *slots = [pool.acquire() for _ in range(n + 1)]
    rng = np.random.default_rng(26)
    k, v = (wl.normal(rng, (prompt, hkv, d), "bf16") for _ in range(2))
    kn, vn = (wl.normal(rng, (n, hkv, d), "bf16") for _ in range(2))
    q = wl.normal(rng, (n, hq, d), "bf16")
    to = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to("cuda", torch.bfloat16)
    pool.append([root], [0, prompt], to(k), to(v))
    for s in slots:
        pool.alias(root, s, prompt)
    cu = np.arange(n + 1, dtype=np.int32)
    pool.append(slots, cu, to(kn), to(vn))
    lse = torch.empty((n, hq), dtype=torch.float32, device="cuda")
    got = pool.shared_attend(slots, cu, to(q), 0.125, lse=lse).float().cpu().numpy()
    assert dk.last_plan(pool.handle)["merges"] == n
    lse = lse.cpu().numpy()
    s0 = np.einsum("nhd,kd->nhk", q.astype(np.float64), k[:, 0].astype(np.float64)) * 0.125
    s1 = np.einsum("nhd,nd->nh", q.astype(np.float64), kn[:, 0].astype(np.float64)) * 0.125
    top = np.maximum(s0.max(-1), s1)
    p0, p1 = np.exp(s0 - top[..., None]), np.exp(s1 - top)
    z = p0.sum(-1) + p1
    new = vn[:, 0].astype(np.float64)[:, None]
    o = (p0 @ v[:, 0].astype(np.float64) + p1[..., None] * new) / z[..., None]
    mag = (p0 @ np.abs(v[:, 0]).astype(np.float64) + p1[..., None] * np.abs(new)) / z[..., None]
    size = np.maximum((np.abs(q).astype(np.float64) @ np.abs(k[:, 0]).astype(np.float64).T).max(-1),
                      np.einsum("nhd,nd->nh", np.abs(q).astype(np.float64), np.abs(kn[:, 0]).astype(np.float64))) * 0.125
    tol, ltol = bounds((o, top + np.log(z), mag, size), "bf16", prompt + 1, d)
    assert (np.abs(got - o) <= tol).all()
    assert (np.abs(lse - (top + np.log(z))) <= ltol).all()


def test_probes_see_shared_attention():
    t = Tree(22, 4, 2, 64, "bf16", [(None, 0, 900)] + [(0, 900, 3) for _ in range(6)])
    dk.set_attend_timing(t.pool.handle, 8)
    dk.host_times(t.pool.handle, reset=True)
    for delta in (1, 30):
        t.run_and_check(list(range(1, 7)), [delta] * 6, True)
        plan = dk.last_plan(t.pool.handle)
        assert plan["route"] == "shared" and plan["bytes"] == dk.shared_workspace_bytes(t.pool.handle, t.call_slots, t.cu, True)
    with pytest.raises(dk.DeltaKVError):  # refused: the plan stays that of the last call that was enqueued
        t.run(float("nan"))
    assert dk.last_plan(t.pool.handle) == plan
    ms = dk.attend_times(t.pool.handle)
    assert len(ms) == 2 and (ms > 0).all()
    us, calls = dk.host_times(t.pool.handle)
    assert calls == (2, 0) and us["plan"] > 0 and us["launch"] > 0


def test_cells_beyond_two_gib():
    """K and V of 2.6 GB each: what lies in between is reserved, never written or read."""
    hq, hkv, d, far = 16, 8, 128, 1200000
    pool = DevicePool(6, far + 60000, hq, hkv, d, "bf16")
    filler, root, *beams = [pool.acquire() for _ in range(6)]
    rng = np.random.default_rng(23)
    dk.kv_reserve(pool.handle, [filler], [0, far])
    n = 700
    k, v = (wl.normal(rng, (n, hkv, d), "bf16") for _ in range(2))
    to = lambda x: torch.from_numpy(np.ascontiguousarray(x)).to("cuda", torch.bfloat16)
    pool.append([root], [0, n], to(k), to(v))
    assert min(pool.cells(root)) * d * 2 + (hkv - 1) * (far + 60000) * d * 2 > 1 << 31
    for s in beams:
        pool.alias(root, s, n)
    pool.append(beams[:1], [0, 40], to(k[:40]), to(v[:40]))
    pool.reorder(beams, [0, 0, 2, 0])
    cu = np.arange(5, dtype=np.int32)
    q = wl.normal(rng, (4, hq, d), "bf16")
    lse = torch.empty((4, hq), dtype=torch.float32, device="cuda")
    kn, vn = (wl.normal(rng, (4, hkv, d), "bf16") for _ in range(2))
    got = pool.shared_attend(beams, cu, to(q), 0.09, to(kn), to(vn), lse=lse)
    torch.cuda.synchronize()
    for i in range(4):
        own = 0 if i == 2 else 40
        keys, values = (np.concatenate([x, x[:own], new[i:i + 1]]) for x, new in ((k, kn), (v, vn)))
        ref = oracle.scored_attend(q[i:i + 1], keys, values, n + own, 0.09)
        tol, ltol = bounds(ref, "bf16", n + own + 1, d)
        assert (np.abs(got[i:i + 1].float().cpu().numpy() - ref[0]) <= tol).all()
        assert (np.abs(lse[i:i + 1].cpu().numpy() - ref[1]) <= ltol).all()


def test_a_captured_reorder_replays_its_copies():
    b = Beams((8, 2, 128, "bf16"), 4, 0, granule=16)
    b.append(b.slots, [21, 3, 45, 7])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        dk.seq_reorder(b.pool.handle, b.slots, [0, 0, 2, 2], stream=torch.cuda.current_stream())
    b.model.reorder(b.slots, [0, 0, 2, 2])
    cells = [b.pool.cells(s)[-1] for s in b.slots]
    for _ in range(3):
        for c in (cells[1], cells[3]):  # what was copied is copied again
            b.pool.k_arena.view(2, -1, 128)[:, c] = NAN
        g.replay()
        torch.cuda.synchronize()
        b.check()


def test_reorder_on_another_stream():
    b = Beams((8, 2, 128, "bf16"), 5, 37)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.append(b.slots, [3, 1, 4, 1, 5])
        b.reorder([4, 4, 0, 2, 1])
        b.append(b.slots, [1] * 5)
        b.reorder([1, 1, 1, 3, 3])
        b.check()


def test_selection_on_another_stream_and_two_at_once():
    """Two calls on two streams, each with a workspace of its own."""
    rng = np.random.default_rng(24)
    inputs = [(wl.normal(rng, (12, 30001), "f32") * np.float32(2.5), (rng.standard_normal(12) - 9).astype(np.float32)) for _ in range(2)]
    cu = torch.tensor([0, 5, 12], dtype=torch.int32, device="cuda")
    want = [select(x, s, [0, 5, 12], 9, "f32") for x, s in inputs]
    calls = []
    for x, s in inputs:
        buf = torch.full((12, 30004), NAN, device="cuda")
        buf[:, :30001] = torch.from_numpy(x).cuda()
        outs = [torch.empty((2, 9), dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
        ws = torch.empty(dk.beam_workspace_bytes(12, 30001, dk.F32, 9), dtype=torch.uint8, device="cuda")
        calls.append((torch.cuda.Stream(), buf, torch.from_numpy(s).cuda(), outs, ws))
    torch.cuda.synchronize()
    for _ in range(20):
        for stream, buf, s, outs, ws in calls:
            dk.beam_select(2, 12, cu, buf, dk.F32, 30001, 30004, s, 9, *outs, ws, stream=stream)
    torch.cuda.synchronize()
    for (_, _, _, outs, _), w in zip(calls, want):
        for o, x in zip(outs, w):
            assert np.array_equal(o.cpu().numpy(), x)


def test_more_logits_than_31_bits_count():
    """2.2e9 logits in 4.4 GB; the last group is looked at, and one in the middle."""
    rows, vocab, size, n = 17200, 128256, 8, 12
    g = torch.Generator(device="cuda").manual_seed(25)
    x = torch.empty((rows, vocab), dtype=torch.bfloat16, device="cuda")
    for r in range(0, rows, 1720):
        x[r:r + 1720] = torch.randn((1720, vocab), generator=g, device="cuda", dtype=torch.bfloat16)
    scores = torch.randn((rows,), generator=g, device="cuda") - 30
    groups = rows // size
    cu = torch.arange(groups + 1, dtype=torch.int32, device="cuda") * size
    outs = [torch.full((groups, n), -5, dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
    ws = torch.empty(dk.beam_workspace_bytes(rows, vocab, dk.BF16, n), dtype=torch.uint8, device="cuda")
    dk.beam_select(groups, rows, cu, x, dk.BF16, vocab, vocab, scores, n, *outs, ws)
    torch.cuda.synchronize()
    for group in (groups // 2, groups - 1):
        r = slice(group * size, (group + 1) * size)
        want = oracle.beam_select(x[r].float().cpu().numpy(), scores[r].cpu().numpy(), [0, size], n)
        got = [o[group].cpu().numpy() for o in outs]
        assert (np.abs(got[2] - want[2][0]) <= SUM_TOL + 2.0 ** -24 * (np.abs(want[2][0]) + 1)).all()
        pairs = {(int(a) - r.start, int(b)) for a, b in zip(got[0], got[1])}
        gaps = want[2][0][:-1] - want[2][0][1:]
        if (gaps > 2 * SUM_TOL).all():  # (no two too close to tell apart)
            assert pairs == set(zip(want[0][0].tolist(), want[1][0].tolist()))
        full = x[r].double().log_softmax(-1).cpu().numpy() + scores[r].double().cpu().numpy()[:, None]
        for (a, b), s in zip(zip(got[0] - r.start, got[1]), got[2]):
            assert abs(full[a, b] - s) <= SUM_TOL + 2.0 ** -24 * (abs(s) + 1)
