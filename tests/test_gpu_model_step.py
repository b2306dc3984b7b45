"""The operators as a model's step uses them, together: one layer and an output projection, sessions on a shared prefix.

rotate_append (norms, rotation, K and V into the pool) -> scored_attend -> output rows -> logits -> verify_greedy and
token_logprobs -> trim to what was accepted; three steps, every one against the same step in float64 on the host."""
import numpy as np
import pytest
import torch

import oracle
from paper_2605_26289_amd import DevicePool
from paper_2605_26289_amd import binding as dk
from paper_2605_26289_amd import workloads as wl

pytestmark = pytest.mark.gpu


def test_speculative_steps_of_a_layer():
    hq, hkv, d, dtype, vocab, window, cap = 8, 2, 128, "bf16", 1000, 60, 20.0
    heads = hq + 2 * hkv
    rng = np.random.default_rng(1)
    f, amplitude = dk.rotary_freqs(d, 10000.0, dk.ROTARY_RAMP, [4, 1, 32, 64])
    w = wl.normal(rng, (2, d), dtype)
    wd = [torch.from_numpy(x.copy()).to("cuda", torch.bfloat16) for x in w]
    rotary = dk.Rotary(d, torch.from_numpy(f).cuda(), False, amplitude, 1e-6, *wd)
    scores = dk.Scores(cap=cap, window=window)
    pool = DevicePool(3, 2048, hq, hkv, d, dtype, granule_cells=16)
    slots = [pool.acquire() for _ in range(3)]
    project = torch.from_numpy(wl.normal(rng, (hq * d, vocab), "f32")).cuda() / 8
    k_host, v_host = [np.zeros((0, hkv, d))] * 3, [np.zeros((0, hkv, d))] * 3

    def append(which, deltas):
        cu = np.concatenate([[0], np.cumsum(deltas)]).astype(np.int32)
        x = wl.normal(rng, (int(cu[-1]), heads, d), dtype)
        rows = torch.from_numpy(x).to("cuda", torch.bfloat16)
        q = pool.rotate_append(which, cu, rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:], rotary)
        for b, s in enumerate(which):
            i = slots.index(s)
            r = slice(int(cu[b]), int(cu[b + 1]))
            n = len(k_host[i])
            turned = oracle.rotate(x[r, hq:hq + hkv], n + np.arange(deltas[b]), f, d, False, amplitude, 1e-6, w[1])[0]
            k_host[i] = np.concatenate([k_host[i], wl.round_to_bf16(turned.astype(np.float32))])
            v_host[i] = np.concatenate([v_host[i], x[r, hq + hkv:]])
        return cu, q

    append(slots[:1], [37])  # a shared preamble
    for i in (1, 2):
        pool.alias(slots[0], slots[i], 37)
        k_host[i], v_host[i] = k_host[0], v_host[0]
    append(slots, [5, 50, 11])
    for step in range(3):
        deltas = [3, 1, 4]
        before = [pool.length(s) for s in slots]
        cu, q = append(slots, deltas)
        out = pool.scored_attend(slots, cu, q, d ** -0.5, scores)
        logits = (out.float().reshape(int(cu[-1]), -1) @ project)
        rows = logits.shape[0]
        batch = torch.randint(0, vocab, (rows,), device="cuda", dtype=torch.int32)
        batch[1] = logits[0].argmax()  # the first draft of the first session holds
        i32 = lambda n: torch.empty(n, dtype=torch.int32, device="cuda")  # noqa: E731
        keep, nxt, am, rank, ids = i32(3), i32(3), i32(rows), i32(rows), i32((rows, 3))
        lp, ent, tlp = (torch.empty(s, device="cuda") for s in (rows, rows, (rows, 3)))
        ws = torch.empty(dk.verify_workspace_bytes(rows, vocab, dk.F32), dtype=torch.uint8, device="cuda")
        dk.verify_greedy(3, rows, torch.from_numpy(cu).cuda(), logits, dk.F32, vocab, vocab, batch, keep, nxt, ws, argmax_out=am)
        ws2 = torch.empty(dk.logprobs_workspace_bytes(rows, vocab, dk.F32, 3), dtype=torch.uint8, device="cuda")
        dk.token_logprobs(rows, logits, dk.F32, vocab, vocab, am, lp, ws2, rank_out=rank, entropy_out=ent, n_top=3, top_ids_out=ids,
                          top_logprobs_out=tlp)
        # attention against the host's rows, Q as the device has it (its own rounding is tested elsewhere)
        qh = q.float().cpu().numpy()
        for b, n in enumerate(before):
            r = slice(int(cu[b]), int(cu[b + 1]))
            o, _, mag, _ = oracle.scored_attend(qh[r], k_host[b], v_host[b], n, d ** -0.5, cap, window=window)
            # K on the host may be the neighbouring bf16 of the device's where a value lies between two: a step of a key's
            # element moves a score by at most 2^-7 scale sum |q k|, for all elements at once below 2^-7 times 16 here
            assert (np.abs(out[r].float().cpu().numpy() - o) <= 2.0 ** -7 * np.abs(o) + mag * 2.0 ** -3).all()
            kg, vg = pool.gather(slots[b])
            assert np.array_equal(vg.float().cpu().numpy(), v_host[b])
            assert np.allclose(kg.float().cpu().numpy(), k_host[b], rtol=2.0 ** -7, atol=1e-5)
        wlp, wrank, went, wids, wtlp = oracle.token_logprobs(logits.cpu().numpy(), am.cpu().numpy(), 1.0, 3)
        assert np.array_equal(rank.cpu().numpy(), wrank) and (wrank == 0).all() and np.array_equal(ids.cpu().numpy(), wids)
        assert np.array_equal(ids.cpu().numpy()[:, 0], am.cpu().numpy())
        for got, want in ((lp, wlp), (ent, went), (tlp, wtlp)):
            assert np.allclose(got.cpu().numpy(), want, atol=1e-4)
        assert torch.equal(lp, tlp[:, 0])
        kept = keep.cpu().numpy()
        assert kept[0] >= 2
        pool.trim_batch(slots, [n + int(c) for n, c in zip(before, kept)])
        for i in range(3):
            k_host[i], v_host[i] = k_host[i][:before[i] + int(kept[i])], v_host[i][:before[i] + int(kept[i])]
