"""A layer's steps put together, with the attention held to element-wise bounds.

rotate_append -> scored_attend over the pool, and rotate_rows -> scored_attend over staged rows -> append of what was accepted.
The oracle gets the keys and values as the device holds them, so that the bounds are those of test_gpu_scored (the roundings of a
correct kernel) and a step that left out the cap or the window is told from one that did not: both are checked to be far outside."""
import numpy as np
import pytest
import torch

import oracle
from paper_2605_26289_amd import DevicePool
from paper_2605_26289_amd import binding as dk
from paper_2605_26289_amd import workloads as wl
from test_gpu_rotary import TORCH
from test_gpu_scored import _bounds

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mode", ["appended", "staged"])
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "bf16"), (64, "f32")])
def test_speculative_steps_within_the_roundings(d, dtype, mode):
    hq, hkv, window, cap, scale = 8, 2, 30, 4.0, d ** -0.5
    heads = hq + 2 * hkv
    rng = np.random.default_rng(2)
    f, amplitude = dk.rotary_freqs(d, 10000.0, dk.ROTARY_RAMP, [4, 1, 32, 64])
    w = np.float32(1.5) + wl.normal(rng, (2, d), dtype) / 4
    wd = [torch.from_numpy(x.copy()).to("cuda", TORCH[dtype]) for x in w]
    rotary = dk.Rotary(d, torch.from_numpy(f).cuda(), False, amplitude, 1e-6, *wd)
    scores = dk.Scores(cap=cap, window=window)
    pool = DevicePool(3, 2048, hq, hkv, d, dtype, granule_cells=16)
    slots = [pool.acquire() for _ in range(3)]

    def rows(n):
        x = torch.from_numpy(wl.normal(rng, (n, heads, d), dtype)).to("cuda", TORCH[dtype])
        return x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:]

    pool.rotate_append(slots[:1], [0, 37], *rows(37), rotary)  # a shared preamble
    for s in slots[1:]:
        pool.alias(slots[0], s, 37)
    pool.rotate_append(slots, [0, 5, 55, 66], *rows(66), rotary)
    for deltas in ([3, 1, 4], [1, 1, 1], [40, 2, 9]):
        cu = np.concatenate([[0], np.cumsum(deltas)]).astype(np.int32)
        before = [pool.length(s) for s in slots]
        assert min(before) > window
        x = rows(int(cu[-1]))
        lse = torch.empty((int(cu[-1]), hq), dtype=torch.float32, device="cuda")
        if mode == "appended":
            q = pool.rotate_append(slots, cu, *x, rotary)
            out = pool.scored_attend(slots, cu, q, scale, scores, lse=lse)
        else:
            pos = torch.cat([torch.arange(n, n + m, device="cuda") for n, m in zip(before, deltas)])
            q, k = [torch.empty(t.shape, dtype=t.dtype, device="cuda") for t in x[:2]]
            v = x[2].contiguous()
            dk.rotate_rows(pos, x[0], x[1], rotary, q, k)
            out = pool.scored_attend(slots, cu, q, scale, scores, k, v, lse=lse)
            pool.append(slots, cu, k, v)
        qh, oh, lh = q.float().cpu().numpy(), out.float().cpu().numpy(), lse.cpu().numpy()
        for b, n in enumerate(before):
            r = slice(int(cu[b]), int(cu[b + 1]))
            kg, vg = [t.float().cpu().numpy() for t in pool.gather(slots[b])]
            want = oracle.scored_attend(qh[r], kg, vg, n, scale, cap, window=window)
            tol, ltol = _bounds(want, dtype, n + deltas[b], d, cap, 0.0)
            assert (np.abs(oh[r] - want[0]) <= tol).all() and (np.abs(lh[r] - want[1]) <= ltol).all()
            for wrong in (dict(cap=0.0, window=window), dict(cap=cap / 2, window=window), dict(cap=cap, window=0), dict(cap=cap, window=window + 1)):
                other = oracle.scored_attend(qh[r], kg, vg, n, scale, **wrong)
                assert (np.abs(other[0] - want[0]) > 2 * tol).any() and (np.abs(other[1] - want[1]) > 2 * ltol).any(), wrong
        pool.trim_batch(slots, [n + max(1, m // 2) for n, m in zip(before, deltas)])
