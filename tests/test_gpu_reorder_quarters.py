"""dk_seq_reorder with granules of 256 cells and more, of which children share whole quarters: copies that begin inside a granule, chains
that part inside one, and dk_shared_attend on what comes of it."""
import numpy as np
import pytest
import torch

import oracle
from gpu_util import to_dev
from test_gpu_reorder import Beams
from test_gpu_shared import bounds
from paper_2605_26289_amd import binding as dk
from paper_2605_26289_amd import workloads as wl

pytestmark = pytest.mark.gpu


def attend_and_check(b, dtype, seed):
    hq, hkv, d = b.shape.n_q_heads, b.shape.n_kv_heads, b.shape.head_dim
    n = len(b.slots)
    q = wl.normal(np.random.default_rng(seed), (n, hq, d), dtype)
    lse = torch.empty((n, hq), dtype=torch.float32, device="cuda")
    got = b.pool.shared_attend(b.slots, np.arange(n + 1, dtype=np.int32), to_dev(q, dtype), b.shape.scale, lse=lse).float().cpu().numpy()
    lse = lse.cpu().numpy()
    for i, s in enumerate(b.slots):
        k, v = b.cache(s)
        ref = oracle.scored_attend(q[i:i + 1], k, v, len(k) - 1, b.shape.scale)
        tol, ltol = bounds(ref, dtype, len(k), d)
        assert (np.abs(got[i:i + 1] - ref[0]) <= tol).all()
        assert (np.abs(lse[i:i + 1] - ref[1]) <= ltol).all()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 64), ("f32", 128)])
@pytest.mark.parametrize("granule", [256, 512])
@pytest.mark.parametrize("own", [70, 129, 200, 255])
def test_children_share_whole_quarters_and_copy_the_rest(dtype, d, granule, own):
    b = Beams((4, 2, d, dtype), 4, 37, granule, seed=own)
    b.append(b.slots, [own, own + 1, 3, 0])
    before = [dk.seq_cells(b.pool.handle, s) for s in b.slots]
    b.reorder([0, 0, 1, 0])
    now = [dk.seq_cells(b.pool.handle, s) for s in b.slots]
    unit = granule // 4
    shared = 37 + own // unit * unit
    assert np.array_equal(now[0], before[0]) and np.array_equal(now[2], before[1])
    for i in (1, 3):
        assert np.array_equal(now[i][:shared], before[0][:shared]) and not set(now[i][shared:]) & set(before[0])
    assert before[0][shared] % granule == own // unit * unit % granule  # (where the copies came from: inside a granule, where any quarter is full)
    b.check()
    attend_and_check(b, dtype, 1)
    b.append(b.slots, [1, 2, 65, 130])
    b.reorder([3, 2, 1, 3])
    b.check()
    attend_and_check(b, dtype, 2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("granule", [256, 512])
def test_a_search_of_many_quarters(dtype, granule):
    b = Beams((4, 2, 64, dtype), 5, 300, granule, seed=9)
    rng = np.random.default_rng(10)
    for step in range(3 * granule // 4 + 40):
        b.append(b.slots, [1] * 5)
        b.reorder(rng.integers(0, 5, size=5).tolist())
    b.check()
    attend_and_check(b, dtype, 3)
    for s in b.slots:  # the prompt, a run and a node a quarter, the newest one
        runs, depth = dk.seq_stats(b.pool.handle, s)
        steps = 3 * granule // 4 + 40
        assert 3 <= depth <= 3 + 4 * steps // granule and runs <= 4 + 4 * steps // granule
    held = dk.pool_stats(b.pool.handle)[0]
    seen = {int(c) // granule for s in [b.prompt] + b.slots for c in dk.seq_cells(b.pool.handle, s)}
    assert held == granule * len(seen)  # no granule that no slot sees
    for s in [b.prompt] + b.slots:
        b.pool.release(s)
    assert dk.pool_stats(b.pool.handle)[0] == 0
