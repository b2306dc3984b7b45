"""The probes of a pool's calls (dk_last_plan, dk_attend_times, dk_host_times) see scored attention and rotary appends too."""
import pytest
import torch

from paper_2605_26289_amd import DevicePool
from paper_2605_26289_amd import binding as dk

pytestmark = pytest.mark.gpu


def _rows(n, heads, d=64):
    return torch.randn((n, heads, d), device="cuda", dtype=torch.bfloat16)


def test_probes_see_scored_attention():
    pool = DevicePool(2, 8192, 4, 2, 64, "bf16")
    slots = [pool.acquire() for _ in range(2)]
    pool.append(slots, [0, 3000, 3040], _rows(3040, 2), _rows(3040, 2))
    dk.set_attend_timing(pool.handle, 8)
    dk.host_times(pool.handle, reset=True)
    pool.attend(slots, [0, 1, 2], _rows(2, 4), 0.1)
    plain = dk.last_plan(pool.handle)
    assert plain["route"] != "scored"
    pool.scored_attend(slots, [0, 1, 2], _rows(2, 4), 0.1, dk.Scores(cap=20.0))  # few rows, the longer one's keys cut
    few = dk.last_plan(pool.handle)
    assert few["route"] == "scored" and few["row_items"] == 0 and few["stream_items"] > 2 and few["merges"] == 1
    assert few["bytes"] == dk.scored_workspace_bytes(pool.handle, slots, [0, 1, 2], False, dk.Scores(cap=20.0))
    pool.scored_attend(slots, [0, 100, 140], _rows(140, 4), 0.1, dk.Scores(window=64))
    many = dk.last_plan(pool.handle)
    assert many["route"] == "scored" and many["row_items"] > 0 and many["stream_items"] == 0
    with pytest.raises(dk.DeltaKVError):  # refused: the plan stays that of the last call that was enqueued
        pool.scored_attend(slots, [0, 1, 2], _rows(2, 4), float("nan"), dk.Scores())
    assert dk.last_plan(pool.handle) == many
    ms = dk.attend_times(pool.handle)
    assert len(ms) == 3 and (ms > 0).all() and dk.last_attend_ms(pool.handle) == ms[2]
    us, calls = dk.host_times(pool.handle)
    assert calls == (3, 0) and all(us[k] > 0 for k in ("plan", "stage", "upload", "launch"))


def test_probes_see_rotary_appends():
    pool = DevicePool(1, 1024, 4, 2, 64, "bf16")
    slot = pool.acquire()
    dk.host_times(pool.handle, reset=True)
    x = _rows(5, 8)
    pool.rotate_append([slot], [0, 5], x[:, :4], x[:, 4:6], x[:, 6:], dk.Rotary(64, torch.ones(32, device="cuda")))
    us, calls = dk.host_times(pool.handle)
    assert calls == (0, 1) and us["append_bookkeeping"] > 0 and us["append_launch"] > 0
    torch.cuda.synchronize()
