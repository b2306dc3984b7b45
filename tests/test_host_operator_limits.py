"""Calls of the operators around delta attention that are too large, or whose tensors do not fit them, are turned down (no GPU).

Nothing here launches: every call is turned down before it would."""
import numpy as np
import pytest

from paper_2605_26289_amd import binding as dk


def _i32(*values):
    return np.asarray(values, dtype=np.int32).tobytes()


@pytest.mark.parametrize("d", [64, 128])
def test_rotate_append_refuses_more_tokens_than_a_launch_holds(d):
    most = 1 << 26
    pool = dk.pool_create(dk.PoolDesc(2, 0, 1 << 27, 1 << 25, 2, 1, d, dk.BF16, 256 * 10, 256 * 20, 256 * 30, 1 << 20))
    slots = [dk.seq_acquire(pool) for _ in range(2)]
    held = dk.pool_stats(pool)
    r = dk.Rotary(0)
    for cu in ((0, most + 1, most + 1), (0, 5, most + 1), (0, 0, (1 << 27) - 1)):
        rc = dk.lib().dk_rotate_append(pool, 2, _i32(*slots), _i32(*cu), r.address, 1 << 40, 2 * d, 2 << 40, d, 3 << 40, d, 4 << 40, None)
        assert rc == -6
        assert dk.pool_stats(pool) == held and all(dk.seq_len(pool, s) == 0 for s in slots)
    dk.pool_destroy(pool)
