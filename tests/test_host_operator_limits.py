"""Calls of the operators around delta attention that are too large, or whose tensors do not fit them, are turned down (no GPU).

Nothing here launches: every call is turned down before it would."""
import numpy as np
import pytest
import torch

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


class OnGpu(torch.Tensor):
    """Host memory that says it is on a GPU: what the binding would hand on goes to `calls`, not to the library."""

    gpu = 0

    def get_device(self):
        return self.gpu


def _gpu(*shape, dtype=torch.bfloat16, at=0):
    t = torch.zeros(shape, dtype=dtype).as_subclass(OnGpu)
    t.gpu = at
    return t


@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(dk, "_launch", lambda call, args, where, pool: made.append(args))
    return made


@pytest.fixture
def pool():
    p = dk.pool_create(dk.PoolDesc(4, 0, 4096, 16, 8, 2, 64, dk.BF16, 256 * 10, 256 * 20, 256 * 30, 1 << 20))
    yield p
    dk.pool_destroy(p)


def _refused(call, **kw):
    with pytest.raises(dk.DeltaKVError) as e:
        call(**kw)
    assert e.value.status == -1


F32, BF16, I32, I64 = torch.float32, torch.bfloat16, torch.int32, torch.int64


def test_scores_are_of_their_types():
    dk.Scores(slopes=_gpu(8, dtype=F32))
    for slopes in (_gpu(8), _gpu(8, dtype=torch.float64), _gpu(16, dtype=F32)[::2]):
        _refused(dk.Scores, slopes=slopes)
    for window in (1 << 31, 1 << 32, -(1 << 40)):  # (an int32 argument would take the lower half)
        _refused(dk.Scores, window=window)


def test_scored_attend_takes_rows_as_the_pool_has_them(pool, calls):
    def call(q=_gpu(5, 8, 64), out=_gpu(5, 8, 64), slopes=None, cu=(0, 2, 5), **kw):
        dk.scored_attend(pool, [0, 1], cu, q, out, 1.0, dk.Scores(slopes=slopes), stream=0, **kw)

    new = dict(k_new=_gpu(5, 2, 64), v_new=_gpu(5, 2, 64))
    call()
    call(slopes=_gpu(8, dtype=F32), lse=_gpu(5, 8, dtype=F32), workspace=_gpu(1 << 12, dtype=torch.uint8), **new)
    call(q=_gpu(7, 8, 64), out=_gpu(6, 512))  # rows behind the batch's
    assert len(calls) == 3 and calls[1][12] == 1 << 12
    fused = _gpu(5, 12, 64)
    for q in (_gpu(4, 8, 64), _gpu(5, 8, 64, dtype=F32), _gpu(5, 8, 64, dtype=torch.float16), fused[:, :8], _gpu(8, 5, 64).transpose(0, 1),
              torch.zeros((5, 8, 64), dtype=BF16)):
        _refused(call, q=q)
        _refused(call, out=q)
    for k in (_gpu(5, 1, 64), _gpu(5, 2, 64, dtype=F32), fused[:, 8:10], _gpu(5, 2, 64, at=1)):
        _refused(call, **{**new, "k_new": k})
        _refused(call, **{**new, "v_new": k})
    for lse in (_gpu(5, 8), _gpu(4, 8, dtype=F32), torch.zeros((5, 8))):
        _refused(call, lse=lse)
    _refused(call, slopes=_gpu(7, dtype=F32))
    _refused(call, slopes=torch.zeros(8))
    _refused(call, workspace=torch.zeros(1 << 12, dtype=torch.uint8))
    _refused(call, cu=(0, 5))  # offsets of one sequence for two
    _refused(dk.scored_workspace_bytes, pool=pool, slots=[0, 1], cu_delta=[0, 5], staged=False, scores=dk.Scores())
    assert len(calls) == 3


def test_a_rotary_is_of_types_that_fit():
    w = _gpu(64)
    dk.Rotary(64, _gpu(32, dtype=F32), norm_eps=1e-6, q_weight=w, k_weight=w)
    for freqs in (_gpu(31, dtype=F32), _gpu(32), _gpu(32, dtype=I32), _gpu(64, dtype=F32)[::2]):
        _refused(dk.Rotary, rotary_dim=64, inv_freq=freqs)
    for other in (_gpu(64, dtype=F32), _gpu(128)[::2], _gpu(64, at=1)):
        _refused(dk.Rotary, rotary_dim=0, norm_eps=1e-6, q_weight=w, k_weight=other)
    _refused(dk.Rotary, rotary_dim=0, inv_freq=_gpu(32, dtype=F32, at=1), norm_eps=1e-6, q_weight=w)
    _refused(dk.Rotary, rotary_dim=(1 << 32) + 64)


def test_rotate_append_takes_rows_as_the_pool_has_them(pool, calls):
    fused = _gpu(5, 12, 64)
    rows = dict(q=fused[:, :8], k=fused[:, 8:10], v=fused[:, 10:])

    def call(q_out=_gpu(5, 8, 64), rotary=dk.Rotary(0), cu=(0, 2, 5), **kw):
        dk.rotate_append(pool, [0, 1], cu, *{**rows, **kw}.values(), rotary, q_out, stream=0)

    call()
    call(q_out=_gpu(5, 512), rotary=dk.Rotary(64, _gpu(32, dtype=F32), norm_eps=0.0, q_weight=_gpu(64)))
    call(q=_gpu(6, 8, 64), k=_gpu(9, 2, 64))
    call(rotary=dk.Rotary(0, q_weight=_gpu(64, dtype=F32)))  # (without a norm no weight is looked at)
    assert len(calls) == 4
    for name, heads in (("q", 8), ("k", 2), ("v", 2)):
        for bad in (_gpu(4, heads, 64), _gpu(5, heads, 64, dtype=F32), _gpu(5, heads, 64, dtype=torch.float16), _gpu(5, heads + 1, 64),
                    _gpu(5, heads, 128), torch.zeros((5, heads, 64), dtype=BF16), _gpu(5, heads, 128)[:, :, ::2]):
            _refused(call, **{name: bad})
    for bad in (_gpu(4, 8, 64), _gpu(5, 8, 64, dtype=F32), fused[:, :8], torch.zeros((5, 8, 64), dtype=BF16), _gpu(5, 8, 64, at=1)):
        _refused(call, q_out=bad)
    for kw in (dict(q_weight=_gpu(64, dtype=F32)), dict(k_weight=_gpu(32)), dict(q_weight=torch.zeros(64, dtype=BF16)),
               dict(inv_freq=torch.zeros(32), rotary_dim=64)):
        _refused(call, rotary=dk.Rotary(**{"rotary_dim": 0, "norm_eps": 0.0, **kw}))
    _refused(call, cu=(0, 5))
    assert len(calls) == 4


def test_tensors_of_another_gpu_than_the_current_one_are_refused(pool, calls, monkeypatch):
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 77, raising=False)
    for at in (0, 1):
        def attend():
            dk.scored_attend(pool, [0], [0, 5], _gpu(5, 8, 64, at=at), _gpu(5, 8, 64, at=at), 1.0, dk.Scores())

        def append():
            dk.rotate_append(pool, [0], [0, 5], _gpu(5, 8, 64, at=at), *[_gpu(5, 2, 64, at=at)] * 2, dk.Rotary(0), _gpu(5, 8, 64, at=at))

        for call in (attend, append):
            _refused(call) if at else call()
    assert [args[-1] for args in calls] == [77, 77]


class _Recorder:
    """A library whose calls are kept and succeed."""

    def __init__(self, **answers):
        self.made, self.answers = [], answers

    def __getattr__(self, name):
        def call(*args):
            self.made.append(args)
            return 0
        return call


def test_rotate_rows_takes_rows_of_one_kind(monkeypatch):
    lib = _Recorder()
    monkeypatch.setattr(dk, "lib", lambda: lib)
    fused = _gpu(5, 12, 64)

    def call(positions=_gpu(5, dtype=I64), q=fused[:, :8], k=fused[:, 8:], q_out=_gpu(5, 8, 64), k_out=_gpu(5, 4, 64), rotary=dk.Rotary(0)):
        dk.rotate_rows(positions, q, k, rotary, q_out, k_out, stream=0)

    call()
    call(q=None, q_out=None)
    call(k=None, k_out=None, rotary=dk.Rotary(64, _gpu(32, dtype=F32), norm_eps=0.0, q_weight=_gpu(64)))
    call(q=_gpu(5, 8, 64, dtype=F32), k=None, q_out=_gpu(5, 8, 64, dtype=F32), positions=_gpu(7, dtype=I64))
    assert [a[0] for a in lib.made] == [dk.BF16, dk.BF16, dk.BF16, dk.F32] and lib.made[1][5:9] == (0, None, 0, None)
    for positions in (_gpu(5, dtype=I32), _gpu(4, dtype=I64), _gpu(10, dtype=I64)[::2], torch.zeros(5, dtype=I64), _gpu(5, dtype=F32)):
        _refused(call, positions=positions)
    for k in (_gpu(4, 4, 64), _gpu(6, 4, 64), _gpu(5, 2, 128), _gpu(5, 4, 64, dtype=F32), _gpu(5, 256), torch.zeros((5, 4, 64), dtype=BF16)):
        _refused(call, k=k)
    half = _gpu(5, 8, 64, dtype=torch.float16)
    _refused(call, q=half, k=None, q_out=half)
    _refused(call, q=None, k=None)
    for bad in (_gpu(4, 8, 64), _gpu(5, 8, 64, dtype=F32), fused[:, :8], torch.zeros((5, 8, 64), dtype=BF16)):
        _refused(call, q_out=bad)
        _refused(call, k_out=bad[:, :3])
    _refused(call, rotary=dk.Rotary(0, norm_eps=0.0, k_weight=_gpu(64, dtype=F32)))
    assert len(lib.made) == 4


def test_token_logprobs_takes_logits_and_outputs_as_they_are_described(monkeypatch):
    lib = _Recorder()
    monkeypatch.setattr(dk, "lib", lambda: lib)
    good = dict(logits=_gpu(3, 104)[:, :100], tokens=_gpu(3, dtype=I32), logprob_out=_gpu(3, dtype=F32), workspace=_gpu(4096, dtype=torch.uint8),
                rank_out=_gpu(3, dtype=I32), entropy_out=_gpu(3, dtype=F32), top_ids_out=_gpu(3, 2, dtype=I32), top_logprobs_out=_gpu(3, 2, dtype=F32))

    def call(rows=3, dtype=dk.BF16, vocab=100, row_stride=104, n_top=2, **kw):
        t = {**good, **kw}
        logits, rest = t.pop("logits"), t
        dk.token_logprobs(rows, logits, dtype, vocab, row_stride, n_top=n_top, stream=0, **rest)

    call()
    call(logits=_gpu(3 * 104))
    call(logits=_gpu(4, 104))
    call(rows=1, logits=_gpu(100), row_stride=104)
    call(rows=0, logits=_gpu(0, 100), row_stride=104)
    call(tokens=None, logprob_out=None, rank_out=None)
    assert len(lib.made) == 6 and lib.made[0][14] == 4096
    for logits in (_gpu(2, 104), _gpu(3, 96), _gpu(3, 112), _gpu(104, 3).t(), _gpu(3, 208)[:, ::2], _gpu(3, 104, dtype=F32),
                   _gpu(3, 104, dtype=torch.float16), torch.zeros((3, 104), dtype=BF16), _gpu(2 * 104 + 99)):
        _refused(call, logits=logits)
    _refused(call, dtype=dk.F32)
    for name in ("tokens", "rank_out", "logprob_out", "entropy_out", "top_ids_out", "top_logprobs_out"):
        t = good[name]
        other = I64 if t.dtype is I32 else torch.float64
        for bad in (t[:2], t.to(other), t.to(F32 if t.dtype is I32 else I32), torch.zeros(t.shape, dtype=t.dtype),
                    _gpu(6 * t.numel(), dtype=t.dtype)[::2], _gpu(*t.shape, dtype=t.dtype, at=1)):
            _refused(call, **{name: bad})
    _refused(call, workspace=torch.zeros(4096, dtype=torch.uint8))
    _refused(call, n_top=3)  # longer lists than there is room for
    assert len(lib.made) == 6
