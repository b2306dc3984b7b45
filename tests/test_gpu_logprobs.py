"""dk_token_logprobs against the fp64 oracle: ids and ranks bit for bit, the rest within bounds on fp32 arithmetic.

A term exp(y) is off by 2^-24 of |y| (the scaled difference, three roundings) and 2^-22 (exp2); sums of at most `depth` additions
in a line are off by depth 2^-24.  `depth` is vocab / 256 + 64: a kernel that adds more in a line is not careful enough.  A log
probability is then off by 4 2^-24 |y| + 2^-21 + depth 2^-24, the entropy by that times the mean of |ln p| + 1, twice."""
import numpy as np
import pytest
import torch

import oracle
from paper_2605_26289_amd import binding as dk
from paper_2605_26289_amd import workloads as wl

pytestmark = pytest.mark.gpu


def _call(x, dtype, tokens, scale=1.0, n_top=0, gap=0, outputs="lrecp"):
    rows, vocab = x.shape
    tdt = torch.bfloat16 if dtype == "bf16" else torch.float32
    unit = 8 if dtype == "bf16" else 4
    stride = (vocab + unit - 1) // unit * unit + gap
    buf = torch.full((max(rows, 1), stride), float("nan"), dtype=tdt, device="cuda")  # what is behind a row counts for nothing
    buf[:rows, :vocab] = torch.from_numpy(x).to("cuda", tdt)
    f = lambda *s: torch.full(s, -77.0, dtype=torch.float32, device="cuda")  # noqa: E731
    i = lambda *s: torch.full(s, -77, dtype=torch.int32, device="cuda")  # noqa: E731
    lp, rank, ent = f(rows), i(rows), f(rows)
    ids, tlp = (i(rows, n_top), f(rows, n_top)) if n_top else (None, None)
    code = dk.BF16 if dtype == "bf16" else dk.F32
    ws = torch.full((dk.logprobs_workspace_bytes(rows, vocab, code, n_top),), 255, dtype=torch.uint8, device="cuda")
    tok = torch.from_numpy(np.asarray(tokens, dtype=np.int32)).cuda()
    dk.token_logprobs(rows, buf, code, vocab, stride, tok if "l" in outputs or "r" in outputs else None, lp if "l" in outputs else None, ws,
                      scale=scale, rank_out=rank if "r" in outputs else None, entropy_out=ent if "e" in outputs else None, n_top=n_top,
                      top_ids_out=ids, top_logprobs_out=tlp if "p" in outputs else None)
    torch.cuda.synchronize()
    return [None if t is None else t.cpu().numpy() for t in (lp, rank, ent, ids, tlp)]


def _near(got, want, tol):
    same = (got == want) | (np.isnan(got) & np.isnan(want))
    fine = np.isfinite(want) & np.isfinite(got)
    return same | (fine & (np.abs(np.where(fine, got, 0.0) - np.where(fine, want, 0.0)) <= tol))


def _check(x, dtype, tokens, scale=1.0, n_top=0, gap=0):
    lp, rank, ent, ids, tlp = _call(x, dtype, tokens, scale, n_top, gap)
    s32 = float(np.float32(scale))
    wl_, wr, we, wi, wt = oracle.token_logprobs(x, tokens, s32, n_top)
    eps = 2.0 ** -24
    depth = x.shape[1] / 256 + 64
    with np.errstate(invalid="ignore"):
        reach = lambda y: 4 * eps * np.abs(np.where(np.isfinite(y), y, 0.0)) + 2.0 ** -21 + depth * eps  # noqa: E731
        # |y| of a term is its distance from the maximum: |ln p| at most, as ln Z >= 0
        assert _near(lp, wl_, reach(wl_)).all(), (lp, wl_)
        assert _near(ent, we, 2 * (np.abs(np.where(np.isfinite(we), we, 0.0)) + 1) * (depth * eps + 2.0 ** -20)).all(), (ent, we)
        assert np.array_equal(rank, wr), (rank, wr)
        if n_top:
            assert np.array_equal(ids, wi), (ids, wi)
            assert _near(tlp, wt, reach(wt)).all(), (tlp, wt)


def _tokens(rng, x):
    best = oracle.greedy_argmax(x)
    return np.where(rng.random(x.shape[0]) < 0.5, best, rng.integers(0, x.shape[1], size=x.shape[0]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,vocab,n_top", [(1, 1, 1), (3, 2, 2), (2, 7, 3), (5, 64, 32), (4, 255, 1), (3, 256, 5), (2, 1000, 20), (7, 4099, 32),
                                             (3, 16384, 5), (2, 16385, 20), (2, 32003, 8), (1, 128256, 20), (2, 128256, 0), (300, 50, 4), (1, 1 << 24, 32),
                                             (1, 3 << 20, 7)])
def test_rows_of_all_widths(rows, vocab, n_top, dtype):
    rng = np.random.default_rng(rows * vocab)
    x = wl.normal(rng, (rows, vocab), dtype) * np.float32(2)
    _check(x, dtype, _tokens(rng, x), 1.0, n_top, gap=0 if rows % 2 else 64)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [1 / 0.7, 0.1, 30.0])
def test_temperatures(scale, dtype):
    rng = np.random.default_rng(3)
    x = wl.normal(rng, (6, 5003), dtype) * np.float32(4)
    _check(x, dtype, _tokens(rng, x), scale, 5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_top", [1, 20, 32])
def test_ties_infinities_and_broken_rows(dtype, n_top):
    rng = np.random.default_rng(4)
    vocab = 20011
    low = float(torch.finfo(torch.bfloat16 if dtype == "bf16" else torch.float32).min)
    x = wl.round_to_bf16(np.round(wl.normal(rng, (14, vocab), dtype) * 2) / 2)  # few distinct values
    x[1] = -np.inf
    x[2, 17] = np.nan
    x[3, [5, 19000]] = np.inf
    x[4] = 0.25  # all alike
    x[5] = low  # the type's lowest value everywhere: still a distribution
    x[6] = -np.inf
    x[6, [3, 7000, 20010]] = [1.0, 2.0, 1.0]
    x[7, : vocab // 2] = -np.inf
    x[8] = np.linspace(-3, 3, vocab, dtype=np.float32) if dtype == "f32" else wl.round_to_bf16(np.linspace(-3, 3, vocab, dtype=np.float32))
    x[9] = x[8][::-1]
    x[10] = np.where(np.arange(vocab) % 2 == 0, 0.0, -0.0)
    x[11] = low
    x[11, 12345] = 3.0
    x[12, 4] = -np.nan
    x[13] = 0.0
    x[13, 8192:8192 + 2000] = 5.0  # a run of equal maxima
    tokens = _tokens(rng, x)
    tokens[[0, 7]] = [-1, vocab]  # no token
    tokens[6] = 4  # a token that cannot be
    _check(x, dtype, tokens, 1.0, n_top)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_logits(dtype):
    """Logits around 10^4: the distribution is in their differences."""
    rng = np.random.default_rng(5)
    x = wl.normal(rng, (4, 3001), dtype) * np.float32(100) + np.float32(10000)
    x = wl.round_to_bf16(x) if dtype == "bf16" else x.astype(np.float32)
    _check(x, dtype, _tokens(rng, x), 0.05, 7)


def test_outputs_may_be_left_out():
    rng = np.random.default_rng(6)
    x = wl.normal(rng, (5, 3000), "f32")
    t = _tokens(rng, x)
    full = _call(x, "f32", t, 1.0, 4)
    for outputs in ("l", "r", "e", "", "lp", "ep"):
        got = _call(x, "f32", t, 1.0, 4, outputs=outputs)
        for name, a, b in zip("lre", got, full):
            assert np.array_equal(a, b) if name in outputs else (a == -77).all()
        assert np.array_equal(got[3], full[3]) and (np.array_equal(got[4], full[4]) if "p" in outputs else (got[4] == -77).all())


def test_the_same_rows_give_the_same_bits_on_any_stream_and_in_a_graph():
    rng = np.random.default_rng(7)
    rows, vocab, n_top = 9, 40000, 6
    x = torch.from_numpy(wl.normal(rng, (rows, vocab), "bf16")).to("cuda", torch.bfloat16)
    tok = torch.randint(0, vocab, (rows,), device="cuda", dtype=torch.int32)
    new = lambda: [torch.empty(rows, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda"),  # noqa: E731
                   torch.empty((rows, n_top), dtype=torch.int32, device="cuda"), torch.empty((rows, n_top), device="cuda")]
    ws = torch.empty(dk.logprobs_workspace_bytes(rows, vocab, dk.BF16, n_top), dtype=torch.uint8, device="cuda")

    def call(o):
        dk.token_logprobs(rows, x, dk.BF16, vocab, vocab, tok, o[0], ws, 1.3, o[1], o[2], n_top, o[3], o[4])

    want = new()
    call(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = new()
    with torch.cuda.stream(side):
        call(got)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    got = new()
    with torch.cuda.graph(graph, stream=side):
        call(got)
    for _ in range(3):
        for g in got:
            g.zero_()
        ws.fill_(170)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
