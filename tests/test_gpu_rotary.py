"""dk_rotate_append and dk_rotate_rows against the fp64 oracle, element by element.

Bounds: the stored value half a step (2^-8 or 2^-24 of it); the norm D + 10 roundings of 2^-24; an angle half a turn's fp32
rounding (2^-25 turns: 2 pi 2^-25 < 2^-22) and sine and cosine good to 2^-22, together 2^-21 of amplitude (|a| + |b|)."""
import numpy as np
import pytest
import torch

import oracle
from paper_2605_26289_amd import DevicePool
from paper_2605_26289_amd import binding as dk
from paper_2605_26289_amd import workloads as wl

pytestmark = pytest.mark.gpu

TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}


def _fused(rng, tokens, heads, d, dtype, gap=0):
    """[tokens, heads * d + gap] rows, as a fused projection leaves them: (device tensor, host copy)"""
    x = wl.normal(rng, (tokens, heads * d + gap), dtype) * np.float32(3)
    if dtype == "bf16":
        x = wl.round_to_bf16(x)
    return torch.from_numpy(x).to("cuda", TORCH[dtype]), x


def _weights(rng, d, dtype):
    w = wl.normal(rng, (2, d), dtype)
    return w, [torch.from_numpy(x.copy()).to("cuda", TORCH[dtype]) for x in w]


def _check(got, want, before, rotary, amplitude, pairs, dtype, d):
    got = got.float().cpu().numpy().astype(np.float64)
    half = rotary // 2
    part = np.zeros_like(before)
    a, b = (before[..., 0:rotary:2], before[..., 1:rotary:2]) if pairs else (before[..., :half], before[..., half:rotary])
    both = abs(amplitude) * (np.abs(a) + np.abs(b))
    if pairs:
        part[..., 0:rotary:2] = part[..., 1:rotary:2] = both
    else:
        part[..., :half] = part[..., half:rotary] = both
    part[..., rotary:] = np.abs(before[..., rotary:])
    tol = (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(want) + part * ((d + 10) * 2.0 ** -24 + 2.0 ** -21) * 1.01 + 1e-30
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), got[bad][:4], want[bad][:4], tol[bad][:4])


CASES = [  # head width, rotary part, pairs, norm, weights, amplitude
    (128, 128, False, True, True, 1.0), (128, 128, True, True, True, 1.0), (128, 64, False, False, False, 1.0), (128, 20, False, True, False, 1.25),
    (128, 6, True, False, False, 1.0), (128, 0, False, True, True, 1.0), (128, 126, False, False, False, 0.5),
    (64, 64, False, True, True, 1.0), (64, 64, True, False, False, 1.1), (64, 16, False, True, True, 1.0), (64, 2, False, False, False, 1.0),
    (64, 50, True, True, True, 1.0), (64, 50, False, True, True, 1.0), (64, 0, True, False, False, 1.0), (128, 24, False, True, True, 1.0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,rotary,pairs,norm,weighted,amplitude", CASES)
def test_rows_at_given_positions(d, rotary, pairs, norm, weighted, amplitude, dtype):
    rng = np.random.default_rng(d + rotary)
    hq, hk, tokens = 5, 2, 37
    dev, host = _fused(rng, tokens, hq + hk, d, dtype, gap=16)
    q, k = dev[:, :hq * d].view(tokens, hq, d), dev[:, hq * d:(hq + hk) * d].view(tokens, hk, d)
    pos = rng.integers(0, 1 << 22, size=tokens)
    pos[:4] = [0, 1, -5, 1 << 30]
    f = (10000.0 ** (-np.arange(rotary // 2) / max(rotary // 2, 1))).astype(np.float32)
    w, wd = _weights(rng, d, dtype)
    r = dk.Rotary(rotary, torch.from_numpy(f).cuda(), pairs, amplitude, 1e-5 if norm else None, *(wd if weighted else (None, None)))
    qo, ko = (torch.full((tokens, h, d), float("nan"), dtype=TORCH[dtype], device="cuda") for h in (hq, hk))
    dk.rotate_rows(torch.from_numpy(pos).cuda(), q, k, r, qo, ko)
    for got, x, ww in ((qo, host[:, :hq * d].reshape(tokens, hq, d), w[0]), (ko, host[:, hq * d:(hq + hk) * d].reshape(tokens, hk, d), w[1])):
        want, before = oracle.rotate(x, pos, f, rotary, pairs, amplitude, 1e-5 if norm else None, ww if weighted else None)
        _check(got, want, before, rotary, amplitude, pairs, dtype, d)
    assert torch.equal(dev, torch.from_numpy(host).to("cuda", TORCH[dtype]))  # the input stays


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_in_place_and_one_kind_of_rows(dtype):
    rng = np.random.default_rng(2)
    x, host = _fused(rng, 33, 4, 64, dtype)
    x = x.view(33, 4, 64)
    f = torch.from_numpy((100.0 ** (-np.arange(32) / 32)).astype(np.float32)).cuda()
    pos = torch.arange(33, device="cuda", dtype=torch.int64)
    r = dk.Rotary(64, f)
    out = torch.empty_like(x)
    dk.rotate_rows(pos, x, None, r, out, None)
    dk.rotate_rows(pos, None, x, r, None, x)  # as keys, over themselves
    assert torch.equal(out, x)


@pytest.mark.parametrize("rotary,pairs", [(16, False), (16, True), (18, False), (6, True)])
def test_what_is_not_turned_stays_whatever_its_neighbours_hold(rotary, pairs):
    x = torch.randn((3, 2, 64), device="cuda", dtype=torch.bfloat16)
    x[:, :, rotary::3] = float("nan")
    x[:, 1, rotary + 1::5] = float("inf")
    out = torch.empty_like(x)
    dk.rotate_rows(torch.tensor([3, 9, 1000], device="cuda"), x, None, dk.Rotary(rotary, torch.ones(rotary // 2, device="cuda"), pairs), out, None)
    assert torch.equal(out[:, :, rotary:].view(torch.int16), x[:, :, rotary:].view(torch.int16))
    assert torch.isfinite(out[:, :, :rotary]).all()


def test_no_rows_and_many_rows():
    r = dk.Rotary(64, torch.ones(32, device="cuda"))
    none = torch.empty((0, 4, 64), device="cuda")
    dk.rotate_rows(torch.empty(0, dtype=torch.int64, device="cuda"), none, None, r, none, None)
    n = 70000
    x = torch.randn((n, 1, 64), device="cuda")
    pos = torch.arange(n, device="cuda", dtype=torch.int64)
    out = torch.empty_like(x)
    dk.rotate_rows(pos, x, None, r, out, None)
    a, b = x[:, 0, :32].double(), x[:, 0, 32:].double()
    c, s = torch.cos(pos.double())[:, None], torch.sin(pos.double())[:, None]
    want = torch.cat([a * c - b * s, b * c + a * s], dim=1)
    bound = 2.0 ** -24 * want.abs() + torch.cat([a.abs() + b.abs()] * 2, dim=1) * 2.0 ** -20
    assert ((out[:, 0].double() - want).abs() <= bound).all()


@pytest.mark.parametrize("granule", [4, 256])
@pytest.mark.parametrize("hq,hkv,d,dtype", [(8, 2, 128, "bf16"), (6, 2, 64, "bf16"), (4, 1, 64, "f32"), (4, 4, 128, "f32")])
@pytest.mark.parametrize("deltas", [[1], [9, 0, 1, 30], [400, 3, 700]], ids=["one", "few", "many"])
def test_append_is_rotation_then_append(hq, hkv, d, dtype, granule, deltas):
    """Sessions of different lengths, one through an alias; with granules of 4 the larger batches go to more runs of cells than
    the kernel arguments hold."""
    rng = np.random.default_rng(sum(deltas))
    n_slots = len(deltas)
    hist = [int(h) for h in rng.integers(0, 50, size=n_slots)]
    pool = DevicePool(n_slots, 8192, hq, hkv, d, dtype, granule_cells=granule)
    slots = [pool.acquire() for _ in deltas]
    old = {}
    for s, n in zip(slots, hist):
        kv = [torch.from_numpy(wl.normal(rng, (n, hkv, d), dtype)).to("cuda", TORCH[dtype]) for _ in range(2)]
        old[s] = kv
        if n:
            pool.append([s], [0, n], *kv)
    cu = np.concatenate([[0], np.cumsum(deltas)]).astype(np.int32)
    total = int(cu[-1])
    heads = hq + 2 * hkv
    dev, host = _fused(rng, total, heads, d, dtype)
    rows = dev.view(total, heads, d)
    f = (10000.0 ** (-np.arange(d // 2) / (d // 2))).astype(np.float32)
    w, wd = _weights(rng, d, dtype)
    rotary = dk.Rotary(d, torch.from_numpy(f).cuda(), False, 1.0, 1e-6, *wd)
    out = pool.rotate_append(slots, cu, rows[:, :hq], rows[:, hq:hq + hkv], rows[:, hq + hkv:], rotary)
    x = host.reshape(total, heads, d)
    pos = np.concatenate([n + np.arange(m) for n, m in zip(hist, deltas)])
    want, before = oracle.rotate(x[:, :hq], pos, f, d, False, 1.0, 1e-6, w[0])
    _check(out, want, before, d, 1.0, False, dtype, d)
    want, before = oracle.rotate(x[:, hq:hq + hkv], pos, f, d, False, 1.0, 1e-6, w[1])
    for b, s in enumerate(slots):
        r = slice(int(cu[b]), int(cu[b + 1]))
        assert pool.length(s) == hist[b] + deltas[b]
        kg, vg = pool.gather(s)
        assert torch.equal(kg[:hist[b]], old[s][0]) and torch.equal(vg[:hist[b]], old[s][1])
        _check(kg[hist[b]:], want[r], before[r], d, 1.0, False, dtype, d)
        assert np.array_equal(vg[hist[b]:].float().cpu().numpy(), x[r, hq + hkv:])


def test_append_writes_nothing_else():
    pool = DevicePool(2, 64, 2, 1, 64, "f32", granule_cells=16)
    pool.k_arena.fill_(7.0)
    pool.v_arena.fill_(7.0)
    a, b = pool.acquire(), pool.acquire()
    x = torch.randn((5, 4, 64), device="cuda")
    pool.rotate_append([a, b], [0, 3, 5], x[:, :2], x[:, 2:3], x[:, 3:], dk.Rotary(64, torch.ones(32, device="cuda")))
    cells = sorted(pool.cells(a).tolist() + pool.cells(b).tolist())
    free = [c for c in range(64) if c not in cells]
    assert (pool.k_arena[:, free] == 7).all() and (pool.v_arena[:, free] == 7).all()
    assert len(cells) == 5 and not (pool.k_arena[:, cells] == 7).any()


def test_append_past_four_gigabytes():
    cells, hkv, d = 5 * 2 ** 20, 4, 128
    pool = DevicePool(2, cells, 4, hkv, d, "bf16", granule_cells=4096)
    filler, slot = pool.acquire(), pool.acquire()
    dk.kv_reserve(pool.handle, [filler], [0, cells - 4096])
    x = torch.randn((7, 12, d), device="cuda", dtype=torch.bfloat16)
    pool.rotate_append([slot], [0, 7], x[:, :4], x[:, 4:8], x[:, 8:], dk.Rotary(0))
    k, v = pool.gather(slot)
    assert torch.equal(k, x[:, 4:8]) and torch.equal(v, x[:, 8:])  # nothing is turned: exact


def test_captured_and_replayed_on_another_stream():
    pool = DevicePool(1, 512, 4, 2, 64, "bf16")
    slot = pool.acquire()
    x = torch.randn((6, 8, 64), device="cuda", dtype=torch.bfloat16)
    rotary = dk.Rotary(64, torch.linspace(0.01, 1, 32, device="cuda"), norm_eps=1e-6)
    args = ([slot], [0, 6], x[:, :4], x[:, 4:6], x[:, 6:], rotary)
    want = pool.rotate_append(*args).clone()
    kw, vw = pool.gather(slot)
    pool.trim(slot, 0)
    out = torch.empty((6, 4, 64), device="cuda", dtype=torch.bfloat16)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        pool.rotate_append(*args, out=out)
    for _ in range(3):
        pool.k_arena.zero_(), pool.v_arena.zero_(), out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        k, v = pool.gather(slot)
        assert torch.equal(out, want) and torch.equal(k, kw) and torch.equal(v, vw)
