"""The operators around delta attention that a model's step needs: what they compute, in plain torch, and how they are called.

A case is a dict of plain values.  `listed()` names some, `draw()` gives more from the same ranges; `prepare` makes what a
serving loop holds before the call, `run` is one pass -- with `own` through the framework's entry points, without it in
elementary torch operations -- and `exact` the same results in float64, written from the definitions.

Kinds of case:
  attend    attention of a batch's new tokens over their cached ones, with a capped score, a bias by distance, a sliding
            window, a prefix that every row sees, documents that rows may not look out of, rows that see nothing
  append    norms of Q and K for each head, rotation by position, K and V into the cache, for a batch of sessions
  rows      the same norms and rotation for rows at given positions, without a cache
  logprobs  log probability and rank of given tokens, entropy, best alternatives
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

EPS = 1e-6


def _attend(name, **kw):
    case = {"kind": "attend", "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "slots": 1, "n_lo": 0, "n_hi": 0,
            "delta_lo": 1, "delta_hi": 1, "chunks": 0, "chunk": 0, "cap": 0.0, "alibi": False, "window": 0, "prefix": False,
            "docs": 0, "pad": False, "lens": 1}
    case.update(kw)
    if name:
        case["name"] = name
    return case


def _append(name, **kw):
    case = {"kind": "append", "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "slots": 1, "n_lo": 0, "n_hi": 0,
            "delta_lo": 1, "delta_hi": 1, "rotary": 128, "pairs": False, "norm": True, "theta": 500000.0, "stretch": 1.0,
            "amplitude": 1.0, "lens": 1}
    case.update(kw)
    if name:
        case["name"] = name
    return case


def _logprobs(name, **kw):
    case = {"kind": "logprobs", "rows": 1, "vocab": 128256, "dtype": "bf16", "top": 0, "temperature": 1.0, "guided": False}
    case.update(kw)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # One user of a model with capped scores, token by token: the smallest call, latency and launches.
        _attend("attend_decode_one", n_lo=3000, n_hi=3000, cap=50.0),
        # Speculative verification in a layer with capped scores and a sliding window: 64 sessions, long caches.
        _attend("attend_verify_window", slots=64, n_lo=4096, n_hi=16384, delta_lo=1, delta_hi=9, cap=50.0, window=4096, lens=2),
        # Interleaved agents' turns with capped scores: the large products.
        _attend("attend_turns_capped", slots=16, n_lo=1024, n_hi=8192, delta_lo=64, delta_hi=512, cap=30.0, lens=3),
        # Models with 64-wide heads and a bias by distance: two prefill chunks among decoding sessions.
        _attend("attend_heads64_bias", d=64, slots=16, n_lo=512, n_hi=4096, delta_lo=1, delta_hi=9, chunks=2, chunk=256,
                alibi=True, lens=4),
        # Documents behind a shared instruction, in fp32 (validation runs): rows see their own document, padding sees nothing.
        _attend("attend_documents_f32", hq=8, hkv=2, dtype="f32", slots=4, n_lo=300, n_hi=2000, delta_lo=100, delta_hi=300,
                docs=200, pad=True, lens=5),
        # One token of one session into the cache: latency and launches.
        _append("append_decode_one", n_lo=3000, n_hi=3000),
        # The candidate rows of 24 verifying sessions.
        _append("append_verify", slots=24, n_lo=4096, n_hi=16384, delta_lo=9, delta_hi=9, lens=6),
        # 16 agents' turns of 512 tokens at far positions, frequencies stretched for a long context.
        _append("append_turns_far", slots=16, n_lo=20000, n_hi=30000, delta_lo=512, delta_hi=512, stretch=8.0,
                amplitude=1.2079441541679836, lens=7),
        # Rows for a staged call: neighbouring pairs of a quarter of the head, no norm, fp32, an odd number of tokens.
        {"name": "rows_pairs_f32", "kind": "rows", "hq": 16, "hkv": 4, "d": 64, "dtype": "f32", "tokens": 1003, "far": 1 << 20,
         "rotary": 16, "pairs": True, "norm": False, "theta": 10000.0, "stretch": 1.0, "amplitude": 1.0},
        # A sampled token's log probability with five alternatives, one user.
        _logprobs("logprobs_one", top=5, temperature=0.7),
        # 64 sessions of nine verified rows: what each answer token was worth.
        _logprobs("logprobs_verify", rows=576, top=0),
        # A prompt scored with 20 alternatives a token: fp32 logits, an odd vocabulary, some rows held to a grammar.
        _logprobs("logprobs_prompt_f32", rows=1500, vocab=50003, dtype="f32", top=20, guided=True),
    ]


def _between(rng, lo, hi):
    """A whole number spread evenly over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


HEADS = [(32, 8, 128), (32, 8, 64), (16, 4, 64), (14, 2, 64), (12, 2, 128), (28, 4, 128), (8, 8, 128), (16, 2, 128), (16, 1, 128)]
HEADS_F32 = [(4, 1, 64), (4, 2, 64), (8, 2, 64), (8, 2, 128), (16, 4, 128)]


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "append", "append", "rows", "logprobs", "logprobs"])
    lens = rng.randrange(1, 1 << 30)
    if kind == "attend":
        f32 = rng.random() < 0.25
        hq, hkv, d = rng.choice(HEADS_F32 if f32 else HEADS)
        mods = {"cap": rng.choice([0.0, 30.0, 50.0, rng.uniform(5.0, 60.0)]), "alibi": rng.random() < 0.3,
                "window": rng.choice([0, 0, _between(rng, 1, 6000)]), "prefix": rng.random() < 0.2,
                "docs": rng.choice([0, 0, _between(rng, 20, 2000)]), "pad": rng.random() < 0.2}
        if rng.random() < 0.5:  # decoding and verification
            slots = _between(rng, 1, 8 if f32 else 64)
            n = _between(rng, 100, min(8000 if f32 else 32000, 500000 // slots))
            return _attend(None, hq=hq, hkv=hkv, d=d, dtype="f32" if f32 else "bf16", slots=slots, n_lo=n // 4, n_hi=n,
                           delta_hi=rng.choice([1, rng.randint(1, 9)]), lens=lens, **mods)
        slots = _between(rng, 1, 4 if f32 else 12)
        n = _between(rng, 30, 2000 if f32 else 20000 // slots)
        return _attend(None, hq=hq, hkv=hkv, d=d, dtype="f32" if f32 else "bf16", slots=slots, n_lo=0, n_hi=n,
                       delta_hi=_between(rng, 2, 300 if f32 else 3000 // slots), lens=lens, **mods)
    if kind == "logprobs":
        dtype = rng.choice(["bf16", "f32"])
        vocab = rng.choice([8 * rng.randint(4000, 16032), rng.randint(1000, 128256)])
        rows = _between(rng, 1, min(2000, 75000000 // vocab))
        return _logprobs(None, rows=rows, vocab=vocab, dtype=dtype, top=rng.choice([0, 1, 5, 20, rng.randint(2, 32)]),
                         temperature=rng.choice([1.0, 0.7, rng.uniform(0.3, 1.5)]), guided=rng.random() < 0.3)
    f32 = rng.random() < 0.3
    hq, hkv, d = rng.choice(HEADS_F32 if f32 else HEADS)
    rotation = {"rotary": rng.choice([d, d, d // 2, 2 * rng.randint(0, d // 2)]), "pairs": rng.random() < 0.4,
                "norm": rng.random() < 0.6, "theta": rng.choice([10000.0, 500000.0, 1000000.0]),
                "stretch": rng.choice([1.0, 1.0, 4.0, 32.0]), "amplitude": rng.choice([1.0, 1.0, rng.uniform(1.0, 1.4)])}
    if kind == "rows":
        return {"kind": "rows", "hq": hq, "hkv": hkv, "d": d, "dtype": "f32" if f32 else "bf16", "tokens": _between(rng, 1, 6000),
                "far": _between(rng, 100, 1 << 22), **rotation}
    slots = _between(rng, 1, 24)
    n = _between(rng, 1, 400000 // slots)
    return _append(None, hq=hq, hkv=hkv, d=d, dtype="f32" if f32 else "bf16", slots=slots, n_lo=n // 4, n_hi=n,
                   delta_hi=_between(rng, 1, 6000 // slots), lens=lens, **rotation)


# ---- inputs ----------------------------------------------------------------------------------------------------------
def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _lengths(case):
    """(cached tokens, new tokens) of every session, by the case alone."""
    rng = random.Random(case["lens"])
    hist = [rng.randint(case["n_lo"], case["n_hi"]) for _ in range(case["slots"])]
    delta = [rng.randint(case["delta_lo"], case["delta_hi"]) for _ in range(case["slots"])]
    for i in rng.sample(range(case["slots"]), min(case.get("chunks", 0), case["slots"])):
        delta[i] = case["chunk"]
    return hist, delta


def _offsets(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def _masks(case):
    """(prefix of every session or None, first position that every new token sees or None), by the case alone."""
    hist, delta = _lengths(case)
    rng = random.Random(case["lens"] + 1)
    prefix = [rng.randint(0, n + new) for n, new in zip(hist, delta)] if case["prefix"] else None
    if not case["docs"] and not case["pad"]:
        return prefix, None
    first = []
    for n, new in zip(hist, delta):
        starts, at = [0], 0
        while case["docs"] and at < n + new:
            at += rng.randint(1, 2 * case["docs"])
            starts.append(at)
        padding = new // 16 if case["pad"] else 0
        k = 0
        for i in range(new):
            while k + 1 < len(starts) and starts[k + 1] <= n + i:
                k += 1
            first.append(n + new if i >= new - padding else starts[k])
    return prefix, first


def _slopes(case):
    """Biases by distance: a geometric series over the heads, from 1/2 down to 2^-8."""
    return torch.tensor([2.0 ** (-8.0 * (h + 1) / case["hq"]) for h in range(case["hq"])], dtype=torch.float32, device="cuda")


def _attend_inputs(case, seed):
    gen, dt = _generator(seed), _type(case)
    hist, delta = _lengths(case)
    hkv, hq, d = case["hkv"], case["hq"], case["d"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dt)

    # queries of twice the keys' size: scores that reach into the bend of the cap
    return {"k": normal(sum(hist), hkv, d), "v": normal(sum(hist), hkv, d), "k_new": normal(sum(delta), hkv, d),
            "v_new": normal(sum(delta), hkv, d), "q": normal(sum(delta), hq, d) * 2}


def _tokens_of(case):
    return case["tokens"] if case["kind"] == "rows" else sum(_lengths(case)[1])


def _rotary_inputs(case, seed):
    """The rows as a fused projection leaves them, norm weights, frequencies, positions."""
    gen, dt = _generator(seed), _type(case)
    hkv, hq, d = case["hkv"], case["hq"], case["d"]
    t = _tokens_of(case)
    fused = torch.randn((t, (hq + 2 * hkv) * d), generator=gen, device="cuda", dtype=dt) * 3
    weights = [1 + 0.2 * torch.randn((d,), generator=gen, device="cuda") for _ in range(2)]
    half = case["rotary"] // 2
    freqs = [case["theta"] ** (-i / half) / case["stretch"] for i in range(half)]
    if case["kind"] == "rows":
        position = torch.randint(0, case["far"], (t,), generator=gen, device="cuda", dtype=torch.int64)
    else:
        hist, delta = _lengths(case)
        position = torch.cat([torch.arange(n, n + new, device="cuda", dtype=torch.int64) for n, new in zip(hist, delta)])
    return {"fused": fused, "wq": weights[0].to(dt), "wk": weights[1].to(dt), "position": position,
            "freqs": torch.tensor(freqs, dtype=torch.float64, device="cuda").float()}


def _split(case, fused):
    hkv, hq, d = case["hkv"], case["hq"], case["d"]
    t = fused.shape[0]
    return (fused[:, :hq * d].view(t, hq, d), fused[:, hq * d:(hq + hkv) * d].view(t, hkv, d),
            fused[:, (hq + hkv) * d:].view(t, hkv, d))


def _logit_inputs(case, seed):
    gen, dt = _generator(seed), _type(case)
    rows, vocab = case["rows"], case["vocab"]
    stride = (vocab + 7) // 8 * 8  # rows start at whole 16 bytes
    buf = torch.randn((rows, stride), generator=gen, device="cuda", dtype=dt) * 2.5
    logits = buf[:, :vocab]
    if case["guided"]:  # every third row: only a few tokens are allowed
        allowed = torch.rand((rows, vocab), generator=gen, device="cuda") < 0.002
        allowed[:, 0] = True
        shut = (torch.arange(rows, device="cuda") % 3 == 1)[:, None] & ~allowed
        logits.masked_fill_(shut, float("-inf"))
    tokens = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    likely = torch.rand((rows,), generator=gen, device="cuda") < 0.7
    tokens = torch.where(likely, logits.float().argmax(dim=1).to(torch.int32), tokens)
    return buf, logits, tokens


def prepare(case, seed):
    if case["kind"] == "logprobs":
        buf, logits, tokens = _logit_inputs(case, seed)
        state = {"case": case, "logits": logits, "tokens": tokens}
        if own:
            from paper_2605_26289_amd import binding as dk
            rows, top = case["rows"], case["top"]
            code = dk.BF16 if case["dtype"] == "bf16" else dk.F32

            def empty(dtype, *shape):
                return torch.empty(shape, dtype=dtype, device="cuda")

            state.update(code=code, stride=buf.shape[1], logprob=empty(torch.float32, rows), rank=empty(torch.int32, rows),
                         entropy=empty(torch.float32, rows), top_ids=empty(torch.int32, rows, top) if top else None,
                         top_logprobs=empty(torch.float32, rows, top) if top else None,
                         ws=empty(torch.uint8, dk.logprobs_workspace_bytes(rows, case["vocab"], code, top)))
        return state
    if case["kind"] in ("rows", "append"):
        t = _rotary_inputs(case, seed)
        state = {"case": case, **t}
        if own:
            from paper_2605_26289_amd import DevicePool
            from paper_2605_26289_amd import binding as dk
            q, k, v = _split(case, t["fused"])
            state.update(q=q, k=k, v=v, q_out=torch.empty(q.shape, dtype=q.dtype, device="cuda"),
                         rotary=dk.Rotary(case["rotary"], t["freqs"], pairs=case["pairs"], amplitude=case["amplitude"],
                                          norm_eps=EPS if case["norm"] else None, q_weight=t["wq"] if case["norm"] else None,
                                          k_weight=t["wk"] if case["norm"] else None))
            if case["kind"] == "rows":
                state.update(k_out=torch.empty(k.shape, dtype=k.dtype, device="cuda"))
                return state
            # granules as long as a session: a session's cells are one run, so what was appended is a slice of the arena
            hist, delta = _lengths(case)
            granule = max(n + new for n, new in zip(hist, delta))
            pool = DevicePool(case["slots"], granule * case["slots"], case["hq"], case["hkv"], case["d"], case["dtype"],
                              granule_cells=granule)
            slots = np.array([pool.acquire() for _ in range(case["slots"])], dtype=np.int32)
            cu, n_past = _offsets(delta), np.array(hist, dtype=np.int64)
            dk.kv_reserve(pool.handle, slots, _offsets(hist))
            cells = dk.kv_reserve(pool.handle, slots, cu)
            pool.trim_batch(slots, n_past)
            new = [slice(int(cells[a]), int(cells[b - 1]) + 1) for a, b in zip(cu[:-1], cu[1:])]
            state.update(pool=pool, slots=slots, cu=cu, n_past=n_past,
                         written=[[arena[:, s] for s in new] for arena in (pool.k_arena, pool.v_arena)])
        return state
    t = _attend_inputs(case, seed)
    hist, delta = _lengths(case)
    prefix, first = _masks(case)
    state = {"case": case, "q": t["q"], "scale": 1.0 / math.sqrt(case["d"]), "slopes": _slopes(case) if case["alibi"] else None}
    if own:
        from paper_2605_26289_amd import DevicePool
        from paper_2605_26289_amd import binding as dk
        n_slots = case["slots"]
        pool = DevicePool(n_slots, sum(hist) + sum(delta) + 512 * (n_slots + 2), case["hq"], case["hkv"], case["d"], case["dtype"])
        slots = np.array([pool.acquire() for _ in range(n_slots)], dtype=np.int32)
        pool.append(slots, _offsets(hist), t["k"], t["v"])
        pool.append(slots, _offsets(delta), t["k_new"], t["v_new"])
        state.update(pool=pool, slots=slots, cu=_offsets(delta), out=torch.empty_like(t["q"]),
                     lse=torch.empty((sum(delta), case["hq"]), dtype=torch.float32, device="cuda"),
                     scores=dk.Scores(cap=case["cap"], slopes=state["slopes"], window=case["window"], prefix=prefix, first=first))
        return state
    cu, ch = _offsets(delta), _offsets(hist)
    state["sessions"] = []
    for b in range(case["slots"]):
        old, new = slice(int(ch[b]), int(ch[b + 1])), slice(int(cu[b]), int(cu[b + 1]))
        lo, hi = _visible(case, b, hist[b], delta[b], prefix, None if first is None else first[new])
        state["sessions"].append((new, torch.cat([t["k"][old], t["k_new"][new]]), torch.cat([t["v"][old], t["v_new"][new]]),
                                  hist[b], lo, hi))
    return state


def _visible(case, b, n, new, prefix, first):
    """First and last position that each of a session's new tokens sees."""
    p = torch.arange(n, n + new, dtype=torch.int64)
    lo, hi = torch.zeros_like(p), p.clone()
    if prefix is not None:
        hi = torch.maximum(p, torch.tensor(prefix[b] - 1))
    if case["window"]:
        lo = torch.maximum(lo, p - case["window"] + 1)
    if first is not None:
        lo = torch.maximum(lo, torch.tensor(first, dtype=torch.int64))
    return lo.cuda(), hi.cuda()


# ---- one pass --------------------------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if case["kind"] == "attend":
        if not own:
            return _plain_attend(state)
        state["pool"].scored_attend(state["slots"], state["cu"], state["q"], state["scale"], state["scores"], out=state["out"],
                                    lse=state["lse"])
        return [state["out"], state["lse"]]
    if case["kind"] == "logprobs":
        if not own:
            return _plain_logprobs(state)
        from paper_2605_26289_amd import binding as dk
        dk.token_logprobs(case["rows"], state["logits"], state["code"], case["vocab"], state["stride"], state["tokens"],
                          state["logprob"], state["ws"], scale=1.0 / case["temperature"], rank_out=state["rank"],
                          entropy_out=state["entropy"], n_top=case["top"], top_ids_out=state["top_ids"],
                          top_logprobs_out=state["top_logprobs"])
        best = [state["top_ids"], state["top_logprobs"]] if case["top"] else []
        return [state["logprob"], state["rank"], state["entropy"]] + best
    if not own:
        return _plain_rotary(state)
    if case["kind"] == "rows":
        from paper_2605_26289_amd import binding as dk
        dk.rotate_rows(state["position"], state["q"], state["k"], state["rotary"], state["q_out"], state["k_out"])
        return [state["q_out"], state["k_out"]]
    pool = state["pool"]
    pool.rotate_append(state["slots"], state["cu"], state["q"], state["k"], state["v"], state["rotary"], out=state["q_out"])
    pool.trim_batch(state["slots"], state["n_past"])
    return [state["q_out"], state["written"][0], state["written"][1]]


def _plain_attend(state):
    case, scale = state["case"], state["scale"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    group = hq // hkv
    out = torch.empty_like(state["q"])
    lse = torch.empty(state["q"].shape[:2], dtype=torch.float32, device="cuda")
    for rows, k, v, n, lo, hi in state["sessions"]:
        keys = k.float().permute(1, 2, 0).contiguous()  # head, depth, position
        values = v.float().transpose(0, 1).contiguous()
        where = torch.arange(k.shape[0], device="cuda")
        new = rows.stop - rows.start
        step = max(1, (1 << 27) // max(1, k.shape[0] * hq))
        for a in range(0, new, step):
            b = min(new, a + step)
            q = state["q"][rows][a:b].float().view(b - a, hkv, group, d).transpose(0, 1).reshape(hkv, (b - a) * group, d)
            s = (torch.matmul(q, keys) * scale).view(hkv, b - a, group, -1)
            if case["cap"]:
                s = torch.tanh(s / case["cap"]) * case["cap"]
            if state["slopes"] is not None:
                far = (where[None, :] - torch.arange(n + a, n + b, device="cuda")[:, None]).abs().float()
                s = s - state["slopes"].view(hkv, 1, group, 1) * far[None, :, None, :]
            seen = (where[None, :] >= lo[a:b, None]) & (where[None, :] <= hi[a:b, None])
            s = s.masked_fill(~seen[None, :, None, :], float("-inf"))
            top = s.amax(dim=3, keepdim=True)
            top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
            p = torch.exp(s - top)
            z = p.sum(dim=3, keepdim=True)
            o = torch.matmul(p.view(hkv, (b - a) * group, -1), values).view(hkv, b - a, group, d)
            o = torch.where(z > 0, o / z, torch.zeros_like(o))
            out[rows][a:b] = o.transpose(0, 1).reshape(b - a, hq, d).to(out.dtype)
            lse[rows][a:b] = (top + torch.log(z)).squeeze(3).transpose(0, 1).reshape(b - a, hq)
    return [out, lse]


def _plain_rotary(state):
    case = state["case"]
    q, k, v = _split(case, state["fused"])
    angle = state["position"].double()[:, None] * state["freqs"].double()[None, :]
    cos = (torch.cos(angle) * case["amplitude"]).float()[:, None, :]
    sin = (torch.sin(angle) * case["amplitude"]).float()[:, None, :]
    r, half = case["rotary"], case["rotary"] // 2
    outs = []
    for x, w in ((q, state["wq"]), (k, state["wk"])):
        y = x.float()
        if case["norm"]:
            y = y * torch.rsqrt((y * y).sum(dim=2, keepdim=True) / case["d"] + EPS) * w.float()
        a, b = (y[:, :, 0:r:2], y[:, :, 1:r:2]) if case["pairs"] else (y[:, :, :half], y[:, :, half:r])
        u, t = a * cos - b * sin, b * cos + a * sin
        turned = torch.stack([u, t], dim=3).flatten(2) if case["pairs"] else torch.cat([u, t], dim=2)
        outs.append(torch.cat([turned, y[:, :, r:]], dim=2).to(x.dtype))
    if case["kind"] == "rows":
        return outs
    cu = _offsets(_lengths(case)[1])
    new = [slice(int(a), int(b)) for a, b in zip(cu[:-1], cu[1:])]
    return [outs[0]] + [[x[s].transpose(0, 1).contiguous() for s in new] for x in (outs[1], v)]


def _plain_logprobs(state):
    case = state["case"]
    x = state["logits"].float()
    scale = 1.0 / case["temperature"]
    t = state["tokens"].long()[:, None]
    given = x.gather(1, t)
    top = x.amax(dim=1, keepdim=True)
    y = (x - top) * scale
    p = torch.exp(y)
    z = p.sum(dim=1, dtype=torch.float64)
    ln_z = torch.log(z).float()
    weighted = torch.where(p > 0, p * y, torch.zeros_like(y)).sum(dim=1, dtype=torch.float64)
    outs = [((given - top) * scale).squeeze(1) - ln_z, (x > given).sum(dim=1).to(torch.int32), (torch.log(z) - weighted / z).float()]
    if case["top"]:
        # whole numbers in the order wanted: by value, then the lower id
        bits = (x + 0.0).view(torch.int32)
        order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 32)
        order += (1 << 31) - 1 - torch.arange(x.shape[1], device="cuda")
        ids = []
        for _ in range(case["top"]):
            best = order.amax(dim=1, keepdim=True)
            at = (1 << 31) - 1 - (best & 0xFFFFFFFF)
            ids.append(at)
            order.scatter_(1, at, torch.iinfo(torch.int64).min)
        ids = torch.cat(ids, dim=1)
        outs += [ids.to(torch.int32), (x.gather(1, ids) - top) * scale - ln_z[:, None]]
    return outs


# ---- what a pass cannot do without -----------------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "logprobs":
        cells = case["rows"] * case["vocab"]
        return {"bytes": cells * e + case["rows"] * (16 + 8 * case["top"]), "flops": 5 * cells}
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["kind"] in ("rows", "append"):
        t = _tokens_of(case)
        moved = hq + hkv if case["kind"] == "rows" else hq + 2 * hkv
        per_head = 3 * case["rotary"] + (4 * d if case["norm"] else 0)
        return {"bytes": 2 * t * moved * d * e, "flops": t * (hq + hkv) * per_head}
    hist, delta = _lengths(case)
    prefix, first = _masks(case)
    keys = pairs = at = 0
    for b, (n, new) in enumerate(zip(hist, delta)):
        low, high = n + new, -1  # the positions that some row sees
        for i in range(new):
            lo, hi = 0, n + i
            if prefix is not None:
                hi = max(hi, prefix[b] - 1)
            if case["window"]:
                lo = max(lo, n + i - case["window"] + 1)
            if first is not None:
                lo = max(lo, first[at + i])
            if lo <= hi:
                pairs += hi - lo + 1
                low, high = min(low, lo), max(high, hi)
        keys += max(0, high - low + 1)
        at += new
    return {"bytes": keys * hkv * d * e * 2 + sum(delta) * hq * (2 * d * e + 4), "flops": 4 * hq * d * pairs}


# ---- the same results in 64 bits -------------------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "logprobs":
        return _exact_logprobs(case, seed)
    if case["kind"] == "attend":
        return _exact_attend(case, seed)
    return _exact_rotary(case, seed)


def _exact_attend(case, seed):
    """Key block by key block a whole head group at a time, weights normalised by their log-sum-exp."""
    t = _attend_inputs(case, seed)
    hist, delta = _lengths(case)
    prefix, first = _masks(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    group, total = hq // hkv, sum(delta)
    out = torch.zeros((total, hq, d), dtype=torch.float64, device="cuda")
    lse = torch.full((total, hq), float("-inf"), dtype=torch.float64, device="cuda")
    cu, ch = _offsets(delta), _offsets(hist)
    slope = [2.0 ** (-8.0 * (h + 1) / hq) for h in range(hq)]
    for b in range(case["slots"]):
        n, new = hist[b], delta[b]
        r0 = int(cu[b])
        k = torch.cat([t["k"][int(ch[b]):int(ch[b + 1])], t["k_new"][r0:r0 + new]]).double()
        v = torch.cat([t["v"][int(ch[b]):int(ch[b + 1])], t["v_new"][r0:r0 + new]]).double()
        key = torch.arange(n + new, device="cuda")
        for a in range(0, new, 128):
            c = min(new, a + 128)
            pos = torch.arange(n + a, n + c, device="cuda")
            last = pos if prefix is None else pos.clamp(min=prefix[b] - 1)
            hidden = key[None, :] > last[:, None]
            if case["window"]:
                hidden |= pos[:, None] - key[None, :] >= case["window"]
            if first is not None:
                hidden |= key[None, :] < torch.tensor(first[r0 + a:r0 + c], device="cuda")[:, None]
            apart = (pos[:, None] - key[None, :]).abs().double()
            for h in range(hq):
                s = t["q"][r0 + a:r0 + c, h].double() @ k[:, h // group].t() / math.sqrt(d)
                if case["cap"]:
                    s = case["cap"] * torch.tanh(s / case["cap"])
                if case["alibi"]:
                    s = s - float(np.float32(slope[h])) * apart
                s = s.masked_fill(hidden, float("-inf"))
                norm = torch.logsumexp(s, dim=1)
                lse[r0 + a:r0 + c, h] = norm
                w = torch.exp(s - norm.clamp(min=-1e300)[:, None])
                out[r0 + a:r0 + c, h] = w @ v[:, h // group]
    return [out, lse]


def _exact_rotary(case, seed):
    """Each pair as a complex number times one of modulus `amplitude`."""
    t = _rotary_inputs(case, seed)
    hq, hkv, d, r = case["hq"], case["hkv"], case["d"], case["rotary"]
    x = t["fused"].double().view(-1, hq + 2 * hkv, d)
    turn = torch.polar(torch.full((x.shape[0], r // 2), float(case["amplitude"]), dtype=torch.float64, device="cuda"),
                       t["position"].double()[:, None] * t["freqs"].double()[None, :])[:, None, :]
    outs = []
    for y, w in ((x[:, :hq], t["wq"]), (x[:, hq:hq + hkv], t["wk"])):
        if case["norm"]:
            y = y / torch.sqrt(y.square().mean(dim=2, keepdim=True) + EPS) * w.double()
        else:
            y = y.clone()
        if case["pairs"]:
            z = torch.complex(y[..., 0:r:2], y[..., 1:r:2]) * turn
            y[..., 0:r:2], y[..., 1:r:2] = z.real, z.imag
        else:
            z = torch.complex(y[..., :r // 2], y[..., r // 2:r]) * turn
            y[..., :r // 2], y[..., r // 2:r] = z.real, z.imag
        outs.append(y)
    if case["kind"] == "rows":
        return outs
    cuts = [int(c) for c in _offsets(_lengths(case)[1])]
    return [outs[0]] + [[y[a:b].transpose(0, 1) for a, b in zip(cuts[:-1], cuts[1:])] for y in (outs[1], x[:, hq + hkv:])]


def _exact_logprobs(case, seed):
    _, logits, tokens = _logit_inputs(case, seed)
    rows, top = case["rows"], case["top"]
    logprob, entropy = [torch.empty(rows, dtype=torch.float64, device="cuda") for _ in range(2)]
    best = torch.empty((rows, top), dtype=torch.float64, device="cuda")
    for a in range(0, rows, 256):
        b = min(rows, a + 256)
        ln_p = torch.log_softmax(logits[a:b].double() / case["temperature"], dim=1)
        logprob[a:b] = ln_p[torch.arange(b - a, device="cuda"), tokens[a:b].long()]
        entropy[a:b] = -(torch.exp(ln_p) * ln_p.clamp(min=-1e300)).sum(dim=1)
        if top:
            best[a:b] = torch.sort(ln_p, dim=1, descending=True).values[:, :top]
    return [logprob, None, entropy] + ([None, best] if top else [])
