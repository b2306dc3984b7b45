"""The operators of batches that continue shared prompts: what they compute, in plain torch, and how they are called.

A case is a dict of plain values.  `listed()` names some, `draw()` gives more from the same ranges; `prepare` makes what a
serving loop holds before the call, `run` is one pass -- with `own` through the framework's entry points, without it in
elementary torch operations -- and `exact` the same results in float64, written from the definitions.

Kinds of case:
  attend  attention of a batch whose sessions share the beginnings of their caches: a prefix for each group, perhaps a second one
          for each of its subgroups, then tokens of their own
  step    a step of beam search in the cache: every beam takes over its parent's state, its new token is appended and attended
  select  the best continuations of each request's beams, by cumulative log probability
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False


def _attend(name, **kw):
    case = {"kind": "attend", "hq": 32, "hkv": 8, "d": 128, "dtype": "bf16", "groups": 1, "size_lo": 1, "size_hi": 1,
            "prefix_lo": 0, "prefix_hi": 0, "subs": 0, "sub_lo": 0, "sub_hi": 0, "tail_lo": 0, "tail_hi": 0, "delta_lo": 1,
            "delta_hi": 1, "staged": False, "lens": 1}
    case.update(kw)
    if name:
        case["name"] = name
    return case


def _step(name, **kw):
    return _attend(name, **{"kind": "step", **kw})


def _select(name, **kw):
    case = {"kind": "select", "groups": 1, "size_lo": 4, "size_hi": 4, "vocab": 128256, "dtype": "bf16", "n": 8, "temperature": 1.0,
            "guided": False, "first": False, "lens": 1}
    case.update(kw)
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # Four samples of one answer, token by token, behind one prompt: the smallest call, latency and launches.
        _attend("attend_samples", size_lo=4, size_hi=4, prefix_lo=3000, prefix_hi=3000, tail_lo=20, tail_hi=60),
        # 64 agents decoding behind one preamble, each with a history of its own.
        _attend("attend_agents", size_lo=64, size_hi=64, prefix_lo=8192, prefix_hi=8192, tail_lo=100, tail_hi=1000, lens=2),
        # Speculative verification of 32 sessions about one long document, the candidates' K and V still outside the cache.
        _attend("attend_verify", size_lo=32, size_hi=32, prefix_lo=30000, prefix_hi=30000, tail_lo=50, tail_hi=400, delta_lo=1,
                delta_hi=9, staged=True, lens=3),
        # 64-wide heads: three preambles, tool descriptions for subgroups behind them, decoding and verifying sessions.
        _attend("attend_tree_heads64", d=64, groups=3, size_lo=12, size_hi=20, prefix_lo=1000, prefix_hi=3000, subs=3, sub_lo=300,
                sub_hi=1500, tail_lo=0, tail_hi=300, delta_lo=1, delta_hi=9, lens=4),
        # Turns of 16 agents behind one preamble: the large products.
        _attend("attend_turns", size_lo=16, size_hi=16, prefix_lo=4096, prefix_hi=4096, tail_lo=100, tail_hi=1000, delta_lo=64,
                delta_hi=512, lens=5),
        # Validation in fp32: samples of two prompts.
        _attend("attend_f32", hq=8, hkv=2, dtype="f32", groups=2, size_lo=6, size_hi=12, prefix_lo=500, prefix_hi=2000, tail_lo=0,
                tail_hi=200, delta_lo=1, delta_hi=20, lens=6),
        # One user's beam search, a step of its cache: latency and launches.
        _step("step_one", size_lo=4, size_hi=4, prefix_lo=3000, prefix_hi=3000, tail_lo=60, tail_hi=60, lens=7),
        # 16 requests of eight beams.
        _step("step_many", groups=16, size_lo=8, size_hi=8, prefix_lo=1000, prefix_hi=4000, tail_lo=100, tail_hi=600, lens=8),
        # Wide beams with seven heads to a KV head.
        _step("step_wide", hq=28, hkv=4, groups=4, size_lo=20, size_hi=32, prefix_lo=300, prefix_hi=2000, tail_lo=1, tail_hi=300, lens=9),
        # One request's four beams: latency and launches.
        _select("select_one"),
        # 64 requests of eight beams, twice as many continuations so that ended ones can be set aside.
        _select("select_many", groups=64, size_lo=8, size_hi=8, n=16),
        # Requests of one to ten beams held to a grammar: fp32 logits, an odd vocabulary.
        _select("select_f32", groups=40, size_lo=1, size_hi=10, vocab=50003, dtype="f32", n=20, temperature=0.7, guided=True, lens=10),
    ]


def _between(rng, lo, hi):
    """A whole number spread evenly over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


HEADS = [(32, 8, 128), (32, 8, 64), (16, 4, 64), (14, 2, 64), (12, 2, 128), (28, 4, 128), (8, 8, 128), (16, 2, 128), (16, 1, 128)]
HEADS_F32 = [(4, 1, 64), (4, 2, 64), (8, 2, 64), (8, 2, 128), (16, 4, 128)]


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "step", "step", "select", "select"])
    lens = rng.randrange(1, 1 << 30)
    if kind == "select":
        dtype = rng.choice(["bf16", "f32"])
        vocab = rng.choice([8 * rng.randint(4000, 16032), rng.randint(1000, 128256)])
        size = _between(rng, 1, 32)
        groups = _between(rng, 1, max(1, min(64, 65000000 // (vocab * size))))
        return _select(None, groups=groups, size_lo=rng.randint(1, size), size_hi=size, vocab=vocab, dtype=dtype,
                       n=min(64, rng.choice([size, 2 * size, rng.randint(1, 64)])), temperature=rng.choice([1.0, 0.7, rng.uniform(0.3, 1.5)]),
                       guided=rng.random() < 0.3, first=rng.random() < 0.2, lens=lens)
    f32 = rng.random() < 0.25
    hq, hkv, d = rng.choice(HEADS_F32 if f32 else HEADS)
    shape = {"hq": hq, "hkv": hkv, "d": d, "dtype": "f32" if f32 else "bf16", "lens": lens}
    if kind == "step":
        size = _between(rng, 1, 8 if f32 else 32)
        groups = _between(rng, 1, max(1, (16 if f32 else 128) // size))
        prefix = _between(rng, 20, min(4000 if f32 else 30000, 60000 // groups))
        tail = _between(rng, 1, 400 if f32 else 1000)
        return _step(None, groups=groups, size_lo=rng.randint(1, size), size_hi=size, prefix_lo=prefix // 4 + 1, prefix_hi=prefix,
                     tail_lo=tail // 4, tail_hi=tail, **shape)
    turns = rng.random() < 0.3
    size = _between(rng, 1, 12 if turns else 16 if f32 else 64)
    groups = _between(rng, 1, max(1, (12 if turns else 16 if f32 else 64) // size))
    prefix = _between(rng, 20, min(2000, 8000 // groups) if turns else min(4000, 16000 // groups) if f32 else 32000 // groups)
    subs = rng.choice([0, 0, rng.randint(1, 4)])
    sub = _between(rng, 20, prefix) if subs else 0
    tail = rng.choice([0, _between(rng, 1, 1000 if not f32 else 300)])
    delta = _between(rng, 10, 100 if f32 else 3000 // (size * groups) + 10) if turns else rng.choice([1, rng.randint(1, 9)])
    return _attend(None, groups=groups, size_lo=rng.randint(1, size), size_hi=size, prefix_lo=prefix // 4, prefix_hi=prefix, subs=subs,
                   sub_lo=sub // 4, sub_hi=sub, tail_lo=tail // 8, tail_hi=tail, delta_hi=delta, staged=rng.random() < 0.3, **shape)


# ---- what a case is made of ------------------------------------------------------------------------------------------
def _plan(case):
    """Lengths and places by the case alone.  Sessions are in the batch's order: `group` and `sub` of each (-1: none), lengths of
    the groups' prefixes, the subgroups' and the sessions' own cached tokens, new tokens of each, the steps' parents."""
    rng = random.Random(case["lens"])
    sizes = [rng.randint(case["size_lo"], case["size_hi"]) for _ in range(case["groups"])]
    sessions = [(g, rng.randrange(case["subs"]) if case["subs"] else -1) for g, size in enumerate(sizes) for _ in range(size)]
    if case["kind"] == "attend":  # sessions come as they come; beams are next to one another
        rng.shuffle(sessions)
    prefix = [rng.randint(case["prefix_lo"], case["prefix_hi"]) for _ in sizes]
    sub = [rng.randint(case["sub_lo"], case["sub_hi"]) for _ in sizes for _ in range(case["subs"])]
    if case["kind"] == "step":  # beams of a request are equally long
        same = [rng.randint(case["tail_lo"], case["tail_hi"]) for _ in sizes]
        tail = [same[g] for g, _ in sessions]
    else:
        tail = [rng.randint(case["tail_lo"], case["tail_hi"]) for _ in sessions]
    delta = [rng.randint(case["delta_lo"], case["delta_hi"]) for _ in sessions]
    first = {}
    for i, (g, _) in enumerate(sessions):
        first.setdefault(g, i)
    parents = [[first[g] + min(rng.randrange(sizes[g]), rng.randrange(sizes[g])) for g, _ in sessions] if case["kind"] == "step" else []
               for _ in range(8)]  # the better beams have more children
    return {"group": [g for g, _ in sessions], "sub": [g * case["subs"] + s if s >= 0 else -1 for g, s in sessions], "prefix": prefix,
            "subs": sub, "tail": tail, "delta": delta, "parents": parents}


def _offsets(lengths):
    return np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    return gen


def _attend_inputs(case, seed):
    """Caches as [owner, position, head, depth] of the groups, subgroups and sessions, each as wide as its longest; new rows packed."""
    gen, dt = _generator(seed), _type(case)
    plan = _plan(case)
    hkv, hq, d = case["hkv"], case["hq"], case["d"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dt)

    tokens = sum(plan["delta"])
    t = {"plan": plan, "q": normal(tokens, hq, d) * 2, "k_new": normal(tokens, hkv, d), "v_new": normal(tokens, hkv, d)}
    for name, lengths in (("prefix", plan["prefix"]), ("subs", plan["subs"]), ("tail", plan["tail"])):
        for x in "kv":
            t[name + "_" + x] = normal(len(lengths), max(lengths, default=0), hkv, d)
    return t


def _rows(case):
    """Beams of every request."""
    rng = random.Random(case["lens"])
    return [rng.randint(case["size_lo"], case["size_hi"]) for _ in range(case["groups"])]


def _select_inputs(case, seed):
    gen, dt = _generator(seed), _type(case)
    sizes, vocab = _rows(case), case["vocab"]
    rows = sum(sizes)
    stride = (vocab + 7) // 8 * 8  # rows start at whole 16 bytes
    buf = torch.randn((rows, stride), generator=gen, device="cuda", dtype=dt) * 2.5
    logits = buf[:, :vocab]
    if case["guided"]:  # every third row: only a few tokens are allowed
        allowed = torch.rand((rows, vocab), generator=gen, device="cuda") < 0.002
        allowed[:, 0] = True
        shut = (torch.arange(rows, device="cuda") % 3 == 1)[:, None] & ~allowed
        logits.masked_fill_(shut, float("-inf"))
    scores = torch.randn((rows,), generator=gen, device="cuda") * 2 - 20
    if case["first"]:  # a request's first step: its beams are still alike, one of them counts
        starts = torch.tensor(_offsets(sizes)[:-1].astype(np.int64), device="cuda")
        begun = torch.full_like(scores, float("-inf"))
        begun[starts] = scores[starts]
        scores = begun
    return sizes, buf, logits, scores


def _index(values):
    return torch.tensor(values, dtype=torch.int64, device="cuda")


def prepare(case, seed):
    if case["kind"] == "select":
        sizes, buf, logits, scores = _select_inputs(case, seed)
        state = {"case": case, "logits": logits, "scores": scores, "cu": torch.tensor(_offsets(sizes), device="cuda"),
                 "beam": _index([i for size in sizes for i in range(size)]), "group": _index([g for g, size in enumerate(sizes) for _ in range(size)])}
        if own:
            from paper_2605_26289_amd import binding as dk
            rows, n = len(scores), case["n"]
            code = dk.BF16 if case["dtype"] == "bf16" else dk.F32
            out = [torch.empty((len(sizes), n), dtype=t, device="cuda") for t in (torch.int32, torch.int32, torch.float32)]
            state.update(code=code, stride=buf.shape[1], out=out,
                         ws=torch.empty(dk.beam_workspace_bytes(rows, case["vocab"], code, n), dtype=torch.uint8, device="cuda"))
        return state
    t = _attend_inputs(case, seed)
    plan = t["plan"]
    sessions, cu = len(plan["delta"]), _offsets(plan["delta"])
    state = {"case": case, **t, "scale": 1.0 / math.sqrt(case["d"]), "turn": 0, "parents_dev": [_index(p) for p in plan["parents"]]}
    if own:
        from paper_2605_26289_amd import DevicePool
        n_nodes = len(plan["prefix"]) + len(plan["subs"]) + sessions
        cells = sum(plan["prefix"]) + sum(plan["subs"]) + sum(plan["tail"]) + sum(plan["delta"]) + 512 * (n_nodes + sessions + 4)
        pool = DevicePool(n_nodes, cells, case["hq"], case["hkv"], case["d"], case["dtype"])
        state.update(pool=pool, cu=cu, out=torch.empty_like(t["q"]),
                     lse=torch.empty((int(cu[-1]), case["hq"]), dtype=torch.float32, device="cuda"))
        _fill(state)
        return state
    # where each token is among those of its group, its subgroup and its session
    state["levels"] = []
    for name, of in (("prefix", plan["group"]), ("subs", plan["sub"]), ("tail", range(sessions))):
        if not len(plan[name]) or not max(plan[name]):
            continue
        seen, place = [0] * len(plan[name]), []
        for b, new in enumerate(plan["delta"]):
            place += range(seen[of[b]], seen[of[b]] + new)
            seen[of[b]] += new
        node = [of[b] for b, new in enumerate(plan["delta"]) for _ in range(new)]
        state["levels"].append((name, _index(node), _index(place), max(seen), _index(plan[name])))
    state["session"] = _index([b for b, new in enumerate(plan["delta"]) for _ in range(new)])
    state["turn_of"] = _index([i for new in plan["delta"] for i in range(new)])
    return state


def _fill(state):
    """The pool as a serving loop has it: the groups' prefixes in sequences of their own, everything behind them through aliases."""
    pool, plan, staged = state["pool"], state["plan"], state["case"]["staged"]

    def put(slot, name, i):
        length = plan[name][i]
        if length:
            pool.append([slot], [0, length], state[name + "_k"][i, :length], state[name + "_v"][i, :length])

    roots = [pool.acquire() for _ in plan["prefix"]]
    for g, slot in enumerate(roots):
        put(slot, "prefix", g)
    branches = [pool.acquire() for _ in plan["subs"]]
    per = state["case"]["subs"]
    for i, slot in enumerate(branches):
        pool.alias(roots[i // per], slot, plan["prefix"][i // per])
        put(slot, "subs", i)
    slots = []
    for b, (g, s) in enumerate(zip(plan["group"], plan["sub"])):
        slot, donor = pool.acquire(), branches[s] if s >= 0 else roots[g]
        pool.alias(donor, slot, plan["prefix"][g] + (plan["subs"][s] if s >= 0 else 0))
        put(slot, "tail", b)
        slots.append(slot)
    state["slots"] = np.array(slots, dtype=np.int32)
    state["n_past"] = np.array([pool.length(s) for s in slots], dtype=np.int64)
    if state["case"]["kind"] == "attend" and not staged:
        pool.append(state["slots"], state["cu"], state["k_new"], state["v_new"])


# ---- one pass --------------------------------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    if case["kind"] == "select":
        if not own:
            return _plain_select(state)
        from paper_2605_26289_amd import binding as dk
        row, token, score = state["out"]
        dk.beam_select(case["groups"], len(state["scores"]), state["cu"], state["logits"], state["code"], case["vocab"], state["stride"],
                       state["scores"], case["n"], row, token, score, state["ws"], scale=1.0 / case["temperature"])
        return [row, token, score]
    turn = state["turn"]
    state["turn"] = (turn + 1) % 8
    if not own:
        if case["kind"] == "step":
            for x in ("tail_k", "tail_v"):
                state[x] = state[x][state["parents_dev"][turn]]
        return _plain_attend(state)
    pool, slots, cu = state["pool"], state["slots"], state["cu"]
    if case["kind"] == "step":
        pool.reorder(slots, state["plan"]["parents"][turn])
        pool.append(slots, cu, state["k_new"], state["v_new"])
    new = (state["k_new"], state["v_new"]) if case["staged"] else (None, None)
    pool.shared_attend(slots, cu, state["q"], state["scale"], *new, out=state["out"], lse=state["lse"])
    if case["kind"] == "step":
        pool.trim_batch(slots, state["n_past"])  # the same step again in the next pass
    return [state["out"], state["lse"]]


def _part(case, scale, q, k, v, seen):
    """Largest score, sum of weights and weighted sum of values: q [nodes, tokens, heads, depth] against k, v [nodes, positions, KV
    heads, depth], seen [nodes, tokens or 1, positions]."""
    nodes, tokens, hq, d = q.shape
    hkv, n = k.shape[2], k.shape[1]
    q = q.view(nodes, tokens, hkv, hq // hkv, d).transpose(1, 2).reshape(nodes, hkv, -1, d)
    s = torch.matmul(q, k.float().permute(0, 2, 3, 1).contiguous()) * scale
    s = s.view(nodes, hkv, tokens, hq // hkv, n).masked_fill(~seen[:, None, :, None, :], float("-inf"))
    top = s.amax(dim=4, keepdim=True)
    p = torch.exp(s - torch.where(top == float("-inf"), torch.zeros_like(top), top))
    z = p.sum(dim=4, keepdim=True)
    o = torch.matmul(p.view(nodes, hkv, -1, n), v.float().transpose(1, 2).contiguous()).view(nodes, hkv, tokens, hq // hkv, d)
    return [x.transpose(1, 2).reshape(nodes, tokens, hq, -1) for x in (top, z, o)]


def _plain_attend(state):
    """Prefixes once for all rows behind them, then the sessions' own tokens, joined by their log-sum-exp."""
    case, scale, q = state["case"], state["scale"], state["q"].float()
    parts = []
    for name, node, place, width, lengths in state["levels"]:
        k, v = state[name + "_k"], state[name + "_v"]
        grid = torch.zeros((k.shape[0], width) + q.shape[1:], device="cuda")
        grid[node, place] = q
        seen = torch.arange(k.shape[1], device="cuda")[None, None, :] < lengths[:, None, None]
        parts.append([x[node, place] for x in _part(case, scale, grid, k, v, seen)])
    session, turn = state["session"], state["turn_of"]
    most = max(state["plan"]["delta"])

    def spread(x):
        grid = torch.zeros((len(state["plan"]["delta"]), most) + x.shape[1:], dtype=x.dtype, device="cuda")
        grid[session, turn] = x
        return grid

    where = torch.arange(most, device="cuda")
    causal = (where[None, :] <= where[:, None])[None].expand(len(state["plan"]["delta"]), most, most)
    parts.append([x[session, turn] for x in _part(case, scale, spread(q), spread(state["k_new"]), spread(state["v_new"]), causal)])
    top = torch.stack([m for m, _, _ in parts]).amax(dim=0)
    weights = [torch.exp(m - top) for m, _, _ in parts]
    z = sum(w * x for w, (_, x, _) in zip(weights, parts))
    o = sum(w * x for w, (_, _, x) in zip(weights, parts)) / z
    return [o.to(state["q"].dtype), (top + torch.log(z)).squeeze(2)]


def _plain_select(state):
    case, n = state["case"], state["case"]["n"]
    x, group, beam = state["logits"].float(), state["group"], state["beam"]
    scale = 1.0 / case["temperature"]
    top = x.amax(dim=1, keepdim=True)
    ln_z = torch.log(torch.exp((x - top) * scale).sum(dim=1, dtype=torch.float64))
    # a row's best: whole numbers in the order wanted, by value, then the lower id
    bits = (x + 0.0).view(torch.int32)
    order = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits).long() * (1 << 32) + (1 << 31) - 1 - torch.arange(x.shape[1], device="cuda")
    best = min(n, x.shape[1])
    ids = (1 << 31) - 1 - (torch.topk(order, best, dim=1).values & 0xFFFFFFFF)
    value = state["scores"].double()[:, None] + (x.gather(1, ids) - top).double() * scale - ln_z[:, None]
    # the best of a request's beams, rows and ranks in order
    widest = case["size_hi"] * best
    grid = torch.full((case["groups"], max(widest, n)), float("-inf"), dtype=torch.float64, device="cuda")
    at = beam[:, None] * best + torch.arange(best, device="cuda")[None, :]
    grid[group[:, None], at] = value
    value, place = torch.sort(grid, dim=1, descending=True, stable=True)
    value, place = value[:, :n], place[:, :n]
    none = value == float("-inf")
    row = torch.where(none, torch.zeros_like(place), place // best + state["cu"][:-1].long()[:, None])
    token = ids[row, place % best]
    return [torch.where(none, -1, row).to(torch.int32), torch.where(none, -1, token).to(torch.int32), value.float()]


# ---- what a pass cannot do without -----------------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "select":
        cells = sum(_rows(case)) * case["vocab"]
        return {"bytes": cells * e + sum(_rows(case)) * 4 + case["groups"] * case["n"] * 12, "flops": 4 * cells}
    plan = _plan(case)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    tokens = sum(plan["delta"])
    keys = sum(plan["prefix"]) + sum(plan["subs"][i] for i in set(plan["sub"]) if i >= 0) + sum(plan["tail"]) + tokens
    pairs = 0
    for g, s, tail, new in zip(plan["group"], plan["sub"], plan["tail"], plan["delta"]):
        pairs += new * (plan["prefix"][g] + (plan["subs"][s] if s >= 0 else 0) + tail) + new * (new + 1) // 2
    moved = 2 * tokens * hkv * d * e if case["kind"] == "step" else 0  # the new tokens' K and V into the cache
    return {"bytes": 2 * keys * hkv * d * e + tokens * hq * (2 * d * e + 4) + moved, "flops": 4 * hq * d * pairs}


# ---- the same results in 64 bits -------------------------------------------------------------------------------------
def exact(case, seed):
    return _exact_select(case, seed) if case["kind"] == "select" else _exact_attend(case, seed)


def _exact_attend(case, seed):
    """Session by session and head by head over all it sees, weights normalised by their log-sum-exp."""
    t = _attend_inputs(case, seed)
    plan = t["plan"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    cu = _offsets(plan["delta"])
    out = torch.empty((int(cu[-1]), hq, d), dtype=torch.float64, device="cuda")
    lse = torch.empty((int(cu[-1]), hq), dtype=torch.float64, device="cuda")
    for b, (g, s) in enumerate(zip(plan["group"], plan["sub"])):
        a, c = int(cu[b]), int(cu[b + 1])
        from_whom = plan["parents"][0][b] if case["kind"] == "step" else b
        whole = []
        for x in "kv":
            pieces = [t["prefix_" + x][g, :plan["prefix"][g]]] + ([t["subs_" + x][s, :plan["subs"][s]]] if s >= 0 else [])
            whole.append(torch.cat(pieces + [t["tail_" + x][from_whom, :plan["tail"][b]], t[x + "_new"][a:c]]).double())
        k, v = whole
        n = k.shape[0] - (c - a)
        hidden = torch.arange(k.shape[0], device="cuda")[None, :] > torch.arange(n, n + c - a, device="cuda")[:, None]
        for h in range(hq):
            score = (t["q"][a:c, h].double() @ k[:, h * hkv // hq].t() / math.sqrt(d)).masked_fill(hidden, float("-inf"))
            lse[a:c, h] = torch.logsumexp(score, dim=1)
            out[a:c, h] = torch.exp(score - lse[a:c, h, None]) @ v[:, h * hkv // hq]
    return [out, lse]


def _exact_select(case, seed):
    """Every continuation of a request in one list."""
    sizes, _, logits, scores = _select_inputs(case, seed)
    n, cu = case["n"], _offsets(sizes)
    best = torch.full((len(sizes), n), float("-inf"), dtype=torch.float64, device="cuda")
    for g in range(len(sizes)):
        a, b = int(cu[g]), int(cu[g + 1])
        every = torch.log_softmax(logits[a:b].double() / case["temperature"], dim=1) + scores[a:b].double()[:, None]
        most = min(n, every.numel())
        best[g, :most] = torch.sort(every.reshape(-1), descending=True).values[:most]
    return [None, None, best]
