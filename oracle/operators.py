"""Plain fp64 definitions of the operators around delta attention (test oracle).

  scored_attend    attention of new tokens with capped scores, a bias by distance, and a range of positions for every row
  rotate           norm of a head and its rotation by position
  token_logprobs   log probability and rank of a token, entropy, best alternatives of a logits row
  beam_select      the best continuations of groups of rows

Everything is float64, loop by loop, with no tiling, fusion or reordering.
"""
from __future__ import annotations

import math
from typing import Optional

import numpy as np


def scored_attend(q, k_all, v_all, n: int, scale: float, cap: float = 0.0, slopes=None, window: int = 0, prefix: int = 0, first=None):
    """q [Delta, Hq, D], k_all / v_all [n + Delta, Hkv, D]: row i is position n + i.

    Returns (O, LSE, A, S): A [Delta, Hq, D] is the softmax of the same weights over |V| and S [Delta, Hq] the largest
    |scale| sum |q_d k_d| among the visible keys -- what bounds on rounding are made of."""
    q, k_all, v_all = (np.asarray(x, dtype=np.float64) for x in (q, k_all, v_all))
    delta, hq, d = q.shape
    total, hkv, _ = k_all.shape
    group = hq // hkv
    out, mag = np.zeros((delta, hq, d)), np.zeros((delta, hq, d))
    lse, size = np.full((delta, hq), -np.inf), np.zeros((delta, hq))
    for i in range(delta):
        p = n + i
        lo = 0 if first is None else int(first[i])
        if window:
            lo = max(lo, p - window + 1)
        hi = min(max(p, prefix - 1), total - 1)
        if lo > hi:
            continue
        keys = np.arange(lo, hi + 1)
        for h in range(hq):
            k, v = k_all[lo:hi + 1, h // group], v_all[lo:hi + 1, h // group]
            s = scale * (k @ q[i, h])
            if cap > 0:
                s = cap * np.tanh(s / cap)
            if slopes is not None:
                s = s - float(slopes[h]) * np.abs(p - keys)
            m = s.max()
            w = np.exp(s - m)
            z = w.sum()
            out[i, h] = (w / z) @ v
            mag[i, h] = (w / z) @ np.abs(v)
            lse[i, h] = m + math.log(z)
            size[i, h] = abs(scale) * (np.abs(k) @ np.abs(q[i, h])).max()
    return out, lse, mag, size


def rotate(x, positions, inv_freq, rotary_dim: int, pairs: bool, amplitude: float = 1.0, eps: Optional[float] = None, weight=None):
    """x [tokens, heads, D] -> (turned rows, the rows before the turn)."""
    y = np.array(x, dtype=np.float64)
    if eps is not None:
        y = y / np.sqrt((y ** 2).mean(axis=2, keepdims=True) + eps)
        if weight is not None:
            y = y * np.asarray(weight, dtype=np.float64)
    out = y.copy()
    half = rotary_dim // 2
    for t in range(y.shape[0]):
        for i in range(half):
            # (the product of a whole number and a float32, exactly; then its whole turns are taken out in long arithmetic)
            angle = float(np.longdouble(int(positions[t])) * np.longdouble(np.float32(inv_freq[i])) % (2 * np.longdouble(math.pi)))
            c, s = math.cos(angle), math.sin(angle)
            a, b = (2 * i, 2 * i + 1) if pairs else (i, i + half)
            out[t, :, a] = amplitude * (y[t, :, a] * c - y[t, :, b] * s)
            out[t, :, b] = amplitude * (y[t, :, b] * c + y[t, :, a] * s)
    return out, y


def token_logprobs(logits, tokens, scale: float = 1.0, n_top: int = 0):
    """(log probabilities, ranks, entropies, top ids, top log probabilities) of a [rows, vocab] array."""
    x = np.asarray(logits, dtype=np.float64)
    rows, vocab = x.shape
    key = np.where(np.isnan(x), np.inf, x)
    lp, rank, ent = np.full(rows, -np.inf), np.full(rows, vocab, dtype=np.int64), np.empty(rows)
    ids, tlp = np.zeros((rows, n_top), dtype=np.int64), np.zeros((rows, n_top))
    for r in range(rows):
        sound = np.isfinite(key[r].max())
        if sound:
            y = scale * (x[r] - x[r].max())
            ln_p = y - math.log(np.exp(y).sum())
            keep = np.exp(ln_p) > 0
            ent[r] = -(np.exp(ln_p[keep]) * ln_p[keep]).sum()
        else:
            ln_p = np.full(vocab, np.nan)
            ent[r] = np.nan
        if 0 <= tokens[r] < vocab:
            lp[r] = ln_p[tokens[r]]
            rank[r] = int((key[r] > key[r][tokens[r]]).sum())
        ids[r] = np.lexsort((np.arange(vocab), -key[r]))[:n_top]
        tlp[r] = ln_p[ids[r]]
    return lp, rank, ent, ids, tlp


def beam_select(logits, scores, cu_rows, n_out: int, scale: float = 1.0):
    """(rows, tokens, scores) [groups, n_out]: every continuation of a group's live rows in one list, best first; equal ones by row, then
    logit, then token."""
    x = np.asarray(logits, dtype=np.float64)
    groups = len(cu_rows) - 1
    rows, tokens = np.full((groups, n_out), -1, dtype=np.int64), np.full((groups, n_out), -1, dtype=np.int64)
    best = np.full((groups, n_out), -np.inf)
    for g in range(groups):
        every = []
        for r in range(cu_rows[g], cu_rows[g + 1]):
            if not np.isfinite(scores[r]) or np.isnan(x[r]).any() or not np.isfinite(x[r].max()):
                continue
            y = scale * (x[r] - x[r].max())
            ln_z = math.log(np.exp(y).sum())
            every += [(float(scores[r]) + (y[t] - ln_z), -r, x[r][t], -t) for t in range(x.shape[1]) if x[r][t] > -np.inf]
        every.sort(reverse=True)
        for j, (s, r, _, t) in enumerate(every[:n_out]):
            rows[g, j], tokens[g, j], best[g, j] = -r, -t, s
    return rows, tokens, best
