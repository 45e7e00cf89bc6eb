"""Oracle of the operators around the 4-bit cache and behind the head: rotary positions, weight per cached token, eviction, log probabilities, in numpy and 64 bits.

Written from the definitions of include/bnn.h; caches and plans as in oracle/cache4.py.
"""
from __future__ import annotations

import numpy as np

from . import cache4 as oc


def rotate(x, positions, frequencies, neighbours=False, magnitude=1.0, inverse=False):
    """x [tokens][heads][dim] -> the same in 64 bits."""
    x = np.array(x, np.float64)
    pairs = len(frequencies)
    first = np.arange(pairs) * 2 if neighbours else np.arange(pairs)
    second = first + 1 if neighbours else first + pairs
    angle = np.asarray(positions, np.float64)[:, None] * np.asarray(frequencies, np.float64)[None]
    if inverse:
        angle = -angle
    c, s = magnitude * np.cos(angle)[:, None], magnitude * np.sin(angle)[:, None]
    a, b = x[..., first].copy(), x[..., second].copy()
    x[..., first], x[..., second] = a * c - b * s, a * s + b * c
    return x


def rows_of(lens, start, tokens):
    """(row, sequence, its token) of every row inside a sequence."""
    each = tokens // max(len(lens), 1)
    for b, length in enumerate(lens):
        lo, hi = (b * each, (b + 1) * each) if start is None else (int(start[b]), int(start[b + 1]))
        for t in range(lo, hi):
            yield t, b, int(length) - (hi - lo) + t - lo


def weigh(cache, q, lse, table, lens, start, scale, out, causal=True, window=0, previous=None, decay=1.0):
    """Into out [batch][kv_heads][width]; also returns what bounds the error: for every entry the sum over its rows of weight * (magnitude of the products, and of the logarithm)."""
    tokens, heads = lse.shape
    group = heads // cache.heads
    room = table.shape[1] * cache.page
    spread = np.zeros(out.shape)
    counts = np.zeros(len(lens), int)
    for _, b, _ in rows_of(lens, start, tokens):
        counts[b] += 1
    for b, length in enumerate(lens):
        n = min(max(int(length), 0), room)
        new = max(int(length), 0) - counts[b]
        out[b, :, :n] = 0
        if previous is not None:
            old = min(max(new, 0), n)
            out[b, :, :old] = decay * previous[b, :, :old]
    values = {}
    for t, b, token in rows_of(lens, start, tokens):
        n = min(max(int(lens[b]), 0), room)
        at = np.arange(n)
        seen = np.ones(n, bool)
        if causal:
            seen &= at <= token
        if window:
            seen &= at > token - window
        for h in range(cache.heads):
            if (b, h) not in values:
                records = [cache.record(table, b, j, h) for j in range(n)]
                there = np.array([r is not None for r in records], bool)
                values[b, h] = there, np.array([r.get("k", j % cache.page) if r is not None else np.zeros(cache.dim) for j, r in enumerate(records)]).reshape(n, cache.dim)
            there, k = values[b, h]
            use = np.flatnonzero(seen & there)
            for g in range(group):
                x, log = q[t, h * group + g], lse[t, h * group + g]
                with np.errstate(all="ignore"):
                    w = np.zeros(len(use)) if log == -np.inf else np.exp(scale * (k[use] @ x) - log)
                    out[b, h, use] += w
                    spread[b, h, use] += w * (scale * (np.abs(k[use]) @ np.abs(x)) + abs(log))
    return spread


def heaviest(weights, table, lens, keep, first, last, page, pages):
    """(tokens [batch][kv_heads][keep], ascending, the rest -1; how many of every sequence)."""
    batch, heads, _ = weights.shape
    tokens, kept = np.full((batch, heads, keep), -1, np.int32), np.zeros(batch, np.int32)
    room = table.shape[1] * page
    for b in range(batch):
        length = min(max(int(lens[b]), 0), room)
        there = np.array([j for j in range(length) if 0 <= table[b, j // page] < pages], int)
        kept[b] = min(keep, len(there))
        for h in range(heads):
            w = weights[b, h, there].astype(np.float64)
            w = np.where(np.isnan(w), -np.inf, w)
            rank = np.where(np.isnan(weights[b, h, there]), -1, 0)              # NaN below -infinity
            always = (there < first) | (there >= length - last)
            order = np.lexsort((there, -w, -rank, ~always))
            tokens[b, h, :kept[b]] = np.sort(there[order[:keep]])
    return tokens, kept


def move(cache, tokens, table, into, weights=None):
    """Copies records' tokens; returns the moved weights [batch][kv_heads][into's tokens], 0 past the kept ones."""
    batch, heads, keep = tokens.shape
    room = into.shape[1] * cache.page
    moved = np.zeros((batch, heads, room), np.float32)
    for b, h, i in np.ndindex(batch, heads, keep):
        j = int(tokens[b, h, i])
        if i >= room:
            continue
        source = cache.record(table, b, j, h) if j >= 0 else None
        if weights is not None and source is not None and j < weights.shape[2]:
            moved[b, h, i] = weights[b, h, j]
        target = cache.record(into, b, i, h)
        if source is None or target is None:
            continue
        for name in "kv":
            target.codes[name][i % cache.page] = source.codes[name][j % cache.page]
            target.scales[name][:, i % cache.page] = source.scales[name][:, j % cache.page]
        if source.signs is not None:
            target.signs[i % cache.page] = source.signs[j % cache.page]
    return moved


def token_logprobs(logits, targets, scale, top):
    """(log probability of the targets, entropy, log of the sum of exponentials, the best alternatives' log probabilities, their columns)."""
    x = np.asarray(logits, np.float64)
    rows, cols = x.shape
    lp, entropy, lse = np.zeros(rows), np.zeros(rows), np.zeros(rows)
    best, column = np.zeros((rows, top)), np.zeros((rows, top), np.int32)
    for r in range(rows):
        z = x[r] * scale
        m = z.max() if cols else -np.inf
        if not np.isfinite(m):                               # every logit -infinity, or a NaN or +infinity among them
            lse[r] = -np.inf if m == -np.inf else np.nan
            lp[r], entropy[r], best[r], column[r] = np.nan, np.nan, np.nan, -1
        else:
            e = np.exp(z - m)
            lse[r] = m + np.log(e.sum())
            with np.errstate(invalid="ignore"):
                entropy[r] = np.log(e.sum()) - np.where(e > 0, e * (z - m), 0).sum() / e.sum()
            order = np.lexsort((np.arange(cols), -x[r]))[:top]
            best[r], column[r] = z[order] - m - np.log(e.sum()), order
            if targets is not None:
                lp[r] = z[targets[r]] - m - np.log(e.sum()) if 0 <= targets[r] < cols else 0.0
        if targets is not None and not 0 <= targets[r] < cols:
            lp[r] = 0.0
    return lp, entropy, lse, best, column


assert oc.GRID[-1] == 6
