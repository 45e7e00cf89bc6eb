"""Oracle of the 4-bit key/value cache: the definitions of include/bnn.h in numpy and 64 bits, one token, head and row at a time.

A cache is numpy uint8 [pages][heads][record]; the plan (table, lens, start) is numpy int32 as the library takes it.
"""
from __future__ import annotations

import numpy as np

GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
VALUES = np.concatenate([GRID, -GRID])
LOW, HIGH, NAN = -100, 100, 255


def record_bytes(dim, page, signs=True):
    return page * (dim + dim // 16 + (dim // 8 if signs else 0))


def quantise_group(x):
    """32 numbers -> (codes, byte of the scale)."""
    x = np.asarray(x, np.float64)
    assert x.shape == (32,)
    if not np.isfinite(x).all():
        return np.zeros(32, np.uint8), NAN
    high = np.abs(x).max()
    e = LOW
    while e < HIGH and high > 6 * 2.0 ** e:
        e += 1
    y = np.abs(x) * 2.0 ** -e
    codes = np.zeros(32, np.uint8)
    for i in range(32):
        distance = np.abs(GRID - y[i])
        near = np.flatnonzero(distance == distance.min())
        codes[i] = near[0] if len(near) == 1 else [n for n in near if n % 2 == 0][0]        # between two codes: the even one
    return codes | np.where(np.signbit(x), 8, 0).astype(np.uint8), e + 127


def group_values(codes, byte):
    return np.full(32, np.nan) if byte == NAN else VALUES[codes] * 2.0 ** (int(byte) - 127)


class Record:
    """Views of the parts of one (page, head)."""

    def __init__(self, data, page, dim, signs=True):
        c, e = page * dim // 2, page * dim // 32
        self.codes = {"k": data[:c].reshape(page, dim // 2), "v": data[c:2 * c].reshape(page, dim // 2)}
        self.scales = {"k": data[2 * c:2 * c + e].reshape(dim // 32, page), "v": data[2 * c + e:2 * c + 2 * e].reshape(dim // 32, page)}
        self.signs = data[2 * c + 2 * e:].reshape(page, dim // 8) if signs else None

    def put(self, offset, k, v):
        for name, x in (("k", k), ("v", v)):
            for g in range(len(x) // 32):
                codes, byte = quantise_group(x[32 * g:32 * g + 32])
                if byte != NAN:
                    self.codes[name][offset, 16 * g:16 * g + 16] = codes[0::2] | codes[1::2] << 4
                self.scales[name][g, offset] = byte
        if self.signs is not None:
            self.signs[offset] = np.packbits(np.asarray(k) >= 0, bitorder="little")

    def get(self, name, offset):
        row = self.codes[name][offset]
        codes = np.stack([row & 15, row >> 4], -1).reshape(-1, 32)
        return np.concatenate([group_values(c, b) for c, b in zip(codes, self.scales[name][:, offset])])

    def sign_bits(self, offset):
        return np.unpackbits(self.signs[offset], bitorder="little").astype(bool)


class Cache:
    def __init__(self, data, dim, page, signs=True):
        self.data, self.dim, self.page = data, dim, page
        self.heads = data.shape[1]
        self.records = [[Record(data[p, h], page, dim, signs) for h in range(self.heads)] for p in range(data.shape[0])]

    def record(self, table, b, token, head):
        at = token // self.page
        if token < 0 or at >= table.shape[1] or not 0 <= table[b, at] < len(self.records):
            return None
        return self.records[table[b, at]][head]


def row_places(cache, table, lens, start, tokens):
    """(sequence, position) of every row."""
    batch = table.shape[0]
    start = np.arange(batch + 1) * (tokens // batch) if start is None else start
    out = []
    for b in range(batch):
        n = int(start[b + 1]) - int(start[b])
        out += [(b, int(lens[b]) - n + i) for i in range(n)]
    return out


def write(cache, k, v, table, lens, start=None):
    for t, (b, pos) in enumerate(row_places(cache, table, lens, start, len(k))):
        for h in range(cache.heads):
            rec = cache.record(table, b, pos, h)
            if rec is not None:
                rec.put(pos % cache.page, k[t, h], v[t, h])


def read(cache, table, lens, start, tokens):
    k, v = np.zeros((tokens, cache.heads, cache.dim)), np.zeros((tokens, cache.heads, cache.dim))
    for t, (b, pos) in enumerate(row_places(cache, table, lens, start, tokens)):
        for h in range(cache.heads):
            rec = cache.record(table, b, pos, h)
            if rec is not None:
                k[t, h], v[t, h] = rec.get("k", pos % cache.page), rec.get("v", pos % cache.page)
    return k, v


def select(cache, q, table, lens, keep, start=None, first=1, last=1):
    tokens, heads = q.shape[:2]
    group = heads // cache.heads
    out = np.full((tokens, cache.heads, keep), -1, np.int32)
    for t, (b, pos) in enumerate(row_places(cache, table, lens, start, tokens)):
        for h in range(cache.heads):
            score = {}
            for block in range(pos // cache.page + 1 if pos >= 0 else 0):
                keys = [p for p in range(block * cache.page, min((block + 1) * cache.page, pos + 1))]
                rec = cache.record(table, b, keys[0], h)
                if rec is None:
                    continue
                bits = np.stack([rec.sign_bits(p % cache.page) for p in keys])
                score[block] = sum(int(((q[t, h * group + g] >= 0) == bits).sum(-1).max()) for g in range(group))
            own = pos // cache.page
            kept = {x for x in score if x < first or x > own - last}
            rest = sorted((x for x in score if x not in kept), key=lambda x: (-score[x], x))
            chosen = sorted(kept | set(rest[:keep - len(kept)]))
            out[t, h, :len(chosen)] = chosen
    return out


def attend(cache, q, table, lens, start=None, scale=1.0, causal=True, window=0, blocks=None):
    """(out, lse, magnitude, spread): magnitude is the weighted mean of |v|, spread the largest scale * sum |q| |k| of the row, both for error bounds."""
    tokens, heads = q.shape[:2]
    group = heads // cache.heads
    out, magnitude = np.zeros((tokens, heads, cache.dim)), np.zeros((tokens, heads, cache.dim))
    lse, spread = np.full((tokens, heads), -np.inf), np.zeros((tokens, heads))
    places = row_places(cache, table, lens, start, tokens)
    values = {}
    for t, (b, pos) in enumerate(places):
        top = pos if causal else int(lens[b]) - 1
        low = max(0, pos - window + 1) if window else 0
        for h in range(cache.heads):
            keys = []
            for p in range(low, top + 1):
                if cache.record(table, b, p, h) is None:
                    continue
                times = 1 if blocks is None else int((blocks[t, h] == p // cache.page).sum())
                keys += [p] * times
            if not keys:
                continue
            for p in keys:
                if (b, h, p) not in values:
                    rec = cache.record(table, b, p, h)
                    values[b, h, p] = rec.get("k", p % cache.page), rec.get("v", p % cache.page)
            k, v = np.stack([values[b, h, p][0] for p in keys]), np.stack([values[b, h, p][1] for p in keys])
            for g in range(group):
                x = q[t, h * group + g].astype(np.float64)
                with np.errstate(invalid="ignore", over="ignore"):
                    s = scale * (k @ x)
                    m = s.max()
                    w = np.exp(s - m)
                    out[t, h * group + g] = w @ v / w.sum()
                    magnitude[t, h * group + g] = w @ np.abs(v) / w.sum()
                    lse[t, h * group + g] = m + np.log(w.sum())
                    spread[t, h * group + g] = scale * (np.abs(k) @ np.abs(x)).max()
    return out, lse, magnitude, spread
