"""Without a GPU: what the calls around the cache and behind the head refuse before anything is launched, and the oracle's own pins."""
import ctypes

import numpy as np
import pytest

from oracle import cache4 as oc
from oracle import decoding as od

OK, INVALID, ALIGNMENT, UNSUPPORTED, WORKSPACE = 0, -1, -2, -3, -5
F32, BF16, F16, I32 = range(4)
P = ctypes.c_void_p
A = 4096                                      # an address that nothing follows


@pytest.fixture(scope="module")
def b():
    from paper_2006_16578_amd import binding
    return binding


def rotation(b, frequencies=A, positions=A, pairs=8, neighbours=0, inverse=0, magnitude=1.0):
    return ctypes.byref(b._RotationStruct(frequencies, positions, pairs, neighbours, inverse, magnitude))


def cache(b, data=A, pages=4, kv_heads=2, dim=64, page=16, signs=1):
    return ctypes.byref(b._Cache4Struct(data, pages, kv_heads, dim, page, signs))


def rows(b, table=A, lens=A, start=0, batch=2, pages=3, tokens=4):
    return ctypes.byref(b._Rows4Struct(table, lens, start, batch, pages, tokens))


def i64(*values):
    return [ctypes.c_int64(v) for v in values]


def test_rotary(b):
    def call(x=A, out=A + 4096, dtype=F32, tokens=4, heads=2, dim=16, strides=(32, 16, 32, 16), rot=None, **kw):
        return b.load().bnn_rotary(P(x), P(out), dtype, tokens, heads, dim, *i64(*strides), rotation(b, **kw) if rot is None else rot, None)
    assert call(rot=ctypes.POINTER(b._RotationStruct)()) == INVALID
    for kw in (dict(x=0), dict(out=0), dict(frequencies=0), dict(positions=0), dict(dtype=3), dict(dtype=-1), dict(tokens=-1), dict(heads=-1), dict(dim=15), dict(pairs=0), dict(pairs=-3),
               dict(neighbours=2), dict(inverse=-1), dict(magnitude=float("nan")), dict(magnitude=float("inf")), dict(out=A, strides=(32, 16, 48, 16))):
        assert call(**kw) == INVALID, kw
    for kw in (dict(frequencies=A + 4), dict(positions=A + 2), dict(x=A + 2), dict(out=A + 1), dict(dtype=BF16, x=A + 1)):
        assert call(**kw) == ALIGNMENT, kw
    for kw in (dict(pairs=1025, dim=4096), dict(dim=1 << 20), dict(tokens=2147483647, heads=1)):
        assert call(**kw) == UNSUPPORTED, kw
    assert call(tokens=0) == OK and call(heads=0) == OK


def test_rotary_into_heads_that_overlap(b):
    """Distances by which a head of the output would be written over another: refused.  (Without tokens nothing is launched: what is allowed is checked with frequencies that are refused later.)"""
    def call(tokens, heads, token, head, out=A + (1 << 20), dim=16):
        return b.load().bnn_rotary(P(A), P(out), F32, tokens, heads, dim, *i64(token, head, token, head), rotation(b), None)
    for args in ((4, 2, 32, 0), (4, 2, 0, 16), (4, 2, 32, 15), (4, 2, 15, 64), (4, 2, 16, 16), (4, 3, 32, 16), (100, 7, 16, 1592), (5, 3, 48, 56), (3, 5, -32, 32), (1, 2, 32, -15), (2, 1, 3, 0)):
        assert call(*args) == INVALID, args
        assert call(*args, out=A) == INVALID, args
    assert call(3, 5, 1 << 62, 1 << 61) == INVALID and call(4, 4, 3 << 60, 1 << 61, out=A + (1 << 20) + 2) == INVALID      # products beyond 64 bits
    seen = set()
    for tokens, heads, token, head in ((3, 4, 40, 16), (4, 3, 16, 64), (3, 3, 48, 80), (3, 3, 80, 48), (3, 3, 32, 48), (4, 4, 33, 50), (2, 2, 17, 33), (2, 3, 47, 16), (5, 4, 64, 16)):
        spans = sorted(t * token + h * head for t in range(tokens) for h in range(heads))
        apart = all(y - x >= 16 for x, y in zip(spans, spans[1:]))
        seen.add(apart)                       # (what is apart goes on to the next check: a misaligned pointer)
        assert call(tokens, heads, token, head, out=A + (1 << 20) + 2) == (ALIGNMENT if apart else INVALID), (tokens, heads, token, head)
    assert seen == {True, False}


def test_write_rotary(b):
    def call(c=None, r=None, rot=None, q=A, q_out=2 * A, k=A, v=A, dtype=F32, heads=4, q_d=(256, 64), k_d=(128, 64), v_d=(128, 64)):
        return b.load().bnn_cache4_write_rotary(c or cache(b), r or rows(b), rot or rotation(b), P(q), *i64(*q_d), heads, P(q_out), P(k), P(v), dtype, *i64(*k_d, *v_d), None)
    for kw in (dict(k=0), dict(v=0), dict(q=0), dict(q_out=0), dict(dtype=3), dict(heads=-1), dict(rot=rotation(b, pairs=33)), dict(rot=rotation(b, frequencies=0)),
               dict(q_out=A, q_d=(512, 64)), dict(q_out=A, q_d=(256, 128)), dict(r=rows(b, tokens=5)), dict(r=rows(b, table=0)), dict(c=cache(b, data=0))):
        assert call(**kw) == INVALID, kw
    for kw in (dict(k=A + 4), dict(q=A + 8), dict(q_out=A + 4), dict(k_d=(130, 64)), dict(q_d=(256, 65)), dict(rot=rotation(b, positions=A + 1))):
        assert call(**kw) == ALIGNMENT, kw
    assert call(rot=rotation(b, pairs=1025)) == UNSUPPORTED and call(c=cache(b, dim=80)) == UNSUPPORTED
    assert call(r=rows(b, tokens=0)) == OK


def test_weigh(b):
    def call(c=None, r=None, q=A, dtype=F32, q_d=(256, 64), heads=4, lse=A, scale=0.125, causal=1, window=0, previous=0, decay=1.0, weights=A, width=48, work=0, size=0):
        return b.load().bnn_cache4_weigh(c or cache(b), r or rows(b), P(q), dtype, *i64(*q_d), heads, P(lse), ctypes.c_float(scale), causal, window, P(previous), ctypes.c_float(decay),
                                         P(weights), ctypes.c_int64(width), P(work), ctypes.c_size_t(size), None)
    for kw in (dict(q=0), dict(lse=0), dict(weights=0), dict(width=47), dict(dtype=4), dict(heads=3), dict(heads=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
               dict(scale=float("inf")), dict(window=-1), dict(window=2, causal=0), dict(decay=float("nan")), dict(decay=float("inf")), dict(r=rows(b, lens=0))):
        assert call(**kw) == INVALID, kw
    for kw in (dict(q=A + 4), dict(lse=A + 2), dict(previous=A + 1), dict(weights=A + 2), dict(q_d=(254, 64))):
        assert call(**kw) == ALIGNMENT, kw
    assert call(r=rows(b, pages=(1 << 26) + 1), width=1 << 40) == UNSUPPORTED
    assert call(r=rows(b, tokens=1 << 29), heads=4) == UNSUPPORTED
    assert call(scale=1e-39) == INVALID                              # (its reciprocal is no fp32 number)
    need = b.load().bnn_cache4_weigh_workspace_bytes(cache(b), rows(b, tokens=2000), F32, 4)
    assert need > 0 and b.load().bnn_cache4_weigh_workspace_bytes(cache(b), rows(b), F32, 4) == 0
    assert call(r=rows(b, tokens=2000)) == WORKSPACE and call(r=rows(b, tokens=2000), work=A, size=need - 1) == WORKSPACE and call(r=rows(b, tokens=2000), work=A + 8, size=need) == ALIGNMENT
    for bad in ((cache(b, dim=80), rows(b), F32, 4), (cache(b), rows(b, tokens=5), F32, 4), (cache(b), rows(b), 3, 4), (cache(b), rows(b), F32, 3), (cache(b), rows(b, tokens=1 << 29), F32, 4)):
        assert b.load().bnn_cache4_weigh_workspace_bytes(*bad) == 0
    assert call(r=rows(b, tokens=0)) == OK


@pytest.mark.parametrize("counts,group,kv_heads,dim,page,pages", [([1] * 255 + [4096], 4, 8, 128, 64, 2048), ([1] * 63 + [1024], 4, 8, 128, 64, 2048), ([1, 70, 700, 66, 300, 0, 2], 3, 2, 64, 16, 8192),
                                                                  ([64] * 256, 4, 8, 128, 64, 2048), ([300] * 7 + [2], 1, 4, 256, 256, 512)])
def test_weigh_workspace_of_mixed_runs(b, counts, group, kv_heads, dim, page, pages):
    """Sums of parts are kept for sequences in several parts only, in parts of up to 2048 rows: where a table is as wide as a context allows, a place is kv_heads * its tokens * 4 bytes, 4 MB in the first call.
    A sequence of n rows in parts of P is in fewer than 2 n / P, so there are less than two places for every P rows of the call, P being 128 at least and 2048 where workgroups are many."""
    tokens, room = sum(counts), pages * page
    need = b.load().bnn_cache4_weigh_workspace_bytes(cache(b, kv_heads=kv_heads, dim=dim, page=page), rows(b, start=A, batch=len(counts), pages=pages, tokens=tokens), BF16, kv_heads * group)
    place = kv_heads * room * 4
    tiles = kv_heads * -(-room // (64 * (2 if dim >= 192 else 4)))
    part = next((p for p in (256, 512, 1024) if tokens * group * tiles // p <= 2048), 2048)
    assert need <= max(2 * (tokens * group // part), 0) * place
    if counts[-1] == 4096:
        assert need == 16 * place == 1 << 26


def test_heaviest_and_move(b):
    def heaviest(c=None, table=A, lens=A, batch=2, pages=3, weights=A, width=48, keep=8, first=1, last=2, tokens=A, kept=A, work=0, size=0):
        return b.load().bnn_cache4_heaviest(c or cache(b), P(table), P(lens), batch, pages, P(weights), ctypes.c_int64(width), keep, first, last, P(tokens), P(kept), P(work), ctypes.c_size_t(size), None)
    for kw in (dict(table=0), dict(lens=0), dict(weights=0), dict(tokens=0), dict(kept=0), dict(batch=-1), dict(pages=0), dict(width=47), dict(keep=0), dict(first=-1), dict(last=-1),
               dict(first=4, last=5), dict(first=2147483647, last=2147483647), dict(c=cache(b, kv_heads=0))):
        assert heaviest(**kw) == INVALID, kw
    for kw in (dict(table=A + 1), dict(lens=A + 2), dict(weights=A + 2), dict(tokens=A + 1), dict(kept=A + 3)):
        assert heaviest(**kw) == ALIGNMENT, kw
    assert heaviest(pages=(1 << 26) + 1, width=1 << 40) == UNSUPPORTED and heaviest(batch=1 << 22) == UNSUPPORTED and heaviest(batch=0) == OK

    need = b.load().bnn_cache4_heaviest_workspace_bytes(cache(b), 2, 4000)
    assert need > 0 and b.load().bnn_cache4_heaviest_workspace_bytes(cache(b), 2, 3) == 0 and b.load().bnn_cache4_heaviest_workspace_bytes(cache(b), 20000, 4000) == 0
    assert heaviest(pages=4000, width=64000) == WORKSPACE and heaviest(pages=4000, width=64000, work=A, size=need - 1) == WORKSPACE
    assert heaviest(pages=4000, width=64000, work=A + 8, size=need) == ALIGNMENT
    for bad in ((cache(b, dim=80), 2, 4000), (cache(b), 0, 4000), (cache(b), 2, 0), (cache(b), 2, (1 << 26) + 1)):
        assert b.load().bnn_cache4_heaviest_workspace_bytes(*bad) == 0

    def move(c=None, tokens=A, keep=8, table=A, pages=3, into=A, into_pages=1, batch=2, weights=A, width=48, moved=A):
        return b.load().bnn_cache4_move(c or cache(b), P(tokens), keep, P(table), pages, P(into), into_pages, batch, P(weights), ctypes.c_int64(width), P(moved), None)
    for kw in (dict(tokens=0), dict(keep=0), dict(table=0), dict(pages=0), dict(into=0), dict(into_pages=-1), dict(batch=-1), dict(weights=0), dict(moved=0), dict(width=0), dict(c=cache(b, data=0))):
        assert move(**kw) == INVALID, kw
    for kw in (dict(tokens=A + 2), dict(table=A + 2), dict(into=A + 1), dict(weights=A + 2), dict(moved=A + 1), dict(c=cache(b, data=A + 8))):
        assert move(**kw) == ALIGNMENT, kw
    assert move(pages=(1 << 26) + 1) == UNSUPPORTED and move(into_pages=(1 << 26) + 1) == UNSUPPORTED and move(into_pages=1 << 26, batch=1 << 20) == UNSUPPORTED
    assert move(batch=0) == OK and move(into_pages=0) == OK


def test_cut_back_into_too_few_pages():
    """The newest of the kept tokens would be passed over, and the lengths would count them."""
    import types

    import torch

    from paper_2006_16578_amd import decoder
    calls = []
    cache = types.SimpleNamespace(page=16, heaviest=lambda *a: calls.append(a) or ("tokens", "lens"), move=lambda *a: "weights")
    table = torch.zeros(2, 10, dtype=torch.int32)
    for keep, pages in ((33, 2), (160, 9), (1000, 9), (17, 1)):
        with pytest.raises(ValueError):
            decoder.cut_back(cache, None, table, None, table[:, :pages], keep)
    assert not calls
    for keep, pages in ((32, 2), (160, 10), (1000, 10), (1, 1)):
        assert decoder.cut_back(cache, None, table, None, table[:, :pages], keep) == ("lens", "weights")


def test_token_logprobs(b):
    lib = b.load()

    def call(x=A, dtype=F32, n=4, cols=100, ld=100, scale=1.0, targets=A, top=5, lp=A, entropy=A, lse=A, best=A, tokens=A, work=A, size=1 << 30):
        return lib.bnn_token_logprobs(P(x), dtype, n, cols, ctypes.c_int64(ld), ctypes.c_float(scale), P(targets), top, P(lp), P(entropy), P(lse), P(best), P(tokens), P(work),
                                      ctypes.c_size_t(size), None)
    for kw in (dict(x=0), dict(dtype=4), dict(dtype=-1), dict(n=-1), dict(cols=0), dict(scale=0.0), dict(scale=-2.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38), dict(targets=0),
               dict(lp=0), dict(top=-1), dict(top=5, cols=4), dict(best=0), dict(tokens=0)):
        assert call(**kw) == INVALID, kw
    for kw in (dict(x=A + 2), dict(x=A + 1, dtype=BF16), dict(targets=A + 4), dict(lp=A + 2), dict(entropy=A + 1), dict(best=A + 2), dict(tokens=A + 2), dict(cols=100000, work=A + 8)):
        assert call(**kw) == ALIGNMENT, kw
    assert call(top=65) == UNSUPPORTED and call(cols=1 << 30) == UNSUPPORTED and call(n=1 << 24) == UNSUPPORTED
    assert call(cols=100000, work=0) == WORKSPACE and call(cols=100000, size=lib.bnn_token_logprobs_workspace_bytes(4, 100000, F32, 5) - 1) == WORKSPACE
    assert call(n=0) == OK
    for dtype in (F32, BF16, F16, I32):
        assert lib.bnn_token_logprobs_workspace_bytes(4, 100, dtype, 5) == 0 and lib.bnn_token_logprobs_workspace_bytes(4, 100000, dtype, 5) > 0
    for bad in ((0, 10, F32, 1), (4, 0, F32, 1), (4, 10, 4, 1), (4, 10, F32, 65), (4, 10, F32, -1), (4, 1 << 30, F32, 1)):
        assert lib.bnn_token_logprobs_workspace_bytes(*bad) == 0


def test_the_oracle_itself():
    # a quarter turn exchanges a pair's elements; neighbours and halves; the inverse turns back
    x = np.arange(12.0).reshape(1, 2, 6)
    y = od.rotate(x, [1], [np.pi / 2, np.pi])
    assert np.allclose(y[0, 0], [-2, -1, 0, -3, 4, 5]) and np.allclose(od.rotate(y, [1], [np.pi / 2, np.pi], inverse=True), x)
    assert np.allclose(od.rotate(x, [1], [np.pi / 2, np.pi], neighbours=True, magnitude=2.0)[0, 0], [-2, 0, -4, -6, 4, 5])
    # entropy of equal ones, of one sure token; ties; a row of nothing
    lp, entropy, lse, best, column = od.token_logprobs(np.array([[0.0] * 4, [0, 1000, 0, 0], [-np.inf] * 4, [1, np.nan, 0, 0]]), np.array([1, 1, 0, 9]), 1.0, 2)
    assert np.allclose(entropy[:2], [np.log(4), 0]) and np.allclose(lp[:2], [-np.log(4), 0]) and lse[2] == -np.inf and np.isnan(lp[2]) and lp[3] == 0 and np.isnan(lse[3])
    assert column.tolist() == [[0, 1], [1, 0], [-1, -1], [-1, -1]] and np.allclose(best[1], [0, -1000])
    # the heaviest, with ties, what is always kept, and a page that is gone
    w = np.array([[[5, 1, 1, 9, 0, 3, 3, 2]]], np.float32)
    table = np.array([[0, 1]], np.int32)
    pick = lambda keep, first, last, t=table, n=8: [v.tolist() for v in od.heaviest(w, t, np.array([n], np.int32), keep, first, last, 4, 2)]
    assert pick(3, 0, 0) == [[[[0, 3, 5]]], [3]] and pick(3, 0, 2) == [[[[3, 6, 7]]], [3]] and pick(4, 2, 1) == [[[[0, 1, 3, 7]]], [4]]
    assert pick(3, 0, 0, np.array([[-1, 1]], np.int32)) == [[[[5, 6, 7]]], [3]] and pick(5, 0, 0, n=2) == [[[[0, 1, -1, -1, -1]]], [2]]
    # weights of one row sum to one, and old ones fade
    rng = np.random.default_rng(0)
    c = oc.Cache(np.zeros((1, 1, oc.record_bytes(64, 16)), np.uint8), 64, 16)
    lens, table = np.array([5], np.int32), np.zeros((1, 1), np.int32)
    oc.write(c, rng.standard_normal((5, 1, 64)), rng.standard_normal((5, 1, 64)), table, lens)
    q = rng.standard_normal((1, 2, 64))
    lse = oc.attend(c, q, table, lens, scale=0.125)[1]
    out = np.full((1, 1, 16), 7.0)
    od.weigh(c, q, lse, table, lens, None, 0.125, out)
    assert abs(out[0, 0, :5].sum() - 2) < 1e-12 and (out[0, 0, 5:] == 7).all()
    more = np.zeros((1, 1, 16))
    od.weigh(c, q, lse, table, lens, None, 0.125, more, previous=out, decay=0.5)
    assert np.allclose(more[0, 0, :4], 1.5 * out[0, 0, :4]) and more[0, 0, 4] == out[0, 0, 4]
