"""GPU: rotary positions, alone and on the way into the 4-bit cache, against the oracle in 64 bits."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import cache4 as oc
from oracle import decoding as od

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}


@pytest.fixture(scope="module")
def bnn():
    import paper_2006_16578_amd as b
    b.load()
    return b


def rounded(x, dtype):
    return torch.from_numpy(np.asarray(x, np.float64)).to(TYPES[dtype]).double().numpy()


def dev(x, dtype):
    return torch.from_numpy(np.asarray(x, np.float64)).to(TYPES[dtype]).cuda()


def ints(x):
    return torch.from_numpy(np.asarray(x, np.int32)).cuda()


def frequencies(pairs, base=10000.0):
    return base ** (-np.arange(pairs) / pairs)


def bound(want, x, magnitude, dtype):
    """A result is rounded to fp32 and to its type (half a step each); sine and cosine are off by 2^-46 at most here (series to 4e-17, angles up to 2^31 rounded alike on both sides and
    reduced exactly but for 2^-53 of the remainder, and the oracle's own), times the pair's magnitude."""
    size = abs(magnitude) * 2 * np.abs(x).max(-1, keepdims=True)
    return (HALF_STEP[dtype] + 2.0 ** -24) * np.abs(want) * (1 + 2.0 ** -10) + 2.0 ** -46 * size + (2.0 ** -25 if dtype == "f16" else 1e-44)


def positions_of(rng, tokens):
    p = rng.integers(0, 5000, tokens)
    p[: min(tokens, 5)] = [0, 1, 1000003, 2147483647, -77][: min(tokens, 5)]
    return p


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,dim,pairs", [(1, 1, 64, 32), (5, 3, 96, 16), (37, 5, 80, 20), (3, 2, 7, 3), (2, 9, 2, 1), (600, 2, 128, 64), (9, 40, 320, 160), (2, 1, 2048, 1024), (17, 3, 20, 6)])
def test_rotary(bnn, dtype, interleaved, tokens, heads, dim, pairs):
    rng = np.random.default_rng(tokens + dim)
    x, p, f = rounded(rng.standard_normal((tokens, heads, dim)), dtype), positions_of(rng, tokens), frequencies(pairs)
    for inverse, magnitude in ((False, 1.0), (True, 1.375)):
        want = od.rotate(x, p, f, interleaved, magnitude, inverse)
        got = bnn.rotary(dev(x, dtype), ints(p), torch.from_numpy(f).cuda(), interleaved=interleaved, magnitude=magnitude, inverse=inverse)
        assert got.dtype == TYPES[dtype] and got.shape == x.shape
        got = got.double().cpu().numpy()
        off = np.abs(got - want) > bound(want, x, magnitude, dtype)
        assert not off.any(), (np.argwhere(off)[:5], np.abs(got - want).max())
        assert (got[..., 2 * pairs:] == x[..., 2 * pairs:]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
def test_distances_alignments_and_in_place(bnn, dtype, interleaved):
    rng = np.random.default_rng(5)
    tokens, heads, dim, pairs = 11, 3, 32, 8
    p, f = positions_of(rng, tokens), frequencies(pairs)
    pt, ft = ints(p), torch.from_numpy(f).cuda()
    for shape, take in (((tokens, heads + 2, dim), lambda t: t[:, 1:1 + heads]),                      # heads of a wider row
                        ((tokens, heads, dim + 3), lambda t: t[:, :, 3:]),                            # elements that are not aligned
                        ((heads, tokens, dim), lambda t: t.transpose(0, 1)),                          # heads before tokens
                        ((1, heads, dim), lambda t: t.expand(tokens, heads, dim)),                    # one token's elements for all
                        ((tokens, heads, dim + 8), lambda t: t[:, :, :dim])):
        whole = dev(rng.standard_normal(shape), dtype)
        x = take(whole)
        values = x.double().cpu().numpy()
        want = od.rotate(values, p, f, interleaved)
        got = bnn.rotary(x, pt, ft, interleaved=interleaved).double().cpu().numpy()
        assert (np.abs(got - want) <= bound(want, values, 1.0, dtype)).all()
        if shape[0] != 1:
            before = whole.clone()
            assert bnn.rotary(x, pt, ft, interleaved=interleaved, out=x) is x
            assert (x.double().cpu().numpy() == got).all()
            x.copy_(take(before))
            assert torch.equal(whole, before)                        # nothing beside x was written
    out = torch.full((tokens, 2 * heads, dim), 7.0, dtype=TYPES[dtype], device="cuda")
    x = dev(rng.standard_normal((tokens, heads, dim)), dtype)
    bnn.rotary(x, pt, ft, interleaved=interleaved, out=out[:, ::2])
    assert torch.equal(out[:, ::2], bnn.rotary(x, pt, ft, interleaved=interleaved)) and (out[:, 1::2] == 7).all()
    assert bnn.rotary(x[:0], pt[:0], ft).shape == (0, heads, dim) and bnn.rotary(x[:, :0], pt, ft).shape == (tokens, 0, dim)


def test_the_inverse_is_the_gradient(bnn):
    """Of sum(g * rotary(x)): the inverse rotation of g, against differences (the map is linear: exact but for roundings) and against the turn back."""
    rng = np.random.default_rng(6)
    tokens, heads, dim, pairs = 4, 2, 24, 8
    p, f = ints(positions_of(rng, tokens)), torch.from_numpy(frequencies(pairs)).cuda()
    x, g = (torch.from_numpy(rng.standard_normal((tokens, heads, dim))).float().cuda() for _ in range(2))
    for interleaved in (False, True):
        turn = lambda t, **kw: bnn.rotary(t, p, f, interleaved=interleaved, magnitude=1.25, **kw)
        grad = turn(g, inverse=True).double()
        for _ in range(20):
            d = torch.from_numpy(rng.standard_normal(x.shape)).float().cuda()
            change = ((turn(x + d).double() - turn(x - d).double()) * g.double()).sum() / 2
            # 4 roundings of fp32 an element (x + d, x - d, and the results), of values below 10
            assert abs(change - (grad * d.double()).sum()) <= 4 * 2.0 ** -24 * 10 * g.abs().double().sum()
        back = turn(turn(x), inverse=True).double()
        scale = torch.ones(dim, device="cuda", dtype=torch.float64)
        scale[:2 * pairs] = 1.25 ** 2
        assert ((back - x.double() * scale).abs() <= 4 * 2.0 ** -24 * 10).all()
        assert ((turn(x).double().square().sum() - (x.double() * scale.sqrt()).square().sum()).abs() <= 1e-4)


def test_nan_and_infinity_stay_in_their_pair(bnn):
    x = torch.randn(3, 2, 16, device="cuda")
    x[1, 0, 2], x[2, 1, 5] = float("nan"), float("inf")
    p, f = ints([3, 4, 5]), torch.from_numpy(frequencies(8)).cuda()
    y = bnn.rotary(x, p, f)
    bad = ~torch.isfinite(y)
    assert sorted(map(tuple, bad.nonzero().tolist())) == [(1, 0, 2), (1, 0, 10), (2, 1, 5), (2, 1, 13)]
    f[3] = float("inf")
    y = bnn.rotary(torch.ones(3, 2, 16, device="cuda"), p, f)
    assert torch.isnan(y[:, :, 3]).all() and torch.isnan(y[:, :, 11]).all() and torch.isfinite(y[:, :, 4:11]).all()


def test_frequencies(bnn):
    f = bnn.rotary_frequencies(8, base=100.0)
    assert f.dtype == torch.float64 and f.is_cuda and torch.allclose(f.cpu(), torch.tensor([1, 100 ** -0.25, 0.1, 100 ** -0.75], dtype=torch.float64), rtol=1e-15)
    assert torch.equal(bnn.rotary_frequencies(8, base=100.0, factor=4.0, device="cpu"), bnn.rotary_frequencies(8, base=100.0, device="cpu") / 4)
    g = bnn.rotary_frequencies(8, base=100.0, factor=4.0, scaling="base", device="cpu")
    assert g[0] == 1 and abs(g[-1] * 4 / 100 ** -0.75 - 1) < 1e-14
    plain = bnn.rotary_frequencies(64, device="cpu")
    h = bnn.rotary_frequencies(64, factor=8.0, scaling="parts", context=4096, low=1, high=32, device="cpu")
    turns = 4096 * plain / (2 * np.pi)
    assert torch.equal(h[turns >= 32], plain[turns >= 32]) and torch.allclose(h[turns <= 1], plain[turns <= 1] / 8, rtol=1e-15)
    between = (turns > 1) & (turns < 32)
    assert between.any() and (h[between] < plain[between]).all() and (h[between] > plain[between] / 8).all()
    for bad in (dict(elements=7), dict(elements=0), dict(elements=8, factor=0.5), dict(elements=8, scaling="other"), dict(elements=8, scaling="parts"), dict(elements=2, scaling="base", factor=2.0)):
        with pytest.raises(ValueError):
            bnn.rotary_frequencies(**bad)


# ------------------------------------------------------------------------------------------ into the cache

class Batch:
    def __init__(self, bnn, seed, lens, counts, kv_heads, dim, page, dtype, signs=True, width=None):
        self.rng = rng = np.random.default_rng(seed)
        self.lens, self.counts, self.dtype, self.dim, self.page, self.kv_heads = np.array(lens, np.int32), counts, dtype, dim, page, kv_heads
        need = [-(-int(n) // page) for n in lens]
        self.data = rng.integers(0, 256, (sum(need) + 2, kv_heads, oc.record_bytes(dim, page, signs))).astype(np.uint8)
        order = rng.permutation(len(self.data))
        self.table = np.full((len(lens), width or max(max(need), 1)), -1, np.int32)
        for b, n in enumerate(need):
            m = min(n, self.table.shape[1])
            self.table[b, :m] = order[sum(need[:b]):sum(need[:b]) + m]
        self.tokens = int(sum(counts))
        self.start = None if len(set(counts)) == 1 else np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.oracle = oc.Cache(self.data, dim, page, signs)
        self.gpu = bnn.Cache4(kv_heads=kv_heads, head_dim=dim, page=page, signs=signs, data=torch.from_numpy(self.data.copy()).cuda())

    def plan(self):
        return dict(table=ints(self.table), lens=ints(self.lens), start=None if self.start is None else ints(self.start))

    def elements(self, heads, tokens=None):
        return rounded(self.rng.standard_normal((tokens or self.tokens, heads, self.dim)) * np.exp(0.5 * self.rng.standard_normal(self.dim)), self.dtype)

    def own_positions(self):
        p = np.zeros(self.tokens, np.int64)
        for t, _, token in od.rows_of(self.lens, self.start, self.tokens):
            p[t] = token
        return p


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim,page,kv_heads,heads,pairs,interleaved", [(64, 16, 3, 3, 32, False), (96, 32, 2, 4, 12, False), (96, 16, 1, 5, 48, True), (128, 64, 2, 2, 64, False),
                                                                        (192, 128, 1, 3, 48, True), (256, 256, 2, 2, 128, False), (64, 16, 2, 8, 1, True), (128, 16, 2, 0, 5, False)])
def test_write_rotary(bnn, dtype, dim, page, kv_heads, heads, pairs, interleaved):
    su = Batch(bnn, dim + pairs, [40, 0, 131, 17, 1, 5], [7, 0, 131, 1, 1, 8], kv_heads, dim, page, dtype)
    su.table[2, 1 if su.table.shape[1] > 1 else 0] = -1
    q, k, v = (su.elements(h) if h else None for h in (heads, kv_heads, kv_heads))
    f = frequencies(pairs)
    for positions in (None, positions_of(su.rng, su.tokens)):
        p = su.own_positions() if positions is None else positions
        magnitude = 1.0 if positions is None else 1.25
        turned = np.float32(od.rotate(k, p, f, interleaved, magnitude)).astype(np.float64)
        oc.write(su.oracle, turned, v, su.table, su.lens, su.start)
        got = su.gpu.write_rotary(None if q is None else dev(q, dtype), dev(k, dtype), dev(v, dtype), frequencies=torch.from_numpy(f).cuda(), interleaved=interleaved,
                                  magnitude=magnitude, positions=None if positions is None else ints(positions), **su.plan())
        assert (su.gpu.data.cpu().numpy() == su.data).all()
        if q is None:
            assert got is None
            continue
        want = od.rotate(q, p, f, interleaved, magnitude)
        got = got.double().cpu().numpy()
        assert (np.abs(got - want) <= bound(want, q, magnitude, dtype)).all()


def test_write_rotary_is_rotary_and_write(bnn):
    """Queries, keys and values side by side in one tensor; many tokens, so that workgroups have several; against the two calls it stands for."""
    su = Batch(bnn, 3, [2000, 700, 1], [2000, 523, 1], 4, 128, 64, "bf16", signs=False)
    other = bnn.Cache4(kv_heads=4, head_dim=128, page=64, signs=False, data=su.gpu.data.clone())
    qkv = torch.randn(su.tokens, 12 + 4 + 4, 128, device="cuda", dtype=torch.bfloat16)
    q, k, v = qkv.split((12, 4, 4), dim=1)
    f = bnn.rotary_frequencies(128)
    plan = su.plan()
    turned = su.gpu.write_rotary(q, k, v, frequencies=f, **plan)
    p = ints(su.own_positions())
    assert torch.equal(turned, bnn.rotary(q, p, f))
    k32 = bnn.rotary(k.float(), p, f)                                # (a rotated key is rounded to fp32, not to bf16)
    other.write(k32, v.float(), **plan)
    assert torch.equal(su.gpu.data, other.data)
    flat = q.contiguous()
    assert su.gpu.write_rotary(flat, k, v, frequencies=f, out=flat, **plan) is flat and torch.equal(flat, turned)


def test_rows_outside_sequences_keep_their_queries(bnn):
    su = Batch(bnn, 4, [5, 9], [2, 3], 2, 64, 16, "f32")
    q, k, v = (torch.randn(9, h, 64, device="cuda") for h in (4, 2, 2))
    out = torch.full_like(q, 3.0)
    before = su.gpu.data.clone()
    su.gpu.write_rotary(q, k, v, frequencies=bnn.rotary_frequencies(64), out=out, **su.plan())
    assert (out[5:] == 3).all() and not (out[:5] == 3).any() and not torch.equal(su.gpu.data, before)


def test_a_token_past_the_table_is_rotated_and_dropped(bnn):
    su = Batch(bnn, 5, [40], [3], 1, 64, 16, "f32", width=2)
    q = torch.randn(3, 1, 64, device="cuda")
    before = su.gpu.data.clone()
    f = bnn.rotary_frequencies(64)
    got = su.gpu.write_rotary(q, q, q, frequencies=f, **su.plan())
    assert torch.equal(got, bnn.rotary(q, ints([37, 38, 39]), f)) and torch.equal(su.gpu.data, before)


def test_no_plan_leads_out(bnn):
    """Tables, lengths and starts of any content: nothing outside the cache and the call's own output is written, and the device is fine afterwards."""
    rng = np.random.default_rng(8)
    f = bnn.rotary_frequencies(64)
    guard = torch.full((6, 2, oc.record_bytes(64, 16)), 9, dtype=torch.uint8, device="cuda")
    cache = bnn.Cache4(kv_heads=2, head_dim=64, page=16, data=guard[2:4])
    x = torch.randn(10, 2, 64, device="cuda")
    wild = lambda *shape: torch.from_numpy(rng.choice(np.array([-2147483648, -1, 0, 1, 2, 5, 31, 1000, 2147483647], np.int32), shape)).cuda()
    for _ in range(12):
        cache.write_rotary(x, x, x, wild(3, 2), wild(3), f, start=wild(4))
    torch.cuda.synchronize()
    assert (guard[:2] == 9).all() and (guard[4:] == 9).all()


def test_refusals(bnn):
    x, p, f = torch.randn(4, 2, 16, device="cuda"), ints([0, 1, 2, 3]), bnn.rotary_frequencies(16)
    for error, args, kw in ((TypeError, (x.cpu(), p, f), {}), (TypeError, (x.double(), p, f), {}), (TypeError, (x, p.long(), f), {}), (TypeError, (x, p, f.float()), {}),
                            (TypeError, (x, None, f), {}), (TypeError, (x, p, f.cpu()), {}), (ValueError, (x[0], p, f), {}), (ValueError, (x, p[:3], f), {}),
                            (ValueError, (x.transpose(1, 2), p, f), {}), (ValueError, (x, p, f), dict(out=torch.empty(4, 2, 15, device="cuda"))),
                            (ValueError, (x, p, f), dict(out=x.half())), (bnn.BnnError, (x[:, :, :12], p, f), {}), (bnn.BnnError, (x, p, f[:0]), {}),
                            (bnn.BnnError, (x, p, f), dict(magnitude=float("nan"))), (bnn.BnnError, (torch.empty(1, 1, 4096, device="cuda"), p[:1], bnn.rotary_frequencies(2050)), {})):
        with pytest.raises(error):
            bnn.rotary(*args, **kw)
    cache = bnn.Cache4(2, kv_heads=2, head_dim=64, page=16)
    k, q, f = torch.randn(4, 2, 64, device="cuda"), torch.randn(4, 4, 64, device="cuda"), bnn.rotary_frequencies(64)
    table, lens = ints([[0], [1]]), ints([2, 2])
    for error, args, kw in ((ValueError, (q, k, k[:3]), {}), (ValueError, (q[:3], k, k), {}), (ValueError, (q.half(), k, k), {}), (ValueError, (q, k[:, :1], k[:, :1]), {}),
                            (ValueError, (None, k, k), dict(out=q)), (ValueError, (q, k, k), dict(out=q[:, :2])), (ValueError, (q, k, k), dict(positions=ints([0]))),
                            (bnn.BnnError, (q, k, k), dict(frequencies=bnn.rotary_frequencies(66))), (bnn.BnnError, (q[:3], k[:3], k[:3]), {}),
                            (bnn.BnnError, (q[:, ::2], k, k), dict(out=None, frequencies=f[:0])), (TypeError, (q, k, k), dict(frequencies=f.float()))):
        with pytest.raises(error):
            cache.write_rotary(*args, table, lens, **{"frequencies": f, **kw})


def test_outputs_that_overlap(bnn):
    """One head for all, in place or as an output, would be turned again and again: refused.  Heads that lie between others' are not."""
    x, p, f = torch.randn(4, 2, 16, device="cuda"), ints([0, 1, 2, 3]), bnn.rotary_frequencies(16)
    kept = x.clone()
    for out in (x[:, :1].expand(4, 2, 16), x[:1].expand(4, 2, 16), torch.zeros(80, device="cuda").as_strided((4, 2, 16), (16, 8, 1))):
        with pytest.raises(bnn.BnnError):
            bnn.rotary(x, p, f, out=out)
        with pytest.raises(bnn.BnnError):
            bnn.rotary(out, p, f, out=out)
    assert torch.equal(x, kept)
    want = bnn.rotary(x, p, f)
    between = torch.zeros(2, 4, 16, device="cuda")
    assert torch.equal(bnn.rotary(x, p, f, out=between.transpose(0, 1)), want) and torch.equal(between, want.transpose(0, 1))
    assert torch.equal(bnn.rotary(x[:, :1].expand(4, 2, 16), p, f), bnn.rotary(x[:, :1].repeat(1, 2, 1), p, f))


def test_captured_and_replayed(bnn):
    """A step recorded once serves growing sequences: lengths and elements are read at replay."""
    cache, other = (bnn.Cache4(4, kv_heads=2, head_dim=64, page=16, data=torch.zeros(4, 2, oc.record_bytes(64, 16), dtype=torch.uint8, device="cuda")) for _ in range(2))
    table, lens = ints([[0, 1], [2, 3]]), ints([5, 9])
    f = bnn.rotary_frequencies(64)
    qkv = torch.randn(2, 8, 64, device="cuda")
    step = lambda c: c.write_rotary(*qkv.split((4, 2, 2), dim=1), table, lens, f)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step(cache)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(cache)
    step(other)
    for _ in range(5):
        lens += 1
        qkv.normal_()
        graph.replay()
        want = step(other)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(cache.data, other.data)


def test_another_stream(bnn):
    x, p, f = torch.randn(3000, 8, 128, device="cuda"), torch.arange(3000, dtype=torch.int32, device="cuda"), bnn.rotary_frequencies(128)
    want = bnn.rotary(x, p, f)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        y = x * 2
        got = bnn.rotary(y, p, f)
    torch.cuda.current_stream().wait_stream(stream)
    assert torch.equal(got, want * 2)
