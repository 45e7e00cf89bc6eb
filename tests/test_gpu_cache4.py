"""GPU: the 4-bit key/value cache against the oracle in 64 bits: writing and reading, selection (both exact), attention (within bounds worked out below)."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import cache4 as oc

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


@pytest.fixture(scope="module")
def bnn():
    import paper_2006_16578_amd as b
    b.load()
    return b


def rounded(x, dtype):
    """x as the type holds it, in 64 bits."""
    return torch.from_numpy(np.asarray(x, np.float64)).to(TYPES[dtype]).double().numpy()


def dev(x, dtype):
    return torch.from_numpy(np.asarray(x, np.float64)).to(TYPES[dtype]).cuda()


class Setup:
    """A cache whose unused bytes are noise, on both sides, and the plan of a batch; sequences filled by the oracle."""

    def __init__(self, bnn, seed, lens, counts=None, kv_heads=2, dim=128, page=16, signs=True, spare=2, dtype="bf16", values=None, width=None):
        self.rng = rng = np.random.default_rng(seed)
        self.lens, self.dtype = np.array(lens, np.int32), dtype
        counts = [1] * len(lens) if counts is None else counts
        need = [-(-int(n) // page) for n in lens]
        pages = sum(need) + spare
        self.data = rng.integers(0, 256, (pages, kv_heads, oc.record_bytes(dim, page, signs))).astype(np.uint8)
        order = rng.permutation(pages)
        self.table = np.full((len(lens), width or max(max(need), 1)), -1, np.int32)
        for b, n in enumerate(need):
            self.table[b, :n] = order[sum(need[:b]):sum(need[:b]) + n]
        self.counts, self.tokens = list(counts), int(sum(counts))
        self.start = None if len(set(counts)) == 1 else np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.cache = oc.Cache(self.data, dim, page, signs)
        k, v = [], []
        for n in lens:
            if values is not None:
                a, b = values(rng, int(n))
            else:
                a, b = rng.standard_normal((int(n), kv_heads, dim)) * np.exp(0.5 * rng.standard_normal(dim)), rng.standard_normal((int(n), kv_heads, dim))
            k.append(rounded(a, dtype)); v.append(rounded(b, dtype))
        self.k, self.v = k, v
        for b, n in enumerate(lens):
            if n:
                oc.write(self.cache, k[b], v[b], self.table[b:b + 1], self.lens[b:b + 1])
        self.bnn = bnn
        self.upload(signs)

    def upload(self, signs=True):
        self.gpu = self.bnn.Cache4(kv_heads=self.cache.heads, head_dim=self.cache.dim, page=self.cache.page, signs=signs, data=torch.from_numpy(self.data.copy()).cuda())
        self.replan()

    def replan(self):
        self.plan = dict(table=torch.from_numpy(self.table).cuda(), lens=torch.from_numpy(self.lens).cuda(),
                         start=None if self.start is None else torch.from_numpy(self.start).cuda())

    def queries(self, heads, spread=1.0):
        return rounded(self.rng.standard_normal((self.tokens, heads, self.cache.dim)) * spread, self.dtype)


def check_attend(su, q, scale=None, **kw):
    """Attention on the GPU against the oracle.

    Bounds, relative to the weighted mean of |v| (with u = 2^-24): a score is a sum of D exact products in fp32, in error by at most D u times the sum of
    their magnitudes (`spread`), and the scaled difference to the maximum rounds twice more; a weight's relative error is the scores' absolute one (the maximum's
    counts as well: twice), plus exp2's 2 units; weights enter the second product with 8, 16 or 24 bits; its sums add a unit for every key at most; the
    result rounds to its type.  Two units of everything are left for what is of second order."""
    scale = su.cache.dim ** -0.5 if scale is None else scale
    blocks = kw.pop("blocks", None)
    want, lse, magnitude, spread = oc.attend(su.cache, q, su.table, su.lens, su.start, scale=scale, blocks=blocks, **kw)
    got, got_lse = su.gpu.attend(dev(q, su.dtype), scale=scale, want_lse=True, blocks=None if blocks is None else torch.from_numpy(blocks).cuda(), **su.plan, **kw)
    assert got.dtype == TYPES[su.dtype] and got.shape == want.shape
    got, got_lse = got.double().cpu().numpy(), got_lse.double().cpu().numpy()
    u = 2.0 ** -24
    keys = max(1, int(su.lens.max()))
    score = (su.cache.dim + 8) * u * spread + 4 * u * np.abs(np.where(np.isfinite(lse), lse, 0))
    # rounding to nearest with p significant bits (the leading one counted) is off by at most 2^-p, relatively
    weight = {"bf16": 2.0 ** -8, "f16": 2.0 ** -16, "f32": 2.0 ** -24}[su.dtype]
    out = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": u}[su.dtype]
    bound = (2 * score + 8 * u + weight + keys * u)[..., None] * magnitude * (1 + 2.0 ** -6) + out * np.abs(want) * 1.01 + 1e-30
    if su.dtype == "f16":
        bound = bound + 2.0 ** -25                                   # subnormal results
    same = (np.isnan(want) & np.isnan(got)) | (np.abs(got - want) <= bound)
    assert same.all(), (np.abs(got - want)[~same].max(), np.argwhere(~same)[:5])
    empty = ~np.isfinite(lse) & ~np.isnan(lse)
    assert (got[empty] == 0).all() and (got_lse[empty] == lse[empty]).all()
    ok = np.isfinite(lse)
    assert (np.abs(got_lse[ok] - lse[ok]) <= (2 * score + 8 * u + keys * u + 4 * u * np.abs(lse))[ok] * (1 + 2.0 ** -6)).all()
    assert np.isnan(got_lse[np.isnan(lse)]).all()


# ------------------------------------------------------------------------------------------ writing and reading

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim,page,heads", [(64, 16, 3), (96, 32, 2), (128, 64, 2), (192, 128, 1), (256, 16, 2)])
def test_write_and_read(bnn, dtype, dim, page, heads):
    # sequences of none to many new tokens, one whose table has given a page back, one whose rows reach before its first token
    lens, counts = [40, 0, 131, 17, 1, 5], [7, 0, 131, 1, 1, 8]
    su = Setup(bnn, 1, lens, counts, heads, dim, page, dtype=dtype)
    su.table[2, 1] = -1
    su.table[3, 0] = su.data.shape[0] + 5 if page < 17 else su.table[3, 0]
    su.replan()
    scale = 2.0 ** su.rng.integers(-9, 9, (su.tokens, heads, 1))
    k, v = (rounded(su.rng.standard_normal((su.tokens, heads, dim)) * scale, dtype) for _ in range(2))
    k[3, 0, :32] = 0.0
    k[4, 0, 5], k[5, 0, 6], v[6, heads - 1, 40] = np.inf, np.nan, -np.inf
    k[9, 0, 0::2] = -0.0
    oc.write(su.cache, k, v, su.table, su.lens, su.start)
    su.gpu.write(dev(k, dtype), dev(v, dtype), **su.plan)
    got = su.gpu.data.cpu().numpy()
    nan_codes = np.zeros(su.data.shape, bool)                        # the codes of a group that holds a NaN are not stated
    for p, h in np.ndindex(su.data.shape[:2]):
        rec = oc.Record(nan_codes[p, h], page, dim)
        mine = su.cache.records[p][h]
        for name in "kv":
            rec.codes[name][...] = np.repeat(mine.scales[name].T == 255, 16, axis=1)
    assert (np.where(nan_codes, 0, got) == np.where(nan_codes, 0, su.data)).all()
    su.data[...] = got
    want_k, want_v = oc.read(su.cache, su.table, su.lens, su.start, su.tokens)
    for out in ("f32", "bf16", "f16"):
        a, b = su.gpu.read(tokens=su.tokens, dtype=TYPES[out], **su.plan)
        assert a.dtype == TYPES[out] and torch.equal(torch.nan_to_num(a, 777), torch.nan_to_num(dev(want_k, out), 777))
        assert torch.equal(torch.nan_to_num(b, 777), torch.nan_to_num(dev(want_v, out), 777))
    assert np.isnan(want_k[4, 0, :32]).all() and not np.isnan(want_k[4, 0, 32:]).any()


def test_every_rounding_case(bnn):
    # ties, neighbours of ties, saturation, the ends of the range of scales, subnormals; fp32
    near = lambda x: [np.nextafter(np.float32(x), np.float32(0)), x, np.nextafter(np.float32(x), np.float32(9e9))]
    points = [p for x in (0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6) for p in near(x)]
    groups = []
    for high in near(6.0) + near(3.0) + near(4.5):
        for e in (-140, -101, -100, -99, -3, 0, 50, 99, 100):
            g = np.array(([high] + [p for p in points if p <= high] + [0] * 64)[:64]) * 2.0 ** e
            groups += [g[:32], -g[:32], np.concatenate([g[:1], g[32:63]])]
    groups += [np.full(32, 3e38), np.linspace(-3e38, 3e38, 32), np.full(32, 1e-45), np.full(32, 2.0 ** -103), np.array([2.0 ** -102] + [2.0 ** -103] * 31)]
    x = np.float32(np.concatenate(groups + [np.zeros(32)] * (-len(groups) % 4))).astype(np.float64).reshape(-1, 1, 128)
    lens = [len(x)]
    su = Setup(bnn, 2, lens, lens, 1, 128, 64, dtype="f32")
    oc.write(su.cache, x, -x, su.table, su.lens)
    su.gpu.write(dev(x, "f32"), dev(-x, "f32"), **su.plan)
    assert (su.gpu.data.cpu().numpy() == su.data).all()


def test_strided_inputs_and_no_signs(bnn):
    # k, v and q as slices of one projection's output, and heads before tokens
    su = Setup(bnn, 3, [30, 9], [4, 4], 2, 64, 16, signs=False, dtype="bf16")
    fused = dev(su.rng.standard_normal((8, 8 * 64)), "bf16")
    q, k, v = fused[:, :256].view(8, 4, 64), fused[:, 256:384].view(8, 2, 64), fused[:, 384:].view(8, 2, 64)
    host = lambda t: t.double().cpu().numpy()
    oc.write(su.cache, host(k), host(v), su.table, su.lens)
    su.gpu.write(k, v, **su.plan)
    assert (su.gpu.data.cpu().numpy() == su.data).all()
    a = su.gpu.attend(q, **su.plan)
    assert torch.equal(a, su.gpu.attend(q.contiguous(), **su.plan))
    assert torch.equal(a, su.gpu.attend(q.transpose(0, 1).contiguous().transpose(0, 1), **su.plan))
    check_attend(su, host(q))
    # a dimension of one entry, whatever its stride says
    one = torch.as_strided(q[:1].contiguous(), (1, 4, 64), (3, 64, 1))
    plan = dict(table=su.plan["table"][:1], lens=su.plan["lens"][:1])
    assert torch.equal(su.gpu.attend(one, **plan), su.gpu.attend(q[:1].contiguous(), **plan))
    with pytest.raises(ValueError):
        su.gpu.write(k.transpose(1, 2), v, **su.plan)
    with pytest.raises(bnn.BnnError) as e:                           # no signs were kept
        su.gpu.select(q, keep=2, **su.plan)
    assert e.value.status == -1


# ------------------------------------------------------------------------------------------ selection

@pytest.mark.parametrize("dim,page,heads,group,dtype", [(64, 16, 2, 5, "f32"), (96, 32, 1, 1, "bf16"), (128, 64, 2, 8, "bf16"), (192, 16, 1, 9, "f16"), (256, 128, 1, 17, "f32"), (64, 32, 1, 40, "bf16"),
                                                        (96, 16, 1, 3, "f16")])
def test_select(bnn, dim, page, heads, group, dtype):
    su = Setup(bnn, 4, [page * 9 + 3, page * 4, 1, 0, page * 20 + 1], [3, 2, 1, 1, 4], heads, dim, page, dtype=dtype)
    su.table[4, 3] = su.table[4, 11] = -1
    su.table[4, 0] = 1 << 20
    su.replan()
    q = su.queries(heads * group)
    q[0, 0, 0], q[0, 0, 1] = -0.0, np.nan
    for keep, first, last in ((2, 1, 1), (5, 1, 1), (5, 0, 0), (6, 2, 3), (1, 0, 1), (40, 1, 2), (7, 7, 0)):
        want = oc.select(su.cache, q, su.table, su.lens, keep, su.start, first, last)
        got = su.gpu.select(dev(q, dtype), keep=keep, first=first, last=last, **su.plan).cpu().numpy()
        assert (got == want).all(), (keep, first, last)


@pytest.mark.parametrize("blocks,keep", [(255, 17), (256, 100), (257, 256), (700, 64), (1030, 3), (2100, 40)])
def test_select_among_many_with_ties(bnn, blocks, keep):
    # keys from a few patterns only: long ties, broken by the lowest index
    def values(rng, n):
        patterns = rng.standard_normal((3, 1, 64))
        x = patterns[rng.integers(0, 3, n // 16 + 1).repeat(16)[:n]]
        return x, x
    su = Setup(bnn, 5, [blocks * 16 - 2, 16 * 31], [2, 2], 1, 64, 16, values=values)
    q = su.queries(2)
    want = oc.select(su.cache, q, su.table, su.lens, keep)
    assert (su.gpu.select(dev(q, "bf16"), keep=keep, **su.plan).cpu().numpy() == want).all()
    # a cache where every block scores the same
    q[:] = 1.0
    su.data[...] = 0
    su.upload()
    want = oc.select(su.cache, q, su.table, su.lens, keep, first=0, last=0)
    assert (su.gpu.select(dev(q, "bf16"), keep=keep, first=0, last=0, **su.plan).cpu().numpy() == want).all() and want[0, 0, 0] == 0


def test_select_for_many_tokens(bnn):
    # chunks whose tokens see different numbers of blocks, several tokens to a tile of the products
    su = Setup(bnn, 20, [610, 700, 33], [600, 590, 33], 1, 64, 16)
    for heads, keep in ((3, 7), (1, 20), (6, 3)):
        q = su.queries(heads)
        want = oc.select(su.cache, q, su.table, su.lens, keep, su.start)
        assert (su.gpu.select(dev(q, "bf16"), keep=keep, **su.plan).cpu().numpy() == want).all(), heads


# ------------------------------------------------------------------------------------------ attention

@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim,page,heads,group", [(64, 16, 2, 1), (64, 64, 1, 16), (96, 32, 2, 3), (128, 64, 2, 4), (128, 16, 1, 20), (192, 128, 1, 6), (256, 16, 2, 2)])
def test_attend_single_tokens(bnn, dtype, dim, page, heads, group):
    su = Setup(bnn, 6, [1, 16, 0, 31, 33, 100, 515], None, heads, dim, page, dtype=dtype)
    check_attend(su, su.queries(heads * group))
    check_attend(su, su.queries(heads * group, 6.0), scale=0.5, window=20)
    check_attend(su, su.queries(heads * group), causal=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim,page,heads,group", [(64, 32, 1, 2), (96, 16, 1, 5), (128, 64, 2, 3), (192, 16, 1, 1), (256, 32, 1, 2)])
def test_attend_many_tokens(bnn, dtype, dim, page, heads, group):
    # whole prompts, chunks, more rows than tokens, sequences without rows; ragged
    su = Setup(bnn, 7, [75, 0, 130, 3, 40, 1], [75, 0, 50, 9, 0, 1], heads, dim, page, dtype=dtype)
    q = su.queries(heads * group)
    check_attend(su, q)
    check_attend(su, q, window=11)
    check_attend(su, q, causal=False)
    # the same number of rows everywhere
    su = Setup(bnn, 8, [33, 70, 50], [33, 33, 33], heads, dim, page, dtype=dtype)
    check_attend(su, su.queries(heads * group, 3.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
def test_attend_chunks_of_a_long_cache(bnn, dim, dtype):
    # many rows at the end of a few hundred keys: several steps before any mask, pages given back, a window that starts in the middle; and keys cut into parts
    su = Setup(bnn, 19, [700, 333, 65], [40, 70, 65], 1, dim, 64, dtype=dtype, width=80)
    su.table[0, 3] = su.table[1, 0] = -1
    su.replan()
    q = su.queries(3, 2.0)
    check_attend(su, q)
    check_attend(su, q, window=150)


def test_attend_ragged_batch_of_many_sequences(bnn):
    # more sequences than lanes of a wave
    rng = np.random.default_rng(0)
    counts = rng.integers(0, 5, 150)
    counts[[0, 63, 64, 127, 149]] = [0, 0, 3, 4, 2]
    lens = counts + rng.integers(0, 40, 150)
    su = Setup(bnn, 9, lens, counts, 1, 64, 16)
    check_attend(su, su.queries(3))
    q = su.queries(3)
    want = oc.select(su.cache, q, su.table, su.lens, 2, su.start)
    assert (su.gpu.select(dev(q, "bf16"), keep=2, **su.plan).cpu().numpy() == want).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_attend_long_cache_in_parts(bnn, dtype):
    # long enough that the keys are cut into parts and joined; a short sequence beside it
    su = Setup(bnn, 10, [5003, 300], None, 1, 64, 64, dtype=dtype, width=300)
    check_attend(su, su.queries(4, 2.0))
    check_attend(su, su.queries(4), window=3000)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim,page,heads,group", [(64, 16, 2, 5), (128, 64, 1, 8), (128, 32, 1, 24), (96, 128, 1, 1), (256, 16, 1, 3)])
def test_attend_over_blocks(bnn, dtype, dim, page, heads, group):
    su = Setup(bnn, 11, [page * 12 + 5, page * 3, 0, 7, 2], [4, 2, 1, 7, 3], heads, dim, page, dtype=dtype)
    su.table[0, 4] = -1
    su.replan()
    q = su.queries(heads * group)
    check_attend(su, q, blocks=oc.select(su.cache, q, su.table, su.lens, 5, su.start))
    # any order, entries that are no block, blocks of the future, one listed twice; nothing at all
    blocks = np.full((su.tokens, heads, 7), -1, np.int32)
    blocks[0, 0] = [9, 2, 0, 4, -1, 1 << 20, 12]
    blocks[1, 0] = [3, 3, -7, 2 ** 31 - 1, -2 ** 31, 1, 0]
    blocks[4, heads - 1] = [2, 1, 0, 13, 40, -1, -1]
    check_attend(su, q, blocks=blocks)
    check_attend(su, q, blocks=blocks, window=page + 3)
    check_attend(su, q, blocks=blocks, causal=False)


@pytest.mark.parametrize("counts", [[1, 1, 1], [20, 20, 20], [40, 3, 1], [44, 44, 44], [60, 41, 44]])
def test_what_is_masked_does_not_arrive(bnn, counts):
    # NaN keys and values: rows that see them become NaN, rows before them and other heads and sequences do not
    lens = [60, 50, 44]
    su = Setup(bnn, 12, lens, counts, 2, 128, 16, dtype="bf16")
    for b, pos, h, name, element in ((0, 40, 0, "v", 70), (1, 47, 1, "k", 3), (0, 59, 1, "v", 0), (2, 43, 0, "v", 127), (2, 10, 1, "v", 33)):
        rec = su.cache.record(su.table, b, pos, h)
        rec.scales[name][element // 32, pos % 16] = 255
    su.upload()
    q = su.queries(6)
    check_attend(su, q)
    check_attend(su, q, window=8)
    check_attend(su, q, causal=False)
    blocks = oc.select(su.cache, q, su.table, su.lens, 2, su.start)
    check_attend(su, q, blocks=blocks)


def test_scores_of_any_size(bnn):
    # scores far apart, rising and falling along the keys, and queries that are zero, infinite or NaN
    def values(rng, n):
        k = rng.standard_normal((n, 1, 64)) * np.linspace(0.01, 300, n)[rng.permutation(n) if n % 2 else slice(None), None, None]
        return k, rng.standard_normal((n, 1, 64)) * 2.0 ** rng.integers(-60, 60, (n, 1, 1))
    for dtype in ("f32", "bf16"):
        su = Setup(bnn, 13, [700, 701, 64], None, 1, 64, 16, dtype=dtype, values=values)
        q = su.queries(4, 40.0)
        q[:, 1] = 0
        q[:, 2] = rounded(q[:, 2] * 1e4, dtype)
        check_attend(su, q)
        q[0, 3, 5], q[1, 3, 0] = np.nan, np.nan
        check_attend(su, q)


def test_offsets_beyond_32_bits(bnn):
    # 5 GB of cache, the pages in use at its end
    page, dim = 64, 128
    record = oc.record_bytes(dim, page)
    pages = 5 * 10 ** 9 // record
    su = Setup(bnn, 14, [200, 130], [3, 3], 1, dim, page)
    n = su.data.shape[0]
    big = torch.zeros((pages, 1, record), dtype=torch.uint8, device="cuda")
    big[-n:] = torch.from_numpy(su.data).cuda()
    su.gpu = bnn.Cache4(kv_heads=1, head_dim=dim, page=page, data=big)
    su.plan["table"] = torch.where(su.plan["table"] >= 0, su.plan["table"] + (pages - n), su.plan["table"])
    q = su.queries(2)
    check_attend(su, q)
    assert (su.gpu.select(dev(q, "bf16"), keep=2, **su.plan).cpu().numpy() == oc.select(su.cache, q, su.table, su.lens, 2)).all()
    k = su.rng.standard_normal((6, 1, dim))
    oc.write(su.cache, rounded(k, "bf16"), rounded(k, "bf16"), su.table, su.lens)
    su.gpu.write(dev(k, "bf16"), dev(k, "bf16"), **su.plan)
    assert (big[-n:].cpu().numpy() == su.data).all() and not big[:-n].any()
    a, _ = su.gpu.read(tokens=6, dtype=torch.float32, **su.plan)
    assert torch.equal(a, dev(oc.read(su.cache, su.table, su.lens, None, 6)[0], "f32"))


def test_no_tokens_other_streams_and_repeats(bnn):
    su = Setup(bnn, 15, [1000, 77], [2, 2], 2, 128, 32, width=200)
    q = dev(su.queries(8), "bf16")
    empty = q[:0]
    plan = dict(table=su.plan["table"], lens=su.plan["lens"])
    assert su.gpu.attend(empty, **plan).shape == (0, 8, 128) and su.gpu.select(empty, keep=3, **plan).shape == (0, 2, 3)
    su.gpu.write(empty[:, :2], empty[:, :2], **plan)
    assert su.gpu.read(tokens=0, **plan)[0].shape == (0, 2, 128)
    blocks = su.gpu.select(q, keep=4, **plan)
    want = su.gpu.attend(q, **plan), su.gpu.attend(q, blocks=blocks, **plan), blocks
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):                                               # another stream than the tensors' own; results do not depend on the run
        with torch.cuda.stream(s):
            again = su.gpu.attend(q, **plan), su.gpu.attend(q, blocks=blocks, **plan), su.gpu.select(q, keep=4, **plan)
        s.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, again))


def test_recorded_into_a_graph(bnn):
    # a decoding step recorded once, replayed as the sequences grow: the plan's contents are read by the kernels
    su = Setup(bnn, 16, [300, 40], None, 2, 64, 16, width=64)
    su.table[0] = np.arange(64) % su.data.shape[0]
    su.replan()
    q, k = dev(su.queries(4), "bf16"), dev(su.queries(2), "bf16")
    su.table[1, :3] = su.plan["table"].cpu().numpy()[1, :3]

    def step():
        su.gpu.write(k, k, **su.plan)
        blocks = su.gpu.select(q, keep=5, **su.plan)
        return blocks, su.gpu.attend(q, blocks=blocks, **su.plan), su.gpu.attend(q, **su.plan)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        recorded = step()
    for i in range(4):
        q.copy_(torch.randn_like(q.float()))
        k.copy_(torch.randn_like(k.float()))
        su.plan["lens"].add_(1)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in recorded]
        assert all(torch.equal(torch.nan_to_num(a.float(), 777), torch.nan_to_num(b.float(), 777)) for a, b in zip(got, step())), i


def test_native_module_and_ctypes_agree(bnn, monkeypatch):
    # the native module serves ordinary calls; without it, and for what is out of the ordinary, ctypes gives the same
    from paper_2006_16578_amd import binding
    su = Setup(bnn, 18, [300, 40, 77], [4, 1, 3], 2, 64, 16, width=40)
    q, k = dev(su.queries(4), "bf16"), dev(su.queries(2), "bf16")
    binding._load_native()
    native, served = binding._native, []

    class Counted:
        def __getattr__(self, name):
            return lambda *args: served.append((name, getattr(native, name)(*args))) or served[-1][1]

    def calls(keep=5):
        su.gpu.write(k, k, **su.plan)
        blocks = su.gpu.select(q, keep=keep, **su.plan)
        return (blocks, *su.gpu.read(tokens=8, dtype=torch.float32, **su.plan), su.gpu.attend(q, **su.plan), su.gpu.attend(q, blocks=blocks, **su.plan),
                *su.gpu.attend(q, want_lse=True, window=9, scale=0.3, **su.plan))

    monkeypatch.setattr(binding, "_native", Counted())
    fast = calls()
    assert [n for n, r in served] == ["cache4_write", "cache4_select", "cache4_read"] + ["cache4_attend"] * 3 and all(r is not None for n, r in served)
    slow_too = calls(np.int64(5))                                    # a number that is no int: select goes by ctypes
    assert served[len(served) // 2 + 1][1] is None
    monkeypatch.setattr(binding, "_native", binding._PythonOnly())
    for a, b, c in zip(fast, calls(), slow_too):
        assert a.dtype == b.dtype and torch.equal(torch.nan_to_num(a.float(), 7), torch.nan_to_num(b.float(), 7)) and torch.equal(torch.nan_to_num(a.float(), 7), torch.nan_to_num(c.float(), 7))
    monkeypatch.setattr(binding, "_native", native)
    torch._C._set_throw_on_mutable_data_ptr(q)                       # no pointer: raised, with the interpreter lock held
    with pytest.raises(RuntimeError, match="data pointer"):
        su.gpu.attend(q, **su.plan)


def test_refusals(bnn):
    su = Setup(bnn, 17, [30, 9], None, 2, 64, 16)
    q, k = dev(su.queries(4), "bf16"), dev(su.queries(2), "bf16")
    plan = su.plan
    for fn, error in ((lambda: su.gpu.write(k, k.float(), **plan), ValueError), (lambda: su.gpu.write(k.cpu(), k, **plan), TypeError),
                      (lambda: su.gpu.write(k.double(), k.double(), **plan), TypeError), (lambda: su.gpu.write(q, q, **plan), ValueError),
                      (lambda: su.gpu.attend(q[..., :32], **plan), ValueError), (lambda: su.gpu.attend(q[:, 0], **plan), ValueError),
                      (lambda: su.gpu.attend(q, plan["table"].long(), plan["lens"]), TypeError), (lambda: su.gpu.attend(q, plan["table"], plan["lens"][:1]), ValueError),
                      (lambda: su.gpu.attend(q, plan["table"], plan["lens"], start=plan["lens"]), ValueError),
                      (lambda: su.gpu.attend(q, out=q.float(), **plan), TypeError), (lambda: su.gpu.attend(q, out=q[:1], **plan), ValueError),
                      (lambda: su.gpu.attend(q, blocks=torch.zeros((1, 2, 3), dtype=torch.int32, device="cuda"), **plan), ValueError),
                      (lambda: su.gpu.attend(q[:, :3], **plan), bnn.BnnError), (lambda: su.gpu.attend(q[:1], **plan), bnn.BnnError),
                      (lambda: su.gpu.attend(q, scale=0.0, **plan), bnn.BnnError), (lambda: su.gpu.attend(q, window=3, causal=False, **plan), bnn.BnnError),
                      (lambda: su.gpu.select(q, keep=1, **plan), bnn.BnnError), (lambda: su.gpu.read(dtype=torch.float64, **plan), TypeError),
                      (lambda: bnn.Cache4(kv_heads=2, head_dim=64, page=32, data=su.gpu.data), ValueError), (lambda: bnn.Cache4(kv_heads=2, head_dim=64), ValueError)):
        with pytest.raises(error):
            fn()
    assert (su.gpu.data.cpu().numpy() == su.data).all()


def check_far_scores(su, q, scale, blocks=None):
    """Attention where scores lie so far apart that a row has the value of its best key, or the mean over keys that equal it.  Rows whose best and next score are
    nearer than twice the error of a score (D + 8 units of fp32 of the sum of magnitudes, 4 of itself) plus 60 are left out; returns the share of the others."""
    u, dim, heads = 2.0 ** -24, su.cache.dim, su.cache.heads
    got, got_lse = su.gpu.attend(dev(q, su.dtype), scale=scale, want_lse=True, blocks=None if blocks is None else torch.from_numpy(blocks).cuda(), **su.plan)
    got, got_lse = got.double().cpu().numpy(), got_lse.double().cpu().numpy()
    weight = {"bf16": 2.0 ** -8, "f16": 2.0 ** -16, "f32": 2.0 ** -24}[su.dtype]
    out = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": u}[su.dtype]
    group, sure = q.shape[1] // heads, []
    for t, (b, pos) in enumerate(oc.row_places(su.cache, su.table, su.lens, su.start, su.tokens)):
        for h in range(heads):
            keys = [p for p in range(pos + 1) if blocks is None or p // su.cache.page in blocks[t, h]]
            if not keys:
                continue
            k, v = (np.stack([su.cache.record(su.table, b, p, h).get(name, p % su.cache.page) for p in keys]) for name in "kv")
            for g in range(h * group, (h + 1) * group):
                s = scale * (k @ q[t, g])
                error = (dim + 8) * u * scale * (np.abs(k) @ np.abs(q[t, g])).max() + 4 * u * np.abs(s).max()
                best = np.flatnonzero(s > s.max() - 2 * error - 60)
                sure.append((k[best] == k[best[0]]).all())
                if sure[-1]:
                    want, size = v[best].mean(0), np.abs(v[best]).mean(0)
                    assert (np.abs(got[t, g] - want) <= (weight + (8 + len(best)) * u) * size * 1.02 + out * np.abs(want) * 1.01 + 2.0 ** -25).all(), (t, g)
                    assert abs(got_lse[t, g] - s.max() - np.log(len(best))) <= error + 8 * u * abs(s.max()), (t, g)
    return np.mean(sure)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_scores_beyond_what_fp32_resolves(bnn, dtype):
    same = lambda rng, n: (np.repeat(rng.standard_normal((1, 1, 64)), n, 0), rng.standard_normal((n, 1, 64)))
    for values in (None, same):
        single = Setup(bnn, 21, [1, 40, 700], None, 1, 64, 16, dtype=dtype, values=values)
        parts = Setup(bnn, 22, [2100, 300], None, 1, 64, 64, dtype=dtype, width=100, values=values)
        many = Setup(bnn, 23, [75, 130], [75, 40], 1, 64, 32, dtype=dtype, values=values)
        q = parts.queries(3)
        blocks = oc.select(parts.cache, q, parts.table, parts.lens, 3)
        for power in (20, 33, 70):
            assert check_far_scores(single, single.queries(5), 2.0 ** power) > 0.8
            assert check_far_scores(parts, q, 2.0 ** power) > 0.8
            assert check_far_scores(parts, q, 2.0 ** power, blocks) > 0.8
            assert check_far_scores(many, many.queries(2), 2.0 ** power) > 0.8


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_infinite_queries(bnn, dtype):
    # scores that are all -infinity, all +infinity, or some of each: no weights are defined, the row is NaN; others are not touched
    def values(rng, n):
        k = rng.standard_normal((n, 1, 64))
        k[..., 0] = -2 - rng.random((n, 1))
        return k, rng.standard_normal((n, 1, 64))
    for lens, counts in (([1, 40, 700], None), ([75, 130], [75, 40])):
        su = Setup(bnn, 24, lens, counts, 1, 64, 32, dtype=dtype, values=values)
        q = su.queries(4)
        q[0, 0, 0], q[1, 1, 0], q[-1, 2, 5], q[-1, 0, 0] = np.inf, -np.inf, np.inf, np.inf
        check_attend(su, q)


@pytest.mark.parametrize("counts", [[8, 8], [70, 66]])
def test_more_tokens_than_the_table_holds(bnn, counts):
    # the newest tokens of the first sequence lie past the end of its table: they are dropped, and nothing that the table holds is touched
    su = Setup(bnn, 26, [64, 66], counts, 2, 64, 16, dtype="f32", width=5)
    su.table = np.ascontiguousarray(su.table[:, :4])
    su.lens[:] = 73, 66
    su.replan()
    k, v = (rounded(su.rng.standard_normal((su.tokens, 2, 64)), "f32") for _ in range(2))
    oc.write(su.cache, k, v, su.table, su.lens, su.start)
    su.gpu.write(dev(k, "f32"), dev(v, "f32"), **su.plan)
    assert (su.gpu.data.cpu().numpy() == su.data).all()
    want = oc.read(su.cache, su.table, su.lens, su.start, su.tokens)
    assert all(torch.equal(a, dev(b, "f32")) for a, b in zip(su.gpu.read(tokens=su.tokens, dtype=torch.float32, **su.plan), want)) and (want[0][counts[0] - 1] == 0).all()
    q = su.queries(6)
    check_attend(su, q)
    check_attend(su, q, window=20)
    check_attend(su, q, causal=False)
    for keep, first, last in ((2, 1, 1), (3, 0, 2), (6, 1, 1)):
        blocks = oc.select(su.cache, q, su.table, su.lens, keep, su.start, first, last)
        assert (su.gpu.select(dev(q, "f32"), keep=keep, first=first, last=last, **su.plan).cpu().numpy() == blocks).all(), (keep, first, last)
        check_attend(su, q, blocks=blocks)


@pytest.mark.parametrize("counts", [[8, 8, 3], [70, 66, 64]])
def test_windows_of_any_size(bnn, counts):
    # rows that reach before the first token of their sequence, and a window that no sequence fills
    su = Setup(bnn, 25, [5, 66, 3], counts, 1, 64, 16, dtype="f32")
    q = su.queries(2)
    for window in (2 ** 31 - 1, 2 ** 31 - 60, 2 ** 30):
        check_attend(su, q, window=window)
        check_attend(su, q, window=window, blocks=oc.select(su.cache, q, su.table, su.lens, 3, su.start))


@pytest.mark.parametrize("group", [1, 3, 40])
def test_no_plan_leads_out(bnn, group):
    # tables, lengths and starts of any content: calls end, and bytes around the cache, the outputs and the workspaces stay as they are
    rng, dim, page, heads, pages, batch, tokens, width = np.random.default_rng(30), 64, 16, 2, 12, 5, 40, 6
    record = oc.record_bytes(dim, page)
    memory = torch.full((pages + 8, heads, record), 0xA5, dtype=torch.uint8, device="cuda")
    cache = bnn.Cache4(kv_heads=heads, head_dim=dim, page=page, data=memory[4:-4])
    q = torch.randn(tokens, heads * group, dim, device="cuda")
    outs = torch.full((tokens + 2, heads * group, dim), 7.0, device="cuda")

    def guarded(need):
        whole = torch.full((need + 512,), 0xFF, dtype=torch.uint8, device="cuda")
        return whole, whole[256:-256]

    def untouched(whole):
        return bool((whole[:256] == 0xFF).all() and (whole[-256:] == 0xFF).all())

    plans = [dict(start=rng.choice([-2 ** 31, -3, 0, 7, 20, 40, 41, 2 ** 31 - 1], batch + 1)) for _ in range(8)] + [dict(start=None) for _ in range(4)]
    plans.append(dict(start=np.array([0, 20, 0, 40, 40, 40]), lens=np.full(batch, 96)))          # rows whose scores no workgroup writes
    for plan in plans:
        plan.setdefault("lens", rng.choice([-2 ** 31, -1, 0, 5, 40, 96, 97, 500, 2 ** 31 - 1], batch))
        plan["table"] = rng.choice([-2 ** 31, -1, pages, pages + 1, 2 ** 31 - 1, *range(pages), *range(pages)], (batch, width))
        print(plan, flush=True)
        plan = {name: None if x is None else torch.from_numpy(x.astype(np.int32)).cuda() for name, x in plan.items()}
        cache.write(q[:, :heads], q[:, :heads], **plan)
        cache.read(tokens=tokens, **plan)
        rows = cache._rows(plan["table"], plan["lens"], plan["start"], tokens)
        lists = [None, torch.from_numpy(rng.integers(-2, width + 2, (tokens, heads, 3)).astype(np.int32)).cuda()]
        for keep in (2, 9):
            whole, work = guarded(int(bnn.load().bnn_cache4_select_workspace_bytes(cache._struct(), ctypes.byref(rows))))
            lists.append(cache.select(q, keep=keep, workspace=work, **plan))
            assert untouched(whole)
        for blocks in lists:
            for kw in (dict(), dict(window=30), dict(causal=False)):
                need = int(bnn.load().bnn_cache4_attend_workspace_bytes(cache._struct(), ctypes.byref(rows), 0, heads * group, kw.get("window", 0), 0 if blocks is None else blocks.shape[2]))
                whole, work = guarded(need)
                cache.attend(q, blocks=blocks, out=outs[1:-1], workspace=work, **plan, **kw)
                assert untouched(whole)
        assert (outs[0] == 7).all() and (outs[-1] == 7).all() and (memory[:4] == 0xA5).all() and (memory[-4:] == 0xA5).all()
    assert (lists[2] < width).all() and (lists[3] < width).all()


@pytest.mark.parametrize("native", [True, False])
def test_an_empty_list_of_blocks(bnn, monkeypatch, native):
    # refused: it is not "no list", which attends to every key
    from paper_2006_16578_amd import binding
    if not native:
        monkeypatch.setattr(binding, "_native", binding._PythonOnly())
    su = Setup(bnn, 27, [30, 9], None, 2, 64, 16)
    q = dev(su.queries(4), "bf16")
    blocks = su.gpu.select(q, keep=2, **su.plan)
    with pytest.raises(ValueError, match="keep >= 1"):
        su.gpu.attend(q, blocks=blocks[:, :, :0], **su.plan)
    assert torch.equal(su.gpu.attend(q, blocks=blocks[:, :, :1].contiguous(), **su.plan), su.gpu.attend(q, blocks=torch.cat([blocks[:, :, :1], torch.full_like(blocks, -1)], 2), **su.plan))


@pytest.mark.parametrize("native", [True, False])
def test_blocks_of_no_tokens(bnn, monkeypatch, native):
    from paper_2006_16578_amd import binding
    if not native:
        monkeypatch.setattr(binding, "_native", binding._PythonOnly())
    su = Setup(bnn, 27, [30, 9], None, 2, 64, 16)
    q = dev(su.queries(4), "bf16")[:0]
    blocks = su.gpu.select(q, keep=3, **su.plan)
    out, lse = su.gpu.attend(q, blocks=blocks, want_lse=True, **su.plan)
    assert blocks.shape == (0, 2, 3) and out.shape == (0, 4, 64) and lse.shape == (0, 4)


def test_workspace_and_out_of_the_caller(bnn):
    # the same results in memory that the caller gives; what is no memory of the cache's device, or not enough, is refused before anything runs
    su = Setup(bnn, 31, [5000, 300], None, 1, 64, 64, width=200)
    q = dev(su.queries(4), "bf16")
    rows = su.gpu._rows(su.plan["table"], su.plan["lens"], None, 2)
    need = int(bnn.load().bnn_cache4_select_workspace_bytes(su.gpu._struct(), ctypes.byref(rows)))
    need_attend = int(bnn.load().bnn_cache4_attend_workspace_bytes(su.gpu._struct(), ctypes.byref(rows), 1, 4, 0, 0))
    assert need == 2 * 200 * 2 and need_attend > 0                     # (the keys are cut into parts)
    memory = lambda n, **kw: torch.full((n,), 0xFF, dtype=torch.uint8, **{"device": "cuda", **kw})
    blocks, out = su.gpu.select(q, keep=4, **su.plan), torch.empty_like(q)
    assert torch.equal(su.gpu.select(q, keep=4, workspace=memory(need), **su.plan), blocks)
    assert su.gpu.attend(q, out=out, workspace=memory(need_attend), **su.plan) is out and torch.equal(out, su.gpu.attend(q, **su.plan))
    for bad, error in ((lambda n: memory(n, device="cpu"), TypeError), (lambda n: memory(1).expand(n), ValueError), (lambda n: memory(2 * n)[::2], ValueError),
                       (lambda n: memory(n).view(torch.int16), TypeError), (lambda n: memory(n).view(1, n), ValueError), (lambda n: memory(n - 1), bnn.BnnError),
                       (lambda n: memory(n + 1)[1:], bnn.BnnError), (lambda n: memory(0), bnn.BnnError)):
        with pytest.raises(error):
            su.gpu.select(q, keep=4, workspace=bad(need), **su.plan)
        with pytest.raises(error):
            su.gpu.attend(q, workspace=bad(need_attend), **su.plan)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dim,heads,group", [(64, 2, 3), (96, 1, 40), (128, 1, 4), (192, 1, 6), (256, 1, 35)])
def test_pages_of_256(bnn, dtype, dim, heads, group):
    su = Setup(bnn, 28, [1100, 256, 1, 257, 0], [3, 1, 1, 2, 0], heads, dim, 256, dtype=dtype)
    k = rounded(su.rng.standard_normal((su.tokens, heads, dim)), dtype)
    oc.write(su.cache, k, -k, su.table, su.lens, su.start)
    su.gpu.write(dev(k, dtype), dev(-k, dtype), **su.plan)
    assert (su.gpu.data.cpu().numpy() == su.data).all()
    want = oc.read(su.cache, su.table, su.lens, su.start, su.tokens)
    assert all(torch.equal(a, dev(b, "f32")) for a, b in zip(su.gpu.read(tokens=su.tokens, dtype=torch.float32, **su.plan), want))
    q = su.queries(heads * group)
    for keep, first, last in ((2, 1, 1), (3, 0, 1), (4, 0, 0), (9, 1, 1)):
        blocks = oc.select(su.cache, q, su.table, su.lens, keep, su.start, first, last)
        assert (su.gpu.select(dev(q, dtype), keep=keep, first=first, last=last, **su.plan).cpu().numpy() == blocks).all(), (keep, first, last)
        check_attend(su, q, blocks=blocks)
    check_attend(su, q)
    check_attend(su, q, window=300)
    su = Setup(bnn, 29, [300, 520], [70, 66], heads, dim, 256, dtype=dtype)          # many rows
    q = su.queries(heads * min(group, 4))
    check_attend(su, q)
    assert (su.gpu.select(dev(q, dtype), keep=2, **su.plan).cpu().numpy() == oc.select(su.cache, q, su.table, su.lens, 2, su.start)).all()
