"""GPU: attention weight per cached token, the choice of tokens to keep, and moving them, against the oracle."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import cache4 as oc
from oracle import decoding as od

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24


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


class Batch:
    """A cache whose unused bytes are noise, sequences in it, the newest tokens' queries."""

    def __init__(self, bnn, seed, lens, counts=None, kv_heads=2, group=2, dim=64, page=16, dtype="bf16", signs=True, width=None, spread=1.0):
        self.rng = rng = np.random.default_rng(seed)
        self.lens, self.dtype, self.dim, self.page, self.kv_heads, self.heads = np.array(lens, np.int32), dtype, dim, page, kv_heads, kv_heads * group
        counts = [1] * len(lens) if counts is None else counts
        need = [-(-int(n) // page) for n in lens]
        self.data = rng.integers(0, 256, (sum(need) + 3, kv_heads, oc.record_bytes(dim, page, signs))).astype(np.uint8)
        order = rng.permutation(len(self.data))
        self.table = np.full((len(lens), width or max(max(need), 1)), -1, np.int32)
        for b, n in enumerate(need):
            m = min(n, self.table.shape[1])
            self.table[b, :m] = order[sum(need[:b]):sum(need[:b]) + m]
        self.tokens = int(sum(counts))
        self.start = None if len(set(counts)) == 1 else np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
        self.oracle = oc.Cache(self.data, dim, page, signs)
        for b, n in enumerate(lens):
            if n:
                k, v = (rounded(rng.standard_normal((n, kv_heads, dim)), dtype) for _ in range(2))
                oc.write(self.oracle, k, v, self.table[b:b + 1], self.lens[b:b + 1])
        self.q = rounded(rng.standard_normal((self.tokens, self.heads, dim)) * spread, dtype)
        self.gpu = bnn.Cache4(kv_heads=kv_heads, head_dim=dim, page=page, signs=signs, data=torch.from_numpy(self.data.copy()).cuda())

    def plan(self):
        return dict(table=ints(self.table), lens=ints(self.lens), start=None if self.start is None else ints(self.start))


def check_weigh(su, scale=None, causal=True, window=0, decay=1.0, previous=True, extra=0, q=None):
    """Bounds, with u = 2^-24: a score is a sum of D exact products in fp32, off by D u times the sum of their magnitudes; the difference to the logarithm rounds once more, its
    product with 1 / log 2 and that constant once each, relative to it, and the exponential is off by 2 u: all relative to the weight.  `spread` sums weights times those magnitudes.
    Sums add a unit for every row, the previous weight's product and addition one each."""
    scale = float(np.float32(su.dim ** -0.5 if scale is None else scale))
    q = su.q if q is None else q
    _, lse, _, _ = oc.attend(su.oracle, q, su.table, su.lens, su.start, scale=scale, causal=causal, window=window)
    lse = lse.astype(np.float32)
    room = su.table.shape[1] * su.page + extra
    old = np.exp(su.rng.standard_normal((len(su.lens), su.kv_heads, room))).astype(np.float32)
    old[..., -1] = np.nan                                            # behind every sequence
    want = np.full(old.shape, 5.0)
    before = old.astype(np.float64) if previous else None
    spread = od.weigh(su.oracle, q, lse.astype(np.float64), su.table, su.lens, su.start, scale, want, causal, window, before, float(np.float32(decay)))
    old_gpu = torch.from_numpy(old).cuda() if previous else None
    out = torch.full(old.shape, 5.0, device="cuda")
    got = su.gpu.weigh(dev(q, su.dtype), torch.from_numpy(lse).cuda(), scale=scale, causal=causal, window=window, previous=old_gpu, decay=decay, out=out, **su.plan())
    assert got is out
    got = got.double().cpu().numpy()
    rows = max(1, su.tokens) * su.heads // su.kv_heads
    bound = ((su.dim + 8) * U * spread + (rows + 8) * U * np.abs(want)) * (1 + 2.0 ** -6) + 1e-37
    with np.errstate(invalid="ignore"):
        same = (np.isnan(want) & np.isnan(got)) | (np.abs(got - want) <= bound)
    assert same.all(), (np.argwhere(~same)[:5], got[~same][:5], want[~same][:5])
    if previous:                                                     # in place
        su.gpu.weigh(dev(q, su.dtype), torch.from_numpy(lse).cuda(), scale=scale, causal=causal, window=window, previous=old_gpu, decay=decay, out=old_gpu, **su.plan())
        inside = want != 5.0
        assert (old_gpu.double().cpu().numpy()[inside] == got[inside]).all() or np.isnan(got[inside]).any()
        assert np.array_equal(old_gpu.cpu().numpy()[~inside], old[~inside], equal_nan=True)
    return got


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim,page,kv_heads,group", [(64, 16, 2, 1), (96, 32, 1, 3), (128, 64, 2, 4), (192, 128, 1, 5), (256, 256, 2, 2), (64, 16, 1, 17)])
def test_weigh(bnn, dtype, dim, page, kv_heads, group):
    su = Batch(bnn, dim + group, [70, 0, 33, 1, 16, 5], [3, 0, 33, 1, 1, 8], kv_heads, group, dim, page, dtype, signs=dim != 96)
    if su.table.shape[1] > 2:
        su.table[0, 1] = -1                                          # given back
    check_weigh(su)
    check_weigh(su, window=7, decay=0.75, extra=3)
    check_weigh(su, causal=False, previous=False, scale=0.3)


@pytest.mark.parametrize("lens,counts", [([1], [1]), ([257, 3, 120], [1, 1, 1]), ([300, 280], [300, 5]), ([90] * 5, [2] * 5), ([16, 17, 15, 32], [16, 17, 15, 32])])
def test_weigh_lengths(bnn, lens, counts):
    su = Batch(bnn, sum(lens), lens, counts, dim=64, group=3)
    check_weigh(su)
    check_weigh(su, window=1, decay=0.0)
    check_weigh(su, window=2147483647, previous=False)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("dim,page,kv_heads,group", [(64, 16, 2, 8), (96, 32, 1, 5), (128, 64, 1, 3), (192, 128, 1, 7), (256, 16, 1, 33)])
def test_weigh_many_rows(bnn, dtype, dim, page, kv_heads, group):
    """Rows by the hundred: several steps and parts, rows of other tokens in a step (groups that do not divide it), sequences with few rows beside, missing pages, windows, a wave's keys that no row sees."""
    su = Batch(bnn, dim + group, [170, 300, 5, 0, 90], [170, 61, 1, 0, 90], kv_heads, group, dim, page, dtype)
    if su.table.shape[1] > 2:
        su.table[1, 1] = -1
    check_weigh(su)
    check_weigh(su, window=37, decay=0.5)
    check_weigh(su, causal=False, previous=False, scale=0.2)


@pytest.mark.parametrize("lens,counts", [([40, 25, 210, 30], [3, 0, 2, 0]), ([40, 25, 210, 30], [0, 0, 0, 1]), ([220, 25, 9, 30], [200, 0, 1, 0])])
def test_sequences_without_rows(bnn, lens, counts):
    """Sequences that bring no row, the last among them: their old weights only fade."""
    su = Batch(bnn, 33, lens, counts, group=2)
    check_weigh(su, decay=0.25)
    check_weigh(su, window=4, previous=False)


@pytest.mark.parametrize("dtype,dim,counts", [("bf16", 64, [1] * 3 + [40] + [1] * 62 + [150] + [1, 0, 33]), ("f16", 128, [1, 300, 0, 2, 260]), ("f32", 96, [64, 65, 32, 33, 1]), ("bf16", 192, [0] * 130 + [90, 3]),
                                              ("bf16", 64, [200] + [0] * 70)])
def test_single_tokens_beside_prompts(bnn, dtype, dim, counts):
    """Sequences of few rows and of many in one call, the latter looked for among up to 132; in parts and in one."""
    su = Batch(bnn, 37, [n + 3 + b % 5 for b, n in enumerate(counts)], counts, group=2, dim=dim, dtype=dtype)
    check_weigh(su, decay=0.75)
    check_weigh(su, window=19, previous=False)


@pytest.mark.parametrize("counts,width", [([1, 70, 0, 290, 66, 40, 400, 1, 33, 130], 32), ([1] * 40 + [70, 140, 66] + [1] * 30 + [300, 33, 0, 129], 256)])
def test_weigh_within_its_workspace(bnn, counts, width):
    """Sequences in one part before, between and behind those in several; the workspace exactly as large as it has to be, with all bits set, and what lies behind it left alone; starts of any content too."""
    su = Batch(bnn, 38, [n + 5 for n in counts], counts, group=2, dim=64, width=width)
    plan, q = su.plan(), dev(su.q, "bf16")
    _, lse = su.gpu.attend(q, want_lse=True, **plan)
    rows = bnn.binding._Rows4Struct(plan["table"].data_ptr(), plan["lens"].data_ptr(), plan["start"].data_ptr(), len(counts), width, su.tokens)
    need = bnn.load().bnn_cache4_weigh_workspace_bytes(su.gpu._struct(), ctypes.byref(rows), 1, su.heads)
    assert need > 0
    held = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
    zero = lambda: torch.zeros(len(counts), su.kv_heads, width * su.page, device="cuda")
    check_weigh(su, decay=0.5)
    want = su.gpu.weigh(q, lse, out=zero(), **plan)
    assert torch.equal(su.gpu.weigh(q, lse, out=zero(), workspace=held[:need], **plan), want)
    wild = np.random.default_rng(1)
    for _ in range(10):
        start = wild.choice(np.array([-5, 0, 1, 100, 500, su.tokens, 2147483647], np.int32), len(counts) + 1)
        su.gpu.weigh(q, lse, out=zero(), workspace=held[:need], **{**plan, "start": ints(start)})
    assert (held[need:] == 255).all() and torch.equal(su.gpu.weigh(q, lse, out=zero(), workspace=held[:need], **plan), want)
    with pytest.raises(bnn.BnnError):
        su.gpu.weigh(q, lse, out=zero(), workspace=held[:need - 1], **plan)


def test_weigh_thousands_of_rows(bnn):
    """More rows than lie in LDS at once, against rows a few at a time (bounds: the sums of both, 2 units for every row of a key)."""
    su = Batch(bnn, 31, [1500, 700], [1, 1], kv_heads=2, group=4, dim=64, page=64)
    plan = su.plan()
    q = torch.randn(2000, 8, 64, device="cuda", dtype=torch.bfloat16)
    start = ints([0, 1400, 2000])
    out, lse = su.gpu.attend(q, want_lse=True, **{**plan, "start": start})
    zero = lambda: torch.zeros(2, 2, su.table.shape[1] * 64, device="cuda")
    for window in (0, 333):
        out, lse = su.gpu.attend(q, want_lse=True, window=window, **{**plan, "start": start})
        got = su.gpu.weigh(q, lse, out=zero(), window=window, **{**plan, "start": start})
        want = zero().double()
        for i in range(0, 1400, 2):          # tokens 100 .. 1499 and 100 .. 699, two at a time
            parts = [(0, i)] + ([(1, i)] if i < 600 else [])
            for b, t in parts:
                one = dict(table=plan["table"][b:b + 1].contiguous(), lens=ints([100 + t + 2]))
                rows = slice(1400 * b + t, 1400 * b + t + 2)
                want[b:b + 1] += su.gpu.weigh(q[rows], lse[rows], out=torch.zeros(1, 2, su.table.shape[1] * 64, device="cuda"), window=window, **one).double()
        spread = 64 ** 0.5 * 6 * 4           # scale * sum |q| |k| and |lse|, generously
        assert ((got.double() - want).abs() <= (2 * (64 + 8) * U * spread + 2 * 5600 * U) * want + 1e-30).all()
        assert abs(got[0].sum().item() - 1400 * 8) <= 0.01 and abs(got[1].sum().item() - 600 * 8) <= 0.01


def test_weigh_far_apart_rows(bnn):
    """Distances between tokens that 32-bit offsets of the kernel for many rows do not reach."""
    su = Batch(bnn, 32, [80], [80], kv_heads=1, group=1, dim=64)
    wide = torch.empty(80, 1 << 23, device="cuda", dtype=torch.bfloat16)
    wide[:, :64] = dev(su.q, "bf16")[:, 0]
    view = wide.view(80, 1, 1 << 23)[:, :, :64]
    lse = torch.randn(80, 1, device="cuda")
    zero = lambda: torch.zeros(1, 1, su.table.shape[1] * 16, device="cuda")
    near, far = su.gpu.weigh(dev(su.q, "bf16"), lse, out=zero(), **su.plan()), su.gpu.weigh(view, lse, out=zero(), **su.plan())
    assert ((near - far).abs() <= 2 * 80 * U * near + 2 * 72 * U * 40 * near).all() and near.sum() > 0


def test_weigh_many_rows_far_apart(bnn):
    """16384 rows whose heads lie too far apart for the kernel for many rows: every one gives every key exp(-lse), as its query is zero.  A lane has 4096 of them.  Added one after another to one fp32 sum these
    would be off by 740 to 940 u (u = 2^-24) with the logarithms here, whose weights lie where rounding goes one way.  In runs of 256 rows, 64 a lane, and 64 runs: 64 + 64 u at most, 2 for the four lanes, and for the weight
    itself 2 u of its logarithm for two products, 2 for the exponential and 2 for the reciprocal of scale and its product."""
    su = Batch(bnn, 34, [8200], [1], kv_heads=1, group=2, dim=64, page=256)
    q = torch.zeros(((1 << 24) + 8192 * 64,), device="cuda", dtype=torch.bfloat16).as_strided((8192, 2, 64), (64, 1 << 24, 1))
    for log in (0.104244605, 0.39215827, 0.44179857, -0.28294963):
        lse = torch.full((8192, 2), log, device="cuda")
        w = su.gpu.weigh(q, lse, ints(su.table), ints(su.lens), causal=False, out=torch.zeros(1, 1, su.table.shape[1] * 256, device="cuda"))[0, 0, :8200].double().cpu().numpy()
        want = 16384 * np.exp(-float(lse[0, 0]))
        assert (np.abs(w - want) <= 140 * U * want).all(), (log, np.abs(w / want - 1).max() / U)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_weigh_runs_of_rows_far_apart(bnn, dtype):
    """Sequences of 600, 1 and 259 rows by runs, with masks, against the same rows side by side.  Bounds: the sums of both, of up to 1200 rows, and of scores and logarithms below 192."""
    su = Batch(bnn, 35, [700, 40, 259], [600, 1, 259], kv_heads=1, group=2, dim=64, page=64, dtype=dtype)
    near = dev(su.q, dtype)
    far = torch.empty((1 << 24) + 860 * 64, device="cuda", dtype=TYPES[dtype]).as_strided((860, 2, 64), (64, 1 << 24, 1)).copy_(near)
    zero = lambda: torch.zeros(3, 1, su.table.shape[1] * 64, device="cuda")
    for kw in (dict(), dict(window=77), dict(causal=False)):
        _, lse = su.gpu.attend(near, want_lse=True, **kw, **su.plan())
        a, b = su.gpu.weigh(near, lse, out=zero(), **kw, **su.plan()).double(), su.gpu.weigh(far, lse, out=zero(), **kw, **su.plan()).double()
        assert ((a - b).abs() <= (2 * (64 + 8) * U * 192 + 2 * 1200 * U) * a + 1e-30).all() and (a[0, 0, :700] > 0).sum() > 600
    first = su.gpu.weigh(far, lse, out=zero(), causal=False, **su.plan())
    assert torch.equal(first, b.float())


@pytest.mark.parametrize("dim", [64, 96, 128, 192, 256])
@pytest.mark.parametrize("dtype,group", [("bf16", 32), ("f32", 16), ("bf16", 64), ("f32", 64), ("f16", 40)])
def test_weigh_errors_of_high_scores_average_out(bnn, dtype, dim, group):
    """Scores and logarithms near 100, both up to 0.5 apart, one key that has a weight: 128 sequences of `group` rows, through both kernels.  A row's -lse / scale is rounded to fp32, 2^-24 of itself or less, up to 100 u of the weight:
    rows differ, so their mean, over 2048 rows at least, keeps 1.3 u of it for a standard deviation (a rounding's is 1 / sqrt 3 of the most; 12 u and fewer for a sequence's fp32 sum, over 128 of them, 0.6), and 7 u is five of them.  What all
    rows have alike is the rounding of scale / log 2, e of itself: e (score - lse / 2), and the exponential's own 2 u."""
    rng = np.random.default_rng(dim + group)
    cache = bnn.Cache4(1, kv_heads=1, head_dim=dim, page=16)
    k = torch.zeros(1, 1, dim, device="cuda")
    k[..., 0] = 6.0
    cache.write(k, torch.zeros_like(k), ints([[0]]), ints([1]))
    scale = float(np.float32(dim ** -0.5))
    table, lens = ints(np.zeros((128, 1))), ints(np.ones(128))       # the same token for all
    q = np.zeros((128, group, dim))
    q[..., 0] = rounded(rng.uniform(99.5, 100.5, (128, group)) / scale / 6, dtype)
    score = scale * 6 * q[..., 0]
    lse = (score + rng.uniform(-0.5, 0.5, score.shape)).astype(np.float32)
    w = cache.weigh(dev(q, dtype), torch.from_numpy(lse).cuda(), table, lens, scale=scale, out=torch.zeros(128, 1, 16, device="cuda"))[:, 0, 0].double().cpu().numpy()
    want = np.exp(score - lse.astype(np.float64)).sum(1)
    scale2 = float(np.float32(np.float32(scale) * np.float32(1.4426950408889634)))
    e = abs(scale2 / (scale * 1.4426950408889634) - 1)
    assert abs((w / want).mean() - 1) <= 51 * e + 9 * U, ((w / want).mean() - 1) / U


def test_weights_are_those_of_attention(bnn):
    """Every row gives its whole weight: the sums over keys are the rows' number, and with the cache's values they give attention's outputs."""
    su = Batch(bnn, 9, [500, 130], [1, 1], dim=128, page=64, group=4, spread=2.0)
    q, plan = dev(su.q, "bf16"), su.plan()
    out, lse = su.gpu.attend(q, want_lse=True, **plan)
    w = su.gpu.weigh(q, lse, out=torch.zeros(2, 2, su.table.shape[1] * 64, device="cuda"), **plan)
    # fp32 sums of up to 500 weights and their own bounds as above, of scores below 50
    assert ((w.sum(-1) - 4).abs() <= 4 * (500 + 136 * 50) * U).all()
    one = bnn.Cache4(kv_heads=2, head_dim=128, page=64, data=su.gpu.data)
    for b, n in enumerate((500, 130)):
        _, v = one.read(plan["table"][b:b + 1].contiguous(), plan["lens"][b:b + 1].contiguous(), tokens=n, dtype=torch.float32)
        mean = torch.einsum("hk,khd->hd", w[b, :, :n].double().cpu(), v.double().cpu())
        got = out[b].double().cpu().view(2, 4, 128).sum(1)
        assert ((mean - got).abs() <= 4 * (2.0 ** -8 + 2.0 ** -8) * v.abs().max().item()).all()


def test_rows_that_give_nothing_or_nan(bnn):
    """A row whose lse is -infinity gives nothing; one whose lse is NaN, as attention gives for a query with a NaN or infinity, makes the weights of what it sees NaN, and no others; NaN keys
    where no row looks stay there."""
    su = Batch(bnn, 10, [40, 40, 40], [1, 1, 1], kv_heads=1, group=1, dim=64)
    q = dev(su.q, "bf16")
    lse = torch.zeros(3, 1, device="cuda")
    lse[0] = float("-inf")
    q[1, 0, 3], lse[1] = float("nan"), float("nan")
    w = su.gpu.weigh(q, lse, out=torch.zeros(3, 1, 48, device="cuda"), window=5, **su.plan())
    assert (w[0] == 0).all() and torch.isnan(w[1, 0, 35:40]).all() and (w[1, 0, :35] == 0).all() and (w[2, 0, 35:40] > 0).all() and (w[2, 0, 40:] == 0).all()
    q[1, 0, 3] = float("inf")
    w = su.gpu.weigh(q, lse, out=torch.zeros(3, 1, 48, device="cuda"), window=5, **su.plan())
    assert torch.isnan(w[1, 0, 35:40]).all() and (w[1, 0, :35] == 0).all()
    oc.Record(su.data[su.table[2, 0], 0], 16, 64).scales["k"][:, 3] = 255
    su.gpu = bnn.Cache4(kv_heads=1, head_dim=64, page=16, data=torch.from_numpy(su.data).cuda())
    w = su.gpu.weigh(q, lse, out=torch.zeros(3, 1, 48, device="cuda"), window=36, **su.plan())
    assert torch.isfinite(w[2]).all() and w[2, 0, 3] == 0
    w = su.gpu.weigh(q, lse, out=torch.zeros(3, 1, 48, device="cuda"), **su.plan())
    assert torch.isnan(w[2, 0, 3]) and torch.isfinite(w[2, 0, :3]).all() and torch.isfinite(w[2, 0, 4:]).all()


@pytest.mark.parametrize("lens,counts,group", [([48, 33, 16, 1], [0, 0, 0, 1], 2), ([64, 48, 9], [1, 1, 1], 4), ([128, 96, 40], [100, 33, 5], 2), ([300, 64], [200, 40], 3), ([16, 16], [0, 3], 1)])
@pytest.mark.parametrize("dtype,decay", [("bf16", 0.75), ("f32", 1.0)])
def test_weigh_in_place(bnn, lens, counts, group, dtype, decay):
    """previous as the output, bit for bit what another output gets, NaN and all else included: old weights that are NaN or infinite, in sequences that fill their table too, with rows and without."""
    su = Batch(bnn, sum(lens), lens, counts, group=group, dtype=dtype)
    plan, room = su.plan(), su.table.shape[1] * su.page
    q, lse = dev(su.q, dtype), torch.from_numpy(su.rng.standard_normal((su.tokens, su.heads)).astype(np.float32)).cuda()
    old = torch.from_numpy(np.exp(su.rng.standard_normal((len(lens), su.kv_heads, room + 3))).astype(np.float32)).cuda()
    for at, value in ((0, float("nan")), (5, float("inf")), (room - 1, float("nan")), (room, 3.0)):
        old[:, :, at] = value
    for window in (0, 7):
        out = su.gpu.weigh(q, lse, window=window, previous=old, decay=decay, out=old.clone(), **plan)
        place = old.clone()
        assert su.gpu.weigh(q, lse, window=window, previous=place, decay=decay, out=place, **plan) is place
        assert torch.equal(place.view(torch.int32), out.view(torch.int32))
        for b, n in enumerate(lens):
            assert torch.equal(out[b, :, n:].view(torch.int32), old[b, :, n:].view(torch.int32))         # behind the sequence
            new = n - counts[b]
            assert torch.isnan(out[b, :, 0]).all() == (new > 0) and (new <= 5 or torch.isinf(out[b, :, 5]).all())


def test_weigh_past_the_table(bnn):
    su = Batch(bnn, 11, [50, 20], [3, 3], width=2)
    check_weigh(su)
    check_weigh(su, window=25)


def test_strided_queries(bnn):
    su = Batch(bnn, 12, [60, 33], [2, 2], dim=96, page=32)
    wide = torch.zeros(4, 9, 96, device="cuda", dtype=torch.bfloat16)
    wide[:, 3:7] = dev(su.q, "bf16")
    lse = torch.randn(4, 4, device="cuda")
    zero = lambda: torch.zeros(2, 2, 64, device="cuda")
    assert torch.equal(su.gpu.weigh(wide[:, 3:7], lse, out=zero(), **su.plan()), su.gpu.weigh(dev(su.q, "bf16"), lse, out=zero(), **su.plan()))


# ------------------------------------------------------------------------------------------ the choice

def check_heaviest(bnn, weights, lens, table, keep, first, last, page, pages, kv_heads):
    cache = bnn.Cache4(pages, kv_heads=kv_heads, head_dim=64, page=page)
    want, kept = od.heaviest(weights, table, lens, keep, first, last, page, pages)
    got, got_kept = cache.heaviest(torch.from_numpy(weights).cuda(), ints(table), ints(lens), keep, first, last)
    assert (got_kept.cpu().numpy() == kept).all()
    wrong = got.cpu().numpy() != want
    assert not wrong.any(), (np.argwhere(wrong)[:5], got.cpu().numpy()[wrong][:5], want[wrong][:5])


@pytest.mark.parametrize("keep,first,last", [(1, 0, 0), (1, 0, 1), (7, 2, 3), (64, 4, 60), (100, 0, 0), (333, 5, 9), (2000, 1, 64), (6000, 0, 1)])
def test_heaviest(bnn, keep, first, last):
    rng = np.random.default_rng(keep)
    lens = np.array([0, 1, 33, 333, 334, 1000, 2000, 5001], np.int32)
    page, kv_heads = 16, 3
    table = rng.permutation(8 * 320)[:8 * 313].reshape(8, 313).astype(np.int32)
    weights = np.exp(2 * rng.standard_normal((8, kv_heads, 313 * 16 + 5))).astype(np.float32)
    check_heaviest(bnn, weights, lens, table, keep, first, last, page, 8 * 320, kv_heads)
    few = rng.integers(0, 4, weights.shape).astype(np.float32)       # ties
    few[:, 1] = 0
    check_heaviest(bnn, few, lens, table, keep, first, last, page, 8 * 320, kv_heads)
    signed = rng.standard_normal(weights.shape).astype(np.float32)   # numbers of any kind
    signed[rng.random(weights.shape) < 0.05] = np.nan
    signed[rng.random(weights.shape) < 0.05] = np.inf
    signed[rng.random(weights.shape) < 0.05] = -np.inf
    signed[rng.random(weights.shape) < 0.05] = 0.0
    signed[rng.random(weights.shape) < 0.05] = -0.0
    signed[rng.random(weights.shape) < 0.05] = 1e-42                 # subnormal
    check_heaviest(bnn, signed, lens, table, keep, first, last, page, 8 * 320, kv_heads)
    table[rng.random(table.shape) < 0.2] = -1                        # pages given back
    table[0, 0], table[6, 3] = 8 * 320, -2147483648
    check_heaviest(bnn, signed, lens, table, keep, first, last, page, 8 * 320, kv_heads)
    lens[3] = 2147483647                                             # longer than its table
    check_heaviest(bnn, weights, lens, table, keep, first, last, page, 8 * 320, kv_heads)


@pytest.mark.parametrize("keep,first,last", [(1, 0, 1), (5000, 3, 100), (20000, 0, 0), (39990, 1, 1), (50000, 0, 7)])
def test_heaviest_in_parts(bnn, keep, first, last):
    """Tables with room for more than 32768 tokens: a sequence's workgroups pass on what they counted.  Sequences of every length beside each other, ties, numbers of any kind, pages given back; and tables too many
    for that, which one workgroup each reads several times."""
    rng = np.random.default_rng(keep)
    page, kv_heads, width = 64, 2, 700
    lens = np.array([0, 1, 8191, 8192, 8193, 40000, 44800, 100000], np.int32)
    table = rng.permutation(8 * width).reshape(8, width).astype(np.int32)
    weights = np.exp(2 * rng.standard_normal((8, kv_heads, width * page))).astype(np.float32)
    check_heaviest(bnn, weights, lens, table, keep, first, last, page, 8 * width, kv_heads)
    mixed = rng.integers(-2, 3, weights.shape).astype(np.float32)
    mixed[:, 1] = rng.standard_normal(weights[:, 1].shape)
    mixed[rng.random(weights.shape) < 0.02] = np.nan
    mixed[rng.random(weights.shape) < 0.02] = -np.inf
    mixed[rng.random(weights.shape) < 0.02] = np.inf
    table[rng.random(table.shape) < 0.1] = -1
    check_heaviest(bnn, mixed, lens, table, keep, first, last, page, 8 * width, kv_heads)
    if keep == 5000:                         # 400 sequences, few of them long
        many, lens = np.zeros(400, np.int32), lens[:7]
        many[:7], many[399] = lens, 44801
        table = np.full((400, width), -1, np.int32)
        table[:7], table[399] = rng.permutation(8 * width).reshape(8, width)[:7], rng.permutation(8 * width)[:width]
        w = np.zeros((400, kv_heads, width * page), np.float32)
        w[:7], w[399] = mixed[:7], weights[7]
        assert bnn.load().bnn_cache4_heaviest_workspace_bytes(bnn.Cache4(1, kv_heads=kv_heads, head_dim=64, page=page)._struct(), 400, width) == 0
        check_heaviest(bnn, w, many, table, keep, first, last, page, 8 * width, kv_heads)


def test_heaviest_long(bnn):
    rng = np.random.default_rng(1)
    pages = 300001 // 256 + 1
    weights = np.exp(3 * rng.standard_normal((1, 2, pages * 256))).astype(np.float32)
    weights[0, 1] = np.round(weights[0, 1])
    table = rng.permutation(pages).reshape(1, pages).astype(np.int32)
    for keep in (1, 5000, 150000, 300000):
        check_heaviest(bnn, weights, np.array([300001], np.int32), table, keep, min(keep // 2, 4), keep // 3, 256, pages, 2)


# ------------------------------------------------------------------------------------------ moving

@pytest.mark.parametrize("dim,page,kv_heads,signs", [(64, 16, 3, True), (96, 32, 1, False), (128, 64, 2, True), (192, 128, 1, True), (256, 256, 1, False)])
def test_move(bnn, dim, page, kv_heads, signs):
    rng = np.random.default_rng(dim)
    lens, keep = [5 * page + 3, page, 1, 2 * page + 1], page + 7
    need = [-(-n // page) for n in lens]
    into_pages = 3                                                   # more than `keep` needs
    total = sum(need) + 2 * len(lens) + 3
    data = rng.integers(0, 256, (total, kv_heads, oc.record_bytes(dim, page, signs))).astype(np.uint8)
    order = rng.permutation(total)
    table, into, at = np.full((4, max(need)), -1, np.int32), np.full((4, into_pages), -1, np.int32), 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]; at += n
    for b in range(4):
        into[b, :2] = order[at:at + 2]; at += 2
    tokens = np.full((4, kv_heads, keep), -1, np.int32)
    for b, h in np.ndindex(4, kv_heads):
        n = min(keep, lens[b])
        tokens[b, h, :n] = np.sort(rng.choice(lens[b], n, replace=False))
    tokens[0, 0, 3] = -5
    tokens[0, 0, 4] = 2147483647                                     # past the table
    table[3, 1], into[1, 1] = -1, total + 9
    weights = rng.standard_normal((4, kv_heads, table.shape[1] * page + 3)).astype(np.float32)
    oracle = oc.Cache(data.copy(), dim, page, signs)
    moved = od.move(oracle, tokens, table, into, weights)
    cache = bnn.Cache4(kv_heads=kv_heads, head_dim=dim, page=page, signs=signs, data=torch.from_numpy(data.copy()).cuda())
    got = cache.move(ints(tokens), ints(table), ints(into), weights=torch.from_numpy(weights).cuda())
    assert (cache.data.cpu().numpy() == oracle.data).all() and (got.cpu().numpy() == moved).all()
    assert not (oracle.data == data).all()
    again = bnn.Cache4(kv_heads=kv_heads, head_dim=dim, page=page, signs=signs, data=torch.from_numpy(data.copy()).cuda())
    assert again.move(ints(tokens), ints(table), ints(into)) is None and torch.equal(again.data, cache.data)
    assert again.move(ints(tokens), ints(table), ints(into[:, :0])) is None and torch.equal(again.data, cache.data)


def test_moved_weights_are_of_tokens(bnn):
    """0 where there is no token: a list's -1, a token on a page given back or never there, one past the table though the weights go on.  What has no page to go to has its weight all the same."""
    cache = bnn.Cache4(8, kv_heads=1, head_dim=64, page=16)
    table, into = ints([[0, -1, 2, 8]]), ints([[4, -1, 5]])
    tokens = ints([[[0, 15, 16, 31, 32, -1, 47, 48, 63, 64, 70, 2147483647] + list(range(12))]])
    weights = torch.arange(1.0, 81.0, device="cuda").view(1, 1, 80)
    got = cache.move(tokens, table, into, weights=weights)[0, 0].tolist()
    assert got == [1, 16, 0, 0, 33, 0, 48, 0, 0, 0, 0, 0] + [float(i + 1) for i in range(12)] + [0] * 24
    data = np.zeros((8, 1, oc.record_bytes(64, 16)), np.uint8)
    assert od.move(oc.Cache(data, 64, 16), tokens.cpu().numpy(), table.cpu().numpy(), into.cpu().numpy(), weights.cpu().numpy())[0, 0].tolist() == got


def test_no_plan_leads_out(bnn):
    """Tables, lengths, starts and lists of any content: nothing but the cache and the call's own outputs is written."""
    rng = np.random.default_rng(8)
    guard = torch.full((6, 2, oc.record_bytes(64, 16)), 9, dtype=torch.uint8, device="cuda")
    cache = bnn.Cache4(kv_heads=2, head_dim=64, page=16, data=guard[2:4])
    wild = lambda *shape: torch.from_numpy(rng.choice(np.array([-2147483648, -1, 0, 1, 2, 5, 31, 1000, 2147483647], np.int32), shape)).cuda()
    q, lse = torch.randn(10, 4, 64, device="cuda"), torch.randn(10, 4, device="cuda")
    w = torch.randn(5, 2, 48, device="cuda")
    w[:1], w[4:] = 7, 7
    for _ in range(12):
        cache.weigh(q, lse, wild(3, 3), wild(3), start=wild(4), out=w[1:4], previous=w[1:4], window=int(rng.integers(0, 2)) * 2147483647, causal=True)
        cache.weigh(q, lse, wild(3, 3), wild(3), start=wild(4), out=w[1:4], causal=False)
        cache.heaviest(w[1:4], wild(3, 3), wild(3), 7, 1, 2)
        cache.move(wild(3, 2, 9), wild(3, 3), wild(3, 2), weights=w[1:4])
    torch.cuda.synchronize()
    assert (guard[:2] == 9).all() and (guard[4:] == 9).all() and (w[0] == 7).all() and (w[4] == 7).all()


# ------------------------------------------------------------------------------------------ together

def decode(bnn, cache, table, lens, steps, keep, spare, f, heads, rng_seed, budget):
    """Steps of decoding with rotary positions; when a sequence passes the budget it is cut back to `keep` tokens into its spare pages."""
    gen = torch.Generator(device="cuda").manual_seed(rng_seed)
    weights, positions, outs = None, lens.clone(), []
    for _ in range(steps):
        lens = lens + 1
        qkv = torch.randn(len(lens), heads + 2 * cache.kv_heads, cache.head_dim, generator=gen, device="cuda")
        q, k, v = qkv.split((heads, cache.kv_heads, cache.kv_heads), dim=1)
        q = cache.write_rotary(q, k, v, table, lens, f, positions=positions)
        positions = positions + 1
        out, lse = cache.attend(q, table, lens, want_lse=True)
        weights = cache.weigh(q, lse, table, lens, previous=weights)
        outs.append(out)
        if int(lens.max()) > budget:
            tokens, lens = cache.heaviest(weights, table, lens, keep, first=2, last=8)
            weights = cache.move(tokens, table, spare, weights=weights)
            table, spare = spare, table
    return outs, table, lens, weights


def test_decoding_with_eviction(bnn):
    """What a decoder does with all of it: lengths stay under the budget, and after each cut attention is over the kept tokens, as an oracle cache of them says."""
    page, kv_heads, dim, heads = 16, 2, 64, 4
    table, spare = ints([[0, 1, 2, 3], [4, 5, 6, 7]]), ints([[8, 9, 10, 11], [12, 13, 14, 15]])
    cache = bnn.Cache4(16, kv_heads=kv_heads, head_dim=dim, page=page)
    outs, table, lens, weights = decode(bnn, cache, table, ints([0, 0]), 90, 32, spare, bnn.rotary_frequencies(dim), heads, 1, 48)
    assert all(torch.isfinite(o).all() for o in outs) and int(lens.max()) <= 48 and int(lens.min()) > 32
    # the weights of a sequence cannot pass what its rows gave
    n = int(lens[0])
    assert (weights[0, :, :n] >= 0).all() and weights[0, :, :n].sum() <= 90 * heads * 1.001
    # the kept tokens, read back and attended to by the oracle
    data = cache.data.cpu().numpy().copy()
    oracle = oc.Cache(data, dim, page)
    q = rounded(np.random.default_rng(3).standard_normal((2, heads, dim)), "f32")
    want, _, magnitude, spread = oc.attend(oracle, q, table.cpu().numpy(), lens.cpu().numpy(), scale=dim ** -0.5)
    got = cache.attend(dev(q, "f32"), table, lens).double().cpu().numpy()
    assert (np.abs(got - want) <= ((2 * (dim + 8) * spread)[..., None] + 200) * U * magnitude + 1e-30).all()
    again = decode(bnn, bnn.Cache4(16, kv_heads=kv_heads, head_dim=dim, page=page), ints([[0, 1, 2, 3], [4, 5, 6, 7]]), ints([0, 0]), 90, 32, ints([[8, 9, 10, 11], [12, 13, 14, 15]]),
                   bnn.rotary_frequencies(dim), heads, 1, 48)
    assert all(torch.equal(a, b) for a, b in zip(outs, again[0])) and torch.equal(weights[0, :, :n], again[3][0, :, :n])


def test_captured_and_replayed(bnn):
    """weigh, heaviest and move recorded once: lengths, queries and weights are read at replay."""
    su = Batch(bnn, 20, [60, 45], [1, 1], width=6)
    lens, table = ints(su.lens), ints(su.table)
    into = ints([[int(p)] for p in np.setdiff1d(np.arange(len(su.data)), su.table)[:2]])
    q, previous, lse = dev(su.q, "bf16"), torch.rand(2, 2, 96, device="cuda"), torch.randn(2, 4, device="cuda")
    out = torch.zeros_like(previous)

    def step():
        w = su.gpu.weigh(q, lse, table, lens, previous=previous, out=out)
        tokens, kept = su.gpu.heaviest(w, table, lens, 16, 1, 2)
        return tokens, kept, su.gpu.move(tokens, table, into, weights=w)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(5):
        lens += 1
        q.normal_()
        previous.uniform_()
        graph.replay()
        torch.cuda.synchronize()
        copies, data = [g.clone() for g in got], su.gpu.data.clone()
        want = step()
        assert all(torch.equal(a, b) for a, b in zip(copies, want)) and torch.equal(su.gpu.data, data)


def test_refusals(bnn):
    su = Batch(bnn, 21, [40, 20], [1, 1])
    q, plan = dev(su.q, "bf16"), su.plan()
    lse, w = torch.randn(2, 4, device="cuda"), torch.zeros(2, 2, 48, device="cuda")
    table, lens = plan["table"], plan["lens"]
    for error, args, kw in ((TypeError, (q.cpu(), lse), {}), (TypeError, (q.double(), lse), {}), (TypeError, (q, lse.double()), {}), (ValueError, (q, lse[:1]), {}),
                            (ValueError, (q, lse.t().contiguous().t()), {}), (ValueError, (q, lse), dict(previous=w[:, :1].contiguous())), (ValueError, (q, lse), dict(out=w[:, :, :40].contiguous())),
                            (ValueError, (q, lse), dict(out=w, previous=torch.zeros(2, 2, 64, device="cuda"))), (bnn.BnnError, (q, lse), dict(scale=0.0)),
                            (bnn.BnnError, (q, lse), dict(scale=float("inf"))), (bnn.BnnError, (q, lse), dict(window=-1)), (bnn.BnnError, (q, lse), dict(window=3, causal=False)),
                            (bnn.BnnError, (q, lse), dict(decay=float("nan"), previous=w)), (bnn.BnnError, (q[:, :3], lse[:, :3].contiguous()), {}), (ValueError, (q[:0], lse[:0]), dict(out=w))):
        with pytest.raises(error):
            su.gpu.weigh(*args, table, lens, **kw)
    wide = ints(np.zeros((2, 4000)))
    with pytest.raises(bnn.BnnError):
        su.gpu.heaviest(torch.zeros(2, 2, 64000, device="cuda"), wide, lens, 4, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))
    for error, args, kw in ((TypeError, (w.double(), table, lens, 4), {}), (TypeError, (w, table.long(), lens, 4), {}), (ValueError, (w, table, lens[:1], 4), {}),
                            (ValueError, (w[:, :, :32].contiguous(), table, lens, 4), {}), (ValueError, (w, table, lens, 0), {}), (bnn.BnnError, (w, table, lens, 4, 3, 2), {}),
                            (bnn.BnnError, (w, table, lens, 4, -1), {})):
        with pytest.raises(error):
            su.gpu.heaviest(*args, **kw)
    tokens, into = ints(np.zeros((2, 2, 4))), ints([[0], [1]])
    for error, args, kw in ((TypeError, (tokens.long(), table, into), {}), (ValueError, (tokens[:1], table, into), {}), (ValueError, (tokens[:, :1].contiguous(), table, into), {}),
                            (ValueError, (tokens, table, into[:1]), {}), (ValueError, (tokens[:, :, :0], table, into), {}), (ValueError, (tokens, table, into), dict(weights=w[:1]))):
        with pytest.raises(error):
            su.gpu.move(*args, **kw)
