"""Measured work of the 4-bit key/value cache: writing and reading it, attention over it, and the selection of blocks by sign bits.

``own`` False: the plain form, elementary torch operations in 32 bits.  ``own`` True: the calls of ``Cache4``.

``kind`` of a case says which entry points a pass goes through:

  append  Cache4.write of the newest tokens of every sequence, then Cache4.read of the same tokens (values in the input's type)
  attend  Cache4.attend: the newest n tokens of every sequence against its whole cache
  select  Cache4.select: for every query token and kv head, the blocks (pages) whose keys' signs agree best with the queries'
  step    write, select, and attend over the selected blocks: a step of a decoder layer

Layout of the cache, uint8 [pages][kv_heads][record]; a record is
  K codes [page][D/2] | V codes [page][D/2] | K exponents [D/32][page] | V exponents [D/32][page] | signs of K [page][D/8] (where kept)
Element d of a token is nibble d % 2 (low first) of byte d / 2, an E2M1 number (sign, two bits of exponent, one of mantissa); its
group of 32 has a power of two as scale, 2^(byte - 127); a sign bit is 1 where the element was >= 0, bit d % 8 of byte d / 8.
Token i of sequence b lies in page table[b][i / page], at i % page; the newest tokens of a sequence end at lens[b] - 1.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # the smallest call: one decoder step's new tokens of eight conversations
        {"name": "append_decode_8", "kind": "append", "dtype": "bf16", "batch": 8, "len_min": 1000, "len_max": 1030, "n_min": 1, "n_max": 1,
         "kv_heads": 8, "group": 1, "dim": 128, "page": 64},
        # prompts of every length from one token on, small pages, a head dimension that is no power of two, fp32 as the library's products give it
        {"name": "append_ragged_f32", "kind": "append", "dtype": "f32", "batch": 7, "len_min": 1, "len_max": 1031, "n_min": 1, "n_max": 1031,
         "kv_heads": 2, "group": 1, "dim": 96, "page": 16},
        # four long prompts at once
        {"name": "append_prompts_32768", "kind": "append", "dtype": "bf16", "batch": 4, "len_min": 8192, "len_max": 8192, "n_min": 8192, "n_max": 8192,
         "kv_heads": 8, "group": 1, "dim": 128, "page": 64},
        # one short conversation, queries as the library's products give them
        {"name": "attend_one_777_f32", "kind": "attend", "dtype": "f32", "batch": 1, "len_min": 777, "len_max": 777, "n_min": 1, "n_max": 1,
         "kv_heads": 8, "group": 4, "dim": 64, "page": 32, "window": 0},
        # an ordinary serving batch, conversations of all lengths
        {"name": "attend_batch_64", "kind": "attend", "dtype": "bf16", "batch": 64, "len_min": 500, "len_max": 8192, "n_min": 1, "n_max": 1,
         "kv_heads": 8, "group": 4, "dim": 128, "page": 64, "window": 0},
        # two very long documents
        {"name": "attend_long_131072", "kind": "attend", "dtype": "bf16", "batch": 2, "len_min": 100001, "len_max": 131072, "n_min": 1, "n_max": 1,
         "kv_heads": 8, "group": 8, "dim": 128, "page": 64, "window": 0},
        # a few drafted tokens to be checked at once, a layer with a sliding window, wide heads, fp16
        {"name": "attend_draft_window_f16", "kind": "attend", "dtype": "f16", "batch": 16, "len_min": 40, "len_max": 6001, "n_min": 5, "n_max": 5,
         "kv_heads": 4, "group": 6, "dim": 192, "page": 16, "window": 1000},
        # two prompts against themselves: the matrix cores' case
        {"name": "attend_prompt_4096", "kind": "attend", "dtype": "bf16", "batch": 2, "len_min": 4096, "len_max": 4096, "n_min": 4096, "n_max": 4096,
         "kv_heads": 8, "group": 4, "dim": 128, "page": 64, "window": 0},
        # eight long documents, one token each
        {"name": "select_decode_65536", "kind": "select", "dtype": "bf16", "batch": 8, "len_min": 50001, "len_max": 65536, "n_min": 1, "n_max": 1,
         "kv_heads": 8, "group": 8, "dim": 128, "page": 64, "keep": 64},
        # a chunk of a prompt, every token with its own blocks; odd sizes
        {"name": "select_chunk_f32", "kind": "select", "dtype": "f32", "batch": 2, "len_min": 7001, "len_max": 10007, "n_min": 333, "n_max": 333,
         "kv_heads": 4, "group": 5, "dim": 64, "page": 32, "keep": 32},
        # a decoder layer's step of a batch with long contexts
        {"name": "step_decode_16", "kind": "step", "dtype": "bf16", "batch": 16, "len_min": 4001, "len_max": 32768, "n_min": 1, "n_max": 1,
         "kv_heads": 8, "group": 4, "dim": 128, "page": 64, "keep": 32},
        # chunks of two prompts, ragged, fp16
        {"name": "step_chunk_f16", "kind": "step", "dtype": "f16", "batch": 2, "len_min": 9000, "len_max": 20011, "n_min": 77, "n_max": 200,
         "kv_heads": 2, "group": 8, "dim": 64, "page": 32, "keep": 48},
    ]


# What no drawn case goes over: cached bytes, (query head, key) pairs times the head dimension, elements that are written.
MAX_CACHE_BYTES, MAX_PAIR_DIM, MAX_WRITTEN = 240e6, 6e10, 6e7


def _log(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["append", "attend", "attend", "select", "step"])
        case = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"]), "kv_heads": rng.choice([1, 2, 3, 4, 8]),
                "dim": rng.choice([64, 96, 128, 128, 192, 256]), "page": rng.choice([16, 32, 64, 128])}
        case["group"] = 1 if kind == "append" else rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 16])
        decode = rng.random() < 0.5
        case["batch"] = _log(rng, 1, 64 if decode else 8)
        hi = _log(rng, 2, 131072 if decode else 20000)
        lo = _log(rng, 1, hi)
        case["len_min"], case["len_max"] = lo, hi
        n_hi = _log(rng, 1, min(hi, 8192)) if not decode else min(hi, rng.choice([1, 1, 1, 2, 5]))
        case["n_min"], case["n_max"] = n_hi if decode or rng.random() < 0.3 else _log(rng, 1, n_hi), n_hi
        if kind == "attend":
            case["window"] = rng.choice([0, 0, 0, _log(rng, 1, hi)])
        if kind in ("select", "step"):
            case["keep"] = _log(rng, 3, 128)
        lens, counts = _lens(case), _counts(case)
        if kind in ("select", "step") and hi <= (case["keep"] + 1) * case["page"]:
            continue                # there would be nothing to select
        cached = sum(lens) * case["kv_heads"] * case["dim"] * 1.3
        pairs = _pairs(case, lens, counts, dense=True) * case["dim"]
        if kind in ("select", "step"):
            pairs *= 4              # a token of its own blocks costs more than one of many that share all keys
        if (cached <= MAX_CACHE_BYTES and (kind == "append" or pairs <= MAX_PAIR_DIM) and sum(counts) * case["kv_heads"] * case["dim"] * case["group"] <= MAX_WRITTEN
                and 3 * 1024 not in (lo, hi, n_hi, case["n_min"], case.get("window"), case["kv_heads"] * case["group"] * case["dim"])):
            return case


# ---------------------------------------------------------------------------------------- sizes

def _spread(lo, hi, count):
    """count integers evenly over [lo, hi], both ends among them, in a fixed mixed-up order."""
    if count == 1:
        return [hi]
    values = [lo + (hi - lo) * i // (count - 1) for i in range(count)]
    return sorted(values, key=lambda v: (v * 2654435761) % 4294967296)


def _lens(case):
    return _spread(case["len_min"], case["len_max"], case["batch"])


def _counts(case):
    return [min(n, length) for n, length in zip(_spread(case["n_min"], case["n_max"], case["batch"]), _lens(case))]


def _pairs(case, lens, counts, dense=False):
    """(query head, key) pairs that attention or the score visits."""
    window, total = case.get("window", 0), 0
    for length, n in zip(lens, counts):
        first = length - n
        if not dense and case["kind"] == "step":
            limit = case["keep"] * case["page"]
        else:
            limit = window if window else length
        ramp = max(0, min(limit, length) - first)            # query tokens that see fewer keys than the limit allows
        total += ramp * first + ramp * (ramp + 1) // 2 + (n - ramp) * min(limit, length)
    return total * case["kv_heads"] * case["group"]


def work(case):
    lens, counts = _lens(case), _counts(case)
    size = DTYPES[case["dtype"]].itemsize
    D, H, G, tokens = case["dim"], case["kv_heads"], case["group"], sum(counts)
    record = 2 * (D // 2 + D // 32)                          # K and V of a token and head
    io = 2 * tokens * H * D * size                           # new k and v
    q = tokens * H * G * D * size
    plan = 4 * sum(-(-length // case["page"]) for length in lens) + 4 * len(lens)
    seen = sum(min(length, n + case.get("window", 0)) if case.get("window") else length for length, n in zip(lens, counts))
    if case["kind"] == "append":
        return {"bytes": 2 * io + 2 * tokens * H * record + plan, "flops": 4 * tokens * H * D}
    if case["kind"] == "attend":
        return {"bytes": seen * H * record + 2 * q + 4 * tokens * H * G + plan, "flops": 4 * D * _pairs(case, lens, counts)}
    keep = 4 * tokens * H * case["keep"]
    signs = seen * H * D // 8
    scored = 2 * D * _pairs(case, lens, counts, dense=True)
    if case["kind"] == "select":
        return {"bytes": signs + q + keep + plan, "flops": scored}
    union = sum(min(length, n * case["keep"] * case["page"]) for length, n in zip(lens, counts))
    return {"bytes": io + tokens * H * (record + D // 8) + signs + 2 * q + keep + union * H * record + plan,
            "flops": scored + 4 * D * _pairs(case, lens, counts) + 4 * tokens * H * D}


# ---------------------------------------------------------------------------------------- state

class State:
    pass


def _parts(st):
    """Views of the cache's data: K codes, V codes, K exponents, V exponents, signs."""
    P, H, _ = st.data.shape
    page, D = st.page, st.D
    c, e = page * D // 2, page * D // 32
    d = st.data
    return (d[..., :c].unflatten(-1, (page, D // 2)), d[..., c:2 * c].unflatten(-1, (page, D // 2)),
            d[..., 2 * c:2 * c + e].unflatten(-1, (D // 32, page)), d[..., 2 * c + e:2 * c + 2 * e].unflatten(-1, (D // 32, page)),
            d[..., 2 * c + 2 * e:].unflatten(-1, (page, D // 8)))


def prepare(case, seed):
    """A cache with everything but, for append and step, the newest tokens; those, queries, and the plan of the batch."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]
    st = State()
    st.kind, st.page, st.D, st.H, st.G, st.dtype = case["kind"], case["page"], case["dim"], case["kv_heads"], case["group"], dtype
    st.window, st.keep = case.get("window", 0), case.get("keep", 0)
    st.host_lens, st.host_counts = _lens(case), _counts(case)
    pages = [-(-length // st.page) for length in st.host_lens]
    total = sum(pages)
    width = max(pages)
    st.data = torch.zeros((total, st.H, st.page * (st.D + st.D // 16 + st.D // 8)), dtype=torch.uint8, device="cuda")
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    st.table = torch.full((len(pages), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(pages):
        st.table[b, :n] = order[at:at + n]
        at += n
    st.lens = torch.tensor(st.host_lens, dtype=torch.int32, device="cuda")
    bounds = [0]
    for n in st.host_counts:
        bounds.append(bounds[-1] + n)
    st.tokens, st.bounds = bounds[-1], bounds
    st.start = None if len(set(st.host_counts)) == 1 else torch.tensor(bounds, dtype=torch.int32, device="cuda")
    # Keys have a few channels much wider than the rest and an offset of their own, as projections of a trained layer have; values are even.
    H, D, G = st.H, st.D, st.G
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    wide = torch.exp(0.5 * normal(H, D)) * (1 + 5 * (torch.rand(H, D, generator=gen, device="cuda") < 0.02))
    offset = 0.3 * normal(H, D)
    new_k, new_v, st.q = [], [], None
    queries = []
    for b, (length, n) in enumerate(zip(st.host_lens, st.host_counts)):
        k, v = normal(length, H, D) * wide + offset, 0.6 * normal(length, H, D)
        stored = length - n if st.kind in ("append", "step") else length
        if stored:
            index = torch.arange(stored, device="cuda")
            _store(st, k[:stored].to(dtype), v[:stored].to(dtype), st.table[b, index // st.page].long(), index % st.page)
        new_k.append(k[length - n:].to(dtype))
        new_v.append(v[length - n:].to(dtype))
        # a query looks for some key of the past, more or less
        looked = torch.randint(0, length, (n,), generator=gen, device="cuda")
        strength = torch.rand(n, H, G, 1, generator=gen, device="cuda")
        queries.append((strength * (k[looked] / wide).unsqueeze(2) + normal(n, H, G, D)).reshape(n, H * G, D).to(dtype))
    st.k, st.v, st.q = torch.cat(new_k), torch.cat(new_v), torch.cat(queries)
    st.scale = 1.0 / math.sqrt(D)
    if st.kind == "attend" or st.kind == "select":
        st.k = st.v = None
    if st.kind == "append":
        st.q = None
    if own:
        import paper_2006_16578_amd as bnn
        st.cache = bnn.Cache4(kv_heads=H, head_dim=D, page=st.page, signs=True, data=st.data)
    return st


# ---------------------------------------------------------------------------------------- plain form

def _quantise(x):
    """x [tokens][heads][D] -> codes [..][D/2], exponent bytes [..][D/32]."""
    x = x.float()
    groups = x.unflatten(-1, (-1, 32))
    high = groups.abs().amax(-1)
    mantissa, power = torch.frexp(high)                             # high = mantissa 2^power, mantissa in [1/2, 1)
    e = power.to(torch.int32) - 3 + (mantissa > 0.75).to(torch.int32)   # the smallest e with high <= 6 * 2^e
    e = torch.where(high == 0, torch.full_like(e, -100), e.clamp(-100, 100))
    y = groups.abs() * ((127 - e) << 23).view(torch.float32).unsqueeze(-1)
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5)).to(torch.uint8)
    code = (code | (torch.signbit(groups).to(torch.uint8) << 3)).flatten(-2)
    bad = ~torch.isfinite(high)
    return code[..., 0::2] | (code[..., 1::2] << 4), torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)


def _pack_signs(x):
    bits = (x >= 0).to(torch.uint8).unflatten(-1, (-1, 8))
    return (bits << torch.arange(8, dtype=torch.uint8, device=x.device)).sum(-1).to(torch.uint8)


def _dequantise(codes, exps):
    """codes [..][D/2], exponent bytes [..][D/32] -> fp32 [..][D]."""
    code = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).to(torch.int32)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    scale = (exps.to(torch.int32) << 23).view(torch.float32)
    scale = torch.where(exps > 227, torch.full_like(scale, float("nan")), scale)
    return (grid[code].unflatten(-1, (-1, 32)) * scale.unsqueeze(-1)).flatten(-2)


def _store(st, k, v, pages, offsets):
    kc, vc, ke, ve, signs = _parts(st)
    kc[pages, :, offsets], ke[pages, :, :, offsets] = _quantise(k)
    vc[pages, :, offsets], ve[pages, :, :, offsets] = _quantise(v)
    signs[pages, :, offsets] = _pack_signs(k)


def _places(st):
    """Page and offset of every newest token."""
    pages, offsets = [], []
    for b, (length, n) in enumerate(zip(st.host_lens, st.host_counts)):
        index = torch.arange(length - n, length, device="cuda")
        pages.append(st.table[b, index // st.page].long())
        offsets.append(index % st.page)
    return torch.cat(pages), torch.cat(offsets)


def _sequence(st, b, codes, exps):
    """fp32 [heads][len][D] of sequence b."""
    length = st.host_lens[b]
    pages = st.table[b, :-(-length // st.page)].long()
    values = _dequantise(codes[pages], exps[pages].transpose(-1, -2))              # [pages][heads][page][D]
    return values.transpose(0, 1).flatten(1, 2)[:, :length]


def _plain_select(st):
    signs = _parts(st)[4]
    first, last, out = 1, 1, []
    for b, (length, n) in enumerate(zip(st.host_lens, st.host_counts)):
        blocks = -(-length // st.page)
        packed = signs[st.table[b, :blocks].long()].transpose(0, 1).flatten(1, 2)      # [heads][blocks * page][D/8]
        bits = ((packed.unsqueeze(-1) >> torch.arange(8, dtype=torch.uint8, device="cuda")) & 1).flatten(-2)
        keys = bits.float() * 2 - 1
        q = torch.where(st.q[st.bounds[b]:st.bounds[b + 1]].float() >= 0, 1.0, -1.0)
        q = q.unflatten(1, (st.H, st.G)).transpose(0, 1).flatten(1, 2)                 # [heads][n * G][D]
        agree = (torch.matmul(q, keys.transpose(-1, -2)) + st.D) * 0.5
        position = torch.arange(length - n, length, device="cuda")
        seen = torch.arange(blocks * st.page, device="cuda") <= position.unsqueeze(-1)   # [n][blocks * page]
        agree = agree.unflatten(1, (n, st.G)).masked_fill(~seen.unsqueeze(1), -1)
        score = agree.unflatten(-1, (blocks, st.page)).amax(-1).sum(2)                 # [heads][n][blocks]
        block = torch.arange(blocks, device="cuda")
        own_block = (position // st.page).unsqueeze(-1)
        forced = (block < first) | (block > own_block - last)
        score = torch.where(block > own_block, torch.full_like(score, -1), torch.where(forced, score + 1e6, score))
        if blocks < st.keep:
            score = torch.nn.functional.pad(score, (0, st.keep - blocks), value=-1)
        best, index = torch.sort(score, dim=-1, descending=True, stable=True)
        index = torch.where(best < 0, torch.full_like(index, 1 << 30), index)[..., :st.keep].sort(-1).values
        out.append(torch.where(index == 1 << 30, torch.full_like(index, -1), index).transpose(0, 1).to(torch.int32))
    return torch.cat(out)


def _plain_attend(st, chosen=None):
    kc, vc, ke, ve, _ = _parts(st)
    outs, lses = [], []
    for b, (length, n) in enumerate(zip(st.host_lens, st.host_counts)):
        k, v = _sequence(st, b, kc, ke), _sequence(st, b, vc, ve)
        q = st.q[st.bounds[b]:st.bounds[b + 1]].float().unflatten(1, (st.H, st.G)).transpose(0, 1).flatten(1, 2)     # [heads][n * G][D]
        position = torch.arange(length - n, length, device="cuda").unsqueeze(-1)
        key = torch.arange(length, device="cuda")
        seen = key <= position
        if st.window:
            seen = seen & (key > position - st.window)
        seen = seen.unsqueeze(0).expand(st.H, n, length)
        if chosen is not None:
            blocks = -(-length // st.page)
            picked = chosen[st.bounds[b]:st.bounds[b + 1]].transpose(0, 1).long()                                   # [heads][n][keep]
            member = torch.zeros((st.H, n, blocks + 1), dtype=torch.bool, device="cuda")
            member.scatter_(2, torch.where(picked < 0, torch.full_like(picked, blocks), picked), True)
            seen = seen & member[..., key // st.page]
        step = max(1, min(st.H, (1 << 29) // (n * st.G * length)))
        o, lse = [], []
        for h in range(0, st.H, step):
            s = torch.matmul(q[h:h + step], k[h:h + step].transpose(-1, -2)) * st.scale
            s = s.unflatten(1, (n, st.G)).masked_fill(~seen[h:h + step].unsqueeze(2), float("-inf")).flatten(1, 2)
            m = s.amax(-1, keepdim=True).clamp_min(-1e30)
            p = torch.exp(s - m)
            total = p.sum(-1, keepdim=True)
            o.append(torch.matmul(p, v[h:h + step]) / total.clamp_min(1e-30))
            lse.append((m + torch.log(total)).squeeze(-1))
        outs.append(torch.cat(o).unflatten(1, (n, st.G)).transpose(0, 1).flatten(1, 2))
        lses.append(torch.cat(lse).unflatten(1, (n, st.G)).transpose(0, 1).flatten(1, 2))
    return torch.cat(outs).to(st.dtype), torch.cat(lses)


def _plain(st):
    if st.kind in ("append", "step"):
        pages, offsets = _places(st)
        _store(st, st.k, st.v, pages, offsets)
    if st.kind == "append":
        kc, vc, ke, ve, _ = _parts(st)
        return (_dequantise(kc[pages, :, offsets], ke[pages, :, :, offsets]).to(st.dtype),
                _dequantise(vc[pages, :, offsets], ve[pages, :, :, offsets]).to(st.dtype))
    if st.kind == "attend":
        return _plain_attend(st)
    chosen = _plain_select(st)
    return chosen if st.kind == "select" else (chosen, _plain_attend(st, chosen)[0])


# ---------------------------------------------------------------------------------------- one pass

def run(st):
    if not own:
        return _plain(st)
    cache = st.cache
    if st.kind in ("append", "step"):
        cache.write(st.k, st.v, st.table, st.lens, start=st.start)
    if st.kind == "append":
        return cache.read(st.table, st.lens, start=st.start, tokens=st.tokens, dtype=st.dtype)
    if st.kind == "attend":
        return cache.attend(st.q, st.table, st.lens, start=st.start, scale=st.scale, window=st.window, want_lse=True)
    chosen = cache.select(st.q, st.table, st.lens, st.keep, start=st.start, first=1, last=1)
    if st.kind == "select":
        return chosen
    return chosen, cache.attend(st.q, st.table, st.lens, start=st.start, scale=st.scale, blocks=chosen)


# ---------------------------------------------------------------------------------------- the definition in 64 bits

def _exact_group_values(x):
    """What the cache stands for after x [..][D] was written: the nearest multiples of E2M1's step at each magnitude, times the scale."""
    x = x.double().unflatten(-1, (-1, 32))
    high = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(high / 6)).clamp(-100, 100)
    e = torch.where(high > 6 * torch.exp2(e), e + 1, e)
    e = torch.where(high <= 6 * torch.exp2(e - 1), e - 1, e).clamp(-100, 100)
    y = x / torch.exp2(e)
    step = 0.5 * (1 + (y.abs() >= 2) + 2 * (y.abs() >= 4))
    return (torch.round(y / step) * step * torch.exp2(e)).flatten(-2)


def _exact_values(codes, exps):
    """[..][D] in 64 bits from codes [..][D/2] and exponent bytes [..][D/32]."""
    one = [(-1.0) ** (c >> 3) * ((c & 1) * 0.5 if c & 6 == 0 else (1 + 0.5 * (c & 1)) * 2.0 ** ((c >> 1 & 3) - 1)) for c in range(16)]
    pairs = torch.tensor([[one[byte & 15], one[byte >> 4]] for byte in range(256)], dtype=torch.float64, device=codes.device)
    return (pairs[codes.long()].flatten(-2).unflatten(-1, (-1, 32)) * torch.exp2(exps.double() - 127).unsqueeze(-1)).flatten(-2)


def exact(case, seed):
    st = prepare(case, seed)
    if st.kind == "append":
        return _exact_group_values(st.k), _exact_group_values(st.v)
    D, H, G, page = st.D, st.H, st.G, st.page
    c, e = page * D // 2, page * D // 32
    tokens = [torch.arange(length, device="cuda") for length in st.host_lens]
    all_blocks, all_out, all_lse = [], [], []
    for b, (length, n) in enumerate(zip(st.host_lens, st.host_counts)):
        rows, at = slice(st.bounds[b], st.bounds[b + 1]), tokens[b]
        blocks = -(-length // page)
        record = st.data[st.table[b, :blocks].long()]                              # [blocks][H][record]
        rows_of = lambda h, first, width: record[:, h, first:first + page * width].reshape(-1, width)[:length]
        columns_of = lambda h, first: record[:, h, first:first + e].reshape(blocks, D // 32, page).transpose(1, 2).reshape(-1, D // 32)[:length]
        q = st.q[rows].double().view(n, H, G, D)
        place = torch.arange(length - n, length, device="cuda")
        visible = at.view(1, -1) <= place.view(-1, 1)
        if st.window:
            visible &= at.view(1, -1) > (place - st.window).view(-1, 1)
        chosen = torch.full((n, H, st.keep), -1, dtype=torch.int64, device="cuda")
        out = torch.empty((n, H, G, D), dtype=torch.float64, device="cuda")
        lse = torch.empty((n, H, G), dtype=torch.float64, device="cuda")
        some = max(1, (1 << 27) // (G * length))                                   # query tokens at a time
        for h in range(H):
            k, v = _exact_values(rows_of(h, 0, D // 2), columns_of(h, 2 * c)), _exact_values(rows_of(h, c, D // 2), columns_of(h, 2 * c + e))
            signs = rows_of(h, 2 * c + 2 * e, D // 8)
            positive = torch.stack([signs >> i & 1 for i in range(8)], -1).flatten(-2) == 1
            if st.kind == "step":
                k[length - n:], v[length - n:] = _exact_group_values(st.k[rows, h]), _exact_group_values(st.v[rows, h])
                positive[length - n:] = st.k[rows, h] >= 0
            for t in range(0, n, some):
                part = slice(t, min(n, t + some))
                mask = visible[part]
                if st.kind != "attend":
                    equal = D - torch.matmul((q[part, h] >= 0).double(), (~positive).double().t()) - torch.matmul((q[part, h] < 0).double(), positive.double().t())
                    equal = torch.where(mask.unsqueeze(1), equal, torch.full_like(equal, -1e9))
                    equal = torch.nn.functional.pad(equal, (0, blocks * page - length), value=-1e9)
                    score = equal.view(equal.shape[0], G, blocks, page).amax(-1).sum(1)
                    number = torch.arange(blocks, device="cuda")
                    mine = place[part].view(-1, 1) // page
                    score = torch.where((number == 0) | (number == mine), torch.full_like(score, 1e6), score)
                    score = torch.where(number > mine, torch.full_like(score, -1e6), score)
                    # ties go to the lowest index: a small deduction that grows with it (scores are whole numbers)
                    ranked = score - number / (2.0 * blocks)
                    best, index = ranked.topk(min(st.keep, blocks), dim=-1)
                    index = torch.where(best < -1, torch.full_like(index, 1 << 40), index).sort(-1).values
                    chosen[part, h, :index.shape[1]] = torch.where(index == 1 << 40, torch.full_like(index, -1), index)
                if st.kind == "select":
                    continue
                if st.kind == "step":
                    inside = torch.zeros((mask.shape[0], blocks), dtype=torch.float64, device="cuda")
                    picked = chosen[part, h]
                    inside.scatter_add_(1, picked.clamp_min(0), (picked >= 0).double())
                    mask = mask & (inside > 0)[:, at // page]
                s = torch.matmul(q[part, h], k.t()) * st.scale
                s = torch.where(mask.unsqueeze(1), s, torch.full_like(s, float("-inf")))
                lse[part, h] = torch.logsumexp(s, -1)
                out[part, h] = torch.matmul(torch.exp(s - lse[part, h].unsqueeze(-1)), v)
        all_blocks.append(chosen)
        all_out.append(out.flatten(1, 2))
        all_lse.append(lse.flatten(1, 2))
    if st.kind == "select":
        return torch.cat(all_blocks)
    if st.kind == "step":
        return torch.cat(all_blocks), torch.cat(all_out)
    return torch.cat(all_out), torch.cat(all_lse)
