"""Measured work of what a decoder needs around the 4-bit key/value cache: rotary positions, eviction by accumulated attention weight, log
probabilities of tokens.

``own`` False: the plain form, elementary torch operations in 32 bits (angles and rotations in 64).  ``own`` True: the library's calls.

``kind`` of a case says which entry points a pass goes through:

  rotary    rotary: queries and keys side by side, rotated by their positions
  place     Cache4.write_rotary: rotated queries out, rotated keys and values into the cache, then Cache4.read of the same tokens
  weigh     Cache4.weigh: the attention weight that every cached token gets from the rows, added to what it had
  evict     Cache4.heaviest and Cache4.move: the tokens to keep, moved into fresh pages with their weights; then Cache4.read of them
  logprobs  token_logprobs: log probabilities of given tokens, entropy, log of the sum of exponentials, the best alternatives

Layout of the cache, uint8 [pages][kv_heads][record]; a record is
  K codes [page][D/2] | V codes [page][D/2] | K exponents [D/32][page] | V exponents [D/32][page] | signs of K [page][D/8]
Element d of a token is nibble d % 2 (low first) of byte d / 2, an E2M1 number (sign, two bits of exponent, one of mantissa); its
group of 32 has a power of two as scale, 2^(byte - 127); a sign bit is 1 where the element was >= 0, bit d % 8 of byte d / 8.
Token i of sequence b lies in page table[b][i / page], at i % page; the newest tokens of a sequence end at lens[b] - 1.
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32, "i32": torch.int32}


def listed():
    return [
        # two prompts' queries and keys, 32 + 8 heads
        {"name": "rotary_prompt_16384", "kind": "rotary", "dtype": "bf16", "tokens": 16384, "heads": 40, "dim": 128, "rotated": 128, "interleaved": False,
         "inverse": False, "far": 0, "magnitude": 1.0},
        # a few tokens far out in a long context whose angles are scaled; a third of a head, neighbours in pairs, and backwards (the gradient)
        {"name": "rotary_far_f32", "kind": "rotary", "dtype": "f32", "tokens": 333, "heads": 5, "dim": 96, "rotated": 32, "interleaved": True,
         "inverse": True, "far": 1000000, "magnitude": 1.25},
        # the smallest call: one decoder step's new tokens of eight conversations
        {"name": "place_decode_8", "kind": "place", "dtype": "bf16", "batch": 8, "len_min": 1000, "len_max": 1030, "n_min": 1, "n_max": 1,
         "kv_heads": 8, "group": 4, "dim": 128, "page": 64, "rotated": 128, "interleaved": False, "magnitude": 1.0},
        # chunks of prompts of every length from one token on, half of a head rotated, fp32 as the library's products give it
        {"name": "place_ragged_f32", "kind": "place", "dtype": "f32", "batch": 7, "len_min": 1, "len_max": 4099, "n_min": 1, "n_max": 1031,
         "kv_heads": 2, "group": 3, "dim": 192, "page": 16, "rotated": 96, "interleaved": True, "magnitude": 1.0},
        # an ordinary serving batch, conversations of all lengths
        {"name": "weigh_batch_64", "kind": "weigh", "dtype": "bf16", "batch": 64, "len_min": 500, "len_max": 8192, "n_min": 1, "n_max": 1,
         "kv_heads": 8, "group": 4, "dim": 128, "page": 64, "window": 0, "previous": True, "decay": 1.0},
        # a few drafted tokens, a layer with a sliding window, wide heads, fp16
        {"name": "weigh_draft_window_f16", "kind": "weigh", "dtype": "f16", "batch": 16, "len_min": 40, "len_max": 6001, "n_min": 5, "n_max": 5,
         "kv_heads": 4, "group": 6, "dim": 192, "page": 16, "window": 1000, "previous": True, "decay": 0.96875},
        # two prompts against themselves: the matrix cores' case
        {"name": "weigh_prompt_4096", "kind": "weigh", "dtype": "bf16", "batch": 2, "len_min": 4096, "len_max": 4096, "n_min": 4096, "n_max": 4096,
         "kv_heads": 8, "group": 4, "dim": 128, "page": 64, "window": 0, "previous": False, "decay": 1.0},
        # conversations cut back to a budget
        {"name": "evict_batch_32", "kind": "evict", "dtype": "bf16", "batch": 32, "len_min": 2100, "len_max": 16384, "kv_heads": 8, "group": 1, "dim": 128,
         "page": 64, "keep": 2048, "first": 4, "last": 256},
        # one very long document, and an odd budget
        {"name": "evict_long_131072", "kind": "evict", "dtype": "bf16", "batch": 1, "len_min": 131072, "len_max": 131072, "kv_heads": 4, "group": 1, "dim": 64,
         "page": 32, "keep": 8111, "first": 1, "last": 64},
        # a decoding step of eight conversations
        {"name": "logprobs_step_8", "kind": "logprobs", "dtype": "bf16", "rows": 8, "cols": 131072, "top": 20},
        # the sums of a head of signs as they are, an odd vocabulary
        {"name": "logprobs_sums_333", "kind": "logprobs", "dtype": "i32", "rows": 333, "cols": 50001, "top": 5},
        # a long text scored
        {"name": "logprobs_text_4096", "kind": "logprobs", "dtype": "bf16", "rows": 4096, "cols": 131072, "top": 1},
    ]


# What no drawn case goes over: cached bytes, (query head, key) pairs times the head dimension, elements rotated, elements of logits.
MAX_CACHE_BYTES, MAX_PAIR_DIM, MAX_ROTATED, MAX_LOGITS = 300e6, 6e10, 8e7, 4e8


def _log(rng, lo, hi):
    """An integer spread over the logarithm of [lo, hi]."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["rotary", "place", "weigh", "weigh", "evict", "logprobs", "logprobs"])
        case = {"kind": kind, "dtype": rng.choice(["bf16", "bf16", "f16", "f32"])}
        if kind == "logprobs":
            case["dtype"] = rng.choice(["bf16", "bf16", "f16", "f32", "i32"])
            case.update(rows=_log(rng, 1, 8192), cols=_log(rng, 2, 262144))
            case["top"] = min(case["cols"], rng.choice([0, 1, 2, 5, 20, 64]))
            if case["rows"] * case["cols"] <= MAX_LOGITS:
                return case
            continue
        dims = [64, 96, 128, 128, 192, 256]
        if kind == "rotary":
            case.update(tokens=_log(rng, 1, 20000), heads=_log(rng, 1, 96), dim=rng.choice(dims + [80, 112, 160, 320]), interleaved=rng.random() < 0.5,
                        inverse=rng.random() < 0.25, far=rng.choice([0, 0, 10 ** 5, 10 ** 6, 10 ** 9]), magnitude=rng.choice([1.0, 1.0, 1.25]))
            case["rotated"] = rng.choice([case["dim"], case["dim"], case["dim"] // 2, case["dim"] // 4 * 2, 16])
            if case["tokens"] * case["heads"] * case["dim"] <= MAX_ROTATED:
                return case
            continue
        case.update(kv_heads=rng.choice([1, 2, 3, 4, 8]), dim=rng.choice(dims), page=rng.choice([16, 32, 64, 128, 256]))
        case["group"] = 1 if kind == "evict" else rng.choice([1, 2, 3, 4, 5, 6, 7, 8, 16])
        decode = rng.random() < 0.5
        case["batch"] = _log(rng, 1, 64 if decode or kind == "evict" else 8)
        hi = _log(rng, 2, 131072 if decode or kind == "evict" else 20000)
        lo = _log(rng, 1, hi)
        case["len_min"], case["len_max"] = lo, hi
        if kind == "evict":
            case["keep"] = _log(rng, 1, min(hi, 16384))
            case["first"] = rng.choice([0, 0, 1, 4]) if case["keep"] > 8 else 0
            case["last"] = rng.choice([0, 1, case["keep"] // 8, case["keep"] // 2])
        else:
            n_hi = _log(rng, 1, min(hi, 8192)) if not decode else min(hi, rng.choice([1, 1, 1, 2, 5]))
            case["n_min"], case["n_max"] = n_hi if decode or rng.random() < 0.3 else _log(rng, 1, n_hi), n_hi
        if kind == "weigh":
            case["window"] = rng.choice([0, 0, 0, _log(rng, 1, hi)])
            case["previous"] = rng.random() < 0.6
            case["decay"] = rng.choice([1.0, 0.96875]) if case["previous"] else 1.0
        if kind == "place":
            case["interleaved"], case["magnitude"] = rng.random() < 0.5, rng.choice([1.0, 1.0, 1.25])
            case["rotated"] = rng.choice([case["dim"], case["dim"], case["dim"] // 2, case["dim"] // 4])
        lens, counts = _lens(case), _counts(case)
        cached = sum(lens) * case["kv_heads"] * case["dim"] * 1.3
        written = sum(counts) * case["kv_heads"] * case["dim"] * (case["group"] + 2)
        if kind == "evict":
            written = 2 * case["batch"] * case["keep"] * case["kv_heads"] * case["dim"]
        if cached <= MAX_CACHE_BYTES and written <= MAX_ROTATED and (kind != "weigh" or _pairs(case, lens, counts) * case["dim"] <= MAX_PAIR_DIM):
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
    """New tokens of every sequence; for evict the tokens that are kept."""
    if case["kind"] == "evict":
        return [min(case["keep"], length) for length in _lens(case)]
    return [min(n, length) for n, length in zip(_spread(case["n_min"], case["n_max"], case["batch"]), _lens(case))]


def _pairs(case, lens, counts):
    """(query head, key) pairs that are weighed."""
    window, total = case["window"], 0
    for length, n in zip(lens, counts):
        first = length - n
        limit = window if window else length
        ramp = max(0, min(limit, length) - first)            # query tokens that see fewer keys than the limit allows
        total += ramp * first + ramp * (ramp + 1) // 2 + (n - ramp) * min(limit, length)
    return total * case["kv_heads"] * case["group"]


def work(case):
    size = DTYPES[case["dtype"]].itemsize
    if case["kind"] == "logprobs":
        rows, cols, top = case["rows"], case["cols"], case["top"]
        return {"bytes": rows * cols * size + rows * (4 + 12 + 8 * top), "flops": 6 * rows * cols}
    if case["kind"] == "rotary":
        n = case["tokens"] * case["heads"] * case["dim"]
        return {"bytes": 2 * n * size + 4 * case["tokens"], "flops": 3 * case["tokens"] * case["heads"] * case["rotated"]}
    lens, counts = _lens(case), _counts(case)
    D, H, G, tokens = case["dim"], case["kv_heads"], case["group"], sum(counts)
    record = 2 * (D // 2 + D // 32)                          # K and V of a token and head
    plan = 4 * sum(-(-length // case["page"]) for length in lens) + 4 * len(lens)
    q = tokens * H * G * D * size
    if case["kind"] == "place":
        return {"bytes": 2 * q + 4 * tokens * H * D * size + tokens * H * (2 * record + D // 8) + plan, "flops": 3 * tokens * H * (G + 1) * case["rotated"] + 4 * tokens * H * D}
    if case["kind"] == "evict":
        return {"bytes": 4 * sum(lens) * H + tokens * H * (2 * (record + D // 8) + record + 4 + 4 + 8 + 2 * D * size) + plan, "flops": 2 * tokens * H * D}
    seen = sum(min(length, n + case["window"]) if case["window"] else length for length, n in zip(lens, counts))
    return {"bytes": seen * H * record // 2 + q + 4 * tokens * H * G + 4 * H * sum(lens) * (2 if case["previous"] else 1) + plan,
            "flops": 2 * D * _pairs(case, lens, counts)}


# ---------------------------------------------------------------------------------------- state

class State:
    pass


def _parts(data, page, D):
    """Views of a cache's data: K codes, V codes, K exponents, V exponents, signs."""
    c, e = page * D // 2, page * D // 32
    return (data[..., :c].unflatten(-1, (page, D // 2)), data[..., c:2 * c].unflatten(-1, (page, D // 2)),
            data[..., 2 * c:2 * c + e].unflatten(-1, (D // 32, page)), data[..., 2 * c + e:2 * c + 2 * e].unflatten(-1, (D // 32, page)),
            data[..., 2 * c + 2 * e:].unflatten(-1, (page, D // 8)))


def _table(pages, at, order):
    table = torch.full((len(pages), max(pages)), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(pages):
        table[b, :n] = order[at:at + n]
        at += n
    return table, at


def _frequencies(rotated):
    """Radians a position, 64 bits: a geometric row from 1 down to 1 / 10000."""
    return 10000.0 ** (-torch.arange(0, rotated, 2, dtype=torch.float64, device="cuda") / rotated)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *shape: torch.randn(*shape, generator=gen, device="cuda")
    uniform = lambda *shape: torch.rand(*shape, generator=gen, device="cuda")
    dtype = DTYPES[case["dtype"]]
    st = State()
    st.kind, st.dtype = case["kind"], dtype
    if st.kind == "logprobs":
        rows, cols = case["rows"], case["cols"]
        st.top, st.scale = case["top"], 1.0
        st.logits = torch.empty((rows, cols), dtype=dtype, device="cuda")
        some = max(1, (1 << 26) // cols)
        for r in range(0, rows, some):
            # some rows are sure of a few tokens, some are not
            part = st.logits[r:r + some]
            x = normal(*part.shape) * (0.5 + 2.5 * uniform(part.shape[0], 1))
            if dtype == torch.int32:
                part.copy_((x * 45).round())                 # sums of a few thousand signs
            else:
                # a quarter of the rows are constrained: most tokens are ruled out
                ruled = (uniform(part.shape[0], 1) < 0.25) & (uniform(*part.shape) < 0.9)
                part.copy_(x.masked_fill_(ruled, float("-inf")))
        if dtype == torch.int32:
            st.scale = 1.0 / 45
        else:
            st.logits[:, cols // 2] = 1.5                    # no row without a token
        st.targets = torch.randint(0, cols, (rows,), generator=gen, device="cuda")
        if dtype != torch.int32:
            chosen = st.logits.gather(1, st.targets.unsqueeze(1)).squeeze(1)
            st.targets = torch.where(torch.isinf(chosen), torch.full_like(st.targets, cols // 2), st.targets)
        if own:
            import paper_2006_16578_amd as bnn
            st.bnn = bnn
        return st
    if st.kind == "rotary":
        tokens, heads = case["tokens"], case["heads"]
        st.x = normal(tokens, heads, case["dim"]).to(dtype)
        # a few sequences behind one another, each with its own first position
        cut = max(1, tokens // 3)
        index = torch.arange(tokens, device="cuda")
        st.positions = (case["far"] + (index // cut) * 777 + index % cut).to(torch.int32)
        st.frequencies, st.interleaved, st.inverse, st.magnitude = _frequencies(case["rotated"]), case["interleaved"], case["inverse"], case["magnitude"]
        if own:
            import paper_2006_16578_amd as bnn
            st.bnn = bnn
        return st
    st.page, st.D, st.H, st.G = case["page"], case["dim"], case["kv_heads"], case["group"]
    st.host_lens, st.host_counts = _lens(case), _counts(case)
    pages = [-(-length // st.page) for length in st.host_lens]
    more = [-(-n // st.page) for n in st.host_counts] if st.kind == "evict" else []
    total = sum(pages) + sum(more)
    H, D, G = st.H, st.D, st.G
    st.data = torch.zeros((total, H, st.page * (D + D // 16 + D // 8)), dtype=torch.uint8, device="cuda")
    order = torch.randperm(total, generator=gen, device="cuda").to(torch.int32)
    st.table, at = _table(pages, 0, order)
    st.lens = torch.tensor(st.host_lens, dtype=torch.int32, device="cuda")
    st.bounds = [0]
    for n in st.host_counts:
        st.bounds.append(st.bounds[-1] + n)
    st.tokens = st.bounds[-1]
    st.start = None if len(set(st.host_counts)) == 1 else torch.tensor(st.bounds, dtype=torch.int32, device="cuda")
    width = st.table.shape[1] * st.page
    # Keys have a few channels much wider than the rest and an offset of their own, as projections of a trained layer have; values are even.
    wide = torch.exp(0.5 * normal(H, D)) * (1 + 5 * (uniform(H, D) < 0.02))
    offset = 0.3 * normal(H, D)
    new_k, new_v, queries = [], [], []
    for b, (length, n) in enumerate(zip(st.host_lens, st.host_counts)):
        k, v = normal(length, H, D) * wide + offset, 0.6 * normal(length, H, D)
        if st.kind != "place":
            index = torch.arange(length, device="cuda")
            _store(st, k.to(dtype), v.to(dtype), st.table[b, index // st.page].long(), index % st.page)
        if st.kind == "place":
            new_k.append(k[length - n:].to(dtype))
            new_v.append(v[length - n:].to(dtype))
        if st.kind != "evict":
            # a query looks for some key of the past, more or less
            looked = torch.randint(0, length, (n,), generator=gen, device="cuda")
            strength = uniform(n, H, G, 1)
            queries.append((strength * (k[looked] / wide).unsqueeze(2) + normal(n, H, G, D)).reshape(n, H * G, D).to(dtype))
    st.scale = 1.0 / math.sqrt(D)
    if st.kind == "place":
        st.q, st.k, st.v = torch.cat(queries), torch.cat(new_k), torch.cat(new_v)
        st.frequencies, st.interleaved, st.magnitude = _frequencies(case["rotated"]), case["interleaved"], case["magnitude"]
    if st.kind == "weigh":
        st.q, st.window, st.decay = torch.cat(queries), case["window"], case["decay"]
        # what attention over the same keys gave
        st.lse = torch.empty((st.tokens, H * G), dtype=torch.float32, device="cuda")
        for b, rows, h, s in _scores(st):
            st.lse[rows].view(-1, H, G)[:, h] = torch.logsumexp(s, -1)
        st.previous = torch.exp(2 * normal(len(pages), H, width)) * 0.01 if case["previous"] else None
        st.out = torch.zeros((len(pages), H, width), dtype=torch.float32, device="cuda")
    if st.kind == "evict":
        st.keep, st.first, st.last = case["keep"], case["first"], case["last"]
        st.into, at = _table(more, at, order)
        # few tokens have most of the weight; some got none that fp32 can tell
        st.weights = torch.exp(2.5 * normal(len(pages), H, width)) * (uniform(len(pages), H, width) < 0.9)
    if own:
        import paper_2006_16578_amd as bnn
        st.cache = bnn.Cache4(kv_heads=H, head_dim=D, page=st.page, signs=True, data=st.data)
    return st


# ---------------------------------------------------------------------------------------- plain form

def _quantise(x):
    """x [tokens][heads][D] -> codes [..][D/2], exponent bytes [..][D/32]."""
    groups = x.float().unflatten(-1, (-1, 32))
    high = groups.abs().amax(-1)
    mantissa, power = torch.frexp(high)                             # high = mantissa 2^power, mantissa in [1/2, 1)
    e = power.to(torch.int32) - 3 + (mantissa > 0.75).to(torch.int32)   # the smallest e with high <= 6 * 2^e
    e = torch.where(high == 0, torch.full_like(e, -100), e.clamp(-100, 100))
    y = groups.abs() * ((127 - e) << 23).view(torch.float32).unsqueeze(-1)
    code = ((y > 0.25).to(torch.uint8) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5)).to(torch.uint8)
    code = (code | (torch.signbit(groups).to(torch.uint8) << 3)).flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _dequantise(codes, exps):
    """codes [..][D/2], exponent bytes [..][D/32] -> fp32 [..][D]."""
    code = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).to(torch.int32)
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, -0.0, -0.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
    scale = (exps.to(torch.int32) << 23).view(torch.float32)
    return (grid[code].unflatten(-1, (-1, 32)) * scale.unsqueeze(-1)).flatten(-2)


def _store(st, k, v, pages, offsets):
    kc, vc, ke, ve, signs = _parts(st.data, st.page, st.D)
    kc[pages, :, offsets], ke[pages, :, :, offsets] = _quantise(k)
    vc[pages, :, offsets], ve[pages, :, :, offsets] = _quantise(v)
    bits = (k >= 0).to(torch.uint8).unflatten(-1, (-1, 8))
    signs[pages, :, offsets] = (bits << torch.arange(8, dtype=torch.uint8, device=k.device)).sum(-1).to(torch.uint8)


def _indexes(st):
    """Index of every newest token in its sequence, and the page and offset where it lies."""
    index = [torch.arange(length - n, length, device="cuda") for length, n in zip(st.host_lens, st.host_counts)]
    pages = torch.cat([st.table[b, i // st.page].long() for b, i in enumerate(index)])
    index = torch.cat(index)
    return index, pages, index % st.page


def _rotate(x, positions, frequencies, interleaved, magnitude, inverse=False):
    """x [tokens][heads][D] -> the same in 64 bits."""
    x = x.double()
    angle = positions.double().unsqueeze(-1) * frequencies
    c, s = (torch.cos(angle) * magnitude).unsqueeze(1), (torch.sin(angle) * magnitude).unsqueeze(1)
    if inverse:
        s = -s
    R = 2 * frequencies.shape[0]
    a, b = (x[..., 0:R:2], x[..., 1:R:2]) if interleaved else (x[..., :R // 2], x[..., R // 2:R])
    pair = a * c - b * s, a * s + b * c
    turned = torch.stack(pair, -1).flatten(-2) if interleaved else torch.cat(pair, -1)
    return torch.cat((turned, x[..., R:]), -1)


def _scores(st, wide=False):
    """Pieces (b, rows of the call, kv head, scores [tokens][group][keys], -infinity where a row does not see a key); wide: in 64 bits."""
    kc, _, ke, _, _ = _parts(st.data, st.page, st.D)
    for b, (length, n) in enumerate(zip(st.host_lens, st.host_counts)):
        pages = st.table[b, :-(-length // st.page)].long()
        key = torch.arange(length, device="cuda")
        some = max(1, (1 << 28) // (st.G * length))                                # query tokens at a time
        for h in range(st.H):
            k = _dequantise(kc[pages, h], ke[pages, h].transpose(-1, -2)).flatten(0, 1)[:length]
            k = k.double() if wide else k
            for t in range(0, n, some):
                rows = slice(st.bounds[b] + t, st.bounds[b] + min(n, t + some))
                position = torch.arange(length - n + t, length - n + min(n, t + some), device="cuda").unsqueeze(-1)
                seen = key <= position
                if st.window:
                    seen = seen & (key > position - st.window)
                q = st.q[rows, h * st.G:(h + 1) * st.G]
                s = torch.matmul((q.double() if wide else q.float()).flatten(0, 1), k.t()).unflatten(0, (-1, st.G)) * st.scale
                yield b, rows, h, s.masked_fill_(~seen.unsqueeze(1), float("-inf"))


def _weigh(st, wide=False):
    out = st.out.to(torch.float64 if wide else torch.float32, copy=True)
    previous, lse = (x if x is None or not wide else x.double() for x in (st.previous, st.lse))
    for b, (length, n) in enumerate(zip(st.host_lens, st.host_counts)):
        out[b, :, :length] = 0
        if previous is not None:                             # new tokens had nothing before
            out[b, :, :length - n] = previous[b, :, :length - n] * st.decay
    for b, rows, h, s in _scores(st, wide):
        p = torch.exp(s - lse[rows].unflatten(1, (st.H, st.G))[:, h].unsqueeze(-1))
        out[b, h, :s.shape[-1]] += p.sum((0, 1))
    return out


def _heaviest(st):
    tokens = torch.full((len(st.host_lens), st.H, st.keep), -1, dtype=torch.int32, device="cuda")
    for b, (length, n) in enumerate(zip(st.host_lens, st.host_counts)):
        index = torch.arange(length, device="cuda")
        if length > st.keep:
            w = st.weights[b, :, :length].masked_fill((index < st.first) | (index >= length - st.last), float("inf"))
            index = torch.sort(w, dim=-1, descending=True, stable=True).indices[:, :st.keep].sort(-1).values
        tokens[b, :, :n] = index.to(torch.int32)
    return tokens, st.lens.clamp_max(st.keep)


def _move(st, tokens):
    moved = torch.zeros((len(st.host_lens), st.H, st.into.shape[1] * st.page), dtype=torch.float32, device="cuda")
    head = torch.arange(st.H, device="cuda").unsqueeze(-1)
    keys, values = [], []
    for b, n in enumerate(st.host_counts):
        source = tokens[b, :, :n].long()
        target = torch.arange(n, device="cuda").expand(st.H, n)
        moved[b, :, :n] = st.weights[b].gather(1, source)
        p, o = st.table[b].long()[source // st.page], source % st.page
        r, i = st.into[b].long()[target // st.page], target % st.page
        kc, vc, ke, ve, signs = _parts(st.data, st.page, st.D)
        for part in (kc, vc, signs):
            part[r, head, i] = part[p, head, o]
        for part in (ke, ve):
            part[r, head, :, i] = part[p, head, :, o]
        keys.append(_dequantise(kc[r, head, i], ke[r, head, :, i]).transpose(0, 1))
        values.append(_dequantise(vc[r, head, i], ve[r, head, :, i]).transpose(0, 1))
    return moved, torch.cat(keys).to(st.dtype), torch.cat(values).to(st.dtype)


def _best(x, top):
    """Columns of the `top` largest of every row of x (fp32), ties to the lower column."""
    bits = (x + 0.0).contiguous().view(torch.int32).long()   # (no -0)
    order = torch.where(bits < 0, -(bits & 0x7fffffff), bits)        # whole numbers in the order of the values
    column = torch.arange(x.shape[1], device="cuda")
    return torch.topk((order << 20) - column, top, dim=1).indices


def _plain_logprobs(st):
    outs = []
    some = max(1, (1 << 27) // st.logits.shape[1])
    for r in range(0, st.logits.shape[0], some):
        x = st.logits[r:r + some].float() * st.scale
        m = x.amax(1, keepdim=True)
        d = x - m
        e = torch.exp(d)
        total = e.sum(1)
        log = torch.log(total)
        entropy = log - (e * d.clamp_min(-1e30)).sum(1) / total
        best = _best(x, st.top)
        outs.append((d.gather(1, st.targets[r:r + some].unsqueeze(1)).squeeze(1) - log, entropy, m.squeeze(1) + log,
                     d.gather(1, best) - log.unsqueeze(1), best.to(torch.int32)))
    return tuple(torch.cat(parts) for parts in zip(*outs))


def _plain(st):
    if st.kind == "rotary":
        return _rotate(st.x, st.positions, st.frequencies, st.interleaved, st.magnitude, st.inverse).to(torch.float32).to(st.dtype)
    if st.kind == "logprobs":
        return _plain_logprobs(st)
    if st.kind == "weigh":
        return _weigh(st)
    if st.kind == "evict":
        tokens, lens = _heaviest(st)
        return (tokens, lens, *_move(st, tokens))
    index, pages, offsets = _indexes(st)
    q, k = (_rotate(x, index, st.frequencies, st.interleaved, st.magnitude).to(torch.float32) for x in (st.q, st.k))
    _store(st, k, st.v, pages, offsets)
    kc, vc, ke, ve, _ = _parts(st.data, st.page, st.D)
    return (q.to(st.dtype), _dequantise(kc[pages, :, offsets], ke[pages, :, :, offsets]).to(st.dtype),
            _dequantise(vc[pages, :, offsets], ve[pages, :, :, offsets]).to(st.dtype))


# ---------------------------------------------------------------------------------------- one pass

def run(st):
    if not own:
        return _plain(st)
    if st.kind == "rotary":
        return st.bnn.rotary(st.x, st.positions, st.frequencies, interleaved=st.interleaved, magnitude=st.magnitude, inverse=st.inverse)
    if st.kind == "logprobs":
        return tuple(st.bnn.token_logprobs(st.logits, st.targets, scale=st.scale, top=st.top))
    cache = st.cache
    if st.kind == "weigh":
        return cache.weigh(st.q, st.lse, st.table, st.lens, start=st.start, scale=st.scale, window=st.window, previous=st.previous, decay=st.decay, out=st.out)
    if st.kind == "evict":
        tokens, lens = cache.heaviest(st.weights, st.table, st.lens, st.keep, first=st.first, last=st.last)
        moved = cache.move(tokens, st.table, st.into, weights=st.weights)
        return (tokens, lens, moved, *cache.read(st.into, lens, start=st.start, tokens=st.tokens, dtype=st.dtype))
    q = cache.write_rotary(st.q, st.k, st.v, st.table, st.lens, st.frequencies, start=st.start, interleaved=st.interleaved, magnitude=st.magnitude)
    return (q, *cache.read(st.table, st.lens, start=st.start, tokens=st.tokens, dtype=st.dtype))


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


def _exact_rotation(x, positions, frequencies, interleaved, magnitude, inverse):
    """Pairs as complex numbers, times magnitude * exp(i t)."""
    R = 2 * frequencies.shape[0]
    x = x.double()
    turned = x[..., :R].unflatten(-1, (R // 2, 2) if interleaved else (2, R // 2))
    if not interleaved:
        turned = turned.transpose(-1, -2)
    t = positions.double().view(-1, 1, 1) * frequencies * (-1 if inverse else 1)
    z = torch.view_as_complex(turned.contiguous()) * torch.polar(torch.full_like(t, magnitude), t)
    turned = torch.view_as_real(z)
    return torch.cat(((turned if interleaved else turned.transpose(-1, -2)).flatten(-2), x[..., R:]), -1)


def exact(case, seed):
    st = prepare(case, seed)
    if st.kind == "rotary":
        return _exact_rotation(st.x, st.positions, st.frequencies, st.interleaved, st.magnitude, st.inverse)
    if st.kind == "place":
        index = torch.cat([torch.arange(length - n, length, device="cuda") for length, n in zip(st.host_lens, st.host_counts)])
        turn = lambda x: _exact_rotation(x, index, st.frequencies, st.interleaved, st.magnitude, False)
        return turn(st.q), _exact_group_values(turn(st.k).float()), _exact_group_values(st.v)      # (a rotated key is rounded to fp32 once)
    if st.kind == "logprobs":
        outs = []
        some = max(1, (1 << 26) // st.logits.shape[1])
        for r in range(0, st.logits.shape[0], some):
            z = st.logits[r:r + some].double() * st.scale
            lp = torch.log_softmax(z, 1)
            outs.append((lp.gather(1, st.targets[r:r + some].unsqueeze(1)).squeeze(1), -(lp.exp() * lp.clamp_min(-1e30)).sum(1), torch.logsumexp(z, 1),
                         lp.topk(st.top, 1).values))
        return (*(torch.cat(parts) for parts in zip(*outs)), None)
    if st.kind == "weigh":
        pairs = _pairs(case, st.host_lens, st.host_counts)
        return None if pairs * st.D > 4e11 else _weigh_by_keys(st)
    out, keys, values = torch.zeros((len(st.host_lens), st.H, st.into.shape[1] * st.page), dtype=torch.float64, device="cuda"), [], []
    tokens, _ = _heaviest(st)
    one = [(-1.0) ** (c >> 3) * ((c & 1) * 0.5 if c & 6 == 0 else (1 + 0.5 * (c & 1)) * 2.0 ** ((c >> 1 & 3) - 1)) for c in range(16)]
    pairs = torch.tensor([[one[byte & 15], one[byte >> 4]] for byte in range(256)], dtype=torch.float64, device="cuda")
    D, page = st.D, st.page
    for b, n in enumerate(st.host_counts):
        k, v = (torch.empty((n, st.H, D), dtype=torch.float64, device="cuda") for _ in range(2))
        for h in range(st.H):
            kept = tokens[b, h, :n].long()
            out[b, h, :n] = st.weights[b, h, kept].double()
            record, o = st.data[st.table[b, kept // page].long(), h], (kept % page).unsqueeze(-1)
            code, group = torch.arange(D // 2, device="cuda"), torch.arange(D // 32, device="cuda")
            for where, first, exps in ((k, 0, page * D), (v, page * D // 2, page * D + page * D // 32)):
                mantissa = pairs[record.gather(1, first + o * (D // 2) + code).long()].flatten(1)
                power = record.gather(1, exps + group * page + o).double() - 127
                where[:, h] = (mantissa.unflatten(1, (-1, 32)) * torch.exp2(power).unsqueeze(-1)).flatten(1)
        keys.append(k)
        values.append(v)
    return None, None, out, torch.cat(keys), torch.cat(values)


def _weigh_by_keys(st):
    """Key by key: what every key gets from the rows that see it, in 64 bits."""
    D, page, H, G = st.D, st.page, st.H, st.G
    out = st.out.double()
    grid = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64, device="cuda")
    for b, (length, n) in enumerate(zip(st.host_lens, st.host_counts)):
        place = torch.arange(length - n, length, device="cuda").repeat_interleave(G)
        rows = slice(st.bounds[b], st.bounds[b + 1])
        record = st.data[st.table[b, :-(-length // page)].long()]
        some = max(1, (1 << 27) // (n * G))
        for h in range(H):
            code = record[:, h, :page * D // 2].reshape(-1, D // 2)[:length].long()
            code = torch.stack((code % 16, code // 16), -1).flatten(1)
            power = record[:, h, page * D:page * D + page * D // 32].reshape(-1, D // 32, page).transpose(1, 2).reshape(-1, D // 32)[:length].double() - 127
            k = grid[code % 8] * torch.where(code >= 8, -1.0, 1.0) * torch.exp2(power).repeat_interleave(32, 1)
            q = st.q[rows, h * G:(h + 1) * G].double().flatten(0, 1)
            lse = st.lse[rows, h * G:(h + 1) * G].double().flatten()
            for j in range(0, length, some):
                key = torch.arange(j, min(length, j + some), device="cuda").unsqueeze(1)
                sees = key <= place
                if st.window:
                    sees &= key + st.window > place
                p = torch.exp(torch.matmul(k[j:j + some], q.t()) * st.scale - lse)
                got = torch.where(sees, p, torch.zeros_like(p)).sum(1)
                if st.previous is not None:
                    got = got + torch.where(key.squeeze(1) < length - n, st.previous[b, h, j:j + got.shape[0]].double() * st.decay, torch.zeros_like(got))
                out[b, h, j:j + got.shape[0]] = got
    return out
