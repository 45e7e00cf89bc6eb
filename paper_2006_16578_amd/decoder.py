"""A decoder layer of a binarized language model on this library: products of signs around attention over the 4-bit cache.

    python -m paper_2006_16578_amd.decoder [--context 8192] [--steps 32] [--keep 32] [--budget 4096]

Every projection multiplies the signs of its input with packed +1/-1 weights (``sign_pack_f32``, ``bmm``), the hidden layer of the feed-forward part goes from bits to
bits (``bmm_thr``).  Signs do not depend on the length of a vector, so there is no norm to compute in front of them.  Keys and values go into a ``Cache4``;
queries attend to all of it or, with ``keep``, to the pages that ``Cache4.select`` chooses.  With ``rotary_base`` queries and keys are turned by their tokens' positions on their way
(``Cache4.write_rotary``).  Where the attention weight of every cached token is kept (``Cache4.weigh``), ``cut_back`` evicts the lightest tokens (``Cache4.heaviest``, ``Cache4.move``).
``Head`` multiplies signs with a vocabulary's and says what the sums mean for tokens (``token_logprobs``).  Weights are random: the module shows the calls.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as bnn


class DecoderLayer:
    """x [tokens][width] fp32 -> the same.  Weights are +1/-1, drawn from `seed`."""

    def __init__(self, width: int, heads: int, kv_heads: int, head_dim: int, hidden: int, seed: int = 0, device="cuda",
                 rotary_base: float | None = None):
        gen = torch.Generator(device=device).manual_seed(seed)
        weights = lambda rows, cols: bnn.sign_pack_f32(torch.randn(rows, cols, device=device, generator=gen), bnn.round_up(bnn.nwords(cols), 4))
        self.width, self.heads, self.kv_heads, self.head_dim, self.hidden = width, heads, kv_heads, head_dim, hidden
        self.w_qkv = weights((heads + 2 * kv_heads) * head_dim, width)
        self.w_out = weights(width, heads * head_dim)
        self.w_up, self.w_down = weights(hidden, width), weights(width, hidden)
        self.thresholds = torch.randint(-32, 33, (hidden,), dtype=torch.int32, device=device, generator=gen)
        self.frequencies = None if rotary_base is None else bnn.rotary_frequencies(head_dim, rotary_base, device=device)

    @staticmethod
    def _bits(x):
        return bnn.sign_pack_f32(x.contiguous(), bnn.round_up(bnn.nwords(x.shape[1]), 4))

    def _project(self, bits, weights, inputs: int):
        """Products of signs, brought back to unit variance."""
        return bnn.bmm(bits, weights, inputs).float() * inputs ** -0.5

    def attention(self, x, cache, table, lens, start=None, keep: int | None = None, positions=None, weights=None):
        """The attention part before its output projection, [tokens][heads][head_dim] fp32; the new keys and values go into the cache.  positions: of the rows' tokens, where these are not their places in the
        cache (after an eviction).  weights: fp32 [batch][kv_heads][tokens of the table], to which the weight that every token gets is added."""
        if keep is not None and weights is not None:
            raise ValueError("weights are added up by attention to the whole cache only")
        tokens = x.shape[0]
        qkv = self._project(self._bits(x), self.w_qkv, self.width).view(tokens, self.heads + 2 * self.kv_heads, self.head_dim)
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), dim=1)
        if self.frequencies is None:
            cache.write(k, v, table, lens, start)
        else:
            q = cache.write_rotary(q, k, v, table, lens, self.frequencies, start, positions)
        blocks = None if keep is None else cache.select(q, table, lens, keep, start)
        if weights is None:
            return cache.attend(q, table, lens, start, blocks=blocks)
        out, lse = cache.attend(q, table, lens, start, want_lse=True)
        cache.weigh(q, lse, table, lens, start, previous=weights, out=weights)
        return out

    def forward(self, x, cache, table, lens, start=None, keep: int | None = None, positions=None, weights=None):
        o = self.attention(x, cache, table, lens, start, keep, positions, weights).flatten(1)
        x = x + self._project(self._bits(o), self.w_out, self.heads * self.head_dim)
        hidden = bnn.bmm_thr(self._bits(x), self.w_up, self.thresholds, self.width)
        return x + self._project(hidden, self.w_down, self.hidden)


class Head:
    """x [tokens][width] fp32 -> what it says of a vocabulary's tokens: products of signs, brought to unit variance and divided by the temperature, as logits."""

    def __init__(self, width: int, vocabulary: int, seed: int = 0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        self.width = width
        self.w = bnn.sign_pack_f32(torch.randn(vocabulary, width, device=device, generator=gen), bnn.round_up(bnn.nwords(width), 4))

    def forward(self, x, targets=None, top: int = 0, temperature: float = 1.0):
        return bnn.token_logprobs(bnn.bmm(DecoderLayer._bits(x), self.w, self.width), targets, scale=self.width ** -0.5 / temperature, top=top)


def cut_back(cache, weights, table, lens, into, keep: int, first: int = 4, last: int = 64):
    """Evicts the lightest tokens of every sequence longer than `keep`: what stays moves into the pages of `into`.  Returns (lens, weights) of the sequences there; positions go on as before."""
    if into.shape[1] * cache.page < min(keep, table.shape[1] * cache.page):
        raise ValueError("into must have room for the tokens that are kept")
    tokens, lens = cache.heaviest(weights, table, lens, keep, first, last)
    return lens, cache.move(tokens, table, into, weights)


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--batch", type=int, default=8)
    parser.add_argument("--context", type=int, default=8192, help="tokens of every sequence before the timed steps")
    parser.add_argument("--steps", type=int, default=32)
    parser.add_argument("--keep", type=int, default=32, help="pages a query attends to in the second run")
    parser.add_argument("--budget", type=int, default=4096, help="tokens that sequences are cut back to in the third")
    args = parser.parse_args(argv)
    width, heads, kv_heads, head_dim, page = 4096, 32, 8, 128, 64
    layer = DecoderLayer(width, heads, kv_heads, head_dim, 4 * width)
    longest = args.context + 2 * (args.steps + 1)
    pages = -(-longest // page)
    table = torch.arange(args.batch * pages, dtype=torch.int32, device="cuda").view(args.batch, pages)
    cache = bnn.Cache4(args.batch * pages, kv_heads=kv_heads, head_dim=head_dim, page=page)
    lens = torch.zeros(args.batch, dtype=torch.int32, device="cuda")

    def prompts(layer, cache, lens, **kw):
        for first in range(0, args.context, 1024):                     # in chunks
            n = min(1024, args.context - first)
            lens += n
            layer.forward(torch.randn(args.batch * n, width, device="cuda"), cache, table, lens, **kw)

    def timed(one_step, what):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for step in range(args.steps + 1):
            if step == 1:                                              # the first loads the kernels
                begin.record()
            tokens = one_step()
        end.record()
        end.synchronize()
        print("%d sequences of %d tokens, attention to %s: %.1f us a step" % (args.batch, int(tokens[0]), what, begin.elapsed_time(end) * 1e3 / args.steps))

    prompts(layer, cache, lens)
    x = torch.randn(args.batch, width, device="cuda")
    for keep in (None, args.keep):
        def step():
            nonlocal x
            lens.add_(1)
            x = layer.forward(x, cache, table, lens, keep=keep)
            return lens
        timed(step, "the whole cache" if keep is None else "%d pages of %d tokens" % (keep, page))

    # With positions, and the weight that every token got from the prompts' attention on; then cut back to the budget, into other pages.
    layer = DecoderLayer(width, heads, kv_heads, head_dim, 4 * width, rotary_base=10000.0)
    fewer = -(-(args.budget + args.steps + 1) // page)
    cache = bnn.Cache4(args.batch * (pages + fewer), kv_heads=kv_heads, head_dim=head_dim, page=page)
    into = torch.arange(args.batch * pages, args.batch * (pages + fewer), dtype=torch.int32, device="cuda").view(args.batch, fewer)
    weights = torch.zeros(args.batch, kv_heads, pages * page, device="cuda")
    lens.zero_()
    prompts(layer, cache, lens, weights=weights)
    positions = lens.clone()
    lens, weights = cut_back(cache, weights, table, lens, into, args.budget)

    def step():
        nonlocal x
        lens.add_(1)
        x = layer.forward(x, cache, into, lens, positions=positions, weights=weights)
        positions.add_(1)
        return lens
    timed(step, "what is left of %d, with positions and weights added up" % args.context)
    said = Head(width, 32768).forward(x, top=1)
    print("the likeliest next tokens: %s" % ", ".join("%d (%.2f)" % t for t in zip(said.top_tokens[:, 0].tolist(), said.top_logprobs[:, 0].tolist())))


if __name__ == "__main__":
    main()
