"""A decoder layer of a binarized language model on this library: products of signs around attention over the 4-bit cache.

    python -m paper_2006_16578_amd.decoder [--context 8192] [--steps 32] [--keep 32]

Every projection multiplies the signs of its input with packed +1/-1 weights (``sign_pack_f32``, ``bmm``), the hidden layer of the feed-forward part goes from bits to
bits (``bmm_thr``).  Signs do not depend on the length of a vector, so there is no norm to compute in front of them.  Keys and values go into a ``Cache4``;
queries attend to all of it or, with ``keep``, to the pages that ``Cache4.select`` chooses.  Weights are random: the module shows the calls.
"""
from __future__ import annotations

import argparse

import torch

from . import binding as bnn


class DecoderLayer:
    """x [tokens][width] fp32 -> the same.  Weights are +1/-1, drawn from `seed`."""

    def __init__(self, width: int, heads: int, kv_heads: int, head_dim: int, hidden: int, seed: int = 0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        weights = lambda rows, cols: bnn.sign_pack_f32(torch.randn(rows, cols, device=device, generator=gen), bnn.round_up(bnn.nwords(cols), 4))
        self.width, self.heads, self.kv_heads, self.head_dim, self.hidden = width, heads, kv_heads, head_dim, hidden
        self.w_qkv = weights((heads + 2 * kv_heads) * head_dim, width)
        self.w_out = weights(width, heads * head_dim)
        self.w_up, self.w_down = weights(hidden, width), weights(width, hidden)
        self.thresholds = torch.randint(-32, 33, (hidden,), dtype=torch.int32, device=device, generator=gen)

    @staticmethod
    def _bits(x):
        return bnn.sign_pack_f32(x.contiguous(), bnn.round_up(bnn.nwords(x.shape[1]), 4))

    def _project(self, bits, weights, inputs: int):
        """Products of signs, brought back to unit variance."""
        return bnn.bmm(bits, weights, inputs).float() * inputs ** -0.5

    def attention(self, x, cache, table, lens, start=None, keep: int | None = None):
        """The attention part before its output projection, [tokens][heads][head_dim] fp32; the new keys and values go into the cache."""
        tokens = x.shape[0]
        qkv = self._project(self._bits(x), self.w_qkv, self.width).view(tokens, self.heads + 2 * self.kv_heads, self.head_dim)
        q, k, v = qkv.split((self.heads, self.kv_heads, self.kv_heads), dim=1)
        cache.write(k, v, table, lens, start)
        blocks = None if keep is None else cache.select(q, table, lens, keep, start)
        return cache.attend(q, table, lens, start, blocks=blocks)

    def forward(self, x, cache, table, lens, start=None, keep: int | None = None):
        o = self.attention(x, cache, table, lens, start, keep).flatten(1)
        x = x + self._project(self._bits(o), self.w_out, self.heads * self.head_dim)
        hidden = bnn.bmm_thr(self._bits(x), self.w_up, self.thresholds, self.width)
        return x + self._project(hidden, self.w_down, self.hidden)


def main(argv=None):
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--batch", type=int, default=8)
    parser.add_argument("--context", type=int, default=8192, help="tokens of every sequence before the timed steps")
    parser.add_argument("--steps", type=int, default=32)
    parser.add_argument("--keep", type=int, default=32, help="pages a query attends to in the second run")
    args = parser.parse_args(argv)
    width, heads, kv_heads, head_dim, page = 4096, 32, 8, 128, 64
    layer = DecoderLayer(width, heads, kv_heads, head_dim, 4 * width)
    longest = args.context + 2 * (args.steps + 1)
    pages = -(-longest // page)
    table = torch.arange(args.batch * pages, dtype=torch.int32, device="cuda").view(args.batch, pages)
    cache = bnn.Cache4(args.batch * pages, kv_heads=kv_heads, head_dim=head_dim, page=page)
    lens = torch.zeros(args.batch, dtype=torch.int32, device="cuda")
    for first in range(0, args.context, 1024):                         # the prompts, in chunks
        n = min(1024, args.context - first)
        lens += n
        layer.forward(torch.randn(args.batch * n, width, device="cuda"), cache, table, lens)
    x = torch.randn(args.batch, width, device="cuda")
    for keep in (None, args.keep):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        for step in range(args.steps + 1):
            if step == 1:                                              # the first loads the kernels
                begin.record()
            lens += 1
            x = layer.forward(x, cache, table, lens, keep=keep)
        end.record()
        end.synchronize()
        what = "the whole cache" if keep is None else "%d pages of %d tokens" % (keep, page)
        print("%d sequences of %d tokens, attention to %s: %.1f us a step" % (args.batch, int(lens[0]), what, begin.elapsed_time(end) * 1e3 / args.steps))


if __name__ == "__main__":
    main()
