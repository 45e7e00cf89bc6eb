// Rotary positions: queries and keys, rotated by their tokens' positions; and the same on the way into the 4-bit cache.
//
// Pair p of a head, at position n, is turned by the angle n * frequency[p]: (a, b) -> (a cos - b sin, a sin + b cos).  A pair is two neighbours, or element p and element p + pairs;
// what lies behind the pairs is copied.  A workgroup has some tokens and some heads: their sines and cosines are computed once, a pair and token to a thread, and wait in LDS.
// What bounds it is memory; the 64-bit arithmetic (two instructions an element, and conversions) hides behind it: 16384 tokens of 40 heads of 128 bf16 elements, 70 us, 4.8 TB/s.
#include "bnn_rotary.h"

namespace bnn {
namespace {

template <class T, int V, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void rotary_kernel(const T* x, T* out, int tokens, int heads, long long x_token, long long x_head, long long out_token,
                                                     long long out_head, Rotation rot, int tile, int block_heads, int items, FastDiv div_items, FastDiv div_heads, FastDiv div_pairs) {
    __shared__ double2 turns[ROTARY_TURNS];
    const int t0 = (int)blockIdx.x * tile, have = min(tile, tokens - t0);
    const int h0 = (int)blockIdx.y * block_heads, some = min(block_heads, heads - h0);
    for (int i = (int)threadIdx.x; i < have * rot.pairs; i += 256) {
        const int t = fast_div(i, div_pairs);
        turns[i] = turn_of((double)rot.positions[t0 + t] * rot.frequencies[i - t * rot.pairs], rot.magnitude, rot.sign);
    }
    __syncthreads();
    for (int i = (int)threadIdx.x; i < have * block_heads * items; i += 256) {
        const int rest = fast_div(i, div_items), t = fast_div(rest, div_heads), h = rest - t * block_heads;
        if (h >= some) continue;
        rotate_item<V, NEIGHBOURS>(x + (t0 + t) * x_token + (h0 + h) * x_head, out + (t0 + t) * out_token + (h0 + h) * out_head, i - rest * items, rot.pairs,
                                   turns + t * rot.pairs);
    }
}

// Eight consecutive elements of a key from `at` on, rotated.  V < 8: pairs lie anywhere.
template <int V, bool NEIGHBOURS, class T>
__device__ __forceinline__ void rotated8(const T* x, int at, int pairs, const double2* turns, float (&y)[8]) {
    c4_load8(x + at, y);
    if (at >= 2 * pairs) return;
    if constexpr (V == 8 && NEIGHBOURS) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const double2 t = turns[at / 2 + i];
            const float a = y[2 * i], b = y[2 * i + 1];
            y[2 * i] = turned(a, b, t.x, t.y);
            y[2 * i + 1] = turned(b, a, t.x, -t.y);
        }
    } else if constexpr (V == 8) {
        const bool first = at < pairs;
        float other[8];
        c4_load8(x + (first ? at + pairs : at - pairs), other);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const double2 t = turns[first ? at + i : at - pairs + i];
            y[i] = turned(y[i], other[i], t.x, first ? t.y : -t.y);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int e = at + i;
            if (e >= 2 * pairs) continue;
            const bool first = NEIGHBOURS ? e % 2 == 0 : e < pairs;
            const double2 t = turns[NEIGHBOURS ? e / 2 : first ? e : e - pairs];
            const float other = (float)x[NEIGHBOURS ? e ^ 1 : first ? e + pairs : e - pairs];
            y[i] = turned(y[i], other, t.x, first ? t.y : -t.y);
        }
    }
}

// Heads of a workgroup: those of q, then the kv heads, a key and its value together.
template <class T, int V, bool NEIGHBOURS>
__global__ __launch_bounds__(256) void write_rotary_kernel(WriteRotary4 a, int tile, int block_heads, int items, FastDiv div_items, FastDiv div_heads, FastDiv div_pairs,
                                                           FastDiv div_lanes, FastDiv div_tile) {
    __shared__ double2 turns[ROTARY_TURNS];
    __shared__ int place[16][3];             // of a token: position, whether it is a row of a sequence, page
    const int t0 = (int)blockIdx.x * tile, have = min(tile, a.r.tokens - t0);
    const int all = a.heads + a.c.kv_heads, h0 = (int)blockIdx.y * block_heads, h1 = min(h0 + block_heads, all);
    if ((int)threadIdx.x < have) {
        const int t = t0 + (int)threadIdx.x;
        const int b = c4_sequence_of(a.r, t);
        const Sequence4 s = c4_sequence(a.r, b);
        const int i = t - s.first, token = s.length - s.rows + i;
        const bool row = i >= 0 && i < s.rows;
        place[threadIdx.x][0] = token;
        place[threadIdx.x][1] = row;
        place[threadIdx.x][2] = row ? c4_page(a.r, a.c, b, token) : -1;
    }
    __syncthreads();
    for (int i = (int)threadIdx.x; i < have * a.rot.pairs; i += 256) {
        const int t = fast_div(i, div_pairs);
        const int n = a.rot.positions ? a.rot.positions[t0 + t] : place[t][0];
        turns[i] = turn_of((double)n * a.rot.frequencies[i - t * a.rot.pairs], a.rot.magnitude, a.rot.sign);
    }
    __syncthreads();
    const int q1 = min(h1, a.heads), qs = max(q1 - h0, 0);           // heads of q here
    for (int i = (int)threadIdx.x; i < have * block_heads * items && qs > 0; i += 256) {
        const int rest = fast_div(i, div_items), t = fast_div(rest, div_heads), h = rest - t * block_heads;
        if (h >= qs || !place[t][1]) continue;
        rotate_item<V, NEIGHBOURS>(static_cast<const T*>(a.q) + (t0 + t) * a.q_token + (h0 + h) * a.q_head,
                                   static_cast<T*>(a.q_out) + ((long long)(t0 + t) * a.heads + h0 + h) * a.c.dim, i - rest * items, a.rot.pairs, turns + t * a.rot.pairs);
    }
    const int lanes = a.c.dim / 8, k0 = max(h0 - a.heads, 0), ks = max(h1 - a.heads, 0) - k0;
    // tokens before heads: bytes of scales of neighbouring tokens lie side by side
    for (int i = (int)threadIdx.x; i < tile * ks * lanes; i += 256) {
        const int rest = fast_div(i, div_lanes), at = i - rest * lanes;
        const int h = fast_div(rest, div_tile), t = rest - h * tile, head = k0 + h;
        if (t >= have || place[t][2] < 0) continue;                  // whole groups of four lanes
        float x[8], y[8];
        rotated8<V, NEIGHBOURS>(static_cast<const T*>(a.k) + (t0 + t) * a.k_token + head * a.k_head, at * 8, a.rot.pairs, turns + t * a.rot.pairs, x);
        c4_load8(static_cast<const T*>(a.v) + (t0 + t) * a.v_token + head * a.v_head + at * 8, y);
        c4_put(a.c, c4_record(a.c, place[t][2], head), place[t][0] & (a.c.page - 1), at, x, y);
    }
}

// How a call is cut up.  Tokens of a workgroup: up to 16, where there are tokens enough to fill the chip; its heads: all, but where workgroups are few only as many
// as give each thread an item.  An item: what a thread moves at once, `items` to a head.
struct Cut {
    int tile, heads;
    dim3 grid;
};
Cut cut(int tokens, int heads, int pairs, int items) {
    Cut c;
    c.tile = std::min(16, ROTARY_TURNS / pairs);
    while (c.tile > 1 && cdiv(tokens, c.tile) < 512) c.tile /= 2;
    c.heads = heads;
    if (cdiv(tokens, c.tile) < 1024) c.heads = (int)std::min<long long>(heads, cdiv(256, (long long)items * c.tile));
    c.heads = std::min(c.heads, std::max(1, 65536 / items));
    c.grid = dim3((unsigned)cdiv(tokens, c.tile), (unsigned)cdiv(heads, c.heads));
    return c;
}

}  // namespace

int launch_rotary(const void* x, void* out, int dtype, int tokens, int heads, int dim, long long x_token, long long x_head, long long out_token, long long out_head, int width,
                  const Rotation& rot, int neighbours, hipStream_t s) {
    const int items = rot.pairs / width + (dim - 2 * rot.pairs) / width;
    const Cut c = cut(tokens, heads, rot.pairs, items);
    if (c.grid.y > 65535 || c.grid.x >= C4_THREADS / 256) return BNN_ERR_UNSUPPORTED;
    auto go = [&](auto type, auto v, auto nb) {
        using T = decltype(type);
        launch(rotary_kernel<T, decltype(v)::value, decltype(nb)::value>, c.grid, dim3(256), 0, s, static_cast<const T*>(x), static_cast<T*>(out), tokens, heads, x_token, x_head,
               out_token, out_head, rot, c.tile, c.heads, items, make_fastdiv((uint32_t)items), make_fastdiv((uint32_t)c.heads),
               make_fastdiv((uint32_t)rot.pairs));
    };
    auto types = [&](auto v, auto nb) {
        if (dtype == BNN_BF16) go(__bf16{}, v, nb);
        else if (dtype == BNN_F16) go(_Float16{}, v, nb);
        else go(float{}, v, nb);
    };
    auto widths = [&](auto nb) {
        if (width == 8) types(std::integral_constant<int, 8>{}, nb);
        else if (width == 4) types(std::integral_constant<int, 4>{}, nb);
        else if (width == 2) types(std::integral_constant<int, 2>{}, nb);
        else types(std::integral_constant<int, 1>{}, nb);
    };
    if (neighbours) widths(std::true_type{});
    else widths(std::false_type{});
    return check_launch();
}

int launch_cache4_write_rotary(const WriteRotary4& a, int dtype, int neighbours, int width, hipStream_t s) {
    const int items = a.rot.pairs / width + (a.c.dim - 2 * a.rot.pairs) / width, lanes = a.c.dim / 8;
    const Cut c = cut(a.r.tokens, a.heads + a.c.kv_heads, a.rot.pairs, std::max(items, lanes));
    if (c.grid.y > 65535 || c.grid.x >= C4_THREADS / 256) return BNN_ERR_UNSUPPORTED;
    auto go = [&](auto type, auto v, auto nb) {
        using T = decltype(type);
        launch(write_rotary_kernel<T, decltype(v)::value, decltype(nb)::value>, c.grid, dim3(256), 0, s, a, c.tile, c.heads, items, make_fastdiv((uint32_t)items),
               make_fastdiv((uint32_t)c.heads), make_fastdiv((uint32_t)a.rot.pairs), make_fastdiv((uint32_t)lanes), make_fastdiv((uint32_t)c.tile));
    };
    auto types = [&](auto v, auto nb) {
        if (dtype == BNN_BF16) go(__bf16{}, v, nb);
        else if (dtype == BNN_F16) go(_Float16{}, v, nb);
        else go(float{}, v, nb);
    };
    auto widths = [&](auto nb) {
        if (width == 8) types(std::integral_constant<int, 8>{}, nb);
        else if (width == 4) types(std::integral_constant<int, 4>{}, nb);
        else if (width == 2) types(std::integral_constant<int, 2>{}, nb);
        else types(std::integral_constant<int, 1>{}, nb);
    };
    if (neighbours) widths(std::true_type{});
    else widths(std::false_type{});
    return check_launch();
}

}  // namespace bnn
