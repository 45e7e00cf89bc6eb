// Attention over the 4-bit cache; instantiated per head dimension in bnn_cache4_attend*.hip.  attend_kernel: single tokens, drafts, selected blocks (up to 32 rows of queries a
// workgroup, whose waves share the keys); attend_rows_kernel, further down: chunks and prompts (64 or 128 rows, whose waves share what is converted).
//
// Rows of queries that share a kv head -- its query heads, for one token or for several -- are the columns of the products, keys their rows:
//   S^T [keys][rows] = K Q^T,   O^T [dim][rows] += V^T P^T   (v_mfma_f32_16x16x32_bf16).
// A lane then holds, of 32 keys, the scores of ONE row at 8 keys, and exactly those eight are its operand of the second product: softmax weights never cross
// lanes.  Eight or four waves share the 16 * QT rows of a workgroup and take steps of 32 keys in turn, each with a running maximum and sum of its own; they meet in LDS once, at the end.
// What bounds it is memory: the next step's codes are under way while one is computed, and page addresses are read 32 steps ahead, a lane each.  Two documents of 100001 and
// 131072 tokens (8 kv heads of 128, 251 MB): 42 us, 5.9 TB/s; 64 conversations of 500 to 8192 tokens (304 MB): 58 us, 5.3 TB/s.  A step is about 195 vector instructions, half
// of them conversions, and 17 MFMAs of 16 cycles.
// The cache's values are exact in bf16: the conversion instruction applies the scale.
//
// K: lane l supplies key l % 16 of a step's half and, of every 128 elements, the 32 of group l / 16: one 16-byte load and one scale.  Which elements a matrix
// instruction contracts together does not matter as long as Q agrees.  V: its operand wants eight keys of one element in a lane, memory has the elements of
// a key side by side; lane l loads, for its eight keys, the elements 8 (l % 16) .. + 7, converts pairs and interleaves the halves of registers.
// Element 8 i + j is then row i of product j.  64 and 32 elements that are left over of a head dimension work alike with 4 and 2 elements.
//
// The reference point of the weights follows the maximum in steps: it is raised, to 8 (as powers of two) above the highest score, and the sums rescaled, only when a score
// passes it by more than 8, which a wave tests without any exchange between lanes; weights are at most 2^8 then, and nothing is lost, as weights and sums scale alike.
// A weight's exponent is one multiply-add of the score, exact up to its own rounding, while the reference point is rounded: from 2^26 on by enough for the weights of a
// row to overflow or to vanish together.  A wave that meets such a point multiplies its scores first from then on, which rounds them as it rounded the point.
//
// Weights of one bf16 term are divided by the sum of the rounded weights, a product with ones, so that where one key has nearly all the weight its rounding cancels
// (error against 64 bits 0.0016 of the result's size, 0.0015 from rounding the result; 0.0021 without); the logarithm of the sum is of the unrounded ones.
// Queries and weights enter the products as sums of 1 (bf16), 2 (fp16) or 3 (fp32) bf16 terms: queries exactly; weights to 8, 16 and 24 bits.
#ifndef BNN_CACHE4_ATTEND_H
#define BNN_CACHE4_ATTEND_H

#include "bnn_cache4.h"

namespace bnn {
namespace {

constexpr float C4_LOW = -3.0e38f;           // below every score: a row that has seen nothing
constexpr float C4_SLACK = 8.f;
constexpr float C4_FAR = 67108864.f;         // 2^26: fp32 numbers lie 8 apart from here on

template <int DTYPE> struct C4Type { using type = float; static constexpr int terms = 3; };
template <> struct C4Type<BNN_BF16> { using type = __bf16; static constexpr int terms = 1; };
template <> struct C4Type<BNN_F16> { using type = _Float16; static constexpr int terms = 2; };

// The largest over the four lanes of a row (lanes l, l + 16, l + 32, l + 48).
__device__ __forceinline__ float row_max(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ __forceinline__ float row_sum(float v) {
    auto a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(a[0]) + __uint_as_float(a[1]);
    auto b = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(b[0]) + __uint_as_float(b[1]);
}

// The largest of a lane's eight scores; NaN if there is one.  (fmaxf passes over NaN, for which every result of a matrix instruction takes an instruction more.)
__device__ __forceinline__ float max8(const f32x4& a, const f32x4& b) {
    const float v = __builtin_elementwise_maximum(__builtin_elementwise_maximum(a[0], a[1]), a[2]);
    const float w = __builtin_elementwise_maximum(__builtin_elementwise_maximum(v, a[3]), b[0]);
    return __builtin_elementwise_maximum(__builtin_elementwise_maximum(__builtin_elementwise_maximum(w, b[1]), b[2]), b[3]);
}

// The reference point of a row's weights, 2^(score - m): raised to C4_SLACK above the highest score when one has passed it by more than C4_SLACK.  Returns what sums are
// scaled by.
__device__ __forceinline__ float raise_maximum(float& m, float high) {
    const float to = high > m + C4_SLACK ? high + C4_SLACK : m;
    const float factor = __builtin_amdgcn_exp2f(m - to);
    m = to;
    return factor;
}

// Products that stay products: fused with the subtraction that follows they would not be rounded as the reference point is.
__device__ __forceinline__ float product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}
__device__ __forceinline__ void multiply(f32x4& score, float scale) {
#pragma unroll
    for (int i = 0; i < 4; ++i) score[i] = product(score[i], scale);
}
// Whether some row of the wave has a reference point (not that of a row that has seen nothing) beside which scores have to be multiplied before it is subtracted.
__device__ __forceinline__ bool any_far(float m) { return __ballot(fabsf(m) > C4_FAR && m > C4_LOW) != 0; }

__device__ __forceinline__ bf16x8 as_bf16x8(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    const u32x4 v = {a, b, c, d};
    return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ bf16x8 ones() { return as_bf16x8(0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u); }
__device__ __forceinline__ uint32_t pair_bits(bf16x2 v) { return __builtin_bit_cast(uint32_t, v); }

// x as a sum of TERMS bf16 numbers, the largest first.
template <int TERMS>
__device__ __forceinline__ void split_terms(float x, __bf16 (&t)[TERMS]) {
#pragma unroll
    for (int i = 0; i < TERMS; ++i) {
        t[i] = (__bf16)x;
        x -= (float)t[i];
    }
}

// The row tile of a workgroup: rows `row0 ..` of sequence b, counted over (token, head of the group), heads fastest.
struct Tile4 {
    int b, row0, rows;                       // rows of this tile, 0: nothing to do
    Sequence4 s;
};

// ROWS: rows of a tile.  Tiles never span sequences, and with blocks of their own (sparse) never tokens.
template <int ROWS, bool SPARSE>
__device__ __forceinline__ Tile4 find_tile(const Attend4& a, int tile) {
    Tile4 t = {};
    if constexpr (SPARSE) {
        const int per = (a.group + ROWS - 1) / ROWS, token = per == 1 ? tile : tile / per, part = tile - token * per;
        t.b = c4_sequence_of(a.r, token);
        t.s = c4_sequence(a.r, t.b);
        const int i = token - t.s.first;
        if (i < 0 || i >= t.s.rows) return t;
        t.row0 = i * a.group + part * ROWS;
        t.rows = min(ROWS, a.group - part * ROWS);
        return t;
    } else {
        int local;
        if (!c4_find_tile(a.r, a.group, ROWS, tile, a.seq_tiles, a.div_seq_tiles, t.b, local)) return t;
        t.s = c4_sequence(a.r, t.b);
        const int all = t.s.rows * a.group;
        t.row0 = local * ROWS;
        t.rows = max(0, min(ROWS, all - t.row0));
        if (a.causal) {                      // the rows with the most keys first: short ones fill the gaps at the end
            const int last = (all - 1) / ROWS - local;
            t.row0 = max(last, 0) * ROWS;
            t.rows = max(0, min(ROWS, all - t.row0));
            if (last < 0) t.rows = 0;
        }
        return t;
    }
}

// Steps of 32 keys that a tile visits.  Dense: step i covers keys 32 i .. + 31.  Sparse: halves of 16 keys of the listed blocks, in the list's order.
struct Range4 {
    int first, count;
};
template <bool SPARSE>
__device__ __forceinline__ Range4 tile_steps(const Attend4& a, const Tile4& t) {
    Range4 r = {0, 0};
    if (t.rows <= 0) return r;
    if constexpr (SPARSE) {
        r.count = (int)((((long long)a.keep << (a.c.page_shift - 4)) + 1) >> 1);
        return r;
    } else {
        const int base = t.s.length - t.s.rows;
        const int top = min(a.causal ? base + fast_div(t.row0 + t.rows - 1, a.div_group) + 1 : t.s.length, c4_room(a.r, a.c));      // keys below it are visited
        const int low = a.window > 0 ? max(0, max(base + fast_div(t.row0, a.div_group), 0) - a.window + 1) : 0;      // (rows before token 0 see nothing; any window may be theirs)
        if (top <= low) return r;
        r.first = low >> 5;
        r.count = ((top - 1) >> 5) + 1 - r.first;
        return r;
    }
}

// Eight values of K for one matrix instruction from a dword of codes.
__device__ __forceinline__ bf16x8 eight_of(uint32_t codes, float scale) {
    return as_bf16x8(pair_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)), pair_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
                     pair_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)), pair_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3)));
}

// How a head dimension is cut up: pieces of 128, then 64, then 32 elements.
template <int D>
struct Pieces {
    static constexpr int n128 = D / 128, n64 = D % 128 / 64, n32 = D % 64 / 32;
    static constexpr int count = n128 + n64 + n32;
    static constexpr int width(int p) { return p < n128 ? 128 : p < n128 + n64 ? 64 : 32; }
    static constexpr int base(int p) { return p < n128 ? 128 * p : p < n128 + n64 ? 128 * n128 : 128 * n128 + 64 * n64; }
};

// Memory of the cache by an address that lanes hold and hand over as two 32-bit halves.
typedef const uint8_t __attribute__((address_space(1))) * Global4;
template <class T>
__device__ __forceinline__ T load_at(Global4 base, uint32_t offset) {
    return *reinterpret_cast<const T __attribute__((address_space(1))) *>(base + offset);
}

// Where the 16 keys of half a step lie, all in one page.  Uniform over a wave.
struct Half4 {
    Global4 record;
    int offset;                              // of the first key in the page
    int key;                                 // its number in the sequence
    bool there;
};

// What a lane holds of a step's codes and scales between the loads and the products.
template <int D>
struct Raw4 {
    using P = Pieces<D>;
    uint32_t k[2][D / 32];
    uint32_t k_exp[2][P::count];
    uint32_t v[P::count][8];
    uint32_t v_exp[P::count][2];
};

// (Scalar: the record; a lane's offset in it is one addition to a number that no step changes.  Exponents come four keys at a time, and k_scale() takes the lane's: a byte loaded
// alone is widened where it arrives, not where it is used, and that waits for the next step's loads within this one.)
template <int D>
__device__ __forceinline__ void load_k_half(const Cache4& c, const Half4& half, int lane, uint32_t (&codes)[D / 32], uint32_t (&exp)[Pieces<D>::count]) {
    using P = Pieces<D>;
    const uint32_t col = lane & 15, h4 = lane >> 4;
    const uint32_t row = col * (D / 2) + (uint32_t)half.offset * (D / 2);
    static_for<P::count>([&](auto pc) {
        constexpr int p = pc.value, W = P::width(p), B = P::base(p);
        if constexpr (W == 128) {
            const u32x4 v = load_at<u32x4>(half.record, row + 16 * h4 + B / 2);
#pragma unroll
            for (int i = 0; i < 4; ++i) codes[B / 32 + i] = v[i];
        } else if constexpr (W == 64) {
            const u32x2 v = load_at<u32x2>(half.record, row + 8 * h4 + B / 2);
            codes[B / 32] = v[0];
            codes[B / 32 + 1] = v[1];
        } else {
            codes[B / 32] = load_at<uint32_t>(half.record, row + 4 * h4 + B / 2);
        }
        exp[p] = load_at<uint32_t>(half.record, (uint32_t)c.k_exps + (B / 32 + h4 * W / 128) * (uint32_t)c.page + (col & 12u) + (uint32_t)half.offset);
    });
}
__device__ __forceinline__ float k_scale(uint32_t exp, int lane) {
    return __uint_as_float(__builtin_amdgcn_perm(exp, exp, (uint32_t)(lane & 3) << 24 | 0x0c0c0cu) >> 1);
}
// codes[p][0..3] and exp[p]: of the keys 4 (lane / 16) .. + 3 of the half.
template <int D, int N>
__device__ __forceinline__ void load_v_half(const Cache4& c, const Half4& half, int lane, uint32_t (&codes)[Pieces<D>::count][N], uint32_t (&exp)[Pieces<D>::count][N / 4],
                                            int s) {
    using P = Pieces<D>;
    const uint32_t col = lane & 15, h4 = lane >> 4;
    static_for<P::count>([&](auto pc) {
        constexpr int p = pc.value, W = P::width(p), B = P::base(p), E = W / 16;           // E elements of each of 4 keys
        const uint32_t from = (uint32_t)c.v_codes + 4 * h4 * (D / 2) + B / 2 + E / 2 * col + (uint32_t)half.offset * (D / 2);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (E == 8) codes[p][4 * s + i] = load_at<uint32_t>(half.record, from + i * (D / 2));
            else if constexpr (E == 4) codes[p][4 * s + i] = load_at<uint16_t>(half.record, from + i * (D / 2));
            else codes[p][4 * s + i] = load_at<uint8_t>(half.record, from + i * (D / 2));
        }
        exp[p][s] = load_at<uint32_t>(half.record, (uint32_t)c.v_exps + (B / 32 + col * E / 32) * (uint32_t)c.page + 4 * h4 + (uint32_t)half.offset);
    });
}
__device__ __forceinline__ Global4 record_of(uint32_t low, uint32_t high, int lane) {
    return reinterpret_cast<Global4>((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)high, lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)low, lane));
}

template <int D>
__device__ __forceinline__ void load_k(const Cache4& c, const Half4 (&half)[2], int lane, Raw4<D>& raw) {
#pragma unroll
    for (int s = 0; s < 2; ++s) load_k_half<D>(c, half[s], lane, raw.k[s], raw.k_exp[s]);
}
template <int D>
__device__ __forceinline__ void load_v(const Cache4& c, const Half4 (&half)[2], int lane, Raw4<D>& raw) {
#pragma unroll
    for (int s = 0; s < 2; ++s) load_v_half<D, 8>(c, half[s], lane, raw.v, raw.v_exp, s);
}

// Q of the lane's row, in the order of elements that K's loads give, as a sum of TERMS bf16 numbers; zero without a row.  An infinite element becomes NaN (a sum of several
// terms makes it one by itself): its products are infinite or NaN for every key, so no weights are defined, also where all scores are -infinity, the mark of keys not seen.
template <int D, int TERMS, class T>
__device__ __forceinline__ void load_q(const T* src, bool valid, int lane, bf16x8 (&q)[TERMS][D / 32]) {
    using P = Pieces<D>;
    static_for<P::count>([&](auto pc) {
        constexpr int p = pc.value, W = P::width(p), B = P::base(p);
#pragma unroll
        for (int i = 0; i < W / 32; ++i) {
            float x[8] = {};
            if (valid) c4_load8(src + B + W / 4 * (lane >> 4) + 8 * i, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                __bf16 terms[TERMS];
                split_terms<TERMS>(TERMS == 1 ? fmaf(x[e], 0.f, x[e]) : x[e], terms);
#pragma unroll
                for (int n = 0; n < TERMS; ++n) q[n][B / 32 + i][e] = terms[n];
            }
        }
    });
}

template <int D, int DTYPE, int QT, bool SPARSE>
__global__ __launch_bounds__(64 * cache4_waves(D, DTYPE, QT), D == 256 && DTYPE == BNN_F32 ? 1 : 2) void attend_kernel(Attend4 a) {
    using T = typename C4Type<DTYPE>::type;
    constexpr int TERMS = C4Type<DTYPE>::terms;
    constexpr int ROWS = 16 * QT, M = D / 32, J = D / 16, WAVES = cache4_waves(D, DTYPE, QT);
    constexpr int LD = D + 4;                // floats of a row in LDS: rows of the 16 lanes fall on different banks
    using P = Pieces<D>;
    __shared__ __align__(16) float sums[WAVES][16][LD];
    __shared__ float stats[WAVES][ROWS][3];  // reference point, sum of the weights, sum of the rounded weights

    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, h4 = lane >> 4;
    // heads fastest: workgroups go to the eight dies in turn, so with eight kv heads (or a divisor) those that share keys share a die's cache
    int unit = (int)blockIdx.x;
    const int rest = fast_div(unit, a.div_heads), head = unit - rest * a.c.kv_heads;
    const int tile = fast_div(rest, a.div_splits), split = rest - tile * a.splits;
    const Tile4 t = find_tile<ROWS, SPARSE>(a, tile);
    if (t.rows <= 0) return;
    const Range4 range = tile_steps<SPARSE>(a, t);
    const int begin = split * a.chunk, end = min(range.count, begin + a.chunk);
    if (split > 0 && begin >= end) return;
    const bool whole = range.count <= a.chunk;

    const int base = t.s.length - t.s.rows;
    const int32_t* list = SPARSE ? a.blocks + ((long long)(t.s.first + fast_div(t.row0, a.div_group)) * a.c.kv_heads + head) * a.keep : nullptr;
    const int per_shift = a.c.page_shift - 4;                        // halves of steps in a page
    // Where the halves of this wave's next 32 steps lie, a lane each: the record's address, the first key's number (sparse), whether there is a page.
    const int turns = (end - begin - wave + WAVES - 1) / WAVES;                  // steps of this wave
    uint32_t low = 0, high = 0;
    int keys = 0;
    unsigned long long present = 0;
    auto locate = [&](int turn) {                                    // turn: a multiple of 32
        const int i = 2 * (range.first + begin + wave + WAVES * (turn + (lane >> 1))) + (lane & 1);
        bool listed = true;
        if constexpr (SPARSE) {
            const int entry = i >> per_shift;
            const int block = list[min(entry, a.keep - 1)];
            listed = entry < a.keep && block >= 0 && block < a.r.table_pages;
            keys = listed ? (block << a.c.page_shift) + 16 * (i & ((1 << per_shift) - 1)) : 0;
        } else {
            keys = 16 * min(i, 2 * (range.first + range.count) - 1);
        }
        const int page = c4_page(a.r, a.c, t.b, keys);
        present = __ballot(listed && page >= 0);
        const uint64_t at = (uint64_t)(uintptr_t)c4_record(a.c, max(page, 0), head);
        low = (uint32_t)at;
        high = (uint32_t)(at >> 32);
    };
    auto fetch = [&](int turn, Half4 (&half)[2]) {
        if (turn % 32 == 0) locate(turn);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int at = 2 * (turn % 32) + s;
            half[s].record = record_of(low, high, at);
            half[s].key = SPARSE ? __builtin_amdgcn_readlane(keys, at) : 32 * (range.first + begin + wave + WAVES * turn) + 16 * s;
            half[s].offset = half[s].key & (a.c.page - 1);
            half[s].there = present >> at & 1;
        }
    };

    Half4 now[2], next[2];
    Raw4<D> raw;
    if (turns > 0) {
        fetch(0, now);
        load_k<D>(a.c, now, lane, raw);
        load_v<D>(a.c, now, lane, raw);
        next[0] = now[0];
        next[1] = now[1];
    }

    // Q, in the order of elements that K's loads give
    bf16x8 q[QT][TERMS][M];
    int pos[QT];                             // position of the lane's row; -1: no row, or one before the first token
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        const int row = t.row0 + 16 * u + c;
        const int token = fast_div(row, a.div_group), g = row - token * a.group;
        const bool valid = 16 * u + c < t.rows;
        pos[u] = valid ? max(base + token, -1) : -1;
        load_q<D, TERMS>(static_cast<const T*>(a.q) + (t.s.first + token) * a.q_token + (long long)(head * a.group + g) * a.q_head, valid, lane, q[u]);
    }

    f32x4 o[QT][J], rounded[QT];
    float m[QT], l[QT];
    bool far = false;                        // scores are multiplied by the scale first, and `times` is 1
    float times = a.scale;
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        m[u] = C4_LOW;
        l[u] = 0.f;
        rounded[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < J; ++j) o[u][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // keys that every row of the tile sees, if none is missing: [low_last, top_first]
    const int top_first = a.causal ? base + fast_div(t.row0, a.div_group) : t.s.length - 1;
    const int low_last = a.window > 0 ? max(base + fast_div(t.row0 + t.rows - 1, a.div_group), 0) - a.window + 1 : 0;

    for (int turn = 0; turn < turns; ++turn) {
        bool full = true;
#pragma unroll
        for (int s = 0; s < 2; ++s) full = full && now[s].there && now[s].key + 15 <= top_first && now[s].key >= low_last;

        // K and the scores
        f32x4 score[QT][2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int u = 0; u < QT; ++u) score[u][s] = f32x4{0.f, 0.f, 0.f, 0.f};
            static_for<P::count>([&](auto pc) {
                constexpr int p = pc.value, W = P::width(p), B = P::base(p);
                const float scale = k_scale(raw.k_exp[s][p], lane);
#pragma unroll
                for (int i = 0; i < W / 32; ++i) {
                    const bf16x8 k = eight_of(raw.k[s][B / 32 + i], scale);
#pragma unroll
                    for (int u = 0; u < QT; ++u)
#pragma unroll
                        for (int n = 0; n < TERMS; ++n) score[u][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[u][n][B / 32 + i], score[u][s], 0, 0, 0);
                }
            });
        }
        // the next step's K into the same registers (the last step's once more at the end)
        if (turn + 1 < turns) fetch(turn + 1, next);
        load_k<D>(a.c, next, lane, raw);

        if (!full) {
#pragma unroll
            for (int u = 0; u < QT; ++u) {
                const int top = a.causal ? pos[u] : t.s.length - 1, low = a.window > 0 ? pos[u] - a.window + 1 : 0;
#pragma unroll
                for (int s = 0; s < 2; ++s)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int key = now[s].key + 4 * h4 + i;
                        if (!(now[s].there && key <= top && key >= low)) score[u][s][i] = -__builtin_inff();
                    }
            }
        }

        if (far) {
#pragma unroll
            for (int u = 0; u < QT; ++u)
#pragma unroll
                for (int s = 0; s < 2; ++s) multiply(score[u][s], a.scale);
        }

        // weights
        bf16x8 w[QT][TERMS];
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            const float high = max8(score[u][0], score[u][1]);
            if (__ballot(high * times > m[u] + C4_SLACK) != 0) {
                const float factor = raise_maximum(m[u], product(row_max(high), times));
                l[u] *= factor;
                rounded[u] *= factor;
#pragma unroll
                for (int j = 0; j < J; ++j) o[u][j] *= factor;
                if (!far && any_far(m[u])) {
                    far = true;
                    times = 1.f;
#pragma unroll
                    for (int v = u; v < QT; ++v)
#pragma unroll
                        for (int s = 0; s < 2; ++s) multiply(score[v][s], a.scale);
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = __builtin_amdgcn_exp2f(fmaf(score[u][i >> 2][i & 3], times, -m[u]));
                l[u] += x;
                __bf16 terms[TERMS];
                split_terms<TERMS>(x, terms);
#pragma unroll
                for (int n = 0; n < TERMS; ++n) w[u][n][i] = terms[n];
            }
            if constexpr (TERMS == 1) rounded[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones(), w[u][0], rounded[u], 0, 0, 0);
        }

        // V
        static_for<P::count>([&](auto pc) {
            constexpr int p = pc.value, W = P::width(p), B = P::base(p), E = W / 16;       // E elements of each of 8 keys
            float scale[8];
            uint32_t bad = 0;                // keys with a NaN group
            if (!full) {
                // Where a mask is at work, a NaN must reach the rows that see its key and no other: its values are taken as finite here, and every row
                // counts the NaN groups among the keys that it sees.
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if ((raw.v_exp[p][i >> 2] >> 8 * (i & 3) & 255u) > C4_EXP_MAX) {
                        bad |= 1u << i;
                        raw.v_exp[p][i >> 2] &= ~(255u << 8 * (i & 3));
                    }
                if (__ballot(bad != 0) != 0) {
                    bf16x8 marks;
#pragma unroll
                    for (int i = 0; i < 8; ++i) marks[i] = (bad >> i & 1u) ? (__bf16)1.f : (__bf16)0.f;
#pragma unroll
                    for (int u = 0; u < QT; ++u) {
                        bf16x8 seen;
#pragma unroll
                        for (int i = 0; i < 8; ++i) seen[i] = score[u][i >> 2][i & 3] == -__builtin_inff() ? (__bf16)0.f : (__bf16)1.f;
                        const f32x4 count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(marks, seen, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                        for (int j = 0; j < E; ++j)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (count[i] > 0.f) o[u][B / 16 + j][i] = __builtin_nanf("");
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) scale[i] = c4_scale(raw.v_exp[p][i >> 2] >> 8 * (i & 3) & 255u);
            static_for<E / 2>([&](auto ec) {
                constexpr int e = ec.value;
                uint32_t v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = pair_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw.v[p][i], scale[i], e));
                const bf16x8 even = as_bf16x8(__builtin_amdgcn_perm(v[1], v[0], 0x05040100u), __builtin_amdgcn_perm(v[3], v[2], 0x05040100u),
                                              __builtin_amdgcn_perm(v[5], v[4], 0x05040100u), __builtin_amdgcn_perm(v[7], v[6], 0x05040100u));
                const bf16x8 odd = as_bf16x8(__builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u),
                                             __builtin_amdgcn_perm(v[5], v[4], 0x07060302u), __builtin_amdgcn_perm(v[7], v[6], 0x07060302u));
#pragma unroll
                for (int u = 0; u < QT; ++u)
#pragma unroll
                    for (int n = 0; n < TERMS; ++n) {
                        o[u][B / 16 + 2 * e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(even, w[u][n], o[u][B / 16 + 2 * e], 0, 0, 0);
                        o[u][B / 16 + 2 * e + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(odd, w[u][n], o[u][B / 16 + 2 * e + 1], 0, 0, 0);
                    }
            });
        });
        load_v<D>(a.c, next, lane, raw);
#pragma unroll
        for (int s = 0; s < 2; ++s) now[s] = next[s];
    }

    // The waves meet: 16 rows at a time.
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        const float sum = row_sum(l[u]);
        if (h4 == 0) {
            stats[wave][16 * u + c][0] = m[u];
            stats[wave][16 * u + c][1] = sum;
            stats[wave][16 * u + c][2] = TERMS == 1 ? rounded[u][0] : sum;
        }
    }
    const long long slot = ((long long)tile * a.c.kv_heads + head) * a.splits + split;
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        if (16 * u >= t.rows) break;
        if (u > 0) __syncthreads();
        static_for<P::count>([&](auto pc) {
            constexpr int p = pc.value, W = P::width(p), B = P::base(p), E = W / 16;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < E; ++j) sums[wave][c][B + E * (4 * h4 + i) + j] = o[u][B / 16 + j][i];
        });
        __syncthreads();
        for (int x = (int)threadIdx.x; x < 16 * (D / 8); x += 64 * WAVES) {
            const int row = x / (D / 8), d = x % (D / 8) * 8, r = 16 * u + row;
            if (r >= t.rows) continue;
            float high = C4_LOW, total = 0.f, divisor = 0.f, y[8] = {};
#pragma unroll
            for (int v = 0; v < WAVES; ++v) high = fmaxf(high, stats[v][r][0]);
#pragma unroll
            for (int v = 0; v < WAVES; ++v) {
                const float f = __builtin_amdgcn_exp2f(stats[v][r][0] - high);
                total = fmaf(stats[v][r][1], f, total);
                divisor = fmaf(stats[v][r][2], f, divisor);
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = fmaf(sums[v][row][d + e], f, y[e]);
            }
            if (whole) {
                const int token = fast_div(t.row0 + r, a.div_group), g = t.row0 + r - token * a.group;
                const long long at = ((long long)(t.s.first + token) * a.c.kv_heads + head) * a.group + g;
                const float f = 1.f / divisor;
#pragma unroll
                for (int e = 0; e < 8; ++e) y[e] = divisor == 0.f ? 0.f : y[e] * f;
                c4_store8(static_cast<T*>(a.out) + at * D + d, y);
                if (a.lse != nullptr && d == 0) a.lse[at] = total == 0.f ? -__builtin_inff() : (high + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
            } else {
                c4_store8(a.part + (slot * ROWS + r) * D + d, y);
                if (d == 0) a.part_sums[slot * ROWS + r] = f32x4{high, total, divisor, 0.f};
            }
        }
    }
}

// Many rows: a workgroup's four waves have 16 * QT rows each and share keys.  32 keys at a time are converted once for all and left in LDS as finished operands (a
// lane's 16 bytes side by side: reads and writes without conflicts): two waves have a half each of the keys, K two steps ahead of its use and V in turn; one barrier a step.
// In step i a wave forms the scores of step i + 1, the weights of step i and the sums of step i - 1: three pieces of work that do not wait for each other, so that matrix
// and vector instructions of one wave alternate.  A maximum that is raised in step i scales the sums at the step's end, when those of step i - 1 are in.
// Two prompts of 4096 tokens (32 heads of 128 on 8 kv heads, bf16): 336 to 350 us, 0.8 PFLOP/s; every wave converting for itself 416.  Bounded by what a SIMD issues: an MFMA
// takes 16.3 cycles of it, a plain vector instruction beside MFMAs 2.1, an exponential 5.5, a read of LDS 7 (each measured), so a step of 34, 109, 16 and 16 of them 1080 at least, 2160 for two waves, which take
// 2830.  More than two do not fit: 32 rows of sums, queries, scores and weights are 232 registers.  16 rows a wave at three or four waves a SIMD read twice the operands from LDS for a row: 424 us;
// eight waves to what is converted, 512 threads: 358.
template <int D, int DTYPE, int QT>
__global__ __launch_bounds__(256, 2) void attend_rows_kernel(Attend4 a) {
    using T = typename C4Type<DTYPE>::type;
    constexpr int TERMS = C4Type<DTYPE>::terms;
    constexpr int ROWS = 64 * QT, M = D / 32, J = D / 16;
    using P = Pieces<D>;
    __shared__ u32x4 k_ops[2][2][M][64];     // [step % 2][half][..]
    __shared__ u32x4 v_ops[2][J][64];
    __shared__ int nans[2][2];               // [step % 2][half]: values that are NaN and were taken as finite

    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, h4 = lane >> 4;
    const int rest = fast_div((int)blockIdx.x, a.div_heads), head = (int)blockIdx.x - rest * a.c.kv_heads;
    const int tile = fast_div(rest, a.div_splits), split = rest - tile * a.splits;
    const Tile4 t = find_tile<ROWS, false>(a, tile);
    if (t.rows <= 0) return;
    const Range4 range = tile_steps<false>(a, t);
    const int begin = split * a.chunk, end = min(range.count, begin + a.chunk);
    if (split > 0 && begin >= end) return;
    const bool whole = range.count <= a.chunk;
    const int steps = max(end - begin, 0), key_first = 32 * (range.first + begin);
    const int own = wave >> 1;               // the half of every step that this wave converts, K and V in turn with its neighbour

    // Where the halves of 32 steps lie, a lane each (2 * step + half); whole: all that are asked for are in pages.  K's turn is ahead of V's.
    struct Pages {
        uint32_t low, high;
        bool whole;
    };
    auto locate = [&](Pages& p, int step) {  // step: a multiple of 32
        const int page = c4_page(a.r, a.c, t.b, key_first + 32 * step + 16 * lane);
        p.whole = __ballot(page < 0 && step + lane / 2 < steps) == 0;
        const uint64_t at = (uint64_t)(uintptr_t)c4_record(a.c, max(page, 0), head);
        p.low = (uint32_t)at;
        p.high = (uint32_t)(at >> 32);
    };
    auto place = [&](const Pages& p, int step) {                     // of this wave's half
        const int at = 2 * (step % 32) + own;
        Half4 half;
        half.record = record_of(p.low, p.high, at);
        half.key = key_first + 32 * step + 16 * own;
        half.offset = half.key & (a.c.page - 1);
        half.there = true;
        return half;
    };

    const int base = t.s.length - t.s.rows;
    const int wave_rows = min(16 * QT, t.rows - 16 * QT * wave), wave_row0 = t.row0 + 16 * QT * wave;
    // Steps whose keys every row of some rows sees, [from, from + count), if all are in pages: of the workgroup's rows, and of this wave's
    struct Steps {
        int from;
        unsigned count;
        __device__ bool operator()(int step) const { return (unsigned)(step - from) < count; }
    };
    auto seen_by_all = [&](int row0, int rows) {
        const int first = base + fast_div(row0, a.div_group), last = base + fast_div(row0 + max(rows, 1) - 1, a.div_group);
        const int top = a.causal ? first : t.s.length - 1, bottom = a.window > 0 ? max(max(last, 0) - a.window + 1, 0) : 0;
        Steps r;
        r.from = max((bottom - key_first + 31) >> 5, 0);
        r.count = (unsigned)max(((top + 1 - key_first) >> 5) - r.from, 0);
        return r;
    };
    const Steps clear = seen_by_all(t.row0, t.rows), wave_clear = seen_by_all(wave_row0, wave_rows);

    uint32_t k_codes[M], k_exp[P::count], v_codes[P::count][4], v_exp[P::count][1];
    Pages k_pages = {}, v_pages = {};
    auto convert_k = [&](int step) {         // what was loaded
        static_for<P::count>([&](auto pc) {
            constexpr int p = pc.value, W = P::width(p), B = P::base(p);
            const float scale = k_scale(k_exp[p], lane);
#pragma unroll
            for (int i = 0; i < W / 32; ++i) k_ops[step & 1][own][B / 32 + i][lane] = __builtin_bit_cast(u32x4, eight_of(k_codes[B / 32 + i], scale));
        });
    };
    auto convert_v = [&](int step, bool masked) {                    // masked: some row of the workgroup does not see some key
        if (masked) {
            bool bad = false;
#pragma unroll
            for (int p = 0; p < P::count; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if ((v_exp[p][0] >> 8 * i & 255u) > C4_EXP_MAX) {
                        bad = true;
                        v_exp[p][0] &= ~(255u << 8 * i);
                    }
            const bool any = __ballot(bad) != 0;
            if (lane == 0) nans[step & 1][own] = any;
        }
        static_for<P::count>([&](auto pc) {
            constexpr int p = pc.value, W = P::width(p), B = P::base(p), E = W / 16;
            float scale[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) scale[i] = c4_scale(v_exp[p][0] >> 8 * i & 255u);
            static_for<E / 2>([&](auto ec) {
                constexpr int e = ec.value;
                uint32_t v[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) v[i] = pair_bits(__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(v_codes[p][i], scale[i], e));
                u32x2* even = reinterpret_cast<u32x2*>(&v_ops[step & 1][B / 16 + 2 * e][lane]) + own;
                u32x2* odd = reinterpret_cast<u32x2*>(&v_ops[step & 1][B / 16 + 2 * e + 1][lane]) + own;
                *even = u32x2{__builtin_amdgcn_perm(v[1], v[0], 0x05040100u), __builtin_amdgcn_perm(v[3], v[2], 0x05040100u)};
                *odd = u32x2{__builtin_amdgcn_perm(v[1], v[0], 0x07060302u), __builtin_amdgcn_perm(v[3], v[2], 0x07060302u)};
            });
        });
    };
    // The page table is read at every 32nd step, whichever wave's turn it is.
    auto load_k_step = [&](int step, bool mine) {
        if (step >= steps) return;
        if (step % 32 == 0) locate(k_pages, step);
        if (mine) load_k_half<D>(a.c, place(k_pages, step), lane, k_codes, k_exp);
    };
    auto load_v_step = [&](int step, bool mine) {
        if (step >= steps) return;
        if (step % 32 == 0) locate(v_pages, step);
        if (mine) load_v_half<D, 4>(a.c, place(v_pages, step), lane, v_codes, v_exp, 0);
    };

    load_k_step(0, (wave & 1) == 0);
    load_k_step(1, (wave & 1) == 1);
    bf16x8 q[QT][TERMS][M];
    int pos[QT];                             // position of the lane's row; -1: no row, or one before the first token
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        const int row = wave_row0 + 16 * u + c;
        const int token = fast_div(row, a.div_group), g = row - token * a.group;
        const bool valid = 16 * u + c < wave_rows;
        pos[u] = valid ? max(base + token, -1) : -1;
        load_q<D, TERMS>(static_cast<const T*>(a.q) + (t.s.first + token) * a.q_token + (long long)(head * a.group + g) * a.q_head, valid, lane, q[u]);
    }
    f32x4 o[QT][J], rounded[QT];
    float m[QT], l[QT];
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        m[u] = C4_LOW;
        l[u] = 0.f;
        rounded[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < J; ++j) o[u][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    bool far = false;                        // scores are multiplied by the scale first, and `times` is 1
    float times = a.scale;
    constexpr int SHARE = (QT * 8 * (2 + 2 * TERMS) + J + 2 * M - 1) / (J + 2 * M);
    using Scores = f32x4[QT][2];
    using Weights = bf16x8[QT][TERMS];
    auto visible = [&](int u, int key, bool there) {
        const int top = a.causal ? pos[u] : t.s.length - 1, bottom = a.window > 0 ? pos[u] - a.window + 1 : 0;
        return there && key <= top && key >= bottom;
    };
    auto products = [&](Scores& score, int step) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
#pragma unroll
            for (int u = 0; u < QT; ++u) score[u][s] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < M; ++i) {
                const bf16x8 k = __builtin_bit_cast(bf16x8, k_ops[step & 1][s][i][lane]);
#pragma unroll
                for (int u = 0; u < QT; ++u)
#pragma unroll
                    for (int n = 0; n < TERMS; ++n) score[u][s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[u][n][i], score[u][s], 0, 0, 0);
            }
        }
    };
    auto sums = [&](const Weights& w, int step) {
        if constexpr (TERMS == 1)
#pragma unroll
            for (int u = 0; u < QT; ++u) rounded[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones(), w[u][0], rounded[u], 0, 0, 0);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const bf16x8 v = __builtin_bit_cast(bf16x8, v_ops[step & 1][j][lane]);
#pragma unroll
            for (int u = 0; u < QT; ++u)
#pragma unroll
                for (int n = 0; n < TERMS; ++n) o[u][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, w[u][n], o[u][j], 0, 0, 0);
        }
    };
    // Step i of the loop; whole: its keys are all in pages; now: its scores, next: where those of step i + 1 go; before: the weights of step i - 1, after: where its own go.
    auto turn = [&](auto first, int i, bool whole, Scores& now, Scores& next, const Weights& before, Weights& after) {
        float factor[QT];
        bool raise = false, raised = false;
#pragma unroll
        for (int u = 0; u < QT; ++u) {
            factor[u] = max8(now[u][0], now[u][1]);
            raise = raise || factor[u] * times > m[u] + C4_SLACK;
        }
        const bool masked = !(whole && wave_clear(i));
        if (__ballot(raise) != 0 || masked || far) {
            if (masked) {
                const int key0 = key_first + 32 * i;
                const bool there[2] = {c4_page(a.r, a.c, t.b, key0) >= 0, c4_page(a.r, a.c, t.b, key0 + 16) >= 0};
#pragma unroll
                for (int u = 0; u < QT; ++u)
#pragma unroll
                    for (int x = 0; x < 8; ++x)
                        if (!visible(u, key0 + 16 * (x >> 2) + 4 * h4 + (x & 3), there[x >> 2])) now[u][x >> 2][x & 3] = -__builtin_inff();
            }
            raise = false;
            float most = 0.f;                // of the new reference points' magnitudes
#pragma unroll
            for (int u = 0; u < QT; ++u) {
                factor[u] = product(row_max(max8(now[u][0], now[u][1])), a.scale);
                if (factor[u] > m[u] + C4_SLACK) {
                    raise = true;
                    most = fmaxf(most, fabsf(factor[u]));
                }
            }
            raised = __ballot(raise) != 0;
            if (any_far(most)) {
                far = true;
                times = 1.f;
            }
            if (far) {
#pragma unroll
                for (int u = 0; u < QT; ++u)
#pragma unroll
                    for (int s = 0; s < 2; ++s) multiply(now[u][s], a.scale);
            }
#pragma unroll
            for (int u = 0; u < QT; ++u) {
                factor[u] = raise_maximum(m[u], factor[u]);
                l[u] *= factor[u];
            }
        }
        if constexpr (!first.value) sums(before, i - 1);
#pragma unroll
        for (int u = 0; u < QT; ++u)
#pragma unroll
            for (int x = 0; x < 8; ++x) {
                const float y = __builtin_amdgcn_exp2f(fmaf(now[u][x >> 2][x & 3], times, -m[u]));
                l[u] += y;
                __bf16 terms[TERMS];
                split_terms<TERMS>(y, terms);
#pragma unroll
                for (int n = 0; n < TERMS; ++n) after[u][n][x] = terms[n];
            }
        products(next, i + 1);               // (of the last step: what is left in LDS, and not used)
#pragma unroll
        for (int u = 0; u < QT; ++u)         // the weights are wanted here, among the products, not where they are used
#pragma unroll
            for (int n = 0; n < TERMS; ++n) {
                u32x4 bits = __builtin_bit_cast(u32x4, after[u][n]);
                asm volatile("" : "+v"(bits));
                after[u][n] = __builtin_bit_cast(bf16x8, bits);
            }
        // One read of LDS, two ahead of its use, QT * TERMS matrix and a share of the vector instructions at a time
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
#pragma unroll
        for (int x = 0; x < J + 2 * M; ++x) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, QT * TERMS, 0);
            __builtin_amdgcn_sched_group_barrier(0x402, SHARE, 0);
        }
        if (raised) {
#pragma unroll
            for (int u = 0; u < QT; ++u) {
                rounded[u] *= factor[u];
#pragma unroll
                for (int j = 0; j < J; ++j) o[u][j] *= factor[u];
            }
        }
    };
    // Seldom: NaN values, which must reach the rows that see them (as in the kernel above).
    auto spread_nans = [&](int i, bool was_masked) {
        if (!was_masked || (__builtin_amdgcn_readfirstlane(nans[i & 1][0]) | __builtin_amdgcn_readfirstlane(nans[i & 1][1])) == 0) return;
        const int key0 = key_first + 32 * i;
        static_for<P::count>([&](auto pc) {
            constexpr int p = pc.value, W = P::width(p), B = P::base(p), E = W / 16;
            bf16x8 marks;
            bool there[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int page = c4_page(a.r, a.c, t.b, key0 + 16 * s);
                there[s] = page >= 0;
                const uint8_t* exps = c4_record(a.c, max(page, 0), head) + a.c.v_exps + ((key0 + 16 * s) & (a.c.page - 1));
                const uint32_t bytes = *reinterpret_cast<const uint32_t*>(exps + ((B / 32 + c * E / 32) * a.c.page + 4 * h4));
#pragma unroll
                for (int x = 0; x < 4; ++x) marks[4 * s + x] = (bytes >> 8 * x & 255u) > C4_EXP_MAX ? (__bf16)1.f : (__bf16)0.f;
            }
#pragma unroll
            for (int u = 0; u < QT; ++u) {
                bf16x8 seen;
#pragma unroll
                for (int x = 0; x < 8; ++x) seen[x] = visible(u, key0 + 16 * (x >> 2) + 4 * h4 + (x & 3), there[x >> 2]) ? (__bf16)1.f : (__bf16)0.f;
                const f32x4 count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(marks, seen, f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
                for (int j = 0; j < E; ++j)
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        if (count[x] > 0.f) o[u][B / 16 + j][x] = __builtin_nanf("");
            }
        });
    };

    Scores s0, s1;
    Weights w0, w1;
    // K of steps 0 and 1 before the loop.  Within step i: K of step i + 2 and V of step i, loaded a step earlier, by the two waves of a half in turn.
    const bool odd = (wave & 1) == 1;        // a wave that converts V in even steps
    auto load_for = [&](int i, bool v) {
        load_k_step(i + 2, !v);
        load_v_step(i, v);
    };
    auto prepare = [&](int i, bool v, bool masked) {
        if (v) convert_v(i, masked);
        else if (i + 2 < steps) convert_k(i + 2);
        if (i + 1 < steps) load_for(i + 1, !v);
    };
    if (steps > 0) {
        if (!odd) convert_k(0);
        else if (steps > 1) convert_k(1);
        load_for(0, odd);
        __syncthreads();
        products(s0, 0);
        __syncthreads();                     // step 2's K may take step 0's place
        // (whether step i's keys are in pages is asked before prepare() goes on to the pages of step i + 1)
        bool whole = v_pages.whole, masked = !(whole && clear(0));
        prepare(0, odd, masked);
        turn(std::true_type{}, 0, whole, s0, s1, w1, w0);
        __syncthreads();
        for (int i = 1; i < steps; i += 2) {
            bool was_masked = masked;
            whole = v_pages.whole;
            masked = !(whole && clear(i));
            prepare(i, !odd, masked);
            spread_nans(i - 1, was_masked);
            turn(std::false_type{}, i, whole, s1, s0, w0, w1);
            __syncthreads();
            if (i + 1 < steps) {
                was_masked = masked;
                whole = v_pages.whole;
                masked = !(whole && clear(i + 1));
                prepare(i + 1, odd, masked);
                spread_nans(i, was_masked);
                turn(std::false_type{}, i + 1, whole, s0, s1, w1, w0);
                __syncthreads();
            }
        }
        spread_nans(steps - 1, masked);
        if (steps % 2 == 1) sums(w0, steps - 1);
        else sums(w1, steps - 1);
    }

    const long long slot = ((long long)tile * a.c.kv_heads + head) * a.splits + split;
#pragma unroll
    for (int u = 0; u < QT; ++u) {
        const float total = row_sum(l[u]), divisor = TERMS == 1 ? rounded[u][0] : total;
        if (16 * u + c >= wave_rows) continue;
        const float f = whole ? 1.f / divisor : 1.f;
        const int row = wave_row0 + 16 * u + c, r = 16 * QT * wave + 16 * u + c;
        const int token = fast_div(row, a.div_group), g = row - token * a.group;
        const long long at = ((long long)(t.s.first + token) * a.c.kv_heads + head) * a.group + g;
        static_for<P::count>([&](auto pc) {
            constexpr int p = pc.value, W = P::width(p), B = P::base(p), E = W / 16;       // E elements in a row
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = B + E * (4 * h4 + i);
                float y[E];
#pragma unroll
                for (int j = 0; j < E; ++j) y[j] = whole && divisor == 0.f ? 0.f : o[u][B / 16 + j][i] * f;
                if (whole) c4_store<E>(static_cast<T*>(a.out) + at * D + d, y);
                else c4_store<E>(a.part + (slot * ROWS + r) * D + d, y);
            }
        });
        if (h4 == 0) {
            if (!whole) {
                a.part_sums[slot * ROWS + r] = f32x4{m[u], total, divisor, 0.f};
            } else if (a.lse != nullptr) {
                a.lse[at] = total == 0.f ? -__builtin_inff() : (m[u] + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
            }
        }
    }
}

// Joins the parts of the tiles whose keys were cut up: a workgroup per row of a tile.  D / 8 lanes hold a row's elements, eight each; the groups of so many lanes take
// the parts in turn and meet in LDS.  32 parts of 16 rows x 16 heads (1 MB): 4.9 us, a launch and three dependent loads; one workgroup for all rows of a tile took 42 with 64 parts.
template <int D, int DTYPE, int ROWS, bool SPARSE>
__global__ __launch_bounds__(256) void join_kernel(Attend4 a) {
    using T = typename C4Type<DTYPE>::type;
    constexpr int LANES = D / 8, GROUPS = 256 / LANES;
    __shared__ __align__(16) float sums[GROUPS][D + 4];
    __shared__ float totals[GROUPS][2];
    const int rest = fast_div((int)blockIdx.x, a.div_heads), head = (int)blockIdx.x - rest * a.c.kv_heads, tile = rest, r = (int)blockIdx.y;
    const Tile4 t = find_tile<ROWS, SPARSE>(a, tile);
    if (r >= t.rows) return;
    const Range4 range = tile_steps<SPARSE>(a, t);
    if (range.count <= a.chunk) return;      // written already
    const int parts = (range.count + a.chunk - 1) / a.chunk;
    const long long slot = (((long long)tile * a.c.kv_heads + head) * a.splits) * ROWS + r;
    const int group = (int)threadIdx.x / LANES, d = (int)threadIdx.x % LANES * 8;
    const f32x4* ml = a.part_sums + slot;
    float high = C4_LOW, total = 0.f, divisor = 0.f, y[8] = {};
    for (int p = (int)threadIdx.x & 63; p < parts; p += 64) high = fmaxf(high, ml[(long long)p * ROWS][0]);
    high = row_max(high);
#pragma unroll
    for (int x = 1; x < 16; x <<= 1) high = fmaxf(high, __shfl_xor(high, x));
    if (group < GROUPS) {
        for (int p = group; p < parts; p += GROUPS) {
            const f32x4 v = ml[(long long)p * ROWS];
            const float f = __builtin_amdgcn_exp2f(v[0] - high);
            total = fmaf(v[1], f, total);
            divisor = fmaf(v[2], f, divisor);
            float part[8];
            c4_load8(a.part + (slot + (long long)p * ROWS) * D + d, part);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = fmaf(part[e], f, y[e]);
        }
        c4_store8(&sums[group][d], y);
        if (d == 0) {
            totals[group][0] = total;
            totals[group][1] = divisor;
        }
    }
    __syncthreads();
    if (group > 0) return;
    const int groups = min(GROUPS, parts);
    for (int g = 1; g < groups; ++g) {
        float part[8];
        c4_load8(&sums[g][d], part);
        total += totals[g][0];
        divisor += totals[g][1];
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] += part[e];
    }
    const int token = fast_div(t.row0 + r, a.div_group), g = t.row0 + r - token * a.group;
    const long long at = ((long long)(t.s.first + token) * a.c.kv_heads + head) * a.group + g;
    const float f = 1.f / divisor;
#pragma unroll
    for (int e = 0; e < 8; ++e) y[e] = divisor == 0.f ? 0.f : y[e] * f;
    c4_store8(static_cast<T*>(a.out) + at * D + d, y);
    if (a.lse != nullptr && d == 0) a.lse[at] = total == 0.f ? -__builtin_inff() : (high + __builtin_amdgcn_logf(total)) * 0.6931471805599453f;
}

// kernel: attend_kernel or attend_rows_kernel, whose workgroups carry ROWS rows.
template <int D, int DTYPE, int ROWS, bool SPARSE>
int launch_attend(void (*kernel)(Attend4), int threads, const Attend4& a, hipStream_t s) {
    const unsigned heads = (unsigned)a.c.kv_heads;
    launch(kernel, dim3((unsigned)a.tiles * (unsigned)a.splits * heads), dim3((unsigned)threads), 0, s, a);
    const unsigned rows = (unsigned)(SPARSE && a.group < ROWS ? a.group : ROWS);
    if (a.splits > 1) launch(join_kernel<D, DTYPE, ROWS, SPARSE>, dim3((unsigned)a.tiles * heads, rows), dim3(256), 0, s, a);
    return check_launch();
}

template <int D, int DTYPE>
int launch_attend_rows(const Attend4& a, int rows, hipStream_t s) {
    if (a.blocks != nullptr) return launch_attend<D, DTYPE, 16, true>(attend_kernel<D, DTYPE, 1, true>, 64 * cache4_waves(D, DTYPE, 1), a, s);
    constexpr int QT = cache4_wide_qtiles(D, DTYPE);
    if (rows == 64 * QT) return launch_attend<D, DTYPE, 64 * QT, false>(attend_rows_kernel<D, DTYPE, QT>, 256, a, s);
    if (rows == 16) return launch_attend<D, DTYPE, 16, false>(attend_kernel<D, DTYPE, 1, false>, 64 * cache4_waves(D, DTYPE, 1), a, s);
    if constexpr (cache4_qtiles(D, DTYPE) >= 2) if (rows == 32) return launch_attend<D, DTYPE, 32, false>(attend_kernel<D, DTYPE, 2, false>, 64 * cache4_waves(D, DTYPE, 2), a, s);
    return BNN_ERR_UNSUPPORTED;
}

template <int D>
int launch_attend_type(const Attend4& a, int dtype, int rows, hipStream_t s) {
    if (dtype == BNN_BF16) return launch_attend_rows<D, BNN_BF16>(a, rows, s);
    if (dtype == BNN_F16) return launch_attend_rows<D, BNN_F16>(a, rows, s);
    return launch_attend_rows<D, BNN_F32>(a, rows, s);
}

}  // namespace
}  // namespace bnn
#endif
