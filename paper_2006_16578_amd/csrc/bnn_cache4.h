// Declarations shared by the kernels of the 4-bit key/value cache (not part of the ABI; the layout and the operators are stated in include/bnn.h).
#ifndef BNN_CACHE4_H
#define BNN_CACHE4_H

#include <algorithm>

#include "bnn_internal.h"

namespace bnn {

// What a stored scale may be: 2^(byte - 127), byte in [C4_EXP_MIN, C4_EXP_MAX]; C4_EXP_NAN marks a group that held an infinity or a NaN.
// Six times the largest and half the smallest are ordinary numbers in fp32 and bf16, so no value of the cache overflows or is subnormal there.
constexpr int C4_EXP_MIN = 27, C4_EXP_MAX = 227, C4_EXP_NAN = 255;
constexpr int C4_GROUP = 32;                 // elements that share a scale: the width of the matrix instructions' own block scales

// A cache as the kernels see it.  Offsets of a record's parts are in bytes.
struct Cache4 {
    uint8_t* data;
    int pages, kv_heads, dim, page, page_shift;
    int record;                              // bytes of one (page, head)
    int v_codes, k_exps, v_exps, signs;      // K codes at 0
};

// The rows of a call: sequence b's newest start[b + 1] - start[b] tokens (start == nullptr: `each` of every sequence).
struct Rows4 {
    const int32_t* table;
    const int32_t* lens;
    const int32_t* start;
    int batch, table_pages, tokens, each;
    FastDiv div_each;
};

// One sequence of a call: its first row, its number of rows, its length, which may pass the end of its table.  Row i (of the sequence) is the token at length - rows + i.
struct Sequence4 {
    int first, rows, length;
};

__device__ __forceinline__ Sequence4 c4_sequence(const Rows4& r, int b) {
    Sequence4 s;
    if (r.start == nullptr) {
        s.first = b * r.each;
        s.rows = r.each;
    } else {                                 // clamped: no content of start leads out of the callers' arrays
        s.first = min(max(r.start[b], 0), r.tokens);
        s.rows = min(max(r.start[b + 1], s.first), r.tokens) - s.first;
    }
    s.length = max(r.lens[b], 0);
    return s;
}

// Tokens that a table has room for.
__device__ __forceinline__ int c4_room(const Rows4& r, const Cache4& c) { return (int)((long long)r.table_pages << c.page_shift); }

// The sequence that row t belongs to: the last one that starts at or before t.
__device__ __forceinline__ int c4_sequence_of(const Rows4& r, int t) {
    if (r.start == nullptr) return fast_div(t, r.div_each);
    int lo = 0, hi = r.batch - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (r.start[mid] <= t) lo = mid; else hi = mid - 1;
    }
    return lo;
}

// The page that holds a token of sequence b, or -1: out of the table, or an entry that is no page.  Without branches, so that loads of several can be under way.
__device__ __forceinline__ int c4_page(const Rows4& r, const Cache4& c, int b, int token) {
    const int at = token >> c.page_shift;                    // negative for a negative token
    const int p = r.table[(long long)b * r.table_pages + min(max(at, 0), r.table_pages - 1)];
    return at >= 0 && at < r.table_pages && (uint32_t)p < (uint32_t)c.pages ? p : -1;
}
__device__ __forceinline__ uint8_t* c4_record(const Cache4& c, int page, int head) {
    return c.data + ((long long)page * c.kv_heads + head) * c.record;
}

// Tiles of `rows` rows (units: rows of a token) that never span sequences: the sequence of `tile`, and its number in it; false: there are fewer tiles.
// With start == nullptr every sequence has seq_tiles; else a wave counts the tiles of 64 sequences at a time.
__device__ __forceinline__ bool c4_find_tile(const Rows4& r, int units, int rows, int tile, int seq_tiles, const FastDiv& div_seq_tiles, int& b, int& local) {
    if (r.start == nullptr) {
        b = fast_div(tile, div_seq_tiles);
        local = tile - b * seq_tiles;
        return b < r.batch;
    }
    const int lane = (int)threadIdx.x & 63;
    int before = 0;
    for (int b0 = 0; b0 < r.batch; b0 += 64) {
        int n = 0;
        if (b0 + lane < r.batch) {
            const int first = min(max(r.start[b0 + lane], 0), r.tokens);
            n = (int)(((long long)(min(max(r.start[b0 + lane + 1], first), r.tokens) - first) * units + rows - 1) / rows);
        }
        int sum = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int other = __shfl_up(sum, d);
            if (lane >= d) sum += other;
        }
        const unsigned long long past = __ballot(before + sum > tile);
        if (past != 0) {
            const int at = __ffsll(past) - 1;
            b = b0 + at;
            local = __builtin_amdgcn_readfirstlane(tile - (before + __shfl(sum, at) - __shfl(n, at)));
            return true;
        }
        before += __shfl(sum, 63);
    }
    return false;
}
// How many such tiles a launch needs at most (with start: a partly filled one for every sequence).
inline long long c4_tiles(const Rows4& r, int units, int rows, int* seq_tiles) {
    *seq_tiles = r.start ? 0 : (int)cdiv((long long)r.each * units, rows);
    return r.start ? (long long)r.tokens * units / rows + r.batch : (long long)r.batch * *seq_tiles;
}

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Eight consecutive elements as fp32, from 16-byte aligned memory.
template <class T>
__device__ __forceinline__ void c4_load8(const T* p, float (&x)[8]) {
    if constexpr (sizeof(T) == 4) {
        const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = a[i]; x[4 + i] = b[i]; }
    } else {
        typedef T t8 __attribute__((ext_vector_type(8)));
        const t8 a = *reinterpret_cast<const t8*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)a[i];
    }
}
// N consecutive elements (2, 4 or 8), aligned to their bytes, 16 at most.
template <int N, class T>
__device__ __forceinline__ void c4_store(T* p, const float (&x)[N]) {
    constexpr int W = N * sizeof(T) > 16 ? 16 / sizeof(T) : N;
    typedef T tw __attribute__((ext_vector_type(W)));
#pragma unroll
    for (int b = 0; b < N; b += W) {
        tw a;
#pragma unroll
        for (int i = 0; i < W; ++i) a[i] = (T)x[b + i];
        *reinterpret_cast<tw*>(p + b) = a;
    }
}
template <class T>
__device__ __forceinline__ void c4_store8(T* p, const float (&x)[8]) { c4_store<8>(p, x); }

// Value of the lane whose number in its group of four differs in the bits of X.
template <int X>
__device__ __forceinline__ uint32_t c4_quad_xor(uint32_t v) {
    constexpr int perm = X == 1 ? 0xB1 : 0x4E;          // lanes 1,0,3,2 / 2,3,0,1
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, perm, 0xf, 0xf, true);
}

// Eight elements of a group of 32 that four lanes share: returns the codes, sets the scale's byte.
__device__ __forceinline__ uint32_t c4_quantise(const float (&x)[8], uint32_t& byte) {
    uint32_t high = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) high = max(high, __float_as_uint(x[i]) & 0x7fffffffu);
    high = max(high, c4_quad_xor<1>(high));
    high = max(high, c4_quad_xor<2>(high));
    // 1.m 2^(E - 127) <= 6 2^e: e + 127 = E - 2, one more where 1.m > 1.5
    const int e = (int)(high >> 23) - 2 + ((high & 0x7fffffu) > 0x400000u ? 1 : 0);
    const int clamped = min(max(e, C4_EXP_MIN), C4_EXP_MAX);
    byte = high >= 0x7f800000u ? C4_EXP_NAN : (uint32_t)clamped;
    const float scale = __uint_as_float((uint32_t)clamped << 23);
    uint32_t codes = 0;
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], scale, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], scale, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], scale, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], scale, 3);
    return codes;
}

// Writes a token's key x and value y, eight elements from 8 * at on of each, with the signs of x: the four lanes of a group of 32 elements together.
__device__ __forceinline__ void c4_put(const Cache4& c, uint8_t* rec, int offset, int at, const float (&x)[8], const float (&y)[8]) {
    uint32_t kb, vb;
    const uint32_t kc = c4_quantise(x, kb), vc = c4_quantise(y, vb);
    const int row = c.dim / 2 * offset + at * 4;
    *reinterpret_cast<uint32_t*>(rec + row) = kc;
    *reinterpret_cast<uint32_t*>(rec + c.v_codes + row) = vc;
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) bits |= (x[i] >= 0.f ? 1u : 0u) << i;
    bits <<= 8 * (at & 3);
    bits |= c4_quad_xor<1>(bits);
    bits |= c4_quad_xor<2>(bits);
    if ((at & 3) == 0) {
        const int e = (at >> 2) * c.page + offset;
        rec[c.k_exps + e] = (uint8_t)kb;
        rec[c.v_exps + e] = (uint8_t)vb;
        if (c.signs) *reinterpret_cast<uint32_t*>(rec + c.signs + offset * (c.dim / 8) + at) = bits;
    }
}

// The scale that a byte stands for, for the conversion instructions: with the NaN byte's (the bits of an infinity) they give NaN for every code, 0 included.
__device__ __forceinline__ float c4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// bf16 terms of a query or weight of a type.
constexpr int cache4_terms(int dtype) { return dtype == BNN_BF16 ? 1 : dtype == BNN_F16 ? 2 : 3; }

// The attention call as the kernels see it.
struct Attend4 {
    Cache4 c;
    Rows4 r;
    const void* q;
    long long q_token, q_head;               // elements between tokens and between heads
    int group;                               // query heads of a kv head
    FastDiv div_group;
    float scale;                             // times log2(e): scores are powers of two
    int causal, window;
    const int32_t* blocks;                   // [tokens][kv_heads][keep], or nullptr: every key
    int keep;
    void* out;
    float* lse;
    int tiles;                               // row tiles of the launch
    int seq_tiles;                           // row tiles of a sequence, where all have as many rows
    FastDiv div_seq_tiles;
    int splits, chunk;                       // parts the keys are cut into: of `chunk` steps of 32 keys
    FastDiv div_splits, div_heads;
    float* part;                             // [tiles][kv_heads][splits][rows of a tile][dim]
    f32x4* part_sums;                        // [tiles][kv_heads][splits][rows of a tile]: reference point, sum of the weights, sum of the rounded weights
};

// A launch has fewer threads than this (along a dimension of its grid).
constexpr long long C4_THREADS = 1LL << 32;

// How a call is cut up.  rows: of a workgroup.
struct AttendPlan4 {
    int rows, threads, tiles, seq_tiles, splits, chunk;
    size_t part_bytes, workspace_bytes;
};

// Groups of 16 rows that a wave carries, by what fits 256 registers: per group a lane keeps D / 4 of sums, D / 8 of every term of Q, and scores and weights.  (With twice as
// many, at one wave a SIMD, nothing runs while a wave waits: two prompts of 4096 tokens 631 us instead of 416.)
constexpr int cache4_qtiles(int dim, int dtype) {            // a workgroup's rows, each wave has all
    return 2 * (dim / 4 + cache4_terms(dtype) * (dim / 8) + 4 * cache4_terms(dtype)) < 144 ? 2 : 1;
}
// Waves that share the keys of 16 rows, or of 32 (and of wide heads in fp32, which take more than the 256 registers that eight waves leave each other).  Eight make for half
// as many parts to be joined as four: two long documents 50 -> 48 us, 64 conversations 76 -> 66 (now 60; with sixteen 77).
constexpr int cache4_waves(int dim, int dtype, int qtiles) { return qtiles == 1 && !(dim == 256 && dtype == BNN_F32) ? 8 : 4; }
constexpr int cache4_wide_qtiles(int dim, int dtype) {       // a wave's, of four with different rows
    return 2 * (dim / 4 + cache4_terms(dtype) * (dim / 8) + 8 * cache4_terms(dtype) + 16) <= 170 ? 2 : 1;
}

int launch_cache4_attend64(const Attend4& a, int dtype, int rows, hipStream_t s);
int launch_cache4_attend96(const Attend4& a, int dtype, int rows, hipStream_t s);
int launch_cache4_attend128(const Attend4& a, int dtype, int rows, hipStream_t s);
int launch_cache4_attend192(const Attend4& a, int dtype, int rows, hipStream_t s);
int launch_cache4_attend256(const Attend4& a, int dtype, int rows, hipStream_t s);

// The selection call as the kernels see it.
struct Select4 {
    Cache4 c;
    Rows4 r;
    const void* q;
    long long q_token, q_head;
    int group;
    int keep, first, last;
    int32_t* blocks;                         // [tokens][kv_heads][keep]
    uint16_t* scores;                        // [tokens][kv_heads][table_pages]: score + 1, 0 where the row sees no key of the block
    // of the launch that scores
    int columns, tile_tokens;                // columns of a token, its query heads, and tokens in 32 columns
    FastDiv div_columns;
    int tiles, seq_tiles, parts;
    FastDiv div_seq_tiles, div_parts, div_heads;
};
int launch_cache4_select(Select4 a, int dtype, hipStream_t s);
// The call that sums attention weights, as the kernels see it.
struct Weigh4 {
    Cache4 c;
    Rows4 r;
    const void* q;
    long long q_token, q_head;
    int group;
    FastDiv div_group, div_heads;
    float scale2;                            // scale / log 2
    double unscale;                          // 1 / scale, less half of what scale2 is off by
    int causal, window;
    const float* lse;                        // [tokens][heads]
    const float* previous;                   // [batch][kv_heads][width], or nullptr; may be out
    float* out;
    float decay;
    long long width;
    int few_most;                            // sequences of up to so many rows are the launch's for few rows, others that for many
    int parts;                               // of a launch for few rows: that share a sequence's keys; for many: that share the rows of a tile of keys, where all sequences have as many
    int items, slots, part_shift;            // (sequence, part) pairs of the launch for many rows; slots: those of sequences in several parts; where sequences differ, a part has 2^part_shift rows at most
    FastDiv div_parts, div_items;
    float* partial;                          // [slots][kv_heads][width4]
    long long width4;                        // tokens that the table has room for
};
// How such a call is cut up: a launch for sequences of few rows (row_tiles: tiles of 16 rows that a wave carries, 0: no such launch), one for those of many (items: pairs of a sequence and a part of its rows that there can be, 0: no such launch; slots: of them, those whose sums are joined), or both.
struct WeighPlan4 {
    int few_most, row_tiles, few_parts, items, slots, many_parts, part_shift;
    bool runs;                               // the launch for few rows has sequences of more than 256, too far apart for the other
    long long few_groups, many_groups;
    size_t workspace_bytes;
};
constexpr int cache4_weigh_tiles(int dim) { return dim >= 192 ? 2 : 4; }          // tiles of 16 keys that a wave of that kernel keeps
constexpr bool cache4_weigh_two(int dim, int dtype) { return dim / 32 * cache4_terms(dtype) <= 12; }       // whether two tiles of rows fit a wave's registers
int launch_cache4_weigh(const Weigh4& a, const WeighPlan4& p, int dtype, hipStream_t s);

// The choice of the tokens to keep, and moving them.
struct Heaviest4 {
    Cache4 c;
    const float* weights;                    // [batch][kv_heads][width]
    long long width;
    const int32_t *table, *lens;
    int batch, table_pages, keep, first, last;
    int32_t *tokens, *kept;                  // [batch][kv_heads][keep], [batch]
};
// How the choice is cut up.  parts: of a sequence, of 8192 tokens each, 0: one workgroup has a sequence and kv head.
struct HeaviestPlan4 {
    int parts;
    size_t bins_bytes, borders_bytes, workspace_bytes;
};
HeaviestPlan4 plan_cache4_heaviest(const Cache4& c, int batch, int table_pages);
int launch_cache4_heaviest(const Heaviest4& a, const HeaviestPlan4& plan, void* workspace, hipStream_t s);
struct Move4 {
    Cache4 c;
    const int32_t* tokens;                   // [batch][kv_heads][keep]
    const int32_t *table, *into;             // [batch][table_pages], [batch][into_pages]
    int batch, table_pages, into_pages, keep;
    const float* weights;                    // [batch][kv_heads][width], or nullptr
    long long width;
    float* moved;                            // [batch][kv_heads][into_pages * page]
};
int launch_cache4_move(const Move4& a, hipStream_t s);

// Workgroups of 256 threads of writing and reading, for a kv head: each has the rows whose elements, eight to a thread, fill it.
inline int cache4_block_rows(const Cache4& c) { return 256 / (c.dim / 8); }
inline long long cache4_row_blocks(const Cache4& c, const Rows4& r) { return cdiv(r.tokens, cache4_block_rows(c)); }
int launch_cache4_write(const Cache4& c, const Rows4& r, const void* k, const void* v, int dtype, long long k_token, long long k_head,
                        long long v_token, long long v_head, hipStream_t s);
int launch_cache4_read(const Cache4& c, const Rows4& r, void* k, void* v, int dtype, hipStream_t s);

}  // namespace bnn
#endif
