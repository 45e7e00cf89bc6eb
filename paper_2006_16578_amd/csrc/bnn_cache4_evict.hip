// Eviction: which cached tokens to keep, by their weights, and moving them into other pages.
//
// heaviest_kernel: a workgroup has a sequence and kv head.  Weights in the order of numbers are whole numbers in the order of their bits (negative ones turned round); that of the last token that
// is kept is found digit by digit, from the highest on: a histogram of the digit over what agrees so far, 11 + 11 + 10 bits.  Of those that equal it the lowest tokens are kept.  A wave has a run of
// consecutive tokens, a lane four beside each other, so one exchange of counts gives every wave the place of its first kept token, and the list is ascending.  Weights are read once and stay in
// registers where the table has room for up to 32768 tokens; beyond, heaviest_part_kernel has 8192 of them, or, with many sequences, they are read five times, eight loads under way.
// What bounds it is the chain of barriers, counts and scans: 32 sequences of 2100 to 16384 tokens, 8 kv heads, 23 us, of which reading their 9 MB is 2.
// move_kernel: a workgroup has a kv head and 64 places of the new sequence.  What bounds it is memory, by whole lines: a token's scales are 2 * D / 32 bytes in as many lines, and lines of codes hold the neighbours that
// stay behind.  2048 tokens of each of those sequences, heads of 128: 171 MB come in for 80 MB of tokens, 52 to 69 us.
#include "bnn_cache4.h"

namespace bnn {
namespace {

constexpr int H_THREADS = 1024, H_WAVES = H_THREADS / 64, H_BINS = 2048, H_VECTOR = 256;       // H_VECTOR: tokens of a wave at once

// The order of weights as that of whole numbers; NaN below all.  -0 counts as 0.
__device__ __forceinline__ uint32_t rank_of(float w) {
    if (w != w) return 0;
    const uint32_t bits = __float_as_uint(w + 0.f);
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

// Four tokens of a lane.  (Pages and tables have room for multiples of 16: what begins inside lies inside.)
struct Four {
    f32x4 weight;
    int page;
};
__device__ __forceinline__ Four fetch_four(const float* weights, const int32_t* table, int page_shift, int j, int end) {
    Four f = {f32x4{0.f, 0.f, 0.f, 0.f}, -1};
    if (j < end) {
        __builtin_memcpy(&f.weight, weights + j, 16);
        f.page = table[j >> page_shift];
    }
    return f;
}
// 0: nowhere; kept in any case: the highest; else a number between
__device__ __forceinline__ void rank_four(const Heaviest4& a, const Four& f, int j, int end, int length, uint32_t (&r)[4]) {
    const bool there = (uint32_t)f.page < (uint32_t)a.c.pages;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int t = j + i;
        r[i] = t < a.first || t >= length - a.last ? 0xffffffffu : min(max(rank_of(f.weight[i]), 1u), 0xfffffffeu);
        if (!there || t >= end) r[i] = 0;
    }
}

// What is known of the lowest rank that is kept: its digits so far, and how many of those that agree with them are kept.
struct Border {
    uint32_t rank;
    int count;
};
__device__ __forceinline__ int digit_shift(int digit) { return digit == 0 ? 21 : digit == 1 ? 10 : 0; }
__device__ __forceinline__ int digit_width(int digit) { return digit == 2 ? 10 : 11; }
__device__ __forceinline__ bool digit_counts(uint32_t r, const Border& border, int digit) {
    return r != 0 && (digit == 0 || r >> (digit_shift(digit) + digit_width(digit)) == border.rank >> (digit_shift(digit) + digit_width(digit)));
}
__device__ __forceinline__ int digit_of(uint32_t r, int digit) { return (int)(r >> digit_shift(digit) & ((1u << digit_width(digit)) - 1)); }

// The next digit: from the highest bin down the one in which the count reaches border.count.  A thread has the bins 2047 - 2 t and 2046 - 2 t; there is such a bin.  Begins and ends with a barrier for `shared`.
struct PickShared {
    int wave_sum[H_WAVES], picked[2];
};
__device__ __forceinline__ void pick_digit(Border& border, int digit, int high, int low, PickShared& shared) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, top = H_BINS - 1 - 2 * (int)threadIdx.x;
    int upto = high + low;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int other = __shfl_up(upto, d);
        if (lane >= d) upto += other;
    }
    if (lane == 63) shared.wave_sum[wave] = upto;
    __syncthreads();
    for (int w = 0; w < wave; ++w) upto += shared.wave_sum[w];
    const int before = upto - high - low;
    if (before < border.count && upto >= border.count) {
        const bool first = before + high >= border.count;
        shared.picked[0] = first ? top : top - 1;
        shared.picked[1] = border.count - before - (first ? 0 : high);
    }
    __syncthreads();
    border.rank |= (uint32_t)shared.picked[0] << digit_shift(digit);
    border.count = shared.picked[1];
}

// Writes a wave's kept tokens, vector by vector: place: of the next; equals: how many of the border's rank came before.
struct Emit {
    int32_t* out;
    Border border;
    int place, equals;
    // lanes before this one, in a mask
    __device__ __forceinline__ static int before(unsigned long long mask) {
        return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
    }
    __device__ __forceinline__ void operator()(const uint32_t (&r)[4], int j) {
        bool keep[4];
        unsigned long long e[4], any = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e[i] = __ballot(r[i] == border.rank);
            any |= e[i];
            keep[i] = r[i] > border.rank;
        }
        if (any != 0) {                      // which of those at the border: the lowest
            int n = equals + before(e[0]) + before(e[1]) + before(e[2]) + before(e[3]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (r[i] == border.rank) {
                    keep[i] = n < border.count;
                    ++n;
                }
                equals += __popcll(e[i]);
            }
        }
        unsigned long long k[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) k[i] = __ballot(keep[i]);
        int at = place + before(k[0]) + before(k[1]) + before(k[2]) + before(k[3]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (keep[i]) out[at++] = j + i;
            place += __popcll(k[i]);
        }
    }
};

// E: vectors of a wave that its registers hold; 0: none.
template <int E>
__global__ __launch_bounds__(H_THREADS) void heaviest_kernel(Heaviest4 a) {
    constexpr int LOADS = E == 0 ? 8 : E;    // under way together
    __shared__ int bins[H_BINS];
    __shared__ int wave_above[H_WAVES], wave_equal[H_WAVES], wave_there[H_WAVES];
    __shared__ PickShared shared;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int b = (int)blockIdx.x, head = (int)blockIdx.y;
    const int length = (int)min((long long)max(a.lens[b], 0), (long long)a.table_pages << a.c.page_shift);
    const int run = (length + H_WAVES * H_VECTOR - 1) / (H_WAVES * H_VECTOR);     // vectors of a wave
    const int begin = min(wave * run * H_VECTOR, length), end = min(begin + run * H_VECTOR, length);
    const float* weights = a.weights + ((long long)b * a.c.kv_heads + head) * a.width;
    const int32_t* table = a.table + (long long)b * a.table_pages;
    int32_t* out = a.tokens + ((long long)b * a.c.kv_heads + head) * a.keep;

    auto fetch = [&](int j) { return fetch_four(weights, table, a.c.page_shift, j, end); };
    auto rank = [&](const Four& f, int j, uint32_t (&r)[4]) { rank_four(a, f, j, end, length, r); };
    uint32_t held[E == 0 ? 1 : E][4];
    if constexpr (E > 0) {
        Four f[E];
#pragma unroll
        for (int e = 0; e < E; ++e) f[e] = fetch(begin + e * H_VECTOR + 4 * lane);
#pragma unroll
        for (int e = 0; e < E; ++e) rank(f[e], begin + e * H_VECTOR + 4 * lane, held[e]);
    }
    // f(ranks, first token of the lane) for every vector of the wave
    auto for_each = [&](auto f) {
        if constexpr (E > 0) {
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (begin + e * H_VECTOR < end) f(held[e], begin + e * H_VECTOR + 4 * lane);
        } else {
            for (int j0 = begin; j0 < end; j0 += LOADS * H_VECTOR) {
                Four four[LOADS];
#pragma unroll
                for (int e = 0; e < LOADS; ++e) four[e] = fetch(j0 + e * H_VECTOR + 4 * lane);
#pragma unroll
                for (int e = 0; e < LOADS; ++e) {
                    if (j0 + e * H_VECTOR >= end) break;
                    uint32_t r[4];
                    rank(four[e], j0 + e * H_VECTOR + 4 * lane, r);
                    f(r, j0 + e * H_VECTOR + 4 * lane);
                }
            }
        }
    };

    int there = 0;
    for (int i = (int)threadIdx.x; i < H_BINS; i += H_THREADS) bins[i] = 0;
    __syncthreads();
    for_each([&](const uint32_t (&r)[4], int) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r[i] != 0) {
                ++there;
                atomicAdd(&bins[r[i] >> 21], 1);
            }
    });
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) there += __shfl_xor(there, d);
    if (lane == 0) wave_there[wave] = there;
    __syncthreads();
    there = 0;
#pragma unroll
    for (int w = 0; w < H_WAVES; ++w) there += wave_there[w];
    const int kept = min(there, a.keep);
    if (head == 0 && threadIdx.x == 0) a.kept[b] = kept;

    Border border = {1, 0x7fffffff};         // everything that lies somewhere
    if (there > a.keep) {
        border = {0, a.keep};
        for (int digit = 0; digit < 3; ++digit) {
            if (digit > 0) {
                for (int i = (int)threadIdx.x; i < H_BINS; i += H_THREADS) bins[i] = 0;
                __syncthreads();
                for_each([&](const uint32_t (&r)[4], int) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (digit_counts(r[i], border, digit)) atomicAdd(&bins[digit_of(r[i], digit)], 1);
                });
                __syncthreads();
            }
            const int top = H_BINS - 1 - 2 * (int)threadIdx.x;
            pick_digit(border, digit, bins[top], bins[top - 1], shared);
        }
    }

    int above = 0, equal = 0;
    for_each([&](const uint32_t (&r)[4], int) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            above += r[i] > border.rank ? 1 : 0;
            equal += r[i] == border.rank ? 1 : 0;
        }
    });
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
        above += __shfl_xor(above, d);
        equal += __shfl_xor(equal, d);
    }
    if (lane == 0) {
        wave_above[wave] = above;
        wave_equal[wave] = equal;
    }
    __syncthreads();
    int place = 0, equals = 0;
    for (int w = 0; w < wave; ++w) {
        place += wave_above[w];
        equals += wave_equal[w];
    }
    Emit emit = {out, border, place + min(equals, border.count), equals};
    for_each([&](const uint32_t (&r)[4], int j) { emit(r, j); });
    for (int i = kept + (int)threadIdx.x; i < a.keep; i += H_THREADS) out[i] = -1;
}

// Long sequences, few of them: a workgroup has 8192 tokens of one, in registers, and four launches pass the histograms on through the workspace.  Launch d < 3 counts digit d, having picked digit d - 1 from all
// parts' counts; the last writes the tokens, the place of its first one being what the parts before it keep.  One sequence of 131072 tokens, 4 kv heads: 5 + 9 + 8 + 10 us; in one workgroup for each head 118.
struct Parts4 {
    int parts;
    int* bins;                               // [unit][digit][part][bins]; unit: sequence and kv head
    Border* borders;                         // [unit][digit]: what launch `digit` found before it counted
    int* above;                              // [unit][digit][part]: tokens of the part above the border by that digit
};
template <int LAUNCH>
__global__ __launch_bounds__(H_THREADS) void heaviest_part_kernel(Heaviest4 a, Parts4 p) {
    constexpr int E = 2;
    __shared__ int bins[H_BINS];
    __shared__ int wave_above[H_WAVES], wave_equal[H_WAVES], sums[3][H_WAVES];
    __shared__ PickShared shared;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), tid = (int)threadIdx.x;
    const int part = (int)blockIdx.x, head = (int)blockIdx.y, b = (int)blockIdx.z;
    const int length = (int)min((long long)max(a.lens[b], 0), (long long)a.table_pages << a.c.page_shift);
    constexpr int TOKENS = H_WAVES * E * H_VECTOR;
    const int used = max((length + TOKENS - 1) / TOKENS, 1);         // parts with tokens (an empty sequence's first writes the list)
    if (part >= used) return;
    const int begin = min(part * TOKENS + wave * E * H_VECTOR, length), end = min(begin + E * H_VECTOR, length);
    const long long unit = (long long)b * a.c.kv_heads + head;
    const float* weights = a.weights + unit * a.width;
    const int32_t* table = a.table + (long long)b * a.table_pages;
    int* const my_bins = p.bins + ((unit * 3 + LAUNCH) * p.parts + part) * H_BINS;       // (LAUNCH < 3)
    Four f[E];                               // (ranked once the loads of the counts are under way as well)
#pragma unroll
    for (int e = 0; e < E; ++e) f[e] = fetch_four(weights, table, a.c.page_shift, begin + e * H_VECTOR + 4 * lane, end);
    uint32_t held[E][4];
    auto rank = [&]() {
#pragma unroll
        for (int e = 0; e < E; ++e) rank_four(a, f[e], begin + e * H_VECTOR + 4 * lane, end, length, held[e]);
    };
    // The sum over a workgroup of each thread's n, for all
    auto total = [&](int n, int* scratch) {
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) n += __shfl_xor(n, d);
        if (lane == 0) scratch[wave] = n;
        __syncthreads();
        n = 0;
#pragma unroll
        for (int w = 0; w < H_WAVES; ++w) n += scratch[w];
        return n;
    };

    Border border = {0, a.keep};
    bool all = false;                        // everything is kept
    int there = 0, above_before = 0, high_before = 0, low_before = 0;       // of the parts before this one: above the border by digits 0 and 1; counts of the thread's bins
    if constexpr (LAUNCH == 0) rank();
    if constexpr (LAUNCH > 0) {
        // Digit LAUNCH - 1, from the counts of all parts
        constexpr int digit = LAUNCH - 1;
        if constexpr (LAUNCH > 1) border = p.borders[unit * 3 + LAUNCH - 1];
        const int top = H_BINS - 1 - 2 * tid;
        const int* counts = p.bins + (unit * 3 + digit) * (long long)p.parts * H_BINS + top - 1;
        int high = 0, low = 0, own_high = 0, own_low = 0;
#pragma unroll 8
        for (int q = 0; q < used; ++q) {
            const int2 n = *reinterpret_cast<const int2*>(counts + (long long)q * H_BINS);
            low += n.x;
            high += n.y;
            if (q < part) {
                low_before += n.x;
                high_before += n.y;
            }
            if (q == part) {
                own_low = n.x;
                own_high = n.y;
            }
        }
        if constexpr (LAUNCH == 3)           // (not written where all are kept, and not used there)
            for (int q = tid; q < part; q += H_THREADS) above_before += p.above[unit * 3 * p.parts + q] + p.above[(unit * 3 + 1) * p.parts + q];
        rank();
        if constexpr (LAUNCH == 1) there = total(high + low, sums[0]);
        all = LAUNCH == 1 ? there <= a.keep : border.count == 0x7fffffff;
        if (all) {
            border = {0, LAUNCH == 3 ? 0 : 0x7fffffff};              // (of the rank 0, of what lies nowhere, none)
        } else {
            pick_digit(border, digit, high, low, shared);
            const int picked = digit_of(border.rank, digit);
            const int over = total((top > picked ? own_high : 0) + (top - 1 > picked ? own_low : 0), sums[1]);
            if (LAUNCH < 3 && tid == 0) p.above[(unit * 3 + digit) * p.parts + part] = over;
        }
        if (LAUNCH < 3 && part == 0 && tid == 0) p.borders[unit * 3 + LAUNCH] = border;
        if (LAUNCH == 1 && part == 0 && head == 0 && tid == 0) a.kept[b] = min(there, a.keep);
    }
    if constexpr (LAUNCH < 3) {
        if (all) return;
        for (int i = tid; i < H_BINS; i += H_THREADS) bins[i] = 0;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (digit_counts(held[e][i], border, LAUNCH)) atomicAdd(&bins[digit_of(held[e][i], LAUNCH)], 1);
        __syncthreads();
        for (int i = tid; i < H_BINS; i += H_THREADS) my_bins[i] = bins[i];
    } else {
        // What the parts before this one keep: above the border by one of its digits, and of its own rank
        int over = 0, same = 0;
        const int top = H_BINS - 1 - 2 * tid;
        if (!all) {
            const int picked = digit_of(border.rank, 2);
            over = above_before + (top > picked ? high_before : 0) + (top - 1 > picked ? low_before : 0);
            same = (top == picked ? high_before : 0) + (top - 1 == picked ? low_before : 0);
        } else {                             // all that is counted by the first digit, the last not having been
            const int* counts = p.bins + unit * 3 * (long long)p.parts * H_BINS + top - 1;
#pragma unroll 8
            for (int q = 0; q < part; ++q) {
                const int2 n = *reinterpret_cast<const int2*>(counts + (long long)q * H_BINS);
                over += n.x + n.y;
            }
        }
        __syncthreads();
        over = total(over, sums[0]);
        same = total(same, sums[2]);
        int above = 0, equal = 0;
#pragma unroll
        for (int e = 0; e < E; ++e)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                above += held[e][i] > border.rank ? 1 : 0;
                equal += held[e][i] == border.rank ? 1 : 0;
            }
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) {
            above += __shfl_xor(above, d);
            equal += __shfl_xor(equal, d);
        }
        if (lane == 0) {
            wave_above[wave] = above;
            wave_equal[wave] = equal;
        }
        __syncthreads();
        for (int w = 0; w < wave; ++w) {
            over += wave_above[w];
            same += wave_equal[w];
        }
        int32_t* const out = a.tokens + unit * a.keep;
        Emit emit = {out, border, over + min(same, border.count), same};
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (begin + e * H_VECTOR < end) emit(held[e], begin + e * H_VECTOR + 4 * lane);
        if (part == 0) {                     // the rest of a list that is not full
            const int kept = a.kept[b];
            for (int i = kept + tid; i < a.keep; i += H_THREADS) out[i] = -1;
        }
    }
}

// A thread moves 16 bytes of codes, K's and V's, the lanes of a token side by side; scales and signs go a byte or word at a time.
__global__ __launch_bounds__(256) void move_kernel(Move4 a, FastDiv div_lanes, int lanes, int blocks) {
    __shared__ int source[64], page[64];     // of a place's token, page -1: none
    const int head = (int)blockIdx.y, b = (int)blockIdx.x / blocks, i0 = ((int)blockIdx.x - b * blocks) * 64;
    const int room = a.into_pages << a.c.page_shift;
    const long long list = ((long long)b * a.c.kv_heads + head) * a.keep;
    if (threadIdx.x < 64) {
        const int i = i0 + (int)threadIdx.x;
        const int j = i < a.keep && i < room ? a.tokens[list + i] : -1;
        const bool weighed = a.weights != nullptr && i < room;
        const float w = weighed && j >= 0 && j < a.width ? a.weights[((long long)b * a.c.kv_heads + head) * a.width + j] : 0.f;         // (under way beside the page)
        const int p = j >= 0 && j >> a.c.page_shift < a.table_pages ? a.table[(long long)b * a.table_pages + (j >> a.c.page_shift)] : -1;
        source[threadIdx.x] = j;
        const bool there = (uint32_t)p < (uint32_t)a.c.pages;
        page[threadIdx.x] = there ? p : -1;
        if (weighed) a.moved[((long long)b * a.c.kv_heads + head) * room + i] = there ? w : 0.f;
    }
    __syncthreads();
    for (int n = (int)threadIdx.x; n < 64 * lanes; n += 256) {
        const int t = fast_div(n, div_lanes), at = n - t * lanes, i = i0 + t, j = source[t], p = page[t];
        if (p < 0) continue;
        const int r = a.into[(long long)b * a.into_pages + (i >> a.c.page_shift)];
        if ((uint32_t)r >= (uint32_t)a.c.pages) continue;
        const uint8_t* from = c4_record(a.c, p, head);
        uint8_t* to = c4_record(a.c, r, head);
        const int fo = j & (a.c.page - 1), o = i & (a.c.page - 1), bytes = a.c.dim / 2;
        // lane `at` of a token has its elements 32 at .. + 31: 16 bytes of codes, one scale and four bytes of signs
        *reinterpret_cast<u32x4*>(to + o * bytes + 16 * at) = *reinterpret_cast<const u32x4*>(from + fo * bytes + 16 * at);
        *reinterpret_cast<u32x4*>(to + a.c.v_codes + o * bytes + 16 * at) = *reinterpret_cast<const u32x4*>(from + a.c.v_codes + fo * bytes + 16 * at);
        to[a.c.k_exps + at * a.c.page + o] = from[a.c.k_exps + at * a.c.page + fo];
        to[a.c.v_exps + at * a.c.page + o] = from[a.c.v_exps + at * a.c.page + fo];
        if (a.c.signs) *reinterpret_cast<uint32_t*>(to + a.c.signs + o * (a.c.dim / 8) + 4 * at) = *reinterpret_cast<const uint32_t*>(from + a.c.signs + fo * (a.c.dim / 8) + 4 * at);
    }
}

}  // namespace

HeaviestPlan4 plan_cache4_heaviest(const Cache4& c, int batch, int table_pages) {
    HeaviestPlan4 p = {};
    const long long room = (long long)table_pages << c.page_shift, units = (long long)batch * c.kv_heads, parts = cdiv(room, H_WAVES * 2 * H_VECTOR);
    // (Parts take 17 us and 0.065 for each, one workgroup to a sequence and head 7.6 for every 8192 of its tokens: 8 sequences of 65536, 8 heads, 49 us in parts, 63 without; 16 of them 83 and 67; 64 of them 244 and 171.
    // By the table's room: 8 sequences of 4000 tokens take 9 us in a table of 4096 and 50 in one of 131072.)
    if (room <= 32768 || units > 80) return p;
    p.parts = (int)parts;
    p.bins_bytes = (size_t)units * 3 * parts * H_BINS * sizeof(int);
    p.borders_bytes = (size_t)units * 3 * sizeof(Border);
    p.workspace_bytes = p.bins_bytes + p.borders_bytes + (size_t)units * 3 * parts * sizeof(int);
    return p;
}

int launch_cache4_heaviest(const Heaviest4& a, const HeaviestPlan4& plan, void* workspace, hipStream_t s) {
    if (plan.parts > 0) {
        const Parts4 p = {plan.parts, static_cast<int*>(workspace), reinterpret_cast<Border*>(static_cast<char*>(workspace) + plan.bins_bytes),
                          reinterpret_cast<int*>(static_cast<char*>(workspace) + plan.bins_bytes + plan.borders_bytes)};
        const dim3 grid((unsigned)p.parts, (unsigned)a.c.kv_heads, (unsigned)a.batch);
        launch(heaviest_part_kernel<0>, grid, dim3(H_THREADS), 0, s, a, p);
        launch(heaviest_part_kernel<1>, grid, dim3(H_THREADS), 0, s, a, p);
        launch(heaviest_part_kernel<2>, grid, dim3(H_THREADS), 0, s, a, p);
        launch(heaviest_part_kernel<3>, grid, dim3(H_THREADS), 0, s, a, p);
        return check_launch();
    }
    const dim3 grid((unsigned)a.batch, (unsigned)a.c.kv_heads);
    const long long vectors = cdiv((long long)a.table_pages << a.c.page_shift, H_WAVES * H_VECTOR);
    if (vectors <= 2) launch(heaviest_kernel<2>, grid, dim3(H_THREADS), 0, s, a);
    else if (vectors <= 8) launch(heaviest_kernel<8>, grid, dim3(H_THREADS), 0, s, a);
    else launch(heaviest_kernel<0>, grid, dim3(H_THREADS), 0, s, a);
    return check_launch();
}

int launch_cache4_move(const Move4& a, hipStream_t s) {
    const int lanes = a.c.dim / 32;
    const long long blocks = cdiv((long long)a.into_pages << a.c.page_shift, 64);
    if (blocks * a.batch >= C4_THREADS / 256) return BNN_ERR_UNSUPPORTED;
    launch(move_kernel, dim3((unsigned)(blocks * a.batch), (unsigned)a.c.kv_heads), dim3(256), 0, s, a, make_fastdiv((uint32_t)lanes), lanes, (int)blocks);
    return check_launch();
}

}  // namespace bnn
