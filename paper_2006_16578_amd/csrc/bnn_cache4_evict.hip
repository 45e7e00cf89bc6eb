// Eviction: which cached tokens to keep, by their weights, and moving them into other pages.
//
// heaviest_kernel: a workgroup has a sequence and kv head.  Weights in the order of numbers are whole numbers in the order of their bits (negative ones turned round); that of the last token that
// is kept is found digit by digit, from the highest on: a histogram of the digit over what agrees so far, 11 + 11 + 10 bits.  Of those that equal it the lowest tokens are kept.  A wave has a run of
// consecutive tokens, a lane four beside each other, so one exchange of counts gives every wave the place of its first kept token, and the list is ascending.  Weights are read once and stay in
// registers where the table has room for up to 65536 tokens; beyond, they are read five times, eight loads under way.
// move_kernel: a workgroup has a kv head and 64 places of the new sequence.
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

// E: vectors of a wave that its registers hold; 0: none.
template <int E>
__global__ __launch_bounds__(H_THREADS) void heaviest_kernel(Heaviest4 a) {
    constexpr int LOADS = E == 0 ? 8 : E;    // under way together
    __shared__ int bins[H_BINS];
    __shared__ int wave_above[H_WAVES], wave_equal[H_WAVES], wave_there[H_WAVES], wave_sum[H_WAVES];
    __shared__ int picked[2];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int b = (int)blockIdx.x, head = (int)blockIdx.y;
    const int length = (int)min((long long)max(a.lens[b], 0), (long long)a.table_pages << a.c.page_shift);
    const int run = (length + H_WAVES * H_VECTOR - 1) / (H_WAVES * H_VECTOR);     // vectors of a wave
    const int begin = min(wave * run * H_VECTOR, length), end = min(begin + run * H_VECTOR, length);
    const float* weights = a.weights + ((long long)b * a.c.kv_heads + head) * a.width;
    const int32_t* table = a.table + (long long)b * a.table_pages;
    int32_t* out = a.tokens + ((long long)b * a.c.kv_heads + head) * a.keep;

    // Four tokens of a lane.  (Pages and tables have room for multiples of 16: what begins inside lies inside.)
    struct Four {
        f32x4 weight;
        int page;
    };
    auto fetch = [&](int j) -> Four {
        Four f = {f32x4{0.f, 0.f, 0.f, 0.f}, -1};
        if (j < end) {
            __builtin_memcpy(&f.weight, weights + j, 16);
            f.page = table[j >> a.c.page_shift];
        }
        return f;
    };
    // 0: nowhere; kept in any case: the highest; else a number between
    auto rank = [&](const Four& f, int j, uint32_t (&r)[4]) {
        const bool there = (uint32_t)f.page < (uint32_t)a.c.pages;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int t = j + i;
            r[i] = t < a.first || t >= length - a.last ? 0xffffffffu : min(max(rank_of(f.weight[i]), 1u), 0xfffffffeu);
            if (!there || t >= end) r[i] = 0;
        }
    };
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

    // The lowest rank that is kept, and how many of that rank
    uint32_t border = 1;
    int of_border = 0x7fffffff;
    if (there > a.keep) {
        border = 0;
        of_border = a.keep;                  // of those that agree with border so far
        for (int digit = 0; digit < 3; ++digit) {
            const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, width = digit == 2 ? 10 : 11;
            if (digit > 0) {
                for (int i = (int)threadIdx.x; i < H_BINS; i += H_THREADS) bins[i] = 0;
                __syncthreads();
                for_each([&](const uint32_t (&r)[4], int) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (r[i] != 0 && r[i] >> (shift + width) == border >> (shift + width)) atomicAdd(&bins[r[i] >> shift & ((1u << width) - 1)], 1);
                });
                __syncthreads();
            }
            // From the highest bin down, two to a thread: the one in which the count reaches of_border
            const int top = H_BINS - 1 - 2 * (int)threadIdx.x, high = bins[top], low = bins[top - 1];
            int upto = high + low;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int other = __shfl_up(upto, d);
                if (lane >= d) upto += other;
            }
            if (lane == 63) wave_sum[wave] = upto;
            __syncthreads();
            for (int w = 0; w < wave; ++w) upto += wave_sum[w];
            const int before = upto - high - low;
            if (before < of_border && upto >= of_border) {
                const bool first = before + high >= of_border;
                picked[0] = first ? top : top - 1;
                picked[1] = of_border - before - (first ? 0 : high);
            }
            __syncthreads();
            border |= (uint32_t)picked[0] << shift;
            of_border = picked[1];
        }
    }

    int above = 0, equal = 0;
    for_each([&](const uint32_t (&r)[4], int) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            above += r[i] > border ? 1 : 0;
            equal += r[i] == border ? 1 : 0;
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
    place += min(equals, of_border);
    // lanes before this one, in a mask
    auto before = [](unsigned long long mask) { return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); };
    for_each([&](const uint32_t (&r)[4], int j) {
        bool keep[4];
        unsigned long long e[4], any = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            e[i] = __ballot(r[i] == border);
            any |= e[i];
            keep[i] = r[i] > border;
        }
        if (any != 0) {                      // which of those at the border: the lowest
            int n = equals + before(e[0]) + before(e[1]) + before(e[2]) + before(e[3]);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (r[i] == border) {
                    keep[i] = n < of_border;
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
    });
    for (int i = kept + (int)threadIdx.x; i < a.keep; i += H_THREADS) out[i] = -1;
}

// A thread moves 16 bytes of codes, K's and V's, the lanes of a token side by side; scales and signs go a byte or word at a time.
__global__ __launch_bounds__(256) void move_kernel(Move4 a, FastDiv div_lanes, int lanes, int blocks) {
    __shared__ int source[64];
    const int head = (int)blockIdx.y, b = (int)blockIdx.x / blocks, i0 = ((int)blockIdx.x - b * blocks) * 64;
    const int room = a.into_pages << a.c.page_shift;
    const long long list = ((long long)b * a.c.kv_heads + head) * a.keep;
    if (threadIdx.x < 64) {
        const int i = i0 + (int)threadIdx.x;
        const int j = i < a.keep && i < room ? a.tokens[list + i] : -1;
        source[threadIdx.x] = j;
        if (a.weights != nullptr && i < room)
            a.moved[((long long)b * a.c.kv_heads + head) * room + i] = j >= 0 && j < a.width ? a.weights[((long long)b * a.c.kv_heads + head) * a.width + j] : 0.f;
    }
    __syncthreads();
    for (int n = (int)threadIdx.x; n < 64 * lanes; n += 256) {
        const int t = fast_div(n, div_lanes), at = n - t * lanes, i = i0 + t, j = source[t];
        if (j < 0 || j >> a.c.page_shift >= a.table_pages) continue;
        const int p = a.table[(long long)b * a.table_pages + (j >> a.c.page_shift)], r = a.into[(long long)b * a.into_pages + (i >> a.c.page_shift)];
        if ((uint32_t)p >= (uint32_t)a.c.pages || (uint32_t)r >= (uint32_t)a.c.pages) continue;
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

int launch_cache4_heaviest(const Heaviest4& a, hipStream_t s) {
    const dim3 grid((unsigned)a.batch, (unsigned)a.c.kv_heads);
    const long long vectors = cdiv((long long)a.table_pages << a.c.page_shift, H_WAVES * H_VECTOR);
    if (vectors <= 2) launch(heaviest_kernel<2>, grid, dim3(H_THREADS), 0, s, a);
    else if (vectors <= 8) launch(heaviest_kernel<8>, grid, dim3(H_THREADS), 0, s, a);
    else if (vectors <= 16) launch(heaviest_kernel<16>, grid, dim3(H_THREADS), 0, s, a);
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
