// Eviction: which cached tokens to keep, by their weights, and moving them into other pages.
//
// heaviest_kernel: a workgroup has a sequence and kv head.  Weights in the order of numbers are whole numbers in the order of their bits (negative ones turned round); the weight of the last token that
// is kept is found digit by digit, from the highest on: a histogram of the digit over what agrees so far, 11 + 11 + 10 bits.  Of those that equal it the lowest tokens are kept.  A wave has a run of
// consecutive tokens, so one exchange of counts gives every wave the place of its first kept token, and the list is ascending.
// move_kernel: a workgroup has a kv head and 64 places of the new sequence.
#include "bnn_cache4.h"

namespace bnn {
namespace {

constexpr int H_THREADS = 1024, H_WAVES = H_THREADS / 64, H_BINS = 2048;

// The order of weights as that of whole numbers; NaN below all.  -0 counts as 0.
__device__ __forceinline__ uint32_t rank_of(float w) {
    if (w != w) return 0;
    const uint32_t bits = __float_as_uint(w + 0.f);
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}

__global__ __launch_bounds__(H_THREADS) void heaviest_kernel(Heaviest4 a) {
    __shared__ int bins[H_BINS];
    __shared__ int wave_above[H_WAVES], wave_equal[H_WAVES], wave_there[H_WAVES];
    __shared__ int picked[3];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int b = (int)blockIdx.x, head = (int)blockIdx.y;
    const int length = (int)min((long long)max(a.lens[b], 0), (long long)a.table_pages << a.c.page_shift);
    const int run = (int)(((long long)length + H_WAVES * 64 - 1) / (H_WAVES * 64)) * 64;          // tokens of a wave
    const int begin = (int)min((long long)wave * run, (long long)length), end = (int)min((long long)begin + run, (long long)length);
    const float* weights = a.weights + ((long long)b * a.c.kv_heads + head) * a.width;
    const int32_t* table = a.table + (long long)b * a.table_pages;
    int32_t* out = a.tokens + ((long long)b * a.c.kv_heads + head) * a.keep;
    // 0: nowhere; kept in any case: the highest; else a number between
    auto rank = [&](int j) -> uint32_t {
        if (j >= end || (uint32_t)table[j >> a.c.page_shift] >= (uint32_t)a.c.pages) return 0;
        if (j < a.first || j >= length - a.last) return 0xffffffffu;
        return min(max(rank_of(weights[j]), 1u), 0xfffffffeu);
    };

    int there = 0;
    for (int j = begin + lane; j - lane < end; j += 64) there += __popcll(__ballot(rank(j) != 0));
    if (lane == 0) wave_there[wave] = there;
    __syncthreads();
    there = 0;
    for (int w = 0; w < H_WAVES; ++w) there += wave_there[w];
    const int kept = min(there, a.keep);
    if (head == 0 && threadIdx.x == 0) a.kept[b] = kept;

    // The lowest rank that is kept, and how many of that rank
    uint32_t border = 1;
    int of_border = 0x7fffffff;
    if (there > a.keep) {
        uint32_t prefix = 0;
        int need = a.keep;                   // of those that agree with prefix so far
        for (int digit = 0; digit < 3; ++digit) {
            const int shift = digit == 0 ? 21 : digit == 1 ? 10 : 0, width = digit == 2 ? 10 : 11;
            for (int i = (int)threadIdx.x; i < H_BINS; i += H_THREADS) bins[i] = 0;
            __syncthreads();
            for (int j = begin + lane; j < end; j += 64) {
                const uint32_t r = rank(j);
                if (r != 0 && (digit == 0 || r >> (shift + width) == prefix >> (shift + width))) atomicAdd(&bins[r >> shift & ((1u << width) - 1)], 1);
            }
            __syncthreads();
            if (wave == 0) {                 // from the highest bin down: the one in which the count passes need
                int above = 0;
                for (int top = (1 << width) - 64; top >= 0; top -= 64) {
                    const int n = bins[top + 63 - lane];
                    int upto = n;
#pragma unroll
                    for (int d = 1; d < 64; d <<= 1) {
                        const int other = __shfl_up(upto, d);
                        if (lane >= d) upto += other;
                    }
                    const unsigned long long past = __ballot(above + upto >= need);
                    if (past != 0) {
                        const int at = __ffsll(past) - 1;
                        if (lane == at) {
                            picked[0] = top + 63 - lane;
                            picked[1] = need - (above + upto - n);
                        }
                        break;
                    }
                    above += __shfl(upto, 63);
                }
            }
            __syncthreads();
            prefix |= (uint32_t)picked[0] << shift;
            need = picked[1];
        }
        border = prefix;
        of_border = need;
    }

    int above = 0, equal = 0;
    for (int j = begin + lane; j - lane < end; j += 64) {
        const uint32_t r = rank(j);
        above += __popcll(__ballot(r > border));
        equal += __popcll(__ballot(r == border));
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
    const unsigned long long below = (1ull << lane) - 1;
    for (int j = begin + lane; j - lane < end; j += 64) {
        const uint32_t r = rank(j);
        const unsigned long long e = __ballot(r == border);
        const bool keep = r > border || (r == border && equals + __popcll(e & below) < of_border);
        equals += __popcll(e);
        const unsigned long long k = __ballot(keep);
        if (keep) out[place + __popcll(k & below)] = j;
        place += __popcll(k);
    }
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
    launch(heaviest_kernel, dim3((unsigned)a.batch, (unsigned)a.c.kv_heads), dim3(H_THREADS), 0, s, a);
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
