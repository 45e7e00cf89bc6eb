// What a head's sums say: log probabilities of given tokens, entropy, the best alternatives, in one pass over the logits.
//
// With a reference point m and u = (x - m) scale / log 2, S = sum 2^u and W = sum 2^u u give
//   log p = scale (x - m) - log S,  entropy = log S - log 2 W / S  (both terms >= 0),  lse = scale m + log S,
// and with m the row's largest column no difference of large numbers is left: that column's own term is 1 exactly, S is 1 or more, and a sure row's results are right relative to themselves.  A wave's m is the
// largest column that it has met.  One branch for four vectors raises it: few groups do, as the longer a row is the rarer a new largest one gets (with m let stay behind by up to 16 powers of two, 4096 rows of 131072 take 210 us in
// place of 211, ascending ones 498 in place of 501, but sure rows lose log p and entropy to the difference of two numbers near 11).  Waves and pieces of a row are joined by the same rule.  What bounds it is memory: 10 instruction slots a column (an exponential counts four) take about four fifths of the time that its
// two bytes take.  4096 rows of 131072 bf16 columns (1.07 GB): 194 us, 5.5 TB/s.  (With a piece of a row held in registers between a pass for the maximum and one for the sums 816 us.)  The smallest calls, 8 rows of 131072
// columns in 256 pieces, are two launches: 6.8 us for the pieces and 6 for the join, chains of loads and barriers.
//
// The `top` best: beside that, every thread keeps the largest of each eight of its vectors.  The `top`-th largest of the threads' maxima is a border that at least `top` columns reach and little more do;
// the vectors' maxima tell where those are, and they are read again, collected in LDS and ranked by counting.  Columns are ordered by (value, lower column first) as one 64-bit number.  Where a border is shared
// by many, what is above it is collected, and then what equals it from the lowest column on; where the best lie so close together in one thread's columns that the list overflows, the
// border is found digit by digit over all columns.
#include <math.h>

#include "bnn_cache4.h"

namespace bnn {
namespace {

constexpr int LP_MAX_TOP = 64;
constexpr float LP_LOG2E = 1.4426950408889634f, LP_LN2 = 0.6931471805599453f;

struct Logprobs {
    const void* x;
    int rows, cols;
    long long ld;
    float scale, scale2;                     // scale2: scale / log 2
    const int64_t* targets;
    int top;
    float *logprobs, *entropy, *lse, *top_logprobs;
    int32_t* top_tokens;
    int pieces;                              // of a row
    FastDiv div_pieces;
    int vectors;                             // of 16 bytes, that a thread has of a piece
    f32x4* sums;                             // [rows][pieces]: m, S, W; with several pieces
    uint64_t* best;                          // [rows][pieces][top], descending, the rest 0
};

// Numbers in the order of the values (no NaN), 0 for none; and back.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t bits = __float_as_uint(x + 0.f);                  // (no -0)
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order); }
__device__ __forceinline__ uint64_t key_of(float x, int col) { return (uint64_t)order_of(x) << 32 | (uint32_t)~col; }

template <class T> __device__ __forceinline__ float as_float(T v) { return (float)v; }

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// A row's target.  (The join loads it ahead of its sums.)
struct Judged {
    bool is;                                 // within the columns
    float x;
};
template <class T>
__device__ __forceinline__ Judged load_judged(const Logprobs& a, int row) {
    Judged j = {false, 0.f};
    if (a.targets == nullptr) return j;
    const int64_t t = a.targets[row];
    j.is = t >= 0 && t < a.cols;
    if (j.is) j.x = as_float(static_cast<const T*>(a.x)[row * a.ld + t]);
    return j;
}

// The results of a row from its reference point and sums, by thread 0 of `threads` that have the row; best(i): its alternatives.
template <class Best>
__device__ __forceinline__ void finish_row(const Logprobs& a, int row, const Judged& judged, float m, float S, float W, int thread, int threads, Best best) {
    const bool none = !(S > 0.f);            // S is NaN, or 0: no distribution
    const float log_s = __builtin_amdgcn_logf(S) * LP_LN2, nan = __builtin_nanf("");
    if (thread == 0) {
        if (a.lse != nullptr) a.lse[row] = none ? (S == 0.f ? -__builtin_inff() : nan) : fmaf(m, a.scale, log_s);
        if (a.entropy != nullptr) a.entropy[row] = none ? nan : log_s - LP_LN2 * (W / S);
        if (a.targets != nullptr) a.logprobs[row] = !judged.is ? 0.f : none ? nan : fmaf(judged.x - m, a.scale, -log_s);
    }
    for (int i = thread; i < a.top; i += threads) {
        const uint64_t key = best(i);
        a.top_logprobs[(long long)row * a.top + i] = none ? nan : fmaf(value_of((uint32_t)(key >> 32)) - m, a.scale, -log_s);
        a.top_tokens[(long long)row * a.top + i] = none || key == 0 ? -1 : (int32_t)~(uint32_t)key;
    }
}

// Rows of up to 512 columns, of which few best are wanted: a wave has one, eight columns a lane (or two); the best come one after another, the largest of all lanes each.
// 8000 rows of 7 columns, 2 best: 7.2 us, 25.9 with a workgroup to a row; of 500 columns without any 6.8 and 23, with 16 best 35 and 41; but 20 rows with 16 best 11.5 and 7.7.
constexpr int LP_SHORT = 512;
template <class T, int N, bool TOP>
__global__ __launch_bounds__(256) void logprobs_short_kernel(Logprobs a) {
    const int lane = (int)threadIdx.x & 63, row = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (row >= a.rows) return;
    const T* x = static_cast<const T*>(a.x) + row * a.ld;
    const Judged judged = load_judged<T>(a, row);
    float y[N];
#pragma unroll
    for (int i = 0; i < N; ++i) y[i] = lane + 64 * i < a.cols ? as_float(x[lane + 64 * i]) : -__builtin_inff();
    float m = y[0];
#pragma unroll
    for (int i = 1; i < N; ++i) m = fmaxf(m, y[i]);
    m = wave_max(m);
    if (!(m > -__builtin_inff())) m = 0.f;   // (all NaN too)
    float S = 0.f, W = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float u = (y[i] - m) * a.scale2, e = __builtin_amdgcn_exp2f(u);
        S += e;
        W = fmaf(e, fmaxf(u, -1e30f), W);
    }
    S = wave_sum(S);
    W = wave_sum(W);
    uint64_t mine = 0;                       // the lane's of the best
    if constexpr (TOP) {
        uint64_t key[N];
#pragma unroll
        for (int i = 0; i < N; ++i) key[i] = lane + 64 * i < a.cols && y[i] == y[i] ? key_of(y[i], lane + 64 * i) : 0;
        for (int t = 0; t < a.top; ++t) {
            uint64_t high = key[0];
#pragma unroll
            for (int i = 1; i < N; ++i) high = key[i] > high ? key[i] : high;
#pragma unroll
            for (int d = 32; d > 0; d >>= 1) {
                const uint64_t other = __shfl_xor((unsigned long long)high, d);
                high = other > high ? other : high;
            }
#pragma unroll
            for (int i = 0; i < N; ++i) key[i] = key[i] == high ? 0 : key[i];
            mine = lane == t ? high : mine;
        }
    }
    finish_row(a, row, judged, m, S, W, lane, 64, [&](int) { return mine; });
}

// The `top` largest of list[0 .. n) to out, descending, 0 where there are fewer.  All different.  Called by all 256 threads; out is complete after the next barrier.
__device__ __forceinline__ void rank_keys(const uint64_t* list, int n, int top, uint64_t* out) {
    for (int i = n + (int)threadIdx.x; i < top; i += 256) out[i] = 0;
    for (int i = (int)threadIdx.x; i < n; i += 256) {
        const uint64_t mine = list[i];
        int above = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) above += list[j] > mine ? 1 : 0;
        if (above < top) out[above] = mine;
    }
}

constexpr int LP_VECTORS = 64, LP_SEGMENT = 8, LP_KEYS = 1024;       // vectors of a thread at most; those that share a maximum; the list's places

// A thread's column of a piece: vector v of the piece begins at column first + 256 * V * v.  col may lie before 0 (rows need not begin at 16 bytes) or behind the last.
template <class T, int V>
__device__ __forceinline__ void load_columns(const Logprobs& a, const T* x, int col, float (&y)[V]) {
    typedef T TV __attribute__((ext_vector_type(V)));
    if (col >= 0 && col + V <= a.cols) {
        const TV w = *reinterpret_cast<const TV*>(x + col);
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = as_float(w[j]);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) y[j] = col + j >= 0 && col + j < a.cols ? as_float(x[col + j]) : -__builtin_inff();
    }
}

// The number of threads for which `mine` holds, to all of them; scratch: 4 ints.
__device__ __forceinline__ int block_count(int n, int* scratch) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) n += __shfl_xor(n, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = n;
    __syncthreads();
    return scratch[0] + scratch[1] + scratch[2] + scratch[3];
}

// The best of a piece.  maxima[s][t]: the largest of thread t's vectors 8 s .. + 7.  best: `top` keys in order, 0 where there are fewer.
template <class T>
__device__ __forceinline__ void best_of_piece(const Logprobs& a, const T* x, int piece_first, int vectors, const float (*maxima)[256], uint16_t* pairs, uint64_t* list, uint64_t* best, int* ints) {
    constexpr int V = 16 / sizeof(T);
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), tid = (int)threadIdx.x;
    const int segments = (vectors + LP_SEGMENT - 1) / LP_SEGMENT, first = piece_first + tid * V;
    int &count = ints[0], &pair_count = ints[7], *scan = ints + 1, *found = ints + 5;
    float high = -__builtin_inff();
    for (int s = 0; s < segments; ++s) high = fmaxf(high, maxima[s][tid]);
    const uint32_t mine = first < a.cols ? order_of(high) : 0;       // 0: no columns
    uint32_t* orders = reinterpret_cast<uint32_t*>(list);
    orders[tid] = mine;
    if (tid == 0) count = pair_count = 0;
    __syncthreads();
    // The largest number that `top` of the threads' maxima reach; the search ends early where few more do
    const int few = a.top + a.top / 2 + 1;
    if (wave == 0) {
        uint32_t o[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = orders[lane + 64 * i];
        uint32_t border = 0;
        int reach = 256;
        for (int bit = 31; bit >= 0 && reach > few; --bit) {
            const uint32_t t = border | 1u << bit;
            int n = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) n += __popcll(__ballot(o[i] >= t));
            if (n >= a.top) {
                border = t;
                reach = n;
            }
        }
        if (lane == 0) {
            found[0] = (int)border;
            found[1] = reach;
        }
    }
    __syncthreads();
    uint32_t border = (uint32_t)found[0];
    bool ties = found[1] > few;              // then border is exact, and fewer than `top` threads have more than it
    // What passes the border: first which maxima do, then the columns behind them: a column to a thread, or, where these are many (352 rows of 32410, 64 best,
    // 33 -> 27 us), a vector (8 rows of 131072, 20 best, 12.2 -> 12.9).
    auto collect = [&]() {
        for (int s = 0; s < segments; ++s) {
            const uint32_t o = first < a.cols ? order_of(maxima[s][tid]) : 0;
            if (ties ? o > border : o >= border && o != 0) pairs[atomicAdd(&pair_count, 1)] = (uint16_t)(s << 8 | tid);
        }
        __syncthreads();
        const int wide = vectors > 4 ? 3 : vectors > 2 ? 2 : vectors > 1 ? 1 : 0;      // 2^wide vectors at least are behind a maximum
        const int n = pair_count << wide;
        auto take = [&](float y, int col) {
            const uint32_t o = order_of(y);
            if (y == y && (ties ? o > border : o >= border)) {
                const int at = atomicAdd(&count, 1);
                if (at < LP_KEYS) list[at] = key_of(y, col);
            }
        };
        if (n * V <= 1024) {
            for (int i = tid; i < n * V; i += 256) {
                const int pair = pairs[i / V >> wide], v = (pair >> 8) * LP_SEGMENT + (i / V & ((1 << wide) - 1));
                const int col = piece_first + (v * 256 + (pair & 255)) * V + i % V;
                if (v < vectors && col >= 0 && col < a.cols) take(as_float(x[col]), col);
            }
        } else {
            for (int i = tid; i < n; i += 256) {
                const int pair = pairs[i >> wide], v = (pair >> 8) * LP_SEGMENT + (i & ((1 << wide) - 1));
                const int col = piece_first + (v * 256 + (pair & 255)) * V;
                if (v >= vectors) continue;
                float y[V];
                load_columns<T, V>(a, x, col, y);
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (col + k >= 0 && col + k < a.cols) take(y[k], col + k);
            }
        }
    };
    collect();
    __syncthreads();
    int have = count;
    if (have > LP_KEYS) {                    // the best lie together: the border digit by digit, over all columns
        border = 0;
        ties = true;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t t = border | 1u << bit;
            int n = 0;
            for (int v = 0; v < vectors; ++v) {
                float y[V];
                load_columns<T, V>(a, x, first + 256 * V * v, y);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int col = first + 256 * V * v + j;
                    n += y[j] == y[j] && order_of(y[j]) >= t && col >= 0 && col < a.cols ? 1 : 0;
                }
            }
            if (block_count(n, scan) >= a.top) border = t;
        }
        __syncthreads();
        if (tid == 0) count = pair_count = 0;
        __syncthreads();
        collect();                           // fewer than `top`
        __syncthreads();
        have = count;
    }
    if (ties && have < a.top) {              // what equals the border, from the lowest column on
        for (int v = 0; v < vectors && have < a.top; ++v) {
            float y[V];
            load_columns<T, V>(a, x, first + 256 * V * v, y);
            int n = 0;
            unsigned equal = 0;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const int col = first + 256 * V * v + j;
                if (y[j] == y[j] && order_of(y[j]) == border && col >= 0 && col < a.cols) equal |= 1u << j;
            }
            n = __popc(equal);
            int upto = n;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int other = __shfl_up(upto, d);
                if (lane >= d) upto += other;
            }
            if (lane == 63) scan[wave] = upto;
            __syncthreads();
            int at = have + upto - n;
            for (int w = 0; w < wave; ++w) at += scan[w];
#pragma unroll
            for (int j = 0; j < V; ++j)
                if (equal >> j & 1) {
                    if (at < a.top) list[at] = key_of(y[j], first + 256 * V * v + j);
                    ++at;
                }
            have += scan[0] + scan[1] + scan[2] + scan[3];
            __syncthreads();
        }
        have = min(have, a.top);
    }
    __syncthreads();
    rank_keys(list, have, a.top, best);
    __syncthreads();
}

// NV: vectors of a thread that are computed together, while as many of the next are loaded.
template <class T, int NV, bool TOP>
__global__ __launch_bounds__(256) void logprobs_kernel(Logprobs a) {
    constexpr int V = 16 / sizeof(T);
    typedef T TV __attribute__((ext_vector_type(V)));
    __shared__ float part[3][4];
    __shared__ float maxima[TOP ? LP_VECTORS / LP_SEGMENT : 1][256];
    __shared__ uint64_t list[TOP ? LP_KEYS : 1], best[TOP ? LP_MAX_TOP : 1];
    __shared__ uint16_t pairs[TOP ? 256 * LP_VECTORS / LP_SEGMENT : 1];
    __shared__ int ints[8];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int row = fast_div((int)blockIdx.x, a.div_pieces), piece = (int)blockIdx.x - row * a.pieces;
    const T* x = static_cast<const T*>(a.x) + row * a.ld;
    const int off = (int)(reinterpret_cast<uintptr_t>(x) / sizeof(T) % V);          // columns before the first whole 16 bytes lie in vector 0
    const int piece_first = piece * a.vectors * (256 * V) - off, first = piece_first + (int)threadIdx.x * V;
    const int vectors = min(a.vectors, (a.cols - piece_first + 256 * V - 1) / (256 * V));       // with columns
    const float c = a.scale2;

    float most = -__builtin_inff(), m = 0.f, S = 0.f, W = 0.f;       // most: the largest column so far, m too, but for 0 in place of -infinity
    float segment = -__builtin_inff();
    auto group = [&](const float (&y)[NV][V], int v0) {
        float high = -__builtin_inff();
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float h = y[v][0];
#pragma unroll
            for (int j = 1; j < V; ++j) h = fmaxf(h, y[v][j]);
            high = fmaxf(high, h);
        }
        if (__ballot(high > most) != 0) {
            const float top = wave_max(high), d = most == -__builtin_inff() ? 0.f : (m - top) * c, f = __builtin_amdgcn_exp2f(d);
            W = f * fmaf(S, fmaxf(d, -1e30f), W);
            S *= f;
            m = most = top;
        }
        if constexpr (TOP) {
            segment = fmaxf(segment, high);
            if (v0 % LP_SEGMENT + NV == LP_SEGMENT || v0 + NV >= vectors) {
                maxima[v0 / LP_SEGMENT][threadIdx.x] = segment;
                segment = -__builtin_inff();
            }
        }
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float u = (y[v][j] - m) * c, e = __builtin_amdgcn_exp2f(u);
                S += e;
                W = fmaf(e, fmaxf(u, -1e30f), W);
            }
    };
    // Groups of vectors whose columns all exist: [from, to)
    const int groups = (vectors + NV - 1) / NV, from = piece_first < 0 ? 1 : 0, to = max(from, min(groups, (a.cols - piece_first) / (256 * V * NV)));
    auto edge = [&](int g) {
        float y[NV][V];
#pragma unroll
        for (int v = 0; v < NV; ++v) load_columns<T, V>(a, x, first + (g * NV + v) * 256 * V, y[v]);
        group(y, g * NV);
    };
    if (from > 0 && groups > 0) edge(0);
    if (from < to) {
        TV next[NV];
#pragma unroll
        for (int v = 0; v < NV; ++v) next[v] = *reinterpret_cast<const TV*>(x + first + (from * NV + v) * 256 * V);
        for (int g = from; g < to; ++g) {
            float y[NV][V];
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < V; ++j) y[v][j] = as_float(next[v][j]);
            if (g + 1 < to) {
#pragma unroll
                for (int v = 0; v < NV; ++v) next[v] = *reinterpret_cast<const TV*>(x + first + ((g + 1) * NV + v) * 256 * V);
            }
            group(y, g * NV);
        }
    }
    for (int g = max(from, to); g < groups; ++g) edge(g);

    // Lanes of a wave share m
    S = wave_sum(S);
    W = wave_sum(W);
    if (lane == 0) {
        part[0][wave] = most;
        part[1][wave] = S;
        part[2][wave] = W;
    }
    __syncthreads();
    if constexpr (TOP) best_of_piece<T>(a, x, piece_first, vectors, maxima, pairs, list, best, ints);
    m = fmaxf(fmaxf(part[0][0], part[0][1]), fmaxf(part[0][2], part[0][3]));
    if (m == -__builtin_inff()) m = 0.f;
    S = 0.f;
    W = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (part[1][w] == 0.f) continue;     // (NaN goes on)
        const float d = (part[0][w] - m) * c, f = __builtin_amdgcn_exp2f(d);
        S = fmaf(part[1][w], f, S);
        W = fmaf(f, fmaf(part[1][w], fmaxf(d, -1e30f), part[2][w]), W);
    }
    if (a.pieces == 1) {
        finish_row(a, row, load_judged<T>(a, row), m, S, W, (int)threadIdx.x, 256, [&](int i) { return best[i]; });
    } else {
        if (threadIdx.x == 0) a.sums[blockIdx.x] = f32x4{m, S, W, 0.f};
        if constexpr (TOP)
            for (int i = (int)threadIdx.x; i < a.top; i += 256) a.best[(long long)blockIdx.x * a.top + i] = best[i];
    }
}

constexpr int LP_LIST = 2048;                // keys that are looked at together

// Joins the pieces of a row.  Each piece's best come in order; of L pieces the ceil(top / L) best each are at least `top`, and the `top`-th of those is a border that little more reach.
template <class T>
__global__ __launch_bounds__(256) void logprobs_join_kernel(Logprobs a) {
    __shared__ uint64_t list[LP_LIST], reach[LP_LIST], best[LP_MAX_TOP];
    uint64_t* const heads = reach;           // (before it has what reaches the border)
    __shared__ float part[3][4];
    __shared__ uint64_t border;
    __shared__ int count;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int row = (int)blockIdx.x;
    // What is needed last is loaded first: the target, and the best of as many pieces as are looked at together
    const Judged judged = load_judged<T>(a, row);
    const uint64_t* from = a.best + (long long)row * a.pieces * a.top;
    const int together = a.top > 0 ? LP_LIST / a.top : 0, first_keys = min(together, a.pieces) * a.top;      // pieces, the best so far counting as one
    uint64_t ahead[LP_LIST / 256];
#pragma unroll
    for (int i = 0; i < LP_LIST / 256; ++i) {
        ahead[i] = 0;
        if (256 * i + (int)threadIdx.x < first_keys) ahead[i] = from[256 * i + threadIdx.x];
    }
    const f32x4* sums = a.sums + (long long)row * a.pieces;
    float m = -__builtin_inff();
    for (int i = (int)threadIdx.x; i < a.pieces; i += 256) {
        const f32x4 p = sums[i];
        if (p[1] != 0.f) m = fmaxf(m, p[0]);
    }
    m = wave_max(m);
    if (lane == 0) part[0][wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(part[0][0], part[0][1]), fmaxf(part[0][2], part[0][3]));
    if (m == -__builtin_inff()) m = 0.f;
    float S = 0.f, W = 0.f;
    for (int i = (int)threadIdx.x; i < a.pieces; i += 256) {
        const f32x4 p = sums[i];
        if (p[1] == 0.f) continue;           // (NaN goes on)
        const float d = (p[0] - m) * a.scale2, f = __builtin_amdgcn_exp2f(d);
        S = fmaf(p[1], f, S);
        W = fmaf(f, fmaf(p[1], fmaxf(d, -1e30f), p[2]), W);
    }
    S = wave_sum(S);
    W = wave_sum(W);
    if (lane == 0) {
        part[1][wave] = S;
        part[2][wave] = W;
    }
    if (a.top > 0) {
        int done = 0;
        for (bool more = false; done < a.pieces; more = true) {
            const int some = min(together - (more ? 1 : 0), a.pieces - done), lists = some + (more ? 1 : 0), n = lists * a.top;
            __syncthreads();                 // best is whole
            if (!more) {
#pragma unroll
                for (int i = 0; i < LP_LIST / 256; ++i)
                    if (256 * i + (int)threadIdx.x < first_keys) list[256 * i + threadIdx.x] = ahead[i];
            } else {
                for (int i = (int)threadIdx.x; i < some * a.top; i += 256) list[i] = from[(long long)done * a.top + i];
            }
            if (more)
                for (int i = (int)threadIdx.x; i < a.top; i += 256) list[some * a.top + i] = best[i];
            if (threadIdx.x == 0) {
                count = 0;
                border = 0;
            }
            __syncthreads();
            const int deep = (a.top + lists - 1) / lists, set = lists * deep;      // set < top + lists
            for (int i = (int)threadIdx.x; i < set; i += 256) heads[i] = list[i / deep * a.top + i % deep];
            __syncthreads();
            for (int i = (int)threadIdx.x; i < set; i += 256) {
                const uint64_t mine = heads[i];
                int above = 0;
#pragma unroll 8
                for (int j = 0; j < set; ++j) above += heads[j] > mine ? 1 : 0;
                if (above == a.top - 1) border = mine;
            }
            __syncthreads();
            for (int i = (int)threadIdx.x; i < n; i += 256)
                if (list[i] != 0 && list[i] >= border) reach[atomicAdd(&count, 1)] = list[i];
            __syncthreads();
            rank_keys(reach, count, a.top, best);
            done += some;
        }
    }
    __syncthreads();
    finish_row(a, row, judged, m, part[1][0] + part[1][1] + part[1][2] + part[1][3], part[2][0] + part[2][1] + part[2][2] + part[2][3], (int)threadIdx.x, 256,
               [&](int i) { return best[i]; });
}

inline int size_of(int dtype) { return dtype == BNN_F32 || dtype == BNN_I32 ? 4 : dtype == BNN_BF16 || dtype == BNN_F16 ? 2 : 0; }

// How rows are cut up: into pieces of up to 64 vectors of 16 bytes a thread, as many as make 512 workgroups, but no more than whose best are joined in one turn.  `at` and ld tell whether rows begin at 16 bytes (a vector more else); without them the
// most that a workspace is asked for.
constexpr int LP_GROUPS = 512;
struct LogprobsPlan {
    int group, vectors, pieces;              // group: vectors computed together; 0: a wave has a row
    size_t sums_bytes, bytes;
};
LogprobsPlan plan_logprobs(int rows, int cols, int size, int top, bool aligned) {
    LogprobsPlan p = {};
    const int v = 16 / size;
    if (cols <= LP_SHORT && (top <= 4 || (top <= 16 && rows >= 1024))) {
        p.pieces = 1;
        return p;
    }
    const long long most = cdiv((long long)cols + v - 1, 256LL * v);
    const long long want = std::max(cdiv(most * rows, LP_GROUPS), top > 0 ? cdiv(most, LP_LIST / top) : 1);
    p.group = want < 4 ? 1 : 4;
    p.vectors = (int)std::min<long long>(LP_VECTORS, p.group == 1 ? want : cdiv(want, 4) * 4);
    p.pieces = (int)cdiv(aligned ? cdiv(cols, 256LL * v) : most, p.vectors);
    if (p.pieces > 1) {
        p.sums_bytes = (size_t)rows * p.pieces * sizeof(f32x4);
        p.bytes = p.sums_bytes + (size_t)rows * p.pieces * top * sizeof(uint64_t);
    }
    return p;
}

template <class T>
int launch_logprobs(const Logprobs& a, int group, hipStream_t s) {
    if (group == 0) {
        const dim3 rows((unsigned)cdiv(a.rows, 4));
        if (a.cols <= 128) {
            if (a.top == 0) launch(logprobs_short_kernel<T, 2, false>, rows, dim3(256), 0, s, a);
            else launch(logprobs_short_kernel<T, 2, true>, rows, dim3(256), 0, s, a);
        } else {
            if (a.top == 0) launch(logprobs_short_kernel<T, 8, false>, rows, dim3(256), 0, s, a);
            else launch(logprobs_short_kernel<T, 8, true>, rows, dim3(256), 0, s, a);
        }
        return check_launch();
    }
    const dim3 grid((unsigned)((long long)a.rows * a.pieces));
    if (a.top == 0) {
        if (group == 4) launch(logprobs_kernel<T, 4, false>, grid, dim3(256), 0, s, a);
        else launch(logprobs_kernel<T, 1, false>, grid, dim3(256), 0, s, a);
    } else {
        if (group == 4) launch(logprobs_kernel<T, 4, true>, grid, dim3(256), 0, s, a);
        else launch(logprobs_kernel<T, 1, true>, grid, dim3(256), 0, s, a);
    }
    if (a.pieces > 1) launch(logprobs_join_kernel<T>, dim3((unsigned)a.rows), dim3(256), 0, s, a);
    return check_launch();
}

}  // namespace
}  // namespace bnn

using namespace bnn;

extern "C" {

size_t bnn_token_logprobs_workspace_bytes(int rows, int cols, int dtype, int top) {
    if (rows < 1 || cols < 1 || size_of(dtype) == 0 || top < 0 || top > LP_MAX_TOP || cols >= (1 << 30)) return 0;
    return plan_logprobs(rows, cols, size_of(dtype), top, false).bytes;
}

int bnn_token_logprobs(const void* logits, int dtype, int rows, int cols, int64_t ld, float scale, const int64_t* targets, int top,
                       float* logprobs, float* entropy, float* lse, float* top_logprobs, int32_t* top_tokens, void* workspace, size_t workspace_bytes, void* stream) {
    const int size = size_of(dtype);
    const float scale2 = scale * LP_LOG2E;
    if (size == 0 || rows < 0 || cols < 1 || top < 0 || top > cols || !(scale > 0.f) || !isfinite(scale2) || (targets == nullptr) != (logprobs == nullptr)) return BNN_ERR_INVALID_ARG;
    if (top > LP_MAX_TOP || cols >= (1 << 30)) return BNN_ERR_UNSUPPORTED;
    if (rows == 0) return BNN_OK;
    if (!logits || (top > 0 && (!top_logprobs || !top_tokens))) return BNN_ERR_INVALID_ARG;
    const void* words[] = {logprobs, entropy, lse, top_logprobs, top_tokens};
    for (const void* p : words)
        if (reinterpret_cast<uintptr_t>(p) & 3u) return BNN_ERR_ALIGNMENT;
    if (reinterpret_cast<uintptr_t>(logits) % size || (reinterpret_cast<uintptr_t>(targets) & 7u)) return BNN_ERR_ALIGNMENT;
    const LogprobsPlan p = plan_logprobs(rows, cols, size, top, reinterpret_cast<uintptr_t>(logits) % 16 == 0 && (rows == 1 || ld * size % 16 == 0));
    if ((long long)rows * p.pieces >= C4_THREADS / 256) return BNN_ERR_UNSUPPORTED;
    if (p.bytes != 0 && (!workspace || workspace_bytes < p.bytes)) return BNN_ERR_WORKSPACE;
    if (p.bytes != 0 && (reinterpret_cast<uintptr_t>(workspace) & 15u)) return BNN_ERR_ALIGNMENT;
    Logprobs a = {};
    a.x = logits; a.rows = rows; a.cols = cols; a.ld = ld;
    a.scale = scale; a.scale2 = scale2;
    a.targets = targets; a.top = top;
    a.logprobs = logprobs; a.entropy = entropy; a.lse = lse; a.top_logprobs = top_logprobs; a.top_tokens = top_tokens;
    a.pieces = p.pieces; a.vectors = p.vectors;
    a.div_pieces = make_fastdiv((uint32_t)p.pieces);
    a.sums = static_cast<f32x4*>(workspace);
    a.best = reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + p.sums_bytes);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == BNN_BF16) return launch_logprobs<__bf16>(a, p.group, s);
    if (dtype == BNN_F16) return launch_logprobs<_Float16>(a, p.group, s);
    if (dtype == BNN_I32) return launch_logprobs<int32_t>(a, p.group, s);
    return launch_logprobs<float>(a, p.group, s);
}

}  // extern "C"
