// What a head's sums say: log probabilities of given tokens, entropy, the best alternatives, in one pass over the logits.
//
// A workgroup has a piece of a row, which stays in its registers: with the piece's maximum m it forms S = sum 2^u and W = sum 2^u u, u = (x - m) scale / log 2, from which
//   log p = scale (x - m) - log S,  entropy = log S - log 2 W / S  (both terms >= 0),  lse = scale m + log S,
// so no difference of large numbers is left; pieces of a row are joined by the same rule.  The `top` best of a piece: the threads' maxima give a border that at least `top` elements reach, and
// little more do; those are collected in LDS and ranked by counting.  Elements are ordered by (value, lower column first) as one 64-bit number.
// What bounds it is memory.
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
    float scale, scale2;                     // scale2: for powers of two
    const int64_t* targets;
    int top;
    float *logprobs, *entropy, *lse, *top_logprobs;
    int32_t* top_tokens;
    int pieces;                              // of a row
    FastDiv div_pieces;
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

// The results of a row from its maximum and sums; best: its alternatives, in LDS.  All threads of the workgroup.
template <class T>
__device__ __forceinline__ void finish_row(const Logprobs& a, int row, float m, float S, float W, const uint64_t* best) {
    const bool none = !(S > 0.f);            // S is NaN, or 0: no distribution
    const float log_s = __builtin_amdgcn_logf(S) * LP_LN2, nan = __builtin_nanf("");
    if (threadIdx.x == 0) {
        if (a.lse != nullptr) a.lse[row] = none ? (S == 0.f ? -__builtin_inff() : nan) : fmaf(m, a.scale, log_s);
        if (a.entropy != nullptr) a.entropy[row] = none ? nan : log_s - LP_LN2 * (W / S);
        if (a.targets != nullptr && a.logprobs != nullptr) {
            const int64_t t = a.targets[row];
            float lp = 0.f;
            if (t >= 0 && t < a.cols) {
                const float x = as_float(static_cast<const T*>(a.x)[row * a.ld + t]);
                lp = none ? nan : fmaf(x - m, a.scale, -log_s);
            }
            a.logprobs[row] = lp;
        }
    }
    for (int i = (int)threadIdx.x; i < a.top; i += (int)blockDim.x) {
        const uint64_t key = best[i];
        a.top_logprobs[(long long)row * a.top + i] = none ? nan : fmaf(value_of((uint32_t)(key >> 32)) - m, a.scale, -log_s);
        a.top_tokens[(long long)row * a.top + i] = none || key == 0 ? -1 : (int32_t)~(uint32_t)key;
    }
}

// The `top` largest of list[0 .. n) to out, descending, 0 where there are fewer.  All different.  Called by all 256 threads; out is complete after the next barrier.
__device__ __forceinline__ void rank_keys(const uint64_t* list, int n, int top, uint64_t* out) {
    for (int i = n + (int)threadIdx.x; i < top; i += 256) out[i] = 0;
    for (int i = (int)threadIdx.x; i < n; i += 256) {
        const uint64_t mine = list[i];
        int above = 0;
        for (int j = 0; j < n; ++j) above += list[j] > mine ? 1 : 0;
        if (above < top) out[above] = mine;
    }
}

// NV: 16-byte loads of a thread.
template <class T, int NV, bool TOP>
__global__ __launch_bounds__(256) void logprobs_kernel(Logprobs a) {
    constexpr int V = 16 / sizeof(T);
    typedef T TV __attribute__((ext_vector_type(V)));
    extern __shared__ uint64_t list[];
    __shared__ float part[3][4];
    __shared__ uint32_t maxima[TOP ? 256 : 1];
    __shared__ uint64_t best[TOP ? LP_MAX_TOP : 1];
    __shared__ uint32_t border_s[2];
    __shared__ int count, scan[4];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int row = fast_div((int)blockIdx.x, a.div_pieces), piece = (int)blockIdx.x - row * a.pieces;
    const T* x = static_cast<const T*>(a.x) + row * a.ld;
    const int off = (int)(reinterpret_cast<uintptr_t>(x) / sizeof(T) % V);          // columns before the first whole 16 bytes lie in slot 0
    const int first = piece * (256 * NV * V) - off + (int)threadIdx.x * V;          // column of the thread's first element; its v-th vector begins 256 * V * v later
    float y[NV][V];
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        const int col = first + v * 256 * V;
        if (col >= 0 && col + V <= a.cols) {
            const TV w = *reinterpret_cast<const TV*>(x + col);
#pragma unroll
            for (int j = 0; j < V; ++j) y[v][j] = as_float(w[j]);
        } else {
#pragma unroll
            for (int j = 0; j < V; ++j) y[v][j] = col + j >= 0 && col + j < a.cols ? as_float(x[col + j]) : -__builtin_inff();
        }
    }
    float high = -__builtin_inff();
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < V; ++j) high = fmaxf(high, y[v][j]);
    const float wave_high = wave_max(high);
    if (lane == 0) part[0][wave] = wave_high;
    if constexpr (TOP) maxima[threadIdx.x] = first < a.cols && first + (NV - 1) * 256 * V + V > 0 ? order_of(high) : 0;
    if (threadIdx.x == 0) count = 0;
    __syncthreads();
    const float m = fmaxf(fmaxf(part[0][0], part[0][1]), fmaxf(part[0][2], part[0][3]));
    const float shift = m == -__builtin_inff() ? 0.f : m;
    float S = 0.f, W = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const float u = (y[v][j] - shift) * a.scale2, e = __builtin_amdgcn_exp2f(u);
            S += e;
            W = fmaf(e, fmaxf(u, -1e30f), W);
        }
    S = wave_sum(S);
    W = wave_sum(W);
    if (lane == 0) {
        part[1][wave] = S;
        part[2][wave] = W;
    }

    if constexpr (TOP) {
        // The largest number that `top` of the threads' maxima reach; the search ends early where few more do
        const int few = a.top + a.top / 2 + 1;
        if (wave == 0) {
            uint32_t mine[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[i] = maxima[lane + 64 * i];
            uint32_t border = 0;
            int reach = 256;
            for (int bit = 31; bit >= 0 && reach > few; --bit) {
                const uint32_t t = border | 1u << bit;
                int n = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) n += __popcll(__ballot(mine[i] >= t));
                if (n >= a.top) {
                    border = t;
                    reach = n;
                }
            }
            if (lane == 0) {
                border_s[0] = border;
                border_s[1] = (uint32_t)reach;
            }
        }
        __syncthreads();
        const uint32_t border = border_s[0];
        const bool ties = (int)border_s[1] > few;        // then border is exact, and fewer than `top` threads have more than it: what equals it is taken in the order of columns
        if (maxima[threadIdx.x] >= border) {
#pragma unroll
            for (int v = 0; v < NV; ++v)
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    const int col = first + v * 256 * V + j;
                    const uint32_t o = order_of(y[v][j]);
                    if ((ties ? o > border : o >= border) && col >= 0 && col < a.cols && y[v][j] == y[v][j]) list[atomicAdd(&count, 1)] = key_of(y[v][j], col);
                }
        }
        __syncthreads();
        int have = count;
        if (ties && have < a.top) {
            for (int v = 0; v < NV; ++v) {
                int n = 0;
#pragma unroll
                for (int u = 0; u < NV; ++u)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const int col = first + u * 256 * V + j;
                        n += u == v && order_of(y[u][j]) == border && col >= 0 && col < a.cols ? 1 : 0;
                    }
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
                for (int u = 0; u < NV; ++u)
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const int col = first + u * 256 * V + j;
                        if (u == v && order_of(y[u][j]) == border && col >= 0 && col < a.cols) {
                            if (at < a.top) list[at] = key_of(y[u][j], col);
                            ++at;
                        }
                    }
                have += scan[0] + scan[1] + scan[2] + scan[3];
                __syncthreads();
                if (have >= a.top) break;
            }
            have = min(have, a.top);
        }
        rank_keys(list, have, a.top, best);
    }
    __syncthreads();
    S = part[1][0] + part[1][1] + part[1][2] + part[1][3];
    W = part[2][0] + part[2][1] + part[2][2] + part[2][3];
    if (a.pieces == 1) {
        finish_row<T>(a, row, m, S, W, best);
    } else {
        if (threadIdx.x == 0) a.sums[blockIdx.x] = f32x4{m, S, W, 0.f};
        if constexpr (TOP)
            for (int i = (int)threadIdx.x; i < a.top; i += 256) a.best[(long long)blockIdx.x * a.top + i] = best[i];
    }
}

constexpr int LP_LIST = 1024;                // keys that are looked at together

// Joins the pieces of a row.  Each piece's best come in order; of L pieces the ceil(top / L) best each are at least `top`, and the `top`-th of those is a border that little more reach.
template <class T>
__global__ __launch_bounds__(256) void logprobs_join_kernel(Logprobs a) {
    __shared__ uint64_t list[LP_LIST], reach[LP_LIST], best[LP_MAX_TOP];
    __shared__ float part[3][4];
    __shared__ uint64_t border;
    __shared__ int count;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int row = (int)blockIdx.x;
    const f32x4* sums = a.sums + (long long)row * a.pieces;
    float m = -__builtin_inff();
    for (int i = (int)threadIdx.x; i < a.pieces; i += 256) m = fmaxf(m, sums[i][0]);
    m = wave_max(m);
    if (lane == 0) part[0][wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(part[0][0], part[0][1]), fmaxf(part[0][2], part[0][3]));
    const float shift = m == -__builtin_inff() ? 0.f : m;
    float S = 0.f, W = 0.f;
    for (int i = (int)threadIdx.x; i < a.pieces; i += 256) {
        const f32x4 p = sums[i];
        if (p[1] == 0.f) continue;           // (NaN goes on)
        const float u = (p[0] - shift) * a.scale2, f = __builtin_amdgcn_exp2f(u);
        S = fmaf(p[1], f, S);
        W = fmaf(f, fmaf(p[1], fmaxf(u, -1e30f), p[2]), W);
    }
    S = wave_sum(S);
    W = wave_sum(W);
    if (lane == 0) {
        part[1][wave] = S;
        part[2][wave] = W;
    }
    if (a.top > 0) {
        const uint64_t* from = a.best + (long long)row * a.pieces * a.top;
        const int together = LP_LIST / a.top;                        // pieces, the best so far counting as one
        int done = 0;
        for (bool more = false; done < a.pieces; more = true) {
            const int some = min(together - (more ? 1 : 0), a.pieces - done), lists = some + (more ? 1 : 0), n = lists * a.top;
            __syncthreads();                 // best is whole
            for (int i = (int)threadIdx.x; i < some * a.top; i += 256) list[i] = from[(long long)done * a.top + i];
            if (more)
                for (int i = (int)threadIdx.x; i < a.top; i += 256) list[some * a.top + i] = best[i];
            if (threadIdx.x == 0) {
                count = 0;
                border = 0;
            }
            __syncthreads();
            const int deep = (a.top + lists - 1) / lists, set = lists * deep;      // set < top + lists
            for (int i = (int)threadIdx.x; i < set; i += 256) {
                const uint64_t mine = list[i / deep * a.top + i % deep];
                int above = 0;
                for (int l = 0; l < lists; ++l)
                    for (int j = 0; j < deep; ++j) above += list[l * a.top + j] > mine ? 1 : 0;
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
    finish_row<T>(a, row, m, part[1][0] + part[1][1] + part[1][2] + part[1][3], part[2][0] + part[2][1] + part[2][2] + part[2][3], best);
}

inline int size_of(int dtype) { return dtype == BNN_F32 || dtype == BNN_I32 ? 4 : dtype == BNN_BF16 || dtype == BNN_F16 ? 2 : 0; }

// How rows are cut up: pieces of 256 threads with 8 loads of 16 bytes each, or 2 where that makes too few workgroups.
struct LogprobsPlan {
    int loads, pieces;
    size_t sums_bytes, bytes;
};
LogprobsPlan plan_logprobs(int rows, int cols, int size, int top) {
    LogprobsPlan p = {};
    const int v = 16 / size;
    p.loads = 8;
    if ((long long)rows * cdiv(cols, 256LL * 8 * v) < 1024) p.loads = 2;
    p.pieces = (int)cdiv((long long)cols + v - 1, 256LL * p.loads * v);            // a row may begin within 16 bytes
    if (p.pieces > 1) {
        p.sums_bytes = (size_t)rows * p.pieces * sizeof(f32x4);
        p.bytes = p.sums_bytes + (size_t)rows * p.pieces * top * sizeof(uint64_t);
    }
    return p;
}

template <class T>
int launch_logprobs(const Logprobs& a, int loads, hipStream_t s) {
    const dim3 grid((unsigned)((long long)a.rows * a.pieces));
    const size_t lds = a.top == 0 ? 0 : std::min<size_t>(a.top + a.top / 2 + 1, 256) * loads * (16 / sizeof(T)) * sizeof(uint64_t);
    if (a.top == 0) {
        if (loads == 8) launch(logprobs_kernel<T, 8, false>, grid, dim3(256), 0, s, a);
        else launch(logprobs_kernel<T, 2, false>, grid, dim3(256), 0, s, a);
    } else {
        if (loads == 8) launch(logprobs_kernel<T, 8, true>, grid, dim3(256), lds, s, a);
        else launch(logprobs_kernel<T, 2, true>, grid, dim3(256), lds, s, a);
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
    return plan_logprobs(rows, cols, size_of(dtype), top).bytes;
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
    const LogprobsPlan p = plan_logprobs(rows, cols, size, top);
    if ((long long)rows * p.pieces >= C4_THREADS / 256) return BNN_ERR_UNSUPPORTED;
    if (p.bytes != 0 && (!workspace || workspace_bytes < p.bytes)) return BNN_ERR_WORKSPACE;
    if (p.bytes != 0 && (reinterpret_cast<uintptr_t>(workspace) & 15u)) return BNN_ERR_ALIGNMENT;
    Logprobs a = {};
    a.x = logits; a.rows = rows; a.cols = cols; a.ld = ld;
    a.scale = scale; a.scale2 = scale2;
    a.targets = targets; a.top = top;
    a.logprobs = logprobs; a.entropy = entropy; a.lse = lse; a.top_logprobs = top_logprobs; a.top_tokens = top_tokens;
    a.pieces = p.pieces;
    a.div_pieces = make_fastdiv((uint32_t)p.pieces);
    a.sums = static_cast<f32x4*>(workspace);
    a.best = reinterpret_cast<uint64_t*>(static_cast<char*>(workspace) + p.sums_bytes);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (dtype == BNN_BF16) return launch_logprobs<__bf16>(a, p.loads, s);
    if (dtype == BNN_F16) return launch_logprobs<_Float16>(a, p.loads, s);
    if (dtype == BNN_I32) return launch_logprobs<int32_t>(a, p.loads, s);
    return launch_logprobs<float>(a, p.loads, s);
}

}  // extern "C"
