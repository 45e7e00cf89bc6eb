// Selection of blocks of the 4-bit cache by the signs of queries and keys.
//
// score_kernel: a wave holds the sign words of up to eight query heads in scalar registers and takes four blocks at a time, sixteen lanes to a block; a lane counts, for each
// of its keys and each head, the differing bits (xor and a counting add) and keeps the fewest.  Counting on the vector ALU: 72 instructions a key at eight heads
// of 128 elements, against 16 bytes of memory.
// pick_kernel: a workgroup per (token, kv head) counts the scores into bins, finds the score at which the places run out, and writes the blocks in order;
// of those at that score the lowest.  Everything is whole numbers, so the result does not depend on any order.
#include "bnn_cache4.h"

namespace bnn {
namespace {

constexpr int HEADS = 8;                     // query heads a wave scores at once

// The largest of the 16 lanes of a row.
__device__ __forceinline__ int max16(int v) {
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x128, 0xf, 0xf, true));    // row_ror:8, 4, 2, 1
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x124, 0xf, 0xf, true));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x122, 0xf, 0xf, true));
    v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x121, 0xf, 0xf, true));
    return v;
}

// Score of a block + 1 (0: the row sees none of its keys), for `span` blocks per workgroup.
template <int D, class T>
__global__ __launch_bounds__(256) void score_kernel(Select4 a, int span, FastDiv div_heads, FastDiv div_parts, int parts) {
    constexpr int W = D / 32;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int rest = fast_div((int)blockIdx.x, div_heads), head = (int)blockIdx.x - rest * a.c.kv_heads;
    const int token = fast_div(rest, div_parts), part = rest - token * parts;
    const int b = __builtin_amdgcn_readfirstlane(c4_sequence_of(a.r, token));
    const Sequence4 s = c4_sequence(a.r, a.c, b);
    const int i = token - s.first;
    if (i < 0 || i >= s.rows) return;
    const int pos = s.length - s.rows + i;
    const int blocks = pos < 0 ? 0 : (pos >> a.c.page_shift) + 1;
    const int end = min(blocks, (part + 1) * span);
    uint16_t* scores = a.scores + ((long long)token * a.c.kv_heads + head) * a.r.table_pages;
    const int sub = lane & 15, which = lane >> 4;
    for (int g0 = 0; g0 < a.group; g0 += HEADS) {
        uint32_t q[HEADS][W];
#pragma unroll
        for (int g = 0; g < HEADS; ++g) {
            const bool there = g0 + g < a.group;
            const T* src = static_cast<const T*>(a.q) + (long long)token * a.q_token + (long long)(head * a.group + g0 + (there ? g : 0)) * a.q_head;
#pragma unroll
            for (int w = 0; w < W; w += 2) {
                const int d = 32 * w + lane;
                const unsigned long long bits = __ballot(d < D && (float)src[d < D ? d : 0] >= 0.f);
                q[g][w] = (uint32_t)bits;
                if (w + 1 < W) q[g][w + 1] = (uint32_t)(bits >> 32);
            }
        }
        for (int b0 = part * span + 4 * wave; b0 < end; b0 += 16) {
            const int block = b0 + which;
            const int page = block < end ? c4_page(a.r, a.c, b, block << a.c.page_shift) : -1;
            int best[HEADS];
#pragma unroll
            for (int g = 0; g < HEADS; ++g) best[g] = -1;
            if (page >= 0) {
                const uint32_t* words = reinterpret_cast<const uint32_t*>(c4_record(a.c, page, head) + a.c.signs);
                for (int k = sub; k < a.c.page; k += 16) {
                    if ((block << a.c.page_shift) + k > pos) break;
                    uint32_t x[W];
#pragma unroll
                    for (int w = 0; w < W; ++w) x[w] = words[k * W + w];
#pragma unroll
                    for (int g = 0; g < HEADS; ++g) {
                        int differ = 0;
#pragma unroll
                        for (int w = 0; w < W; ++w) differ += __popc(x[w] ^ q[g][w]);
                        best[g] = max(best[g], D - differ);
                    }
                }
            }
            int score = 0;
#pragma unroll
            for (int g = 0; g < HEADS; ++g) score += g0 + g < a.group ? max16(best[g]) : 0;
            if (sub == 0 && block < end) {
                if (page < 0) scores[block] = 0;
                else scores[block] = (uint16_t)(score + (g0 == 0 ? 1 : scores[block]));
            }
        }
    }
}

// Position of the lane among the lanes of the workgroup whose flag is set, and their number.  scratch: one int per wave.
__device__ __forceinline__ int count_before(bool flag, int* scratch, int& all) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    const unsigned long long mask = __ballot(flag);
    __syncthreads();
    if (lane == 0) scratch[wave] = __popcll(mask);
    __syncthreads();
    int before = __popcll(mask & ((1ull << lane) - 1));
    all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) before += scratch[w];
        all += scratch[w];
    }
    return before;
}

__global__ __launch_bounds__(256) void pick_kernel(Select4 a, FastDiv div_heads, int bins) {
    extern __shared__ int count[];           // [bins], then scratch
    int* scratch = count + bins;             // [0..3], [4]: score at the edge, [5]: places for it
    const int token = fast_div((int)blockIdx.x, div_heads), head = (int)blockIdx.x - token * a.c.kv_heads;
    const int b = c4_sequence_of(a.r, token);
    const Sequence4 s = c4_sequence(a.r, a.c, b);
    const int i = token - s.first;
    if (i < 0 || i >= s.rows) return;
    const int pos = s.length - s.rows + i;
    const int blocks = pos < 0 ? 0 : (pos >> a.c.page_shift) + 1;
    const long long at = (long long)token * a.c.kv_heads + head;
    const uint16_t* scores = a.scores + at * a.r.table_pages;
    int32_t* out = a.blocks + at * a.keep;
    const int tail = blocks - a.last;        // blocks from here on are kept
    for (int x = (int)threadIdx.x; x < bins; x += 256) count[x] = 0;
    __syncthreads();
    int forced = 0;
    for (int x = (int)threadIdx.x; x < blocks; x += 256) {
        const int v = scores[x];
        if (v == 0) continue;
        if (x < a.first || x >= tail) ++forced;
        else atomicAdd(&count[v], 1);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) forced += __shfl_xor(forced, d);
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = forced;
    __syncthreads();
    forced = scratch[0] + scratch[1] + scratch[2] + scratch[3];
    __syncthreads();
    const int places = a.keep - forced;      // >= 0: keep >= first + last
    if (threadIdx.x < 64) {                  // from the highest score down, 64 bins at a time
        const int lane = (int)threadIdx.x;
        int above = 0, edge = 0, left = 0;
        for (int top = bins - 1; top >= 1; top -= 64) {
            const int bin = top - lane, n = bin >= 1 ? count[bin] : 0;
            int sum = n;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int other = __shfl_up(sum, d);
                if (lane >= d) sum += other;
            }
            const unsigned long long past = __ballot(above + sum >= places);
            if (past != 0) {
                const int l = __ffsll(past) - 1;
                edge = top - l;
                left = places - (above + __shfl(sum, l) - __shfl(n, l));
                break;
            }
            above += __shfl(sum, 63);
        }
        if (lane == 0) {
            scratch[4] = edge;               // 0: there are fewer than places
            scratch[5] = left;
        }
    }
    __syncthreads();
    const int edge = scratch[4], left = scratch[5];
    int written = 0, equal = 0;
    for (int x0 = 0; x0 < blocks; x0 += 256) {
        const int x = x0 + (int)threadIdx.x;
        const int v = x < blocks ? scores[x] : 0;
        const bool kept = v != 0 && (x < a.first || x >= tail);
        const bool tie = v != 0 && !kept && v == edge;
        int all;
        const int before = count_before(tie, scratch, all);
        const bool take = kept || (v != 0 && v > edge) || (tie && equal + before < left);
        equal += all;
        const int place = written + count_before(take, scratch, all);
        if (take && place < a.keep) out[place] = x;
        written += all;
    }
    for (int x = written + (int)threadIdx.x; x < a.keep; x += 256) out[x] = -1;
}

template <int D>
int launch_score(const Select4& a, int dtype, hipStream_t s) {
    // Blocks per workgroup: as few as give every compute unit eight waves, but a multiple of 16, what its four waves take at a time
    const long long rows = (long long)a.r.tokens * a.c.kv_heads;
    const long long wanted = cdiv(1024, rows), most = cdiv(a.r.table_pages, 16);
    const int parts = (int)(wanted < most ? wanted : most);
    const int span = (int)(cdiv(cdiv(a.r.table_pages, parts), 16) * 16);
    const dim3 grid((unsigned)(rows * parts));
    auto go = [&](auto type) {
        using T = decltype(type);
        launch(score_kernel<D, T>, grid, dim3(256), 0, s, a, span, make_fastdiv((uint32_t)a.c.kv_heads), make_fastdiv((uint32_t)parts), parts);
    };
    if (dtype == BNN_BF16) go(__bf16{});
    else if (dtype == BNN_F16) go(_Float16{});
    else go(float{});
    return check_launch();
}

}  // namespace

int launch_cache4_select(const Select4& a, int dtype, hipStream_t s) {
    int rc;
    switch (a.c.dim) {
        case 64: rc = launch_score<64>(a, dtype, s); break;
        case 96: rc = launch_score<96>(a, dtype, s); break;
        case 128: rc = launch_score<128>(a, dtype, s); break;
        case 192: rc = launch_score<192>(a, dtype, s); break;
        default: rc = launch_score<256>(a, dtype, s); break;
    }
    if (rc != BNN_OK) return rc;
    const int bins = a.group * a.c.dim + 2;
    launch(pick_kernel, dim3((unsigned)a.r.tokens * (unsigned)a.c.kv_heads), dim3(256), (size_t)(bins + 8) * 4, s, a, make_fastdiv((uint32_t)a.c.kv_heads), bins);
    return check_launch();
}

}  // namespace bnn
