// Selection of blocks of the 4-bit cache by the signs of queries and keys.
//
// score_kernel: signs on the matrix cores (v_mfma_f32_32x32x64_f8f6f4, E2M1).  Rows are 32 keys, columns the query heads of one or several tokens, 32 in all.  A key's
// bits count as {0, 1}, a query's as -1 / +1: sum_d k_d q_d over them is the number of agreeing bits less the query's 0 bits, a constant of the column,
// so it has the same maximum, and a key's word becomes an operand by four ANDs and one shift: product j takes bit j of every nibble, as 0.5, 1, 2 and
// (shifted) 2, and the query's factor, 2, 1, 0.5 and 0.5, makes them count alike.  A lane holds the products of one column with 16 keys of each tile of 32:
// the maximum over a block is taken in registers, then across two half waves, and the sum over the heads of a token as a difference of running sums across lanes.  All numbers are whole and exact.
// A wave takes 128 keys (or a block of 256) at a time and has loaded the next two lots.
// 8 sequences of 50001 to 65536 tokens, 64 query heads on 8 kv heads of 128: 59 MB of signs in 14 to 16 us, where counting with xor and popcount on the vector ALU took 20; 666 query tokens with 20
// heads on 4 of 64 over up to 10007 keys: 20 us (61).  Bounded by issue slots: 5 instructions a word of 32 signs, 8 for the maxima of 32 keys x 32 columns.
// pick_kernel: a workgroup per (token, kv head) counts the scores into bins, finds the score at which the places run out, and writes the blocks in order;
// of those at that score the lowest.  Everything is whole numbers, so the result does not depend on any order.
#include "bnn_cache4.h"

namespace bnn {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float UNSEEN = -1e9f;

// A word of a key's signs as 32 E2M1 numbers in {0, 0.5}, {0, 1}, {0, 2}, {0, 2}.
__device__ __forceinline__ v8i key_operand(uint32_t w) {
    v8i r = {};
    r[0] = (int)(w & 0x11111111u);
    r[1] = (int)(w & 0x22222222u);
    r[2] = (int)(w & 0x44444444u);
    r[3] = (int)((w >> 1) & 0x44444444u);
    return r;
}
// A word of a query's signs as -1 / +1 times 2, 1, 0.5, 0.5.
__device__ __forceinline__ v8i query_operand(uint32_t w) {
    v8i r = {};
    r[0] = (int)(0x44444444u | (~w & 0x11111111u) << 3);
    r[1] = (int)(0x22222222u | (~(w >> 1) & 0x11111111u) << 3);
    r[2] = (int)(0x11111111u | (~(w >> 2) & 0x11111111u) << 3);
    r[3] = (int)(0x11111111u | (~(w >> 3) & 0x11111111u) << 3);
    return r;
}

// The 32 signs from element `at` on.
template <class T>
__device__ __forceinline__ uint32_t sign_word(const T* p) {
    uint32_t w = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float x[8];
        c4_load8(p + 8 * i, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) w |= (x[e] >= 0.f ? 1u : 0u) << (8 * i + e);
    }
    return w;
}

template <int CTRL, int ROWS = 0xf>
__device__ __forceinline__ float dpp(float v) {              // 0 where the lane has no source, or its row of 16 is not in ROWS
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, ROWS, 0xf, true));
}
// Sum over the `group` columns up to the lane's own, for the last lane of each group; columns are the 32 lanes of a half wave.
__device__ __forceinline__ float sum_columns(float v, int group) {
    if (group == 1) return v;
    v += dpp<0x111>(v);                                          // running sums in rows of 16: lanes 1, 2, 4, 8 below
    v += dpp<0x112>(v);
    v += dpp<0x114>(v);
    v += dpp<0x118>(v);
    v += dpp<0x142, 0xa>(v);                                     // the last of a half wave's first row to its second
    const int lane = (int)threadIdx.x & 63, from = lane - group;
    const float before = __uint_as_float((uint32_t)__builtin_amdgcn_ds_bpermute(4 * from, (int)__float_as_uint(v)));
    return v - ((lane & 31) < group ? 0.f : before);
}
// Lower half wave: the larger of x's halves; upper: of y's.
__device__ __forceinline__ float max_halves(float x, float y) {
    auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <int D, int PAGE>
__global__ __launch_bounds__(256, PAGE == 256 && D > 64 ? 2 : D >= 192 || PAGE == 16 ? 3 : 4) void score_kernel(Select4 a, int dtype) {
    constexpr int W = D / 32, M = (W + 1) / 2;                   // words of a key; matrix instructions, of 64 elements, a tile of 32 keys
    constexpr int KEYS = PAGE < 128 ? 128 : PAGE, TILES = KEYS / 32, NB = KEYS / PAGE;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int col = lane & 31, upper = lane >> 5;
    const int rest = fast_div((int)blockIdx.x, a.div_heads), head = (int)blockIdx.x - rest * a.c.kv_heads;
    const int tile = fast_div(rest, a.div_parts), part = rest - tile * a.parts;
    int b, local;
    if (!c4_find_tile(a.r, 1, a.tile_tokens, tile, a.seq_tiles, a.div_seq_tiles, b, local)) return;
    const Sequence4 s = c4_sequence(a.r, b);
    const int i0 = local * a.tile_tokens, tokens = min(a.tile_tokens, s.rows - i0);
    if (tokens <= 0) return;
    const int base = s.length - s.rows + i0;                     // position of the first
    const int last = base + tokens - 1;
    const int blocks = last < 0 ? 0 : min((last >> a.c.page_shift) + 1, a.r.table_pages);
    const int steps = (blocks + NB - 1) / NB;
    // a share of the steps for every part, each wave every fourth of it
    const int share = (steps + a.parts - 1) / a.parts, begin = part * share, end = min(steps, begin + share);
    if (begin >= end) return;

    const int i = fast_div(col, a.div_columns), g1 = col - i * a.columns;
    const bool row = i < tokens;
    const int pos = base + i;
    const long long token = s.first + i0 + (row ? i : 0);
    uint16_t* scores = a.scores + (token * a.c.kv_heads + head) * a.r.table_pages;

    // Where the signs of this wave's next 64 blocks lie, a lane each: the offset in the cache, and whether there is a page.
    const int turns = (end - begin - wave + 3) / 4;              // steps of this wave
    uint32_t low = 0, high = 0;
    unsigned long long present = 0;
    auto locate = [&](int turn) {                                // turn: a multiple of 64 / NB
        const int block = (begin + wave + 4 * (turn + lane / NB)) * NB + lane % NB;
        const int page = c4_page(a.r, a.c, b, min(block, blocks - 1) << a.c.page_shift);
        const uint64_t at = (uint64_t)(c4_record(a.c, max(page, 0), head) + a.c.signs - a.c.data);
        low = (uint32_t)at;
        high = (uint32_t)(at >> 32);
        present = __ballot(page >= 0 && block < blocks);
    };
    // Of a key's words, lanes of the lower half wave take the first M, those of the upper one the rest: neighbours in memory.
    struct Batch {
        uint32_t raw[TILES][M];
        int in;                                                  // bit n: block n is there
    };
    auto fill = [&](Batch& x, int turn) {
        if (turn >= turns) return;
        if (turn % (64 / NB) == 0) locate(turn);
        const int at = turn % (64 / NB) * NB;
        x.in = (int)(present >> at) & ((1 << NB) - 1);
        const uint32_t* block[NB];
#pragma unroll
        for (int n = 0; n < NB; ++n)
            block[n] = reinterpret_cast<const uint32_t*>(a.c.data + ((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)high, at + n) << 32 |
                                                                     (uint32_t)__builtin_amdgcn_readlane((int)low, at + n)));
#pragma unroll
        for (int t = 0; t < TILES; ++t) {
            const uint32_t* words;
            if constexpr (PAGE == 16) words = (col < 16 ? block[2 * t] : block[2 * t + 1]) + (col & 15) * W + upper * M;
            else words = block[32 * t / PAGE] + (32 * t % PAGE * W + col * W + upper * M);
#pragma unroll
            for (int m = 0; m < M; ++m) x.raw[t][m] = words[M + m < W || upper == 0 ? m : 0];      // (of three words the upper half has one)
        }
    };

    for (int g0 = 0; g0 < a.group; g0 += 32) {
        Batch x, y;
        fill(x, 0);
        fill(y, 1);
        // the queries; a column without one, and the half of the last 64 elements that D does not have, are zero
        v8i q[M];
        float zeros = 0.f;                                       // of the column's signs
        const bool there = row && g0 + g1 < a.group;
        const long long at = token * a.q_token + (long long)(head * a.group + (there ? g0 + g1 : 0)) * a.q_head;
#pragma unroll
        for (int m = 0; m < M; ++m) {
            q[m] = v8i{};
            if (there && upper * M + m < W) {
                const long long e = at + 32 * (upper * M + m);
                const uint32_t w = dtype == BNN_F32 ? sign_word(static_cast<const float*>(a.q) + e) : dtype == BNN_BF16 ? sign_word(static_cast<const __bf16*>(a.q) + e)
                                                                                                     : sign_word(static_cast<const _Float16*>(a.q) + e);
                q[m] = query_operand(w);
                zeros += 32 - __popc(w);
            }
        }
        {
            auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(zeros), __float_as_uint(zeros), false, false);
            zeros = __uint_as_float(r[0]) + __uint_as_float(r[1]);
        }

        auto work = [&](Batch& z, int turn) {
            const int step = begin + wave + 4 * turn, in = z.in;
            const int key0 = step * KEYS;
            const bool edge = key0 + KEYS - 1 > base;            // some token does not see all of these keys
            float best[NB];
#pragma unroll
            for (int n = 0; n < NB; ++n) best[n] = UNSEEN;
            auto products = [&](auto masked) {
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    f32x16 acc = {};
#pragma unroll
                    for (int m = 0; m < M; ++m) acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(key_operand(z.raw[t][m]), q[m], acc, 4, 4, 0, 0, 0, 0);
                    if constexpr (masked.value != 0) {
#pragma unroll
                        for (int i = 0; i < 16; ++i)
                            if (key0 + 32 * t + 8 * (i >> 2) + 4 * upper + (i & 3) > pos) acc[i] = UNSEEN;
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        float& v = best[PAGE == 16 ? 2 * t + (i >> 3) : 32 * t / PAGE];      // registers 0 to 7 hold keys 0 to 15 of the tile
                        v = fmaxf(v, acc[i]);
                    }
                    if (t % 2 == 1) __builtin_amdgcn_sched_barrier(0);           // two tiles' products at a time: more do not fit the registers
                }
            };
            if (edge) products(std::integral_constant<int, 1>{});
            else products(std::integral_constant<int, 0>{});
            fill(z, turn + 2);
#pragma unroll
            for (int n = 0; n < NB; n += 2) {
                const int other = n + 1 < NB ? n + 1 : n;
                float v = max_halves(best[n], best[other]) + zeros;
                v = sum_columns(there && v >= 0.f ? v : 0.f, a.columns);             // (below 0: the token sees none of the keys)
                const int block = step * NB + (upper ? other : n);
                if (row && g1 == a.columns - 1 && block < blocks) {
                    const bool seen = (in >> (upper ? other : n) & 1) && block << a.c.page_shift <= pos;
                    scores[block] = (uint16_t)(!seen ? 0 : (int)v + (g0 == 0 ? 1 : scores[block]));
                }
            }
        };
        for (int turn = 0; turn < turns; turn += 2) {
            work(x, turn);
            if (turn + 1 < turns) work(y, turn + 1);
        }
    }
}

// Sums over the lanes of the workgroup before this one, and over all.
template <int WAVES>
__device__ __forceinline__ int2 scan2(int2 v, int2* scratch, int2& all) {
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    int2 sum = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int x = __shfl_up(sum.x, d), y = __shfl_up(sum.y, d);
        if (lane >= d) { sum.x += x; sum.y += y; }
    }
    __syncthreads();
    if (lane == 63) scratch[wave] = sum;
    __syncthreads();
    int2 before = make_int2(sum.x - v.x, sum.y - v.y);
    all = make_int2(0, 0);
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        const int2 x = scratch[w];
        if (w < wave) { before.x += x.x; before.y += x.y; }
        all.x += x.x; all.y += x.y;
    }
    return before;
}

// A score is a bin's number in LDS, so none above the last is taken as it is: where the plan's start falls, rows can be asked for whose scores no workgroup has
// written, and memory may hold anything.
// A thread owns `each` consecutive blocks (at most EACH, held in registers, or, with EACH == 0, read again in every pass) and, from the highest down, an even share of the
// bins.  The scores are asked for before it is known how many blocks there are: 1024 of them picked in 4.8 us, in 5.5 when every pass read its own.
template <int EACH, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void pick_kernel(Select4 a, int bins) {
    constexpr int THREADS = 64 * WAVES;
    extern __shared__ int count[];           // [bins]
    __shared__ int2 scratch[WAVES];
    __shared__ int found[2];                 // score at the edge, places for it
    const int token = fast_div((int)blockIdx.x, a.div_heads), head = (int)blockIdx.x - token * a.c.kv_heads;
    const long long at = (long long)token * a.c.kv_heads + head;
    const uint16_t* scores = a.scores + at * a.r.table_pages;
    const int each = (a.r.table_pages + THREADS - 1) / THREADS, x0 = (int)threadIdx.x * each;
    uint16_t held[EACH > 0 ? EACH : 1];
#pragma unroll
    for (int i = 0; i < EACH; ++i) held[i] = scores[min(x0 + i, a.r.table_pages - 1)];
    const int b = c4_sequence_of(a.r, token);
    const Sequence4 s = c4_sequence(a.r, b);
    const int i = token - s.first;
    if (i < 0 || i >= s.rows) return;
    const int pos = s.length - s.rows + i;
    const int own = pos >> a.c.page_shift, blocks = pos < 0 ? 0 : min(own + 1, a.r.table_pages), x1 = min(blocks, x0 + each);
    int32_t* out = a.blocks + at * a.keep;
    const int tail = own + 1 - a.last;       // blocks from here on are kept
    // f(block, score + 1) for this thread's blocks that can be selected
    auto for_each = [&](auto f) {
        if constexpr (EACH > 0) {
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (x0 + i < x1 && held[i] != 0) f(x0 + i, min((int)held[i], bins - 1));
        } else {
            for (int x = x0; x < x1; ++x) {
                const int v = min((int)scores[x], bins - 1);
                if (v != 0) f(x, v);
            }
        }
    };
    for (int x = (int)threadIdx.x; x < bins; x += THREADS) count[x] = 0;
    if (threadIdx.x < 2) found[threadIdx.x] = 0;
    __syncthreads();
    int2 forced = make_int2(0, 0);
    for_each([&](int x, int v) {
        if (x < a.first || x >= tail) ++forced.x;
        else atomicAdd(&count[v], 1);
    });
    int2 all;
    scan2<WAVES>(forced, scratch, all);
    const int places = a.keep - all.x;       // >= 0: keep >= first + last
    // The edge: the highest score at which `places` blocks are reached (0: never)
    const int span = (bins + THREADS - 1) / THREADS, top = bins - 1 - (int)threadIdx.x * span;
    int2 mine = make_int2(0, 0);
    for (int v = top; v > top - span && v >= 1; --v) mine.x += count[v];
    int above = scan2<WAVES>(mine, scratch, all).x;
    if (above < places && above + mine.x >= places) {
        for (int v = top; v > top - span && v >= 1; --v) {
            if (above + count[v] >= places) {
                found[0] = v;
                found[1] = places - above;
                break;
            }
            above += count[v];
        }
    }
    __syncthreads();
    const int edge = places > 0 ? found[0] : bins, left = found[1];      // no places: nothing beside the kept ones
    auto kept = [&](int x, int v) { return x < a.first || x >= tail || v > edge; };
    int2 chosen = make_int2(0, 0);           // kept or above the edge; at the edge
    for_each([&](int x, int v) {
        if (kept(x, v)) ++chosen.x;
        else if (v == edge) ++chosen.y;
    });
    const int2 before = scan2<WAVES>(chosen, scratch, all);
    int place = before.x + min(before.y, left), ties = before.y;
    for_each([&](int x, int v) {
        const bool above_edge = kept(x, v);
        if (above_edge || (v == edge && ties < left)) {
            if (place < a.keep) out[place] = x;
            ++place;
        }
        if (!above_edge && v == edge) ++ties;
    });
    for (int x = all.x + min(all.y, left) + (int)threadIdx.x; x < a.keep; x += THREADS) out[x] = -1;
}

template <int D>
void launch_score(const Select4& a, int dtype, hipStream_t s) {
    const dim3 grid((unsigned)a.tiles * (unsigned)a.parts * (unsigned)a.c.kv_heads);
    switch (a.c.page) {
        case 16: launch(score_kernel<D, 16>, grid, dim3(256), 0, s, a, dtype); break;
        case 32: launch(score_kernel<D, 32>, grid, dim3(256), 0, s, a, dtype); break;
        case 64: launch(score_kernel<D, 64>, grid, dim3(256), 0, s, a, dtype); break;
        case 128: launch(score_kernel<D, 128>, grid, dim3(256), 0, s, a, dtype); break;
        default: launch(score_kernel<D, 256>, grid, dim3(256), 0, s, a, dtype); break;
    }
}

}  // namespace

int launch_cache4_select(Select4 a, int dtype, hipStream_t s) {
    a.columns = std::min(a.group, 32);
    a.div_columns = make_fastdiv((uint32_t)a.columns);
    a.tile_tokens = 32 / a.columns;
    const long long tiles = c4_tiles(a.r, 1, a.tile_tokens, &a.seq_tiles);
    // parts of the keys: 1024 workgroups if there are so many steps, of which a workgroup takes four at a time
    const long long steps = cdiv((long long)a.r.table_pages * a.c.page, a.c.page > 128 ? 256 : 128);
    const long long parts = std::max(1LL, std::min(cdiv(1024, tiles * a.c.kv_heads), cdiv(steps, 4)));
    if (tiles * parts * a.c.kv_heads >= C4_THREADS / 256) return BNN_ERR_UNSUPPORTED;
    a.tiles = (int)tiles;
    a.parts = (int)parts;
    a.div_seq_tiles = make_fastdiv((uint32_t)std::max(a.seq_tiles, 1));
    a.div_parts = make_fastdiv((uint32_t)a.parts);
    a.div_heads = make_fastdiv((uint32_t)a.c.kv_heads);
    switch (a.c.dim) {
        case 64: launch_score<64>(a, dtype, s); break;
        case 96: launch_score<96>(a, dtype, s); break;
        case 128: launch_score<128>(a, dtype, s); break;
        case 192: launch_score<192>(a, dtype, s); break;
        default: launch_score<256>(a, dtype, s); break;
    }
    const int rc = check_launch();
    if (rc != BNN_OK) return rc;
    const int bins = a.group * a.c.dim + 2;
    // A wave a row where rows fill the chip without more (2664 rows of 313 blocks: 6.0 us, 7.7 with four waves each); else four, up to 2048 blocks in registers
    const long long rows = (long long)a.r.tokens * a.c.kv_heads;
    const bool single = rows >= 1024 && a.r.table_pages <= 512;
    launch(single ? pick_kernel<8, 1> : a.r.table_pages <= 2048 ? pick_kernel<8, 4> : pick_kernel<0, 4>, dim3((unsigned)rows), dim3(single ? 64u : 256u), (size_t)bins * 4, s, a, bins);
    return check_launch();
}

}  // namespace bnn
