// The attention weight that every cached token gets: w[key] = sum over rows and query heads of exp(scale * q . k - lse), with the logarithms that attention gave.
//
// Queries are the rows of the products, keys their columns: S [rows][keys] = Q K^T (v_mfma_f32_16x16x32_bf16).  A lane then holds, of 16 rows, the scores of ONE key at four of them, so the
// sum over rows stays in a lane until the end, where the four lanes of a key add up.  The products' sums begin at -lse / scale, so that a weight is 2^(sum * scale / log 2): one multiplication, one
// exponential, one addition a score.  What scale / log 2 loses by its rounding to 32 bits, e of itself, makes a weight off by e (scale q . k - lse); -lse / scale, in 64 bits until it is stored, takes half of it to
// the middle, e (scale q . k - lse / 2): all rows being off alike, no sum would average it out.  (With 1 / scale in 32 bits, off by as much again, heads of 96 and 192 had twice the plain form's error.)  No sum depends on the order in which workgroups run.
#include "bnn_cache4_attend.h"

namespace bnn {
namespace {

// What a row's sums begin with: -lse / scale, and -infinity (a weight of 0) for no row and for one that saw nothing.
__device__ __forceinline__ float weigh_origin(const Weigh4& a, float lse, bool there) { return there && lse != -__builtin_inff() ? (float)(-(double)lse * a.unscale) : -__builtin_inff(); }
__device__ __forceinline__ float weigh_lse(const Weigh4& a, const Sequence4& s, int head, int row) {
    const int token = fast_div(row, a.div_group), g = row - token * a.group;
    return a.lse[(long long)(s.first + token) * a.c.kv_heads * a.group + head * a.group + g];
}

// Eight elements of a row as TERMS operands of a product: n-th terms to ops[n][m].
template <class T, int TERMS, int LOADS, int M>
__device__ __forceinline__ void weigh_terms(const u32x4 (&raw)[LOADS], bf16x8 (&ops)[TERMS][M], int m) {
    if constexpr (TERMS == 1) {
        ops[0][m] = __builtin_bit_cast(bf16x8, raw[0]);
    } else {
        float x[8];
        if constexpr (LOADS == 2) {
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(raw[i / 4][i % 4]);
        } else {
            typedef T t8 __attribute__((ext_vector_type(8)));
            const t8 y = __builtin_bit_cast(t8, raw[0]);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = (float)y[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            __bf16 terms[TERMS];
            split_terms<TERMS>(x[i], terms);
#pragma unroll
            for (int n = 0; n < TERMS; ++n) ops[n][m][i] = terms[n];
        }
    }
}

// A product of numbers below 2^24, at full rate.
__device__ __forceinline__ uint32_t times24(uint32_t x, uint32_t y) {
    uint32_t z;
    asm("v_mul_u32_u24 %0, %1, %2" : "=v"(z) : "s"(y), "v"(x));
    return z;
}

// Rows [first, last) of a sequence, counted over (token, head of the group), whose token sees one of the keys key0 .. key1; all of them for every row if `all`.
struct Rows4Range {
    int first, last;
};
__device__ __forceinline__ Rows4Range weigh_rows(const Weigh4& a, const Sequence4& s, int base, int key0, int key1) {
    const int t0 = a.causal ? min(max(key0 - base, 0), s.rows) : 0;
    const int t1 = a.window > 0 ? (int)min((long long)s.rows, max((long long)key1 + a.window - base, 0LL)) : s.rows;
    return {t0 * a.group, max(t0, t1) * a.group};
}

// Tiles of 64 rows over such a range, from row `first` on, and how many of them each part has.
struct WeighTiles {
    int first, count, each;
};
__device__ __forceinline__ WeighTiles weigh_row_tiles(const Rows4Range& range, int parts) {
    WeighTiles t = {range.first / 64 * 64, 0, 1};
    if (range.last > range.first) {
        t.count = (range.last - t.first + 63) / 64;
        t.each = (t.count + parts - 1) / parts;
    }
    return t;
}
constexpr int WEIGH_ROWS = 2048;             // rows whose numbers lie in LDS at once

// Few rows: a wave passes over its sequence's keys, 64 at a time, codes of the next 64 under way.  Bounded by memory: 64 single tokens over 500 to 8192 keys, 8 kv heads of 128, 41 us, 4.1 TB/s (a workgroup's first loads
// wait for a length, a page and the rows; 2048 or 8192 workgroups in place of 4096: 57 and 53 us against 52 before pages were looked up ahead; codes loaded two turns ahead leave room for fewer waves: 57).  Few keys, 16 drafts of 5
// tokens within a window of 1000, heads of 192: 13 us, the same chain of loads; 15.8 when every wave loaded its rows.
// RUNS: for rows by the thousand, those too far apart for the kernel below: added up in runs of 256 as there (in every launch, the second sums' registers would cost heads of 128 one of five waves).
template <int D, int DTYPE, int QT, bool RUNS>
__global__ __launch_bounds__(256, 2) void weigh_kernel(Weigh4 a) {
    using T = typename C4Type<DTYPE>::type;
    constexpr int TERMS = C4Type<DTYPE>::terms, M = D / 32, KT = 4;
    using P = Pieces<D>;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, h4 = lane >> 4;
    const int rest = fast_div((int)blockIdx.x, a.div_heads), head = (int)blockIdx.x - rest * a.c.kv_heads;
    const int b = fast_div(rest, a.div_parts), part = rest - b * a.parts;
    const Sequence4 s = c4_sequence(a.r, b);
    const int length = min(s.length, c4_room(a.r, a.c)), base = s.length - s.rows, rows = s.rows * a.group;
    const int stride = a.parts * 4 * 64;
    int key0 = (part * 4 + wave) * 64;
    if (key0 >= length || rows > a.few_most) return;
    const long long weights = ((long long)b * a.c.kv_heads + head) * a.width;

    uint32_t codes[KT][M], exp[KT][P::count];
    unsigned there = 0;
    int pages = 0;                           // of the next 64 keys, one in a lane: their loads' latency passes beside the products
    auto locate = [&](int key) { pages = c4_page(a.r, a.c, b, key + 16 * (lane & 3)); };
    auto load = [&](int key) {
        there = 0;
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            const int p = __builtin_amdgcn_readlane(pages, u);
            there |= p >= 0 ? 1u << u : 0u;
            const Half4 half = {reinterpret_cast<Global4>(reinterpret_cast<uintptr_t>(c4_record(a.c, max(p, 0), head))), (key + 16 * u) & (a.c.page - 1), key + 16 * u, true};
            load_k_half<D>(a.c, half, lane, codes[u], exp[u]);
        }
    };
    // (keys that no row sees, as behind a window, are not loaded)
    auto rows_of = [&](int key) { return weigh_rows(a, s, base, key, min(key + 63, length - 1)); };
    Rows4Range range = rows_of(key0);
    locate(key0);
    bf16x8 q[QT][TERMS][M];
    f32x4 origin[QT];
    // All loads first: the lane's row of every tile (the first of all in place of one that is not there), and the logarithms of four.
    constexpr int LOADS = sizeof(T) == 4 ? 2 : 1;
    u32x4 x[QT][M][LOADS];
    float lse[QT][4];
    auto fetch_rows = [&](int row0) {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const int row = row0 + 16 * t + c < rows ? row0 + 16 * t + c : 0, token = fast_div(row, a.div_group), g = row - token * a.group;
            const T* src = static_cast<const T*>(a.q) + (s.first + token) * a.q_token + (long long)(head * a.group + g) * a.q_head;
            static_for<P::count>([&](auto pc) {
                constexpr int p = pc.value, W = P::width(p), B = P::base(p);
#pragma unroll
                for (int i = 0; i < W / 32; ++i)
#pragma unroll
                    for (int l = 0; l < LOADS; ++l) x[t][B / 32 + i][l] = reinterpret_cast<const u32x4*>(src + B + W / 4 * h4 + 8 * i)[l];
            });
#pragma unroll
            for (int i = 0; i < 4; ++i) lse[t][i] = weigh_lse(a, s, head, min(row0 + 16 * t + 4 * h4 + i, rows - 1));
        }
    };
    auto convert_rows = [&](int row0) {
#pragma unroll
        for (int t = 0; t < QT; ++t) {
            const bool there = row0 + 16 * t + c < rows;
#pragma unroll
            for (int m = 0; m < M; ++m) {
#pragma unroll
                for (int l = 0; l < LOADS; ++l)
#pragma unroll
                    for (int i = 0; i < 4; ++i) x[t][m][l][i] = there ? x[t][m][l][i] : 0u;
                weigh_terms<T, TERMS>(x[t][m], q[t], m);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) origin[t][i] = weigh_origin(a, lse[t][i], row0 + 16 * t + 4 * h4 + i < rows);
        }
    };
    // Rows are loaded, before the first codes, whose pages are waited for, and converted beside those loads, if the wave's last keys are seen (else none of its keys is; a sequence without rows may lie behind the last)
    const Rows4Range of_last = rows_of(key0 + (length - 1 - key0) / stride * stride);
    const bool few = rows <= 16 * QT && of_last.last > of_last.first;
    if (few) fetch_rows(0);
    if (range.last > range.first) load(key0);
    if (few) convert_rows(0);

    for (; key0 < length; key0 += stride) {
        const int key1 = min(key0 + 63, length - 1);
        const float old = a.previous != nullptr && key0 + lane < min(base, length) ? a.decay * a.previous[weights + key0 + lane] : 0.f;
        float sum[KT] = {}, run[KT] = {};    // run: not used without RUNS
        const unsigned present = there;
        locate(min(key0 + stride, length - 1));
        // (almost always one turn: a launch has QT by the mean over its sequences)
        for (int row0 = range.first / (16 * QT) * (16 * QT); row0 < range.last; row0 += 16 * QT) {
            if (rows > 16 * QT) {
                fetch_rows(row0);
                convert_rows(row0);
            }
            const bool full = (!a.causal || key1 <= base + fast_div(row0, a.div_group)) &&
                              (a.window == 0 || base + fast_div(min(row0 + 16 * QT, rows) - 1, a.div_group) - key0 < a.window);
            int pos[QT][4] = {};
            if (!full) {                     // (a row before token 0 sees nothing; differences stay within 32 bits)
#pragma unroll
                for (int t = 0; t < QT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) pos[t][i] = base + fast_div(row0 + 16 * t + 4 * h4 + i, a.div_group);
            }
#pragma unroll
            for (int u = 0; u < KT; ++u) {
                // (codes that seem to change are converted where they are used: taken out of this loop, the operands of 64 keys would fill the registers)
#pragma unroll
                for (int m = 0; m < M; ++m) asm volatile("" : "+v"(codes[u][m]));
                f32x4 score[QT];
#pragma unroll
                for (int t = 0; t < QT; ++t) score[t] = origin[t];
                static_for<P::count>([&](auto pc) {
                    constexpr int p = pc.value, W = P::width(p), B = P::base(p);
                    const float scale = k_scale(exp[u][p], lane);
#pragma unroll
                    for (int i = 0; i < W / 32; ++i) {
                        const bf16x8 k = eight_of(codes[u][B / 32 + i], scale);
#pragma unroll
                        for (int t = 0; t < QT; ++t)
#pragma unroll
                            for (int n = 0; n < TERMS; ++n) score[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[t][n][B / 32 + i], k, score[t], 0, 0, 0);
                    }
                });
                if (!full) {
#pragma unroll
                    for (int t = 0; t < QT; ++t)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int key = key0 + 16 * u + c, at = pos[t][i];
                            if (!((!a.causal || key <= at) && (a.window == 0 || at - key < a.window))) score[t][i] = -__builtin_inff();
                        }
                }
#pragma unroll
                for (int t = 0; t < QT; ++t)
#pragma unroll
                    for (int i = 0; i < 4; ++i) (RUNS ? run : sum)[u] += __builtin_amdgcn_exp2f(score[t][i] * a.scale2);
            }
            if (RUNS && ((row0 + 16 * QT) % 256 == 0 || row0 + 16 * QT >= range.last)) {
#pragma unroll
                for (int u = 0; u < KT; ++u) {
                    sum[u] += run[u];
                    run[u] = 0.f;
                }
            }
        }
        if (key0 + stride < length) {
            range = rows_of(key0 + stride);
            if (range.last > range.first) load(key0 + stride);
        }
        float all = 0.f;
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            const float v = row_sum(sum[u]);
            if (h4 == u && (present >> u & 1)) all = v;
        }
        if (key0 + lane < length) a.out[weights + key0 + lane] = old + all;
    }
}

// A sequence and part of its rows that a launch for many rows has; slot: of its partial sums, counted over the items of sequences in several parts only.
struct WeighItem {
    int b, part, parts, slot;
};
__device__ __forceinline__ int weigh_parts(const Weigh4& a, int b) {         // where sequences differ
    const int rows = c4_sequence(a.r, b).rows * a.group;
    return rows > a.few_most ? max(1, (int)(((long long)rows + (1LL << a.part_shift) - 1) >> a.part_shift)) : 0;
}
// The nth of them, b -1 where there are fewer: a wave counts those of 64 sequences at a time.
__device__ __forceinline__ WeighItem weigh_item(const Weigh4& a, int nth) {
    if (a.r.start == nullptr) {
        const int b = fast_div(nth, a.div_parts);
        return {b, nth - b * a.parts, a.parts, nth};
    }
    const int lane = (int)threadIdx.x & 63;
    int before = 0, single = 0;              // never more than nth; sequences in one part among them
    for (int b0 = 0; b0 < a.r.batch; b0 += 64) {
        const int n = b0 + lane < a.r.batch ? weigh_parts(a, b0 + lane) : 0;
        int sum = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int other = __shfl_up(sum, d);
            if (lane >= d) sum += other;
        }
        const unsigned long long past = __ballot(before + sum > nth);
        if (past != 0) {
            const int at = __ffsll(past) - 1, parts = __builtin_amdgcn_readlane(n, at);
            single += __popcll(__ballot(n == 1) & ((1ULL << at) - 1));
            return {b0 + at, nth - (before + __builtin_amdgcn_readlane(sum, at) - parts), parts, nth - single};
        }
        single += __popcll(__ballot(n == 1));
        before += __builtin_amdgcn_readlane(sum, 63);
    }
    return {-1, 0, 0, 0};
}
// The first slot of sequence b, which is in several parts, or a.slots where its number is no less.
__device__ __forceinline__ int weigh_first_slot(const Weigh4& a, int b) {
    if (a.r.start == nullptr) return b * a.parts;
    const int lane = (int)threadIdx.x & 63;
    int before = 0;
    for (int b0 = 0; b0 < b && before < a.slots; b0 += 64) {
        int n = b0 + lane < b ? weigh_parts(a, b0 + lane) : 0;
        n = n > 1 ? n : 0;
#pragma unroll
        for (int d = 32; d > 0; d >>= 1) n += __shfl_xor(n, d);
        before += n;
    }
    return min(before, a.slots);
}

// Many rows: a workgroup's four waves have 16 * KT keys each, as finished operands in registers, and pass over the same rows, which lie in LDS as finished operands too.  Rows come with whole lines to a load
// (four lanes beside each other a row's 64 bytes: a lane of a matrix operand has a row of its own, and loads of that shape take a cycle of the first cache for every lane), go to registers while the
// step before last is computed and from there to LDS, where the 16-byte places of an operand are exchanged by an exclusive or, so that neither writes nor reads meet.  Numbers that sums begin with lie
// in LDS for 2048 rows at a time.  A tile's exponentials go with the products of the next.
// What bounds it is what a SIMD issues, 96 us (448 cycles for 16 rows and 64 keys, 256 of them exponentials), and waiting: two prompts of 4096 tokens, 32 heads on 8 of 128 elements, bf16, causal, 176 us (0.78 PFLOP/s of what is not masked; the matrix pipe is busy for 36 %).  Without exponentials it would be
// 160, without products 141, without bringing rows 171, without barriers 152.  Rows loaded in the operands' shape, without LDS: 282; every wave with rows of its own, without barriers: 184; steps of 32 rows: 188.
// Rows are cut into parts, so that there are workgroups enough; a part's sums go to the workspace, and weigh_join_kernel adds them up in order.
template <int D, int DTYPE>
__global__ __launch_bounds__(256, D <= 128 && DTYPE != BNN_F32 ? 3 : D == 256 && DTYPE == BNN_F32 ? 1 : 2) void weigh_rows_kernel(Weigh4 a) {
    using T = typename C4Type<DTYPE>::type;
    constexpr int TERMS = C4Type<DTYPE>::terms, M = D / 32, KT = cache4_weigh_tiles(D), LOADS = sizeof(T) == 4 ? 2 : 1;
    constexpr int ROWS = TERMS == 1 ? 64 : 32, TILES = ROWS / 16;    // of a step
    constexpr int CHUNKS = ROWS * D / 8, EACH = (CHUNKS + 255) / 256;        // of eight elements: of a step, of a thread
    __shared__ u32x4 q_ops[2][TERMS][TILES * M][64];
    __shared__ __align__(16) float origins[WEIGH_ROWS];
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, h4 = lane >> 4;
    // heads fastest (rows stay in a die's cache, with eight kv heads or a divisor), the first keys first: causal rows make those the longest
    const int rest = fast_div((int)blockIdx.x, a.div_heads), head = (int)blockIdx.x - rest * a.c.kv_heads;
    const int tile = fast_div(rest, a.div_items), nth = rest - tile * a.items;
    const WeighItem item = weigh_item(a, nth);
    const int b = item.b, part = item.part, parts = item.parts;
    if (b < 0) return;
    const Sequence4 s = c4_sequence(a.r, b);
    const int length = min(s.length, c4_room(a.r, a.c)), base = s.length - s.rows, rows = s.rows * a.group;
    const int block0 = tile * 64 * KT, key0 = block0 + wave * 16 * KT;
    if (block0 >= length) return;

    const WeighTiles all_tiles = weigh_row_tiles(weigh_rows(a, s, base, block0, min(block0 + 64 * KT, length) - 1), parts);
    const int first = all_tiles.first + 64 * all_tiles.each * part, steps = 64 / ROWS * max(min(all_tiles.count - all_tiles.each * part, all_tiles.each), 0);
    if (steps == 0 && parts > 1) return;   // weigh_join_kernel knows

    float sum[KT] = {};
    if (steps > 0) {
        // The thread's chunks of a step: rows line + e * LINES, elements 8 * at on; their bytes are counted from the first row of the 2048 (the host sees to it that 32 bits do).
        constexpr int LINES = 256 / (D / 8);                         // (D of 96: 21 and a third; its chunks are divided each)
        const int line = (int)threadIdx.x / (D / 8), at = (int)threadIdx.x % (D / 8);
        auto chunk_of = [&](int e, int& r, int& column) {
            if constexpr (256 % (D / 8) == 0) {
                r = line + e * LINES;
                column = at;
            } else {
                const int chunk = (int)threadIdx.x + 256 * e;
                r = chunk / (D / 8);
                column = chunk % (D / 8);
            }
        };
        const char* rows_at = nullptr;       // of the 2048
        int rows_from = 0, phase = 0;        // their first step; the first row's query head of the group
        auto begin_rows = [&](int step) {
            const int row = first + ROWS * step, token = fast_div(row, a.div_group);
            rows_from = step;
            phase = row - token * a.group;
            rows_at = reinterpret_cast<const char*>(static_cast<const T*>(a.q) + (long long)(s.first + token) * a.q_token + (long long)head * a.group * a.q_head);
        };
        u32x4 raw[EACH][LOADS];
        uint32_t offsets[EACH];
        // Bytes from rows_at to the thread's chunks of a step.  Of rows that are not there the last is loaded; what comes of it is masked.
        auto locate = [&](int step) {
            const int most = rows - 1 - first - ROWS * step, ahead = ROWS * (step - rows_from) + phase;
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                int r, column;
                chunk_of(e, r, column);
                const uint32_t n = (uint32_t)(ahead + min(r, most));
                const uint32_t token = (a.div_group.m == 0u ? n : __umulhi(n, a.div_group.m)) >> a.div_group.sh, g = n - times24(token, (uint32_t)a.group);
                offsets[e] = (times24(token, (uint32_t)a.q_token) + times24(g, (uint32_t)a.q_head) + 8 * column) * (uint32_t)sizeof(T);
            }
        };
        // Where a step has whole tokens, its chunks lie as those of the first, a step's bytes further on
        const bool whole = ROWS % a.group == 0;
        const long long step_bytes = whole ? (long long)(ROWS / a.group) * a.q_token * (long long)sizeof(T) : 0;
        auto fetch = [&](int step) {
            const bool last = ROWS * (step + 1) > rows - first;
            if (!whole || last) locate(step);
            const char* from = rows_at + (whole && !last ? (step - rows_from) * step_bytes : 0);
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                if (CHUNKS % 256 != 0 && (int)threadIdx.x + 256 * e >= CHUNKS) continue;
#pragma unroll
                for (int l = 0; l < LOADS; ++l) raw[e][l] = reinterpret_cast<const u32x4*>(from + offsets[e])[l];
            }
        };
        auto store = [&](int buffer) {
#pragma unroll
            for (int e = 0; e < EACH; ++e) {
                if (CHUNKS % 256 != 0 && (int)threadIdx.x + 256 * e >= CHUNKS) continue;
                int r, column;
                chunk_of(e, r, column);
                const int m = column / 4, quarter = column % 4;
                u32x4* to = &q_ops[buffer][0][(r / 16) * M + m][16 * quarter + ((r % 16) ^ (12 * (quarter & 1) + (m & 3)))];
                bf16x8 ops[TERMS][1];
                weigh_terms<T, TERMS>(raw[e], ops, 0);
#pragma unroll
                for (int n = 0; n < TERMS; ++n) to[n * TILES * M * 64] = __builtin_bit_cast(u32x4, ops[n][0]);
            }
        };
        begin_rows(0);
        locate(0);
        fetch(0);
        // Keys in the order of elements that rows have: product m contracts elements 32 m .. + 31, eight a lane
        bf16x8 k[KT][M];
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            const int key = key0 + 16 * u;
            const int page = __builtin_amdgcn_readfirstlane(c4_page(a.r, a.c, b, key));
            const Global4 record = reinterpret_cast<Global4>(reinterpret_cast<uintptr_t>(c4_record(a.c, max(page, 0), head)));
            const uint32_t offset = key & (a.c.page - 1);
#pragma unroll
            for (int m = 0; m < M; ++m) {
                const uint32_t codes = load_at<uint32_t>(record, (offset + c) * (D / 2) + 16 * m + 4 * h4);
                const uint32_t exp = load_at<uint32_t>(record, (uint32_t)a.c.k_exps + m * (uint32_t)a.c.page + offset + (c & 12u));
                k[u][m] = eight_of(codes, k_scale(exp, lane));
            }
        }
        const int operand = 16 * h4 + (c ^ (12 * (h4 & 1)));                // the lane's place, but for m
        float some[KT] = {};                 // of 256 rows: thousands of terms in one fp32 sum would lose its last digits
        f32x4 score[KT];                     // of the tile before
#pragma unroll
        for (int u = 0; u < KT; ++u) score[u] = f32x4{-__builtin_inff(), -__builtin_inff(), -__builtin_inff(), -__builtin_inff()};
        auto add_up = [&]() {
#pragma unroll
            for (int u = 0; u < KT; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) some[u] += __builtin_amdgcn_exp2f(score[u][i] * a.scale2);
            // (they stay here: moved to where the sums are used next, nothing would run beside them)
#pragma unroll
            for (int u = 0; u < KT; ++u) asm volatile("" : "+v"(some[u]));
        };
        auto pass_step = [&](int step) {
            __syncthreads();
            store((step + 1) & 1);
            fetch(min(step + 2, steps - 1));
        };
        auto one_step = [&](int local, int step, auto masked) {      // local: of the steps whose rows' numbers lie in LDS
            pass_step(step);
#pragma unroll
            for (int t = 0; t < TILES; ++t) {
                const f32x4 origin = *reinterpret_cast<const f32x4*>(&origins[ROWS * local + 16 * t + 4 * h4]);
                f32x4 next[KT];
#pragma unroll
                for (int u = 0; u < KT; ++u) next[u] = origin;
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int n = 0; n < TERMS; ++n) {
                        const bf16x8 q = __builtin_bit_cast(bf16x8, q_ops[step & 1][n][t * M + m][operand ^ (m & 3)]);
#pragma unroll
                        for (int u = 0; u < KT; ++u) next[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q, k[u][m], next[u], 0, 0, 0);
                    }
                add_up();
                if constexpr (decltype(masked)::value) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = first + ROWS * step + 16 * t + 4 * h4 + i, pos = base + fast_div(r, a.div_group);
#pragma unroll
                        for (int u = 0; u < KT; ++u) {
                            const int key = key0 + 16 * u + c;
                            next[u][i] = r < rows && (!a.causal || key <= pos) && (a.window == 0 || pos - key < a.window) ? next[u][i] : -__builtin_inff();
                        }
                    }
                }
#pragma unroll
                for (int u = 0; u < KT; ++u) score[u] = next[u];
            }
        };
        // Steps whose rows all see all of the wave's keys; and the first with a row that sees one of them
        int clear_from = 0, clear_to = min(steps, (rows - first) / ROWS), begin = 0;
        if (a.causal) {                      // from the first row whose token is at the last key, or the first
            const long long r = (long long)(key0 + 16 * KT - 1 - base) * a.group - first, r0 = (long long)(key0 - base) * a.group - first;
            clear_from = (int)min(max((r + ROWS - 1) / ROWS, 0LL), (long long)steps);
            begin = (int)min(max(r0 / ROWS, 0LL), (long long)steps);
        }
        if (a.window > 0) {                  // up to the last row whose token still sees the first key
            const long long r = ((long long)key0 + a.window - base) * a.group - first;
            clear_to = (int)min(max(r / ROWS, 0LL), (long long)clear_to);
        }
        clear_to = max(clear_to, clear_from);
        store(0);
        fetch(min(1, steps - 1));
        for (int chunk = 0; chunk < steps; chunk += WEIGH_ROWS / ROWS) {
            const int here = min(WEIGH_ROWS / ROWS, steps - chunk);
            if (chunk > 0) {
                begin_rows(chunk);           // (whole: the rows before began with a whole token as well)
                __syncthreads();
            }
            for (int i = (int)threadIdx.x; i < ROWS * here; i += 256) {
                const int row = first + ROWS * chunk + i;
                origins[i] = weigh_origin(a, weigh_lse(a, s, head, min(row, rows - 1)), row < rows);
            }
            // waves go through different kinds of steps, each with one barrier
            for (int i = chunk; i < chunk + here;) {
                const int end = min(chunk + here, i + 256 / ROWS), from = min(max(clear_from, i), end), to = min(max(clear_to, i), end);
                for (; i < min(begin, end); ++i) pass_step(i);
                for (; i < from; ++i) one_step(i - chunk, i, std::true_type{});
                for (; i < to; ++i) one_step(i - chunk, i, std::false_type{});
                for (; i < end; ++i) one_step(i - chunk, i, std::true_type{});
#pragma unroll
                for (int u = 0; u < KT; ++u) {
                    sum[u] += some[u];
                    some[u] = 0.f;
                }
            }
        }
        add_up();
#pragma unroll
        for (int u = 0; u < KT; ++u) sum[u] += some[u];
    }

    const long long sequence = (long long)b * a.c.kv_heads + head;
    float all = 0.f;
#pragma unroll
    for (int u = 0; u < KT; ++u) {
        const float v = row_sum(sum[u]);
        if (h4 == u) all = v;
    }
    const int key = key0 + lane;
    if (lane >= 16 * KT || key >= length) return;
    if (parts > 1) {
        if (item.slot < a.slots) a.partial[((long long)item.slot * a.c.kv_heads + head) * a.width4 + key] = all;     // (as they are, unless sequences' runs overlap)
    } else {
        if (c4_page(a.r, a.c, b, key) < 0) all = 0.f;
        const float old = a.previous != nullptr && key < base ? a.decay * a.previous[sequence * a.width + key] : 0.f;
        a.out[sequence * a.width + key] = old + all;
    }
}

// Adds up the parts' sums, those that have rows for the key's tile (of `tile` keys).
__global__ __launch_bounds__(256) void weigh_join_kernel(Weigh4 a, int tile, int blocks, FastDiv div_blocks) {
    const int rest = fast_div((int)blockIdx.x, div_blocks), head = (int)blockIdx.y;
    const int key = ((int)blockIdx.x - rest * blocks) * 256 + (int)threadIdx.x, b = rest;
    const Sequence4 s = c4_sequence(a.r, b);
    const int length = min(s.length, c4_room(a.r, a.c)), base = s.length - s.rows;
    const int parts = a.r.start == nullptr ? a.parts : weigh_parts(a, b);
    if (parts < 2) return;                   // those that weigh_kernel or one workgroup has
    const int slot = weigh_first_slot(a, b);
    if (key >= length) return;
    const int block0 = key / tile * tile;
    const Rows4Range range = weigh_rows(a, s, base, block0, min(block0 + tile, length) - 1);
    const long long sequence = (long long)b * a.c.kv_heads + head;
    float all = 0.f;
    if (c4_page(a.r, a.c, b, key) >= 0) {
        const WeighTiles tiles = weigh_row_tiles(range, parts);
        for (int p = 0; p * tiles.each < tiles.count && slot + p < a.slots; ++p) all += a.partial[((long long)(slot + p) * a.c.kv_heads + head) * a.width4 + key];
    }
    const float old = a.previous != nullptr && key < base ? a.decay * a.previous[sequence * a.width + key] : 0.f;
    a.out[sequence * a.width + key] = old + all;
}

template <int D, int DTYPE>
int launch_weigh(Weigh4 a, const WeighPlan4& p, hipStream_t s) {
    if (p.row_tiles > 0) {
        a.parts = p.few_parts;
        a.div_parts = make_fastdiv((uint32_t)a.parts);
        const dim3 grid((unsigned)p.few_groups);
        if constexpr (cache4_weigh_two(D, DTYPE)) {
            if (p.row_tiles == 2) launch(weigh_kernel<D, DTYPE, 2, false>, grid, dim3(256), 0, s, a);
        }
        if (p.row_tiles == 1 && !p.runs) launch(weigh_kernel<D, DTYPE, 1, false>, grid, dim3(256), 0, s, a);
        if (p.row_tiles == 1 && p.runs) launch(weigh_kernel<D, DTYPE, 1, true>, grid, dim3(256), 0, s, a);
    }
    if (p.items > 0) {
        a.parts = p.many_parts;
        a.div_parts = make_fastdiv((uint32_t)a.parts);
        launch(weigh_rows_kernel<D, DTYPE>, dim3((unsigned)p.many_groups), dim3(256), 0, s, a);
    }
    if (p.workspace_bytes != 0) {
        const int blocks = (int)cdiv((long long)a.r.table_pages << a.c.page_shift, 256);
        launch(weigh_join_kernel, dim3((unsigned)((long long)blocks * a.r.batch), (unsigned)a.c.kv_heads), dim3(256), 0, s, a, 64 * cache4_weigh_tiles(D), blocks, make_fastdiv((uint32_t)blocks));
    }
    return check_launch();
}
template <int D>
int launch_weigh_type(const Weigh4& a, const WeighPlan4& p, int dtype, hipStream_t s) {
    if (dtype == BNN_BF16) return launch_weigh<D, BNN_BF16>(a, p, s);
    if (dtype == BNN_F16) return launch_weigh<D, BNN_F16>(a, p, s);
    return launch_weigh<D, BNN_F32>(a, p, s);
}

}  // namespace

int launch_cache4_weigh(const Weigh4& a, const WeighPlan4& p, int dtype, hipStream_t s) {
    switch (a.c.dim) {
        case 64: return launch_weigh_type<64>(a, p, dtype, s);
        case 96: return launch_weigh_type<96>(a, p, dtype, s);
        case 128: return launch_weigh_type<128>(a, p, dtype, s);
        case 192: return launch_weigh_type<192>(a, p, dtype, s);
        default: return launch_weigh_type<256>(a, p, dtype, s);
    }
}

}  // namespace bnn
