// The attention weight that every cached token gets: w[key] = sum over rows and query heads of exp(scale * q . k - lse), with the logarithms that attention gave.
//
// Queries are the rows of the products, keys their columns: S [rows][keys] = Q K^T (v_mfma_f32_16x16x32_bf16).  A lane then holds, of 16 rows, the scores of ONE key at four of them, so the
// sum over rows stays in a lane until the end, where the four lanes of a key add up.  A wave keeps 16 * KT keys as finished operands in registers and passes over the rows that see one of
// them; nothing is exchanged between waves, and no sum depends on the order in which workgroups run.
#include "bnn_cache4_attend.h"

namespace bnn {
namespace {

template <int D, int DTYPE, int KT>
__global__ __launch_bounds__(256, 2) void weigh_kernel(Weigh4 a) {
    using T = typename C4Type<DTYPE>::type;
    constexpr int TERMS = C4Type<DTYPE>::terms, M = D / 32;
    using P = Pieces<D>;
    const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int c = lane & 15, h4 = lane >> 4;
    const int rest = fast_div((int)blockIdx.x, a.div_heads), head = (int)blockIdx.x - rest * a.c.kv_heads;
    const int b = fast_div(rest, a.div_key_tiles), tile = rest - b * a.key_tiles;
    const Sequence4 s = c4_sequence(a.r, b);
    const int length = min(s.length, c4_room(a.r, a.c)), base = s.length - s.rows;
    const int key0 = (tile * 4 + wave) * 16 * KT;
    if (key0 >= length) return;

    bf16x8 k[KT][M];
    bool there[KT];
#pragma unroll
    for (int u = 0; u < KT; ++u) {
        const int key = key0 + 16 * u;
        const int page = __builtin_amdgcn_readfirstlane(c4_page(a.r, a.c, b, key));
        there[u] = page >= 0;
        const Half4 half = {reinterpret_cast<Global4>(reinterpret_cast<uintptr_t>(c4_record(a.c, max(page, 0), head))), key & (a.c.page - 1), key, there[u]};
        uint32_t codes[M], exp[P::count];
        load_k_half<D>(a.c, half, lane, codes, exp);
        static_for<P::count>([&](auto pc) {
            constexpr int p = pc.value, W = P::width(p), B = P::base(p);
            const float scale = k_scale(exp[p], lane);
#pragma unroll
            for (int i = 0; i < W / 32; ++i) k[u][B / 32 + i] = eight_of(codes[B / 32 + i], scale);
        });
    }

    // Rows, counted over (token, head of the group), whose token sees one of the keys
    const int key1 = min(key0 + 16 * KT, length) - 1;
    const int t0 = a.causal ? min(max(key0 - base, 0), s.rows) : 0;
    const int t1 = a.window > 0 ? (int)min((long long)s.rows, max((long long)key1 + a.window - base, 0LL)) : s.rows;
    float sum[KT] = {}, part[KT] = {};       // sums of 256 rows are added up apart: thousands of terms in one fp32 sum would lose its last digits
    for (int row0 = t0 * a.group; row0 < t1 * a.group; row0 += 16) {
        bf16x8 q[TERMS][M];
        {
            const int row = row0 + c, token = fast_div(row, a.div_group), g = row - token * a.group;
            load_q<D, TERMS>(static_cast<const T*>(a.q) + (s.first + token) * a.q_token + (long long)(head * a.group + g) * a.q_head, row < s.rows * a.group, lane, q);
        }
        float lse[4];
        int pos[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = row0 + 4 * h4 + i, token = fast_div(row, a.div_group), g = row - token * a.group;
            const bool valid = row < s.rows * a.group;
            lse[i] = valid ? a.lse[(long long)(s.first + token) * a.c.kv_heads * a.group + head * a.group + g] : __builtin_inff();
            if (lse[i] == -__builtin_inff()) lse[i] = __builtin_inff();      // a row that sees nothing gives nothing
            pos[i] = base + token;
        }
#pragma unroll
        for (int u = 0; u < KT; ++u) {
            f32x4 score = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < M; ++m)
#pragma unroll
                for (int n = 0; n < TERMS; ++n) score = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[n][m], k[u][m], score, 0, 0, 0);
            const int key = key0 + 16 * u + c;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float p = __builtin_amdgcn_exp2f(fmaf(score[i], a.scale, -lse[i]) * 1.4426950408889634f);
                const bool seen = (!a.causal || key <= pos[i]) && (a.window == 0 || pos[i] - key < a.window);
                part[u] += seen ? p : 0.f;
            }
        }
        if ((row0 - t0 * a.group) % 256 == 240) {
#pragma unroll
            for (int u = 0; u < KT; ++u) {
                sum[u] += part[u];
                part[u] = 0.f;
            }
        }
    }

#pragma unroll
    for (int u = 0; u < KT; ++u) {
        const float all = row_sum(sum[u] + part[u]);
        const int key = key0 + 16 * u + c;
        if (h4 != u % 4 || key >= length) continue;
        const long long at = ((long long)b * a.c.kv_heads + head) * a.width + key;
        const float old = a.previous != nullptr && key < base ? a.decay * a.previous[at] : 0.f;
        a.out[at] = there[u] ? old + all : old;
    }
}

template <int D, int KT>
int launch_weigh(const Weigh4& a, int dtype, hipStream_t s) {
    const dim3 grid((unsigned)((long long)a.key_tiles * a.r.batch * a.c.kv_heads));
    if (dtype == BNN_BF16) launch(weigh_kernel<D, BNN_BF16, KT>, grid, dim3(256), 0, s, a);
    else if (dtype == BNN_F16) launch(weigh_kernel<D, BNN_F16, KT>, grid, dim3(256), 0, s, a);
    else launch(weigh_kernel<D, BNN_F32, KT>, grid, dim3(256), 0, s, a);
    return check_launch();
}
template <int D>
int launch_weigh_dim(Weigh4& a, int dtype, hipStream_t s) {
    constexpr int KT = D == 256 ? 2 : 4;
    const long long tiles = cdiv((long long)a.r.table_pages << a.c.page_shift, 64 * KT);
    if (tiles * a.r.batch * a.c.kv_heads >= C4_THREADS / 256) return BNN_ERR_UNSUPPORTED;
    a.key_tiles = (int)tiles;
    a.div_key_tiles = make_fastdiv((uint32_t)tiles);
    return launch_weigh<D, KT>(a, dtype, s);
}

}  // namespace

int launch_cache4_weigh(Weigh4 a, int dtype, hipStream_t s) {
    switch (a.c.dim) {
        case 64: return launch_weigh_dim<64>(a, dtype, s);
        case 96: return launch_weigh_dim<96>(a, dtype, s);
        case 128: return launch_weigh_dim<128>(a, dtype, s);
        case 192: return launch_weigh_dim<192>(a, dtype, s);
        default: return launch_weigh_dim<256>(a, dtype, s);
    }
}

}  // namespace bnn
