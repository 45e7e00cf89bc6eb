// The 4-bit key/value cache: writing new tokens and reading them back.
//
// A group of 32 elements has one scale, a power of two: the smallest 2^e that lets its largest magnitude pass as at most 6, E2M1's largest.  No
// element saturates then, and an element is off by at most half a step of E2M1 (an eighth of its own magnitude or a quarter of the
// scale, whichever is more).  Four lanes carry a group, eight elements each: the largest magnitude is found on the bit patterns (order of
// non-negative floats is that of their bits, with infinities and NaN on top), the codes come from the conversion instruction, which rounds to nearest, ties to even.
//
// Both kernels move bytes and compute next to nothing.  A workgroup takes one kv head and 2048 / D consecutive tokens, K and V together, so that the
// bytes of scales of neighbouring tokens, which lie side by side, come from one workgroup.  32768 tokens of 8 heads of 128, bf16: written in 39 us (172 MB, 4.4 TB/s), read
// in 28 (6.2 TB/s); one token each of 8 sequences 3.4 and 3.0.  Two or four tokens a thread, all loads first, made no difference.
#include "bnn_cache4.h"

namespace bnn {
namespace {

// Value of the lane whose number in its group of four differs in the bits of X.
template <int X>
__device__ __forceinline__ uint32_t quad_xor(uint32_t v) {
    constexpr int perm = X == 1 ? 0xB1 : 0x4E;          // lanes 1,0,3,2 / 2,3,0,1
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, perm, 0xf, 0xf, true);
}

struct Place {
    int page, offset;                                   // page < 0: nowhere
};

__device__ __forceinline__ Place place_of_row(const Cache4& c, const Rows4& r, int t) {
    const int b = c4_sequence_of(r, t);
    const Sequence4 s = c4_sequence(r, b);
    const int i = t - s.first;
    const int token = s.length - s.rows + i;
    Place p;
    p.page = i < 0 || i >= s.rows ? -1 : c4_page(r, c, b, token);
    p.offset = token & (c.page - 1);
    return p;
}

// Eight elements of a group of 32 that four lanes share: returns the codes, sets the scale's byte.
__device__ __forceinline__ uint32_t quantise(const float (&x)[8], uint32_t& byte) {
    uint32_t high = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) high = max(high, __float_as_uint(x[i]) & 0x7fffffffu);
    high = max(high, quad_xor<1>(high));
    high = max(high, quad_xor<2>(high));
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

__device__ __forceinline__ void dequantise(uint32_t codes, uint32_t byte, float (&x)[8]) {
    const float scale = c4_scale(byte);
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 1),
                c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, 3);
    x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1]; x[4] = c[0]; x[5] = c[1]; x[6] = d[0]; x[7] = d[1];
}

template <class T>
__global__ __launch_bounds__(256) void write_kernel(Cache4 c, Rows4 r, const T* __restrict__ k, const T* __restrict__ v, long long k_token, long long k_head,
                                                    long long v_token, long long v_head, FastDiv div_lanes, int rows_block) {
    const int lanes = c.dim / 8;
    const int local = fast_div((int)threadIdx.x, div_lanes), at = (int)threadIdx.x - local * lanes;
    const int head = (int)blockIdx.y;
    const int t = (int)blockIdx.x * rows_block + local;
    if (local >= rows_block || t >= r.tokens) return;            // whole groups of four lanes
    const Place p = place_of_row(c, r, t);
    if (p.page < 0) return;
    float x[8], y[8];
    c4_load8(k + t * k_token + head * k_head + at * 8, x);
    c4_load8(v + t * v_token + head * v_head + at * 8, y);
    uint8_t* rec = c4_record(c, p.page, head);
    uint32_t kb, vb;
    const uint32_t kc = quantise(x, kb), vc = quantise(y, vb);
    const int row = c.dim / 2 * p.offset + at * 4;
    *reinterpret_cast<uint32_t*>(rec + row) = kc;
    *reinterpret_cast<uint32_t*>(rec + c.v_codes + row) = vc;
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) bits |= (x[i] >= 0.f ? 1u : 0u) << i;
    bits <<= 8 * (at & 3);
    bits |= quad_xor<1>(bits);
    bits |= quad_xor<2>(bits);
    if ((at & 3) == 0) {
        const int e = (at >> 2) * c.page + p.offset;
        rec[c.k_exps + e] = (uint8_t)kb;
        rec[c.v_exps + e] = (uint8_t)vb;
        if (c.signs) *reinterpret_cast<uint32_t*>(rec + c.signs + p.offset * (c.dim / 8) + at) = bits;
    }
}

template <class T>
__global__ __launch_bounds__(256) void read_kernel(Cache4 c, Rows4 r, T* __restrict__ k, T* __restrict__ v, FastDiv div_lanes, int rows_block) {
    const int lanes = c.dim / 8;
    const int local = fast_div((int)threadIdx.x, div_lanes), at = (int)threadIdx.x - local * lanes;
    const int head = (int)blockIdx.y;
    const int t = (int)blockIdx.x * rows_block + local;
    if (local >= rows_block || t >= r.tokens) return;
    const Place p = place_of_row(c, r, t);
    float x[8] = {}, y[8] = {};
    if (p.page >= 0) {
        const uint8_t* rec = c4_record(c, p.page, head);
        const int row = c.dim / 2 * p.offset + at * 4, e = (at >> 2) * c.page + p.offset;
        const uint32_t kc = *reinterpret_cast<const uint32_t*>(rec + row), vc = *reinterpret_cast<const uint32_t*>(rec + c.v_codes + row);
        dequantise(kc, rec[c.k_exps + e], x);
        dequantise(vc, rec[c.v_exps + e], y);
    }
    const long long out = ((long long)t * c.kv_heads + head) * c.dim + at * 8;
    c4_store8(k + out, x);
    c4_store8(v + out, y);
}

}  // namespace

int launch_cache4_write(const Cache4& c, const Rows4& r, const void* k, const void* v, int dtype, long long k_token, long long k_head, long long v_token,
                        long long v_head, hipStream_t s) {
    const int lanes = c.dim / 8, rows_block = cache4_block_rows(c);
    const dim3 grid((unsigned)cache4_row_blocks(c, r), (unsigned)c.kv_heads);
    auto go = [&](auto type) {
        using T = decltype(type);
        launch(write_kernel<T>, grid, dim3(256), 0, s, c, r, static_cast<const T*>(k), static_cast<const T*>(v), k_token, k_head, v_token, v_head,
               make_fastdiv((uint32_t)lanes), rows_block);
    };
    if (dtype == BNN_BF16) go(__bf16{});
    else if (dtype == BNN_F16) go(_Float16{});
    else go(float{});
    return check_launch();
}

int launch_cache4_read(const Cache4& c, const Rows4& r, void* k, void* v, int dtype, hipStream_t s) {
    const int lanes = c.dim / 8, rows_block = cache4_block_rows(c);
    const dim3 grid((unsigned)cache4_row_blocks(c, r), (unsigned)c.kv_heads);
    auto go = [&](auto type) {
        using T = decltype(type);
        launch(read_kernel<T>, grid, dim3(256), 0, s, c, r, static_cast<T*>(k), static_cast<T*>(v), make_fastdiv((uint32_t)lanes), rows_block);
    };
    if (dtype == BNN_BF16) go(__bf16{});
    else if (dtype == BNN_F16) go(_Float16{});
    else go(float{});
    return check_launch();
}

}  // namespace bnn
