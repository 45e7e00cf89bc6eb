// Rotation of pairs of elements by angles that grow with a token's position: what the stand-alone kernel and the one that writes into the 4-bit cache share.
#ifndef BNN_ROTARY_H
#define BNN_ROTARY_H

#include "bnn_cache4.h"

namespace bnn {

// A rotation as the kernels see it.
struct Rotation {
    const double* frequencies;               // [pairs], radians a position
    const int32_t* positions;                // [tokens], or nullptr: a token's place in its sequence
    int pairs;
    double magnitude, sign;                  // sign: -1 for the inverse
};

// (magnitude cos t, sign magnitude sin t).  t is reduced to [-pi/4, pi/4] by multiples of pi/2 in two parts -- the first subtraction is exact, t and the product being multiples
// of the same power of two far below the difference's leading bit -- and the series of sine and cosine are summed there up to terms of 4e-17 and 2e-18.  Everything is in 64 bits: the angle
// of position 10^6 has 20 bits in front of the point, and a rotated key decides about 4-bit codes, whose borders 32-bit results of another order would pass now and then.
__device__ __forceinline__ double2 turn_of(double t, double magnitude, double sign) {
    const double n = rint(t * 0.63661977236758134308);               // 2 / pi
    double r = fma(-n, 1.57079632679489655800, t);                   // pi / 2, and what it lacks
    r = fma(-n, 6.12323399573676603587e-17, r);
    const double q = r * r;
    double s = -1.0 / 1307674368000.0;
    s = fma(s, q, 1.0 / 6227020800.0);
    s = fma(s, q, -1.0 / 39916800.0);
    s = fma(s, q, 1.0 / 362880.0);
    s = fma(s, q, -1.0 / 5040.0);
    s = fma(s, q, 1.0 / 120.0);
    s = fma(s, q, -1.0 / 6.0);
    s = fma(s * q, r, r);
    double c = 1.0 / 20922789888000.0;
    c = fma(c, q, -1.0 / 87178291200.0);
    c = fma(c, q, 1.0 / 479001600.0);
    c = fma(c, q, -1.0 / 3628800.0);
    c = fma(c, q, 1.0 / 40320.0);
    c = fma(c, q, -1.0 / 720.0);
    c = fma(c, q, 1.0 / 24.0);
    c = fma(c, q, -0.5);
    c = fma(c, q, 1.0);
    const int quarter = (int)(n - 4.0 * floor(n * 0.25));            // n mod 4, n being too large for an integer type perhaps
    const double cs = quarter & 1 ? s : c, sn = quarter & 1 ? c : s;
    return double2{magnitude * (quarter == 1 || quarter == 2 ? -cs : cs), sign * magnitude * (quarter >= 2 ? -sn : sn)};
}

// One element of a pair (a, b) turned: a cos - b sin for the first (with the sine's sign turned for the second, a and b exchanged), rounded to fp32 once.
__device__ __forceinline__ float turned(float a, float b, double c, double s) { return (float)fma((double)a, c, -((double)b * s)); }

// N consecutive elements as fp32; aligned to their bytes, or to 16.
template <int N, class T>
__device__ __forceinline__ void load_elements(const T* p, float (&x)[N]) {
    if constexpr (N == 8) {
        c4_load8(p, x);
    } else {
        typedef T tn __attribute__((ext_vector_type(N)));
        if constexpr (N == 1) {
            x[0] = (float)*p;
        } else {
            const tn a = *reinterpret_cast<const tn*>(p);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = (float)a[i];
        }
    }
}
template <int N, class T>
__device__ __forceinline__ void store_elements(T* p, const float (&x)[N]) {
    if constexpr (N == 1) *p = (T)x[0];
    else c4_store<N>(p, x);
}

// Items of V pairs, or of V elements that are not rotated, of a head; an item is read whole before it is written, so out may be x.  turns: the token's, [pairs].
template <int V, bool NEIGHBOURS, class T>
__device__ __forceinline__ void rotate_item(const T* x, T* out, int item, int pairs, const double2* turns) {
    const int turning = pairs / V;           // V divides
    if (item >= turning) {
        const int at = 2 * pairs + (item - turning) * V;
        float a[V];
        load_elements<V>(x + at, a);
        store_elements<V>(out + at, a);
        return;
    }
    const int p = item * V;
    float a[V], b[V];
    if constexpr (NEIGHBOURS) {
        float lo[V], hi[V];                  // V pairs are 2 V elements
        load_elements<V>(x + 2 * p, lo);
        load_elements<V>(x + 2 * p + V, hi);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            a[i] = 2 * i < V ? lo[2 * i < V ? 2 * i : 0] : hi[2 * i < V ? 0 : 2 * i - V];
            b[i] = 2 * i + 1 < V ? lo[2 * i + 1 < V ? 2 * i + 1 : 0] : hi[2 * i + 1 < V ? 0 : 2 * i + 1 - V];
        }
    } else {
        load_elements<V>(x + p, a);
        load_elements<V>(x + p + pairs, b);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const double2 t = turns[p + i];
        const float u = turned(a[i], b[i], t.x, t.y), v = turned(b[i], a[i], t.x, -t.y);
        a[i] = u;
        b[i] = v;
    }
    if constexpr (NEIGHBOURS) {
        float lo[V], hi[V];
#pragma unroll
        for (int i = 0; i < V; ++i) {
            (2 * i < V ? lo[2 * i < V ? 2 * i : 0] : hi[2 * i < V ? 0 : 2 * i - V]) = a[i];
            (2 * i + 1 < V ? lo[2 * i + 1 < V ? 2 * i + 1 : 0] : hi[2 * i + 1 < V ? 0 : 2 * i + 1 - V]) = b[i];
        }
        store_elements<V>(out + 2 * p, lo);
        store_elements<V>(out + 2 * p + V, hi);
    } else {
        store_elements<V>(out + p, a);
        store_elements<V>(out + p + pairs, b);
    }
}

// The widest V (8, 4, 2, 1) that divides all of these and whose elements' bytes pass no 16 (fp32's eight are two such accesses).
inline int rotary_width(int size, std::initializer_list<long long> divided, std::initializer_list<const void*> pointers) {
    int v = 8;
    for (const long long d : divided)
        while (d % v != 0) v /= 2;
    for (const void* p : pointers)
        while (reinterpret_cast<uintptr_t>(p) % std::min(16, v * size) != 0) v /= 2;
    return v;
}

constexpr int ROTARY_MAX_PAIRS = 1024;
constexpr int ROTARY_TURNS = 1024;           // pairs and tokens of a workgroup, in LDS: 16 KB

int launch_rotary(const void* x, void* out, int dtype, int tokens, int heads, int dim, long long x_token, long long x_head, long long out_token, long long out_head, int width,
                  const Rotation& rot, int neighbours, hipStream_t s);
struct WriteRotary4 {
    Cache4 c;
    Rows4 r;
    Rotation rot;
    const void *q, *k, *v;
    void* q_out;
    long long q_token, q_head, k_token, k_head, v_token, v_head;
    int heads;                               // of q
};
int launch_cache4_write_rotary(const WriteRotary4& a, int dtype, int neighbours, int width, hipStream_t s);

}  // namespace bnn
#endif
