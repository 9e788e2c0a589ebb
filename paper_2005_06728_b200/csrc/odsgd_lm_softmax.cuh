// Maximum and sum of exponentials of rows of logits: shared by the scores, the policy loss and the verification of
// drafted tokens.
#pragma once

#include "odsgd_lm_elements.cuh"

namespace odsgd_lm {

constexpr int kRowVectors = 4;  // vectors a thread has in flight

// Maximum m of a set of z and sum of exp(c (z - m)); m = -inf, s = 0 for the empty set.
struct MaxSum {
    float m, s;
};

// exp(c (z - m)) in the precision the row's type deserves: 32-bit logits through expf; 16-bit ones
// through the base-2 exponential of the special-function unit (2^-22 relative, far below the 2^-8 or
// 2^-11 that the gradient is rounded to).  The difference comes first: the largest element has
// exactly 1, and c m alone would overflow where a mask holds the type's lowest value.
// For 16-bit rows the inverse temperature is bounded where its product with log2 e is still finite, so that
// the largest element's difference of 0 stays 0 (beyond, only logits less than 1e-36 apart would notice).
template <typename T>
struct RowExp {
    float c, m;
    static float bounded(float inv_temp) { return sizeof(T) == 4 ? inv_temp : fminf(inv_temp, 2.3e38f); }
    __device__ __forceinline__ RowExp(float bounded_temp, float m_)
        : c(sizeof(T) == 4 ? bounded_temp : bounded_temp * 1.4426950408889634f), m(m_) {}
    __device__ __forceinline__ F2 exponent(float z0, float z1) const { return (f2(z0, z1) + f2(-m, -m)) * f2(c, c); }
    __device__ __forceinline__ F2 operator()(float z0, float z1) const {
        float t0, t1;
        split(exponent(z0, z1), t0, t1);
        if constexpr (sizeof(T) == 4) return f2(expf(t0), expf(t1));
        float r0, r1;
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r0) : "f"(t0));
        asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r1) : "f"(t1));
        return f2(r0, r1);
    }
};

// Largest element of a vector (NaN is passed over; it comes back through the sum).
template <typename T>
__device__ __forceinline__ float vectors_max(const uint4 (&q)[kRowVectors]);
template <>
__device__ __forceinline__ float vectors_max<float>(const uint4 (&q)[kRowVectors]) {
    float m = -CUDART_INF_F;
#pragma unroll
    for (int k = 0; k < kRowVectors; ++k)
        m = fmaxf(m, fmaxf(fmaxf(__uint_as_float(q[k].x), __uint_as_float(q[k].y)), fmaxf(__uint_as_float(q[k].z), __uint_as_float(q[k].w))));
    return m;
}
template <typename H2>
__device__ __forceinline__ H2 pairs_max(const uint4 (&q)[kRowVectors]) {
    const auto as = [](const uint32_t& u) { return *reinterpret_cast<const H2*>(&u); };
    H2 m = as(q[0].x);
#pragma unroll
    for (int k = 0; k < kRowVectors; ++k) m = __hmax2(m, __hmax2(__hmax2(as(q[k].x), as(q[k].y)), __hmax2(as(q[k].z), as(q[k].w))));
    return m;
}
// The half instructions return NaN where both operands are.
__device__ __forceinline__ float pair_max(float x, float y) { return fmaxf(-CUDART_INF_F, fmaxf(x, y)); }
template <>
__device__ __forceinline__ float vectors_max<bf16>(const uint4 (&q)[kRowVectors]) {
    const __nv_bfloat162 m = pairs_max<__nv_bfloat162>(q);
    return pair_max(__low2float(m), __high2float(m));
}
template <>
__device__ __forceinline__ float vectors_max<f16>(const uint4 (&q)[kRowVectors]) {
    const __half2 m = pairs_max<__half2>(q);
    return pair_max(__low2float(m), __high2float(m));
}

// Factor that moves a sum held against maximum `from` to maximum `to`.  The empty set (-inf) has
// s = 0, or a NaN that has to stay.
__device__ __forceinline__ float rebase(float from, float to, float c) {
    return from == -CUDART_INF_F ? 1.0f : expf((from - to) * c);
}
__device__ __forceinline__ MaxSum join(MaxSum a, MaxSum b, float c) {
    const float m = fmaxf(a.m, b.m);
    return MaxSum{m, a.s * rebase(a.m, m, c) + b.s * rebase(b.m, m, c)};
}
// Over the lanes of a warp; every lane gets the same bits (each step adds the same two numbers on
// both sides).
__device__ __forceinline__ MaxSum warp_join(MaxSum x, float c) {
    float m = x.m;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
    float s = x.s * rebase(x.m, m, c);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    return MaxSum{m, s};
}

// A row as `vectors` whole 16-byte vectors behind `head` elements, and what is left behind those.
// The edges, fewer than 2 L elements, are held one a thread by the first warp of the row.
template <typename T>
struct RowParts {
    static constexpr int L = kLanes<T>;
    int head, vectors, tail;
    __device__ __forceinline__ RowParts(const T* row, int vocab) {
        head = min(vocab, (int)(((16 - (reinterpret_cast<uintptr_t>(row) & 15)) & 15) / sizeof(T)));
        vectors = (vocab - head) / L;
        tail = vocab - head - vectors * L;
    }
    // Element that thread t of the row holds besides its vectors; -1: none.
    __device__ __forceinline__ int edge(int t) const {
        if (t < head) return t;
        if (t >= 16 && t < 16 + tail) return head + vectors * L + t - 16;
        return -1;
    }
};

// x joined with the elements of some vectors.
template <typename T>
__device__ __forceinline__ MaxSum add_vectors(MaxSum x, const uint4 (&q)[kRowVectors], float inv_temp, float exp_temp) {
    constexpr int L = kLanes<T>;
    const float m = fmaxf(x.m, vectors_max<T>(q));
    const RowExp<T> e(exp_temp, m == -CUDART_INF_F ? 0.0f : m);
    F2 sum = f2(0.0f, 0.0f);
#pragma unroll
    for (int k = 0; k < kRowVectors; ++k) {
        float z[L];
        unpack<T>(q[k], z);
        F2 part = e(z[0], z[1]);
#pragma unroll
        for (int i = 2; i < L; i += 2) part = part + e(z[i], z[i + 1]);
        sum = sum + part;
    }
    float s0, s1;
    split(sum, s0, s1);
    return MaxSum{m, fmaf(x.s, rebase(x.m, m, inv_temp), s0 + s1)};
}

// One element as a set: NaN and +inf leave NaN.
__device__ __forceinline__ MaxSum single(float z) { return MaxSum{z, z == -CUDART_INF_F ? 0.0f : z - z + 1.0f}; }

}  // namespace odsgd_lm
