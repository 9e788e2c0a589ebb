// What the kernels of the language-model operators share: elements and 16-byte vectors of the three types, token
// loads, clusters.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <math_constants.h>
#include <stdint.h>

#include "odsgd.h"

namespace odsgd_lm {

using bf16 = __nv_bfloat16;
using f16 = __half;

// Scheduled early, run in order: see the update kernels.  A grid can have begun while the one ahead of it still
// writes, so what is read behind the wait goes through ordinary loads: the read-only path asks for memory
// that nothing writes in all the time the grid exists (it measured no faster: norms, lookups and clips within 0.5 %).
__device__ __forceinline__ void dependent_launch_prologue() {
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
}

// ------------------------------------------------------------------ elements and 16-byte vectors
template <typename T>
__device__ __forceinline__ float to_f32(T x);
template <>
__device__ __forceinline__ float to_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f32<bf16>(bf16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float to_f32<f16>(f16 x) { return __half2float(x); }

template <typename T>
__device__ __forceinline__ T from_f32(float x);
template <>
__device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <>
__device__ __forceinline__ bf16 from_f32<bf16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ f16 from_f32<f16>(float x) { return __float2half_rn(x); }

// Elements of T in 16 bytes.
template <typename T>
constexpr int kLanes = 16 / (int)sizeof(T);

template <typename T>
__device__ __forceinline__ void unpack(const uint4& q, float (&x)[kLanes<T>]);
template <>
__device__ __forceinline__ void unpack<float>(const uint4& q, float (&x)[4]) {
    x[0] = __uint_as_float(q.x);
    x[1] = __uint_as_float(q.y);
    x[2] = __uint_as_float(q.z);
    x[3] = __uint_as_float(q.w);
}
template <>
__device__ __forceinline__ void unpack<bf16>(const uint4& q, float (&x)[8]) {
    const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(u[i] << 16);
        x[2 * i + 1] = __uint_as_float(u[i] & 0xffff0000u);
    }
}
template <>
__device__ __forceinline__ void unpack<f16>(const uint4& q, float (&x)[8]) {
    const uint32_t u[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}

template <typename T>
__device__ __forceinline__ uint4 pack(const float (&x)[kLanes<T>]);
template <>
__device__ __forceinline__ uint4 pack<float>(const float (&x)[4]) {
    return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
template <>
__device__ __forceinline__ uint4 pack<bf16>(const float (&x)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}
template <>
__device__ __forceinline__ uint4 pack<f16>(const float (&x)[8]) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 h = __floats2half2_rn(x[2 * i], x[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

// Eight elements of 16 bits that start `shift` bytes into two 16-byte words.
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, unsigned shift) {
    uint32_t x[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
    for (int i = 0; i < 6; ++i) x[i] = shift & 8 ? x[i + 2] : x[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) x[i] = shift & 4 ? x[i + 1] : x[i];
    const unsigned bits = shift & 2 ? 16 : 0;
    return make_uint4(__funnelshift_r(x[0], x[1], bits), __funnelshift_r(x[1], x[2], bits), __funnelshift_r(x[2], x[3], bits), __funnelshift_r(x[3], x[4], bits));
}
// Eight elements of 16 bits that start anywhere: the two 16-byte words around them, shifted.  (Both words hold elements of
// the eight, so neither reaches into another 16 bytes than the row's own do.)
template <typename T>
__device__ __forceinline__ uint4 load_anywhere(const T* p) {
    static_assert(sizeof(T) == 2, "16 bits");
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    const uint4* const w = reinterpret_cast<const uint4*>(at & ~(uintptr_t)15);
    const uint4 a = w[0];
    const unsigned shift = (unsigned)(at & 15);
    if (shift == 0) return a;
    return shifted(a, w[1], shift);
}

// Eight floats in one store, 32-byte aligned (two of 16 bytes leave every sector half written at a time).
__device__ __forceinline__ void store_eight(float* p, const float* x) {
    asm volatile("st.global.cs.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]),
                 "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
}
__device__ __forceinline__ bool aligned32(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 31) == 0; }

// Two floats in one register pair, added and multiplied by one instruction each.
struct F2 {
    unsigned long long v;
};
__device__ __forceinline__ F2 f2(float x, float y) {
    F2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void split(F2 a, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(a.v)); }
__device__ __forceinline__ F2 operator+(F2 a, F2 b) {
    F2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ F2 operator*(F2 a, F2 b) {
    F2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}

// Negative infinity in every lane.
template <typename T>
__device__ __forceinline__ uint4 neg_inf_vector() {
    constexpr uint32_t w = sizeof(T) == 4 ? 0xff800000u : 0u;
    if constexpr (sizeof(T) == 4) return make_uint4(w, w, w, w);
    const T h = from_f32<T>(-CUDART_INF_F);
    const uint32_t u = *reinterpret_cast<const uint16_t*>(&h) * 0x10001u;
    return make_uint4(u, u, u, u);
}

__device__ __forceinline__ long long load_token(const void* p, bool wide, long long i) {
    return wide ? static_cast<const long long*>(p)[i] : (long long)static_cast<const int*>(p)[i];
}

// ------------------------------------------------------------------ clusters
__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_sync() {
    cluster_arrive();
    cluster_wait();
}
// The address of a variable of this CTA's shared memory in the CTA `rank` of the cluster.
__device__ __forceinline__ uint32_t cluster_address(const void* smem, unsigned rank) {
    uint32_t out;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(out) : "r"((uint32_t)__cvta_generic_to_shared(smem)), "r"(rank));
    return out;
}
__device__ __forceinline__ void cluster_store(uint32_t addr, float x) {
    asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(x) : "memory");
}
__device__ __forceinline__ uint32_t cluster_load(uint32_t addr) {
    uint32_t x;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(x) : "r"(addr) : "memory");
    return x;
}

}  // namespace odsgd_lm
