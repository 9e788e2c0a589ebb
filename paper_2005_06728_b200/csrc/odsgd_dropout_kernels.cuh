// Device code of dropout (sm_100a): y = residual + keep(e) x / (1 - p), with the mask made anew wherever it is needed.
#pragma once

#include "odsgd_lm_elements.cuh"

namespace odsgd_lm {

// Philox4x32 of ten rounds (Salmon, Moraes, Dror, Shaw: Parallel Random Numbers: As Easy as 1, 2, 3, 2011): four
// random words from a counter of 128 bits and a key of 64.
__device__ __forceinline__ uint4 philox(unsigned long long block, unsigned long long offset, unsigned long long seed) {
    uint32_t c0 = (uint32_t)block, c1 = (uint32_t)(block >> 32), c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32);
    uint32_t k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)b;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return make_uint4(c0, c1, c2, c3);
}

struct DropoutArgs {
    const void* x;
    const void* residual;  // or nullptr
    void* out;
    long long x_so, x_si, r_so, r_si, o_so, o_si;
    long long n, dim, n_inner;  // elements, of a row; rows of an outer level
    unsigned long long seed, offset;
    const uint64_t* counter;            // or nullptr: added to offset
    unsigned threshold;                 // kept: 16 random bits of at least this
    float scale;
};

constexpr int kDropoutThreads = 256;

template <typename T>
__device__ __forceinline__ void load_8(const T* p, float (&x)[8]) {
    if constexpr (sizeof(T) == 2) {
        unpack<T>(*reinterpret_cast<const uint4*>(p), x);
    } else {
        float a[4], b[4];
        unpack<T>(reinterpret_cast<const uint4*>(p)[0], a);
        unpack<T>(reinterpret_cast<const uint4*>(p)[1], b);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
    }
}
template <typename T>
__device__ __forceinline__ void store_8(T* p, const float (&x)[8]) {
    if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(p) = pack<T>(x);
    } else {
        const float a[4] = {x[0], x[1], x[2], x[3]}, b[4] = {x[4], x[5], x[6], x[7]};
        reinterpret_cast<uint4*>(p)[0] = pack<T>(a);
        reinterpret_cast<uint4*>(p)[1] = pack<T>(b);
    }
}

// A thread takes eight consecutive elements of the whole, in the order of their index: one block of the generator,
// 16 bits each.  VEC: the eight lie together and on 16 bytes in every tensor (the last block's may be fewer).
// Bound by memory traffic: 134 M bf16 elements onto a bf16 residual take 122 us, the copy rate for their 805 MB.  Ten
// rounds of the generator are some 8 instructions an element; eight elements a block of it rather than four keep
// them below what the SMs issue in that time.
template <typename TX, typename TO, bool VEC>
__global__ void __launch_bounds__(kDropoutThreads) dropout_kernel(const __grid_constant__ DropoutArgs a) {
    dependent_launch_prologue();
    const TX* const x = static_cast<const TX*>(a.x);
    const TO* const residual = static_cast<const TO*>(a.residual);
    TO* const out = static_cast<TO*>(a.out);
    const unsigned long long offset = a.offset + (a.counter != nullptr ? *a.counter : 0);
    const long long blocks = (a.n + 7) / 8;
    for (long long b = (long long)blockIdx.x * kDropoutThreads + threadIdx.x; b < blocks; b += (long long)gridDim.x * kDropoutThreads) {
        const long long e = 8 * b;
        long long row = 0, col = e;
        if (a.dim != a.n) row = e / a.dim, col = e % a.dim;
        // of the row that the first element lies in; the others' where rows are crossed
        const auto place = [&](long long w, long long so, long long si) { return w / a.n_inner * so + w % a.n_inner * si; };
        const bool whole = VEC && e + 8 <= a.n;
        float v[8], r[8] = {};
        if (whole) {
            load_8(x + place(row, a.x_so, a.x_si) + col, v);
            if (residual) load_8(residual + place(row, a.r_so, a.r_si) + col, r);
        } else {
            long long w = row, c = col;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = 0.0f;
                if (e + i < a.n) {
                    v[i] = to_f32<TX>(x[place(w, a.x_so, a.x_si) + c]);
                    if (residual) r[i] = to_f32<TO>(residual[place(w, a.r_so, a.r_si) + c]);
                }
                if (++c == a.dim) c = 0, ++w;
            }
        }
        const uint4 bits = philox((unsigned long long)b, offset, a.seed);
        const uint32_t word[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bool kept = (i % 2 ? word[i / 2] >> 16 : word[i / 2] & 0xffffu) >= a.threshold;
            v[i] = (kept ? v[i] * a.scale : 0.0f) + r[i];  // (chosen, not multiplied: a dropped NaN is gone)
        }
        if (whole) {
            store_8(out + place(row, a.o_so, a.o_si) + col, v);
        } else {
            long long w = row, c = col;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (e + i < a.n) out[place(w, a.o_so, a.o_si) + c] = from_f32<TO>(v[i]);
                if (++c == a.dim) c = 0, ++w;
            }
        }
    }
}

}  // namespace odsgd_lm
