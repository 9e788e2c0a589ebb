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
    long long first;            // row_dropout_kernel: first block of eight
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

__device__ __forceinline__ void drop(const DropoutArgs& a, unsigned long long block, unsigned long long offset, float (&v)[8], const float (&r)[8]) {
    const uint4 bits = philox(block, offset, a.seed);
    const uint32_t word[4] = {bits.x, bits.y, bits.z, bits.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const bool kept = (i % 2 ? word[i / 2] >> 16 : word[i / 2] & 0xffffu) >= a.threshold;
        v[i] = (kept ? v[i] * a.scale : 0.0f) + r[i];  // (chosen, not multiplied: a dropped NaN is gone)
    }
}

// A thread takes eight consecutive elements of the whole, in the order of their index: one block of the generator,
// 16 bits each.  Here the eight lie together and on 16 bytes in every tensor; row_dropout_kernel has the rest.
// Bound by memory traffic: 134 M bf16 elements onto a bf16 residual take 119 us, the copy rate for their 805 MB being 123;
// without a residual 96 for 82, where the generator's ten rounds, some 8 instructions an element, come near.
template <typename TX, typename TO>
__global__ void __launch_bounds__(kDropoutThreads) dropout_kernel(const __grid_constant__ DropoutArgs a) {
    dependent_launch_prologue();
    const TX* const x = static_cast<const TX*>(a.x);
    const TO* const residual = static_cast<const TO*>(a.residual);
    TO* const out = static_cast<TO*>(a.out);
    const unsigned long long offset = a.offset + (a.counter != nullptr ? *a.counter : 0);
    const bool flat = a.dim == a.n;
    for (long long b = (long long)blockIdx.x * kDropoutThreads + threadIdx.x; b < a.n / 8; b += (long long)gridDim.x * kDropoutThreads) {
        const long long e = 8 * b;
        float v[8], r[8] = {};
        long long at_x = e, at_r = e, at_o = e;
        if (!flat) {
            const long long row = e / a.dim, col = e % a.dim, o = row / a.n_inner, i = row % a.n_inner;
            at_x = o * a.x_so + i * a.x_si + col, at_r = o * a.r_so + i * a.r_si + col, at_o = o * a.o_so + i * a.o_si + col;
        }
        load_8(x + at_x, v);
        if (residual) load_8(residual + at_r, r);
        drop(a, (unsigned long long)b, offset, v, r);
        store_8(out + at_o, v);
    }
}

// Eight elements from anywhere, of which those from lo on and below hi are there.
template <typename T>
__device__ __forceinline__ void load_some(const T* p, int lo, int hi, float (&x)[8]) {
    if (lo == 0 && hi == 8) {
        if constexpr (sizeof(T) == 2) {
            unpack<T>(load_anywhere(p), x);
            return;
        } else if ((reinterpret_cast<uintptr_t>(p) & 15) == 0) {
            load_8(p, x);
            return;
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = i >= lo && i < hi ? to_f32<T>(p[i]) : 0.0f;
}

// Row by row, blocks from a.first on: a block that two rows share is made for both.  blockDim = (blocks, rows).
template <typename TX, typename TO>
__global__ void __launch_bounds__(kDropoutThreads) row_dropout_kernel(const __grid_constant__ DropoutArgs a) {
    dependent_launch_prologue();
    const unsigned long long offset = a.offset + (a.counter != nullptr ? *a.counter : 0);
    const long long rows = a.n / a.dim;
    for (long long row = (long long)blockIdx.x * blockDim.y + threadIdx.y; row < rows; row += (long long)gridDim.x * blockDim.y) {
        const long long o = (unsigned)row / (unsigned)a.n_inner, i = (unsigned)row % (unsigned)a.n_inner;  // (at most 2^24 rows)
        const TX* const x = static_cast<const TX*>(a.x) + o * a.x_so + i * a.x_si;
        const TO* const residual = a.residual ? static_cast<const TO*>(a.residual) + o * a.r_so + i * a.r_si : nullptr;
        TO* const out = static_cast<TO*>(a.out) + o * a.o_so + i * a.o_si;
        const long long begin = row * a.dim, end = begin + a.dim;
        for (long long b = max(a.first, begin / 8) + (long long)blockIdx.y * blockDim.x + threadIdx.x; 8 * b < end; b += (long long)gridDim.y * blockDim.x) {
            const long long col = 8 * b - begin;  // of the block's first element; before the row's where that is another row's
            const int lo = (int)max(0ll, -col), hi = (int)min(8ll, a.dim - col);
            float v[8], r[8] = {};
            load_some(x + col, lo, hi, v);
            if (residual) load_some(residual + col, lo, hi, r);
            drop(a, (unsigned long long)b, offset, v, r);
            TO* const to = out + col;
            if (lo == 0 && hi == 8 && (reinterpret_cast<uintptr_t>(to) & 15) == 0) {
                store_8(to, v);
            } else {
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k >= lo && k < hi) to[k] = from_f32<TO>(v[k]);
            }
        }
    }
}

}  // namespace odsgd_lm
