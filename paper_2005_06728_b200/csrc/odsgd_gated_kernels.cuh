// Device code of the gated feed-forward block (sm_100a): act(x Wg^T) * (x Wu^T), and its gradient.
//
// All products run on the tensor cores (tcgen05): operands come to shared memory by TMA, sums stand in tensor
// memory in 32 bits.  One kernel serves the three of them, which differ in how operands lie and what happens to a
// finished tile:
//   forward       rows of x against 128 rows of Wg and the same 128 of Wu: a tile holds both projections of a
//                 token, so that activation and product are taken where the sums are
//   gradient of x         [dg | du] [Wg; Wu]: one sum over both halves, the second begun where the first ends
//   gradient of weights   dg^T x and du^T x: tiles of both in one launch
#pragma once

#include <cuda.h>

#include "odsgd_lm_elements.cuh"

namespace odsgd_lm {

// ------------------------------------------------------------------ barriers, copies, tensor memory
__device__ __forceinline__ uint32_t smem_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void barrier_init(uint32_t bar, unsigned count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint32_t bar, unsigned bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
// One arrival at a barrier that may be another CTA's of the cluster.
__device__ __forceinline__ void barrier_arrive_at(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint32_t bar, unsigned parity) {
    uint32_t done;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(done)
        : "r"(bar), "r"(parity)
        : "memory");
    return done != 0;
}

// Waits that have given up since the library was loaded (odsgd_stalled_waits).  None ever should.
__device__ unsigned int stalled_waits;

// No wait is without an end: after about four seconds it is given up, counted, and `stalled` ends the CTA's other
// waits.  What comes out of that launch is void.
__device__ __forceinline__ unsigned long long nanoseconds() {
    unsigned long long t;
    asm volatile("mov.u64 %0, %globaltimer;" : "=l"(t));
    return t;
}
__device__ __noinline__ bool barrier_wait_long(uint32_t bar, unsigned parity, volatile int* stalled) {
    const unsigned long long until = nanoseconds() + 4000000000ull;
    for (;;) {
        for (int i = 0; i < 64; ++i)
            if (barrier_try(bar, parity)) return true;
        if (*stalled) return false;
        if (nanoseconds() > until) break;
    }
    *stalled = 1;
    atomicAdd(&stalled_waits, 1u);
    return false;
}
__device__ __forceinline__ bool barrier_wait(uint32_t bar, unsigned parity, volatile int* stalled) {
    return barrier_try(bar, parity) || barrier_wait_long(bar, parity, stalled);
}

// A box of a tensor, from column c and row r on, into this CTA's shared memory; counted at `bar`, which is in the
// cluster's first CTA.
__device__ __forceinline__ void load_box(uint32_t dst, const CUtensorMap* map, int c, int r, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
        "l"(map), "r"(c), "r"(r), "r"(bar)
        : "memory");
}

// The same, counted at a barrier of this CTA.
__device__ __forceinline__ void load_box_alone(uint32_t dst, const CUtensorMap* map, int c, int r, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map),
                 "r"(c), "r"(r), "r"(bar)
                 : "memory");
}

template <int CTAS>
__device__ __forceinline__ void tensor_alloc(uint32_t smem_out, unsigned columns) {
    if constexpr (CTAS == 2) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_out), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_out), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}
template <int CTAS>
__device__ __forceinline__ void tensor_free(uint32_t base, unsigned columns) {
    if constexpr (CTAS == 2)
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
    else
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns));
}
__device__ __forceinline__ void tensor_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tensor_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// d (+)= A B^T over 16 of the long axis; the pair's first CTA issues it for both.
__device__ __forceinline__ void multiply_pair(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a),
                 "l"(b), "r"(instr), "r"((uint32_t)add)
                 : "memory");
}
// An arrival at the barrier of this offset in both CTAs, when all products issued so far are done.
__device__ __forceinline__ void commit_pair(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                 "h"((uint16_t)3)
                 : "memory");
}

// Both for a CTA by itself.
__device__ __forceinline__ void multiply_alone(uint32_t d, uint64_t a, uint64_t b, uint32_t instr, bool add) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %4, 0;\n tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d), "l"(a),
                 "l"(b), "r"(instr), "r"((uint32_t)add)
                 : "memory");
}
__device__ __forceinline__ void commit_alone(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

// 32 columns of a warp's 32 lanes: x[i] is column i of the thread's lane.
__device__ __forceinline__ void tensor_load(uint32_t addr, float (&x)[32]) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
        "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
          "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
          "=r"(r[31])
        : "r"(addr));
#pragma unroll
    for (int i = 0; i < 32; ++i) x[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tensor_load(uint32_t addr, float (&x)[16]) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
          "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(addr));
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tensor_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Operands lie in shared memory as TMA's 128-byte swizzle writes them, 1024-byte aligned: rows of 128 bytes (64
// elements of 16 bits), eight rows to a unit of 1024 bytes.
//   long axis inside the rows (`lines` false): a row is one of the tile's rows, units follow one another; 16 further
//     elements of the long axis are 32 bytes on.
//   tile's axis inside the rows (`lines` true): a row is one place of the long axis with 64 of the tile's rows; the
//     next 64 of the tile's rows are kBlockK rows further on, 16 further places of the long axis 16 rows.
constexpr int kBlockK = 64;  // of the long axis, in one stage
__device__ __forceinline__ uint64_t operand(uint32_t addr, bool lines) {
    const uint64_t chunk = lines ? (uint64_t)(kBlockK * 128 >> 4) : 1, unit = 1024 >> 4;
    return (uint64_t)(addr >> 4 & 0x3fff) | chunk << 16 | unit << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__host__ __device__ constexpr uint32_t operand_step(bool lines) { return (lines ? 16 * 128 : 32) >> 4; }  // to the next 16 of the long axis

// 32-bit sums of 16-bit products, rows x columns of the pair's tile.
__host__ __device__ constexpr uint32_t instruction(bool is_bf16, bool a_lines, bool b_lines, int rows, int columns) {
    return 1u << 4 | (is_bf16 ? 1u << 7 | 1u << 10 : 0u) | (a_lines ? 1u << 15 : 0u) | (b_lines ? 1u << 16 : 0u) | (uint32_t)(columns >> 3) << 17 |
           (uint32_t)(rows >> 4) << 24;
}

// ------------------------------------------------------------------ activation
// Both in 32 bits; `slope` is the derivative.  A kernel is built for one of them: code for both, 32 times in a row, did not fit
// the instruction cache (a tile's end took 14.8 thousand cycles instead of 4.4).
struct Activated {
    float value, slope;
};
// The normal distribution function: for t < 0
//     cdf(t) = exp(-t^2 / 2) k r(k),  k = 1 / (1 + 0.37 |t|)
// and 1 - cdf(-t) above; `bell` is exp(-t^2 / 2), which the slope needs too.  r, of degree 8, is the polynomial whose largest relative
// error over all t <= 0 is least (a linear program on 1500 Chebyshev points of k): 1.8e-7.  In 32 bits the whole is off by 6e-7
// relative at -1, 1e-6 at -4 and 8e-6 at -13, where exp(-t^2 / 2) carries the rounding of its argument; h is rounded to 2^-12 at
// best.  (Half the instructions of 1 + erf, and nothing cancels below 0.)
__device__ __forceinline__ float normal_cdf(float t, float& bell) {
    bell = __expf(-0.5f * t * t);
    const float k = __fdividef(1.0f, fmaf(0.37f, fabsf(t), 1.0f));
    float r = fmaf(k, -0.0313809665f, 0.135318485f);
    r = fmaf(k, r, -0.194549723f);
    r = fmaf(k, r, 0.0646818255f);
    r = fmaf(k, r, 0.0133536168f);
    r = fmaf(k, r, 0.0901881908f);
    r = fmaf(k, r, 0.127164879f);
    r = fmaf(k, r, 0.147615132f);
    r = fmaf(k, r, 0.147608617f);
    const float tail = k * r * bell;
    return t < 0.0f ? tail : 1.0f - tail;
}
template <bool GELU>
__device__ __forceinline__ float activate(float t) {
    if constexpr (GELU) {
        float bell;
        return t * normal_cdf(t, bell);
    }
    return __fdividef(t, 1.0f + __expf(-t));
}
template <bool GELU>
__device__ __forceinline__ Activated activate_with_slope(float t) {
    if constexpr (GELU) {
        float bell;
        const float cdf = normal_cdf(t, bell);
        return {t * cdf, cdf + t * 0.39894228f * bell};
    }
    const float s = __fdividef(1.0f, 1.0f + __expf(-t));
    return {t * s, s * (1.0f + t * (1.0f - s))};
}

// ------------------------------------------------------------------ tiles
enum GatedKind { kForward, kGradX, kGradW };

// Rows of an output: row r lies at (r / n_inner) * so + (r % n_inner) * si.
struct RowsOut {
    void* p;
    long long so, si;
};

struct GatedArgs {
    CUtensorMap a[2], b[2];
    RowsOut out[3];          // forward: h, gate, up; gradient of x: dx; of weights: dw_gate, dw_up
    unsigned rows, columns;  // of the product (forward: columns of each projection)
    unsigned n_inner;        // rows of an outer level of the outputs
    unsigned depth;          // the long axis (gradient of x: of one half)
    int is_bf16, out_f32, accumulate, save;
};

constexpr int kTileRows = 256;       // of a pair of CTAs: 128 each
constexpr int kTileColumns = 256;    // sums a row: forward 128 gates and 128 ups
constexpr int kGatedStages = 6;
constexpr int kHalfBytes = 128 * kBlockK * 2;     // 128 rows of an operand, one stage
constexpr int kStageBytes = 2 * kHalfBytes;       // of one CTA: its 128 rows of A, its half of B
constexpr int kFinishWarps = 8;                   // that finish tiles; behind copy, products, tensor memory and an idle one
constexpr int kGatedThreads = 128 + 32 * kFinishWarps;
constexpr int kPatchPitch = 33;                   // words of a row of the patch through which unaligned rows are written
constexpr int kGatedSmem = 1024 + kGatedStages * kStageBytes + kFinishWarps * 32 * kPatchPitch * 4;
constexpr int kGroupTiles = 8;                    // tiles of rows that follow one another before the columns move on

struct GatedBarriers {
    unsigned long long full[kGatedStages], empty[kGatedStages];
    unsigned long long sums_full[2], sums_empty[2];
    uint32_t tensor_base;
    int stalled;
};

// 32 consecutive columns of a row from its thread's registers to memory, where the row starts on 32 bytes.  Out-of-range
// rows have p == nullptr.
__device__ __forceinline__ void store_sector(void* p, const uint4& a, const uint4& b) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y),
                 "r"(b.z), "r"(b.w)
                 : "memory");
}
template <typename T, bool VEC>
__device__ __forceinline__ void store_32(T* p, int valid, const float (&x)[32]) {
    constexpr int L = kLanes<T>;
    if (p == nullptr) return;
#pragma unroll
    for (int i = 0; i < 32; i += 2 * L) {
        if (VEC && i + 2 * L <= valid) {
            float y[L], z[L];
#pragma unroll
            for (int l = 0; l < L; ++l) y[l] = x[i + l], z[l] = x[i + L + l];
            store_sector(p + i, pack<T>(y), pack<T>(z));
        } else {
#pragma unroll
            for (int l = 0; l < 2 * L; ++l)
                if (i + l < valid) p[i + l] = from_f32<T>(x[i + l]);
        }
    }
}

// Rows that do not start on 32 bytes go through a patch of shared memory, 32 rows of 64 columns a warp, and from there as
// the 16-byte words of their own addresses, eight lanes a row; what is left at both ends goes element by element.  (2036
// x 1001 x 2731 f16, kept: 87 us with a row at a time, element by element, 44 so.)
__device__ __forceinline__ void patch_32(uint32_t* patch, unsigned c, unsigned lane, const uint4 (&q)[4]) {
    uint32_t* const to = patch + lane * kPatchPitch + c / 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) to[4 * i] = q[i].x, to[4 * i + 1] = q[i].y, to[4 * i + 2] = q[i].z, to[4 * i + 3] = q[i].w;
}
// Stores behind a predicate rather than a branch, which the loads of the next rows may pass (nothing reads what they write, and the
// patch is written again behind a barrier): 64 columns of 32 rows took a warp 3.5 thousand cycles with branches and take 2.8 so.
// (Rows turned in the patch so that no two lanes meet in a bank took longer by their addresses.)
__device__ __forceinline__ void store_if(void* p, const uint4& q, bool yes) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %5, 0;\n @p st.global.v4.b32 [%0], {%1, %2, %3, %4};\n}\n" ::"l"(p), "r"(q.x), "r"(q.y), "r"(q.z),
                 "r"(q.w), "r"((uint32_t)yes));
}
__device__ __forceinline__ void store_if(void* p, unsigned short x, bool yes) {
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %2, 0;\n @p st.global.b16 [%0], %1;\n}\n" ::"l"(p), "h"(x), "r"((uint32_t)yes));
}
template <typename T>
__device__ __forceinline__ void store_patch(T* p, int valid, const uint32_t* patch, unsigned lane) {
    static_assert(sizeof(T) == 2, "two elements a word");
    const int l = (int)(lane & 7);
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned r = (lane >> 3) + 4 * i;
        const unsigned long long to = __shfl_sync(~0u, reinterpret_cast<unsigned long long>(p), r);
        const uint32_t* const row = patch + r * kPatchPitch;
        const unsigned short* const half = reinterpret_cast<const unsigned short*>(row);
        const int head = min(valid, (int)(-(unsigned)to & 15) / 2), at = head + 8 * l;
        const uint32_t* const w = row + min(at, 56) / 2;  // (what begins later is not stored)
        const unsigned shift = at & 1 ? 16 : 0;
        const uint32_t x[5] = {w[0], w[1], w[2], w[3], w[4]};  // (the last is not used where `shift` is 0; the row has a spare word)
        const uint4 q = make_uint4(__funnelshift_r(x[0], x[1], shift), __funnelshift_r(x[1], x[2], shift), __funnelshift_r(x[2], x[3], shift),
                                   __funnelshift_r(x[3], x[4], shift));
        store_if(reinterpret_cast<void*>(to + 2 * at), q, to != 0 && at + 8 <= valid);
        // fewer than eight elements at each end; of whole eights, eight in all (or none)
        if (valid % 8 == 0) {
            const int e = l < head ? l : valid - 8 + l;
            store_if(reinterpret_cast<void*>(to + 2 * e), half[e], to != 0 && head != 0);
        } else {
            const int tail = head + (valid - head) / 8 * 8 + l;
            store_if(reinterpret_cast<void*>(to + 2 * l), half[l], to != 0 && l < head);
            store_if(reinterpret_cast<void*>(to + 2 * tail), half[min(tail, 63)], to != 0 && tail < valid);
        }
    }
    __syncwarp();
}
template <typename T>
__device__ __forceinline__ void pack_32(const float (&x)[32], uint4 (&q)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float y[8];
#pragma unroll
        for (int l = 0; l < 8; ++l) y[l] = x[8 * i + l];
        q[i] = pack<T>(y);
    }
}

template <typename T>
__device__ __forceinline__ T* row_of(const RowsOut& o, const GatedArgs& a, unsigned row) {
    return static_cast<T*>(o.p) + (row / a.n_inner) * o.so + (row % a.n_inner) * o.si;
}
template <typename T>
__device__ __forceinline__ bool rows_on_32(const RowsOut& o) {
    return ((reinterpret_cast<uintptr_t>(o.p) | (uintptr_t)(o.so * (long long)sizeof(T)) | (uintptr_t)(o.si * (long long)sizeof(T))) & 31) == 0;
}

// A persistent pair of CTAs per two SMs goes over tiles of 256 rows x 256 sums.  In each CTA one thread copies (its own 128 rows of
// A and its half of B: in the forward pass the first CTA's half is Wg's, the second's Wu's) and eight warps finish
// tiles; one thread of the first CTA issues the products of both.  Two sets of sums, so that one tile is finished
// while the next is computed.  Bound by the tensor cores where products are large: 8192 x 4096 x 11008 bf16 forward 930 us
// in a burst, 1.59 PFLOP/s, 0.99 of the library's rate there, 1157 under the power cap (0.92); gradient of x 913, of weights 950.
// A block of 64 of the long axis takes 320 cycles then; 530 to 600 where the long axis is 1024 and tiles are few.
template <int KIND, typename T, bool GELU>
__global__ void __launch_bounds__(kGatedThreads, 1) __cluster_dims__(2, 1, 1) gated_kernel(const __grid_constant__ GatedArgs a) {
    constexpr bool A_LINES = KIND == kGradW, B_LINES = KIND != kForward;
    extern __shared__ unsigned char raw[];
    __shared__ GatedBarriers s;
    const uint32_t stages = (smem_address(raw) + 1023) & ~1023u;
    uint32_t* const patches = reinterpret_cast<uint32_t*>(raw + (stages - smem_address(raw)) + kGatedStages * kStageBytes);
    const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = blockIdx.x & 1;
    const unsigned pairs = gridDim.x / 2, pair = blockIdx.x / 2;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kGatedStages; ++i) {
            barrier_init(smem_address(&s.full[i]), 1);
            barrier_init(smem_address(&s.empty[i]), 1);
        }
        for (int i = 0; i < 2; ++i) {
            barrier_init(smem_address(&s.sums_full[i]), 1);
            barrier_init(smem_address(&s.sums_empty[i]), 2 * kFinishWarps);  // the finishing warps of both CTAs
        }
        s.stalled = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    dependent_launch_prologue();
    if (warp == 2) tensor_alloc<2>(smem_address(&s.tensor_base), 512);
    tensor_fence_before();
    __syncthreads();
    cluster_sync();
    tensor_fence_after();
    const uint32_t base = *reinterpret_cast<volatile uint32_t*>(&s.tensor_base);

    const unsigned col_step = KIND == kForward ? kTileColumns / 2 : kTileColumns;
    const unsigned row_tiles = (a.rows + kTileRows - 1) / kTileRows, col_tiles = (a.columns + col_step - 1) / col_step;
    const unsigned per_product = row_tiles * col_tiles, tiles = per_product * (KIND == kGradW ? 2 : 1);
    const unsigned half_blocks = (a.depth + kBlockK - 1) / kBlockK, blocks = half_blocks * (KIND == kGradX ? 2 : 1);

    // tile t: which product, first row, first column
    struct Tile {
        unsigned product, row, col;
    };
    const auto tile_at = [&](unsigned t) {
        Tile out;
        out.product = t / per_product;
        t -= out.product * per_product;
        const unsigned group = t / (kGroupTiles * col_tiles), first = group * kGroupTiles, many = min((unsigned)kGroupTiles, row_tiles - first);
        t -= first * col_tiles;
        out.row = (first + t % many) * kTileRows;
        out.col = (t / many) * col_step;
        return out;
    };

    if (warp == 0) {
        if (lane == 0) {
            unsigned stage = 0, phase = 0;
            bool ok = true;
            for (unsigned t = pair; t < tiles && ok; t += pairs) {
                const Tile tile = tile_at(t);
                const int row = (int)(tile.row + rank * 128);
                for (unsigned k = 0; k < blocks; ++k) {
                    ok = barrier_wait(smem_address(&s.empty[stage]), phase ^ 1, &s.stalled);
                    if (!ok) break;
                    if (rank == 0) barrier_expect(smem_address(&s.full[stage]), 2 * kStageBytes);
                    const uint32_t bar = cluster_address(&s.full[stage], 0);
                    const uint32_t to_a = stages + stage * kStageBytes, to_b = to_a + kHalfBytes;
                    const bool second = KIND == kGradX && k >= half_blocks;
                    const int at = (int)((second ? k - half_blocks : k) * kBlockK);
                    const CUtensorMap* ma = KIND == kGradW ? &a.a[tile.product] : &a.a[second];
                    const CUtensorMap* mb = KIND == kForward ? &a.b[rank] : KIND == kGradX ? &a.b[second] : &a.b[0];
                    const int col = (int)(KIND == kForward ? tile.col : tile.col + rank * 128);
                    if constexpr (A_LINES) {
                        load_box(to_a, ma, row, at, bar);
                        load_box(to_a + kHalfBytes / 2, ma, row + 64, at, bar);
                    } else {
                        load_box(to_a, ma, at, row, bar);
                    }
                    if constexpr (B_LINES) {
                        load_box(to_b, mb, col, at, bar);
                        load_box(to_b + kHalfBytes / 2, mb, col + 64, at, bar);
                    } else {
                        load_box(to_b, mb, at, col, bar);
                    }
                    if (++stage == kGatedStages) stage = 0, phase ^= 1;
                }
            }
            // every stage free again: the other CTA's arrivals here are in, and no copy is under way
            for (int i = 0; i < kGatedStages && ok; ++i) {
                ok = barrier_wait(smem_address(&s.empty[stage]), phase ^ 1, &s.stalled);
                if (++stage == kGatedStages) stage = 0, phase ^= 1;
            }
            if (!ok) {  // copies under way land within this time
                for (int i = 0; i < 2000; ++i) __nanosleep(1000);
            }
        }
    } else if (warp == 1) {
        if (lane == 0 && rank == 0) {
            const uint32_t instr = instruction(a.is_bf16 != 0, A_LINES, B_LINES, kTileRows, kTileColumns);
            unsigned stage = 0, phase = 0, set = 0, set_phase = 0;
            bool ok = true;
            for (unsigned t = pair; t < tiles && ok; t += pairs) {
                ok = barrier_wait(smem_address(&s.sums_empty[set]), set_phase ^ 1, &s.stalled);
                if (!ok) break;
                tensor_fence_after();
                const uint32_t d = base + set * kTileColumns;
                for (unsigned k = 0; k < blocks; ++k) {
                    ok = barrier_wait(smem_address(&s.full[stage]), phase, &s.stalled);
                    if (!ok) break;
                    tensor_fence_after();
                    const uint64_t da = operand(stages + stage * kStageBytes, A_LINES);
                    const uint64_t db = operand(stages + stage * kStageBytes + kHalfBytes, B_LINES);
#pragma unroll
                    for (int i = 0; i < kBlockK / 16; ++i)
                        multiply_pair(d, da + i * operand_step(A_LINES), db + i * operand_step(B_LINES), instr, k > 0 || i > 0);
                    commit_pair(smem_address(&s.empty[stage]));
                    if (++stage == kGatedStages) stage = 0, phase ^= 1;
                }
                if (!ok) break;
                commit_pair(smem_address(&s.sums_full[set]));
                if (++set == 2) set = 0, set_phase ^= 1;
            }
        }
    } else if (warp >= 4) {
        const unsigned quarter = warp & 3, part = (warp - 4) / 4;  // a quarter of the rows, a share of the columns
        constexpr unsigned PARTS = kFinishWarps / 4;
        uint32_t* const patch = patches + (warp - 4) * 32 * kPatchPitch;
        const bool vec_t = rows_on_32<T>(a.out[0]) && (KIND == kGradX || rows_on_32<T>(a.out[1])) && (KIND != kForward || rows_on_32<T>(a.out[2]));
        const bool vec_f = rows_on_32<float>(a.out[0]) && rows_on_32<float>(a.out[1]);
        unsigned set = 0, set_phase = 0;
        for (unsigned t = pair; t < tiles; t += pairs) {
            const Tile tile = tile_at(t);
            const unsigned row = tile.row + rank * 128 + quarter * 32 + lane;
            if (!__all_sync(~0u, barrier_wait(smem_address(&s.sums_full[set]), set_phase, &s.stalled))) break;
            tensor_fence_after();
            const unsigned first = part * (col_step / PARTS), col = tile.col + first;
            const int valid = col < a.columns ? (int)min(col_step / PARTS, a.columns - col) : 0;
            const uint32_t from = base + set * kTileColumns + (quarter * 32 << 16) + first;
            if constexpr (KIND == kForward) {
                T* const h = row < a.rows ? row_of<T>(a.out[0], a, row) + col : nullptr;
                T* const gate = row < a.rows && a.save ? row_of<T>(a.out[1], a, row) + col : nullptr;
                T* const up = row < a.rows && a.save ? row_of<T>(a.out[2], a, row) + col : nullptr;
                float g[32], u[32];
                if (vec_t) {
#pragma unroll 1
                    for (int c = 0; c < valid; c += 32) {
                        tensor_load(from + c, g);
                        tensor_load(from + 128 + c, u);
                        tensor_load_wait();
                        if (a.save) {
                            store_32<T, true>(gate ? gate + c : nullptr, valid - c, g);
                            store_32<T, true>(up ? up + c : nullptr, valid - c, u);
                        }
#pragma unroll
                        for (int i = 0; i < 32; ++i) g[i] = activate<GELU>(g[i]) * u[i];
                        store_32<T, true>(h ? h + c : nullptr, valid - c, g);
                    }
                } else {
#pragma unroll 1
                    for (int k = a.save ? 0 : 2; k < 3; ++k) {  // gate, up, h
#pragma unroll 1
                        for (int c = 0; c < valid; c += 32) {
                            tensor_load(from + (k == 1 ? 128 : 0) + c, g);
                            if (k == 2) tensor_load(from + 128 + c, u);
                            tensor_load_wait();
                            if (k == 2) {
#pragma unroll
                                for (int i = 0; i < 32; ++i) g[i] = activate<GELU>(g[i]) * u[i];
                            }
                            uint4 q[4];
                            pack_32<T>(g, q);
                            T* const p = k == 0 ? gate : k == 1 ? up : h;
                            const int begin = c & ~63;
                            patch_32(patch, c & 63, lane, q);
                            if (c + 32 >= valid || (c & 63) == 32) store_patch<T>(p ? p + begin : nullptr, min(64, valid - begin), patch, lane);
                        }
                    }
                }
            } else {
                const RowsOut& o = a.out[KIND == kGradW ? tile.product : 0];
                float x[32];
                if (KIND == kGradW && a.out_f32) {
                    float* const p = row < a.rows ? row_of<float>(o, a, row) + col : nullptr;
#pragma unroll 1
                    for (int c = 0; c < valid; c += 32) {
                        tensor_load(from + c, x);
                        tensor_load_wait();
                        if (a.accumulate && p != nullptr) {
#pragma unroll
                            for (int i = 0; i < 32; ++i)
                                if (c + i < valid) x[i] += p[c + i];
                        }
                        if (vec_f) store_32<float, true>(p ? p + c : nullptr, valid - c, x);
                        else store_32<float, false>(p ? p + c : nullptr, valid - c, x);
                    }
                } else {
                    T* const p = row < a.rows ? row_of<T>(o, a, row) + col : nullptr;
#pragma unroll 1
                    for (int c = 0; c < valid; c += 32) {
                        tensor_load(from + c, x);
                        tensor_load_wait();
                        if (vec_t) {
                            store_32<T, true>(p ? p + c : nullptr, valid - c, x);
                        } else {
                            uint4 q[4];
                            pack_32<T>(x, q);
                            const int begin = c & ~63;
                            patch_32(patch, c & 63, lane, q);
                            if (c + 32 >= valid || (c & 63) == 32) store_patch<T>(p ? p + begin : nullptr, min(64, valid - begin), patch, lane);
                        }
                    }
                }
            }
            tensor_fence_before();
            __syncwarp();
            if (lane == 0) barrier_arrive_at(cluster_address(&s.sums_empty[set], 0));
            if (++set == 2) set = 0, set_phase ^= 1;
        }
    }
    __syncwarp();
    tensor_fence_before();
    __syncthreads();
    cluster_sync();
    if (warp == 2) {
        tensor_fence_after();
        tensor_free<2>(base, 512);
    }
}

__device__ __forceinline__ float4 cluster_load4(uint32_t addr) {
    float4 x;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(addr) : "memory");
    return x;
}

// ------------------------------------------------------------------ few tokens
// Few tokens leave most of a tile of 256 of them empty, and their time is that of reading the weights.  Here weights are
// the rows of the product and tokens its columns, as many as there are, rounded up to 16: a cluster takes 64 columns of the block (64
// rows of Wg above 64 of Wu), or 128 columns of x's gradient, its CTAs share the long axis, and the sums meet in shared memory,
// added in the order of the ranks.  Bound by the read of the weights: 48 tokens x 4096 x 11000 36 us, 0.77 of the copy rate
// (57 us by gated_kernel), one token x 2048 x 5440 9.3 us (27.5).
constexpr int kThinThreads = 128;
constexpr int kThinRows = 128;
constexpr int kThinCluster = 8;
constexpr int kThinStages = 8;  // at most
struct ThinArgs {
    CUtensorMap a[2], b[2];
    RowsOut out[3];
    unsigned tokens, n_inner, columns, depth;
    unsigned chunk;  // tokens of a cluster, a multiple of 16
    unsigned stages, cluster, tensor_columns;
    int is_bf16, save;
};
struct ThinBarriers {
    unsigned long long full[kThinStages], empty[kThinStages], done;
    uint32_t tensor_base;
    int stalled;
};

template <int KIND, typename T, bool GELU>
__global__ void __launch_bounds__(kThinThreads) thin_kernel(const __grid_constant__ ThinArgs a) {
    static_assert(KIND != kGradW, "forward, or the gradient of x");
    constexpr bool A_LINES = KIND == kGradX;
    constexpr unsigned WIDE = KIND == kForward ? 64 : 128;  // columns of the output
    extern __shared__ unsigned char raw[];
    __shared__ ThinBarriers s;
    const uint32_t stages = (smem_address(raw) + 1023) & ~1023u;
    float* const sums = reinterpret_cast<float*>(raw + (stages - smem_address(raw)));  // [chunk][kThinRows], behind the last product
    const unsigned warp = threadIdx.x >> 5, cs = a.cluster;
    const unsigned rank = blockIdx.x % cs, col = blockIdx.x / cs * WIDE, first = blockIdx.y * a.chunk, many = min(a.chunk, a.tokens - first);
    const unsigned token_bytes = a.chunk * kBlockK * 2, stage_bytes = kThinRows * kBlockK * 2 + token_bytes;
    if (threadIdx.x == 0) {
        for (unsigned i = 0; i < a.stages; ++i) {
            barrier_init(smem_address(&s.full[i]), 1);
            barrier_init(smem_address(&s.empty[i]), 1);
        }
        barrier_init(smem_address(&s.done), 1);
        s.stalled = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    dependent_launch_prologue();
    if (warp == 2) tensor_alloc<1>(smem_address(&s.tensor_base), a.tensor_columns);
    tensor_fence_before();
    __syncthreads();
    tensor_fence_after();
    const uint32_t base = *reinterpret_cast<volatile uint32_t*>(&s.tensor_base);
    const unsigned half_blocks = (a.depth + kBlockK - 1) / kBlockK, blocks = half_blocks * (KIND == kGradX ? 2 : 1);
    const unsigned k0 = rank * blocks / cs, k1 = (rank + 1) * blocks / cs;  // (at least one: cs is at most `blocks`)

    if (threadIdx.x == 0) {
        unsigned stage = 0, phase = 0;
        for (unsigned k = k0; k < k1; ++k) {
            if (!barrier_wait(smem_address(&s.empty[stage]), phase ^ 1, &s.stalled)) {
                for (int i = 0; i < 2000; ++i) __nanosleep(1000);  // copies under way land within this time
                break;
            }
            const uint32_t bar = smem_address(&s.full[stage]), to = stages + stage * stage_bytes;
            barrier_expect(bar, stage_bytes);
            const bool second = KIND == kGradX && k >= half_blocks;
            const int at = (int)((second ? k - half_blocks : k) * kBlockK);
            if constexpr (A_LINES) {
                load_box_alone(to, &a.a[second], (int)col, at, bar);
                load_box_alone(to + kThinRows * kBlockK, &a.a[second], (int)col + 64, at, bar);
            } else {
                load_box_alone(to, &a.a[0], at, (int)col, bar);
                load_box_alone(to + kThinRows * kBlockK, &a.a[1], at, (int)col, bar);
            }
            load_box_alone(to + kThinRows * kBlockK * 2, &a.b[second], at, (int)first, bar);
            if (++stage == a.stages) stage = 0, phase ^= 1;
        }
    } else if (threadIdx.x == 32) {
        const uint32_t instr = instruction(a.is_bf16 != 0, A_LINES, false, kThinRows, (int)a.chunk);
        unsigned stage = 0, phase = 0;
        bool ok = true;
        for (unsigned k = k0; k < k1 && ok; ++k) {
            ok = barrier_wait(smem_address(&s.full[stage]), phase, &s.stalled);
            if (!ok) break;
            tensor_fence_after();
            const uint64_t da = operand(stages + stage * stage_bytes, A_LINES);
            const uint64_t db = operand(stages + stage * stage_bytes + kThinRows * kBlockK * 2, false);
#pragma unroll
            for (int i = 0; i < kBlockK / 16; ++i) multiply_alone(base, da + i * operand_step(A_LINES), db + i * operand_step(false), instr, k > k0 || i > 0);
            commit_alone(smem_address(&s.empty[stage]));
            if (++stage == a.stages) stage = 0, phase ^= 1;
        }
        commit_alone(smem_address(&s.done));
    }
    __syncwarp();
    const bool ok = __all_sync(~0u, barrier_wait(smem_address(&s.done), 0, &s.stalled));
    tensor_fence_after();
    if (ok) {
        for (unsigned t = 0; t < many; t += 16) {
            float x[16];
            tensor_load(base + (warp * 32 << 16) + t, x);
            tensor_load_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) sums[(t + i) * kThinRows + threadIdx.x] = x[i];
        }
    }
    tensor_fence_before();
    if (cs > 1) cluster_sync();
    else __syncthreads();
    if (warp == 2) {
        tensor_fence_after();
        tensor_free<1>(base, a.tensor_columns);
    }
    // four columns of a token at a time; the ranks' parts are all on their way before the first is added
    const auto total = [&](unsigned at, float (&x)[4]) {
        if (cs == 1) {
            const float4 q = *reinterpret_cast<const float4*>(sums + at);
            x[0] = q.x, x[1] = q.y, x[2] = q.z, x[3] = q.w;
            return;
        }
        float4 q[kThinCluster];
#pragma unroll
        for (unsigned c = 0; c < kThinCluster; ++c)
            if (c < cs) q[c] = cluster_load4(cluster_address(sums + at, c));
        x[0] = q[0].x, x[1] = q[0].y, x[2] = q[0].z, x[3] = q[0].w;
#pragma unroll
        for (unsigned c = 1; c < kThinCluster; ++c)
            if (c < cs) x[0] += q[c].x, x[1] += q[c].y, x[2] += q[c].z, x[3] += q[c].w;
    };
    const auto put = [&](const RowsOut& out, long long at, int valid, bool whole, const float (&x)[4]) {
        T* const p = static_cast<T*>(out.p) + at;
        if (whole) {
            const float y[8] = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
            const uint4 q = pack<T>(y);
            *reinterpret_cast<uint2*>(p) = make_uint2(q.x, q.y);
        } else {
#pragma unroll
            for (int l = 0; l < 4; ++l)
                if (l < valid) p[l] = from_f32<T>(x[l]);
        }
    };
    const auto on_8 = [](const RowsOut& o) { return ((reinterpret_cast<uintptr_t>(o.p) | (uintptr_t)(o.so * 2) | (uintptr_t)(o.si * 2)) & 7) == 0; };
    const bool vec = on_8(a.out[0]) && on_8(a.out[1]) && on_8(a.out[2]);
    for (unsigned i = rank * kThinThreads + threadIdx.x; i < many * (WIDE / 4); i += cs * kThinThreads) {
        const unsigned t = i / (WIDE / 4), c = i % (WIDE / 4) * 4;
        if (col + c >= a.columns) continue;
        const int valid = (int)min(4u, a.columns - col - c);
        const long long o = (first + t) / a.n_inner, n = (first + t) % a.n_inner;
        const auto at = [&](const RowsOut& out) { return o * out.so + n * out.si + col + c; };
        float x[4];
        total(t * kThinRows + c, x);
        if constexpr (KIND == kForward) {
            float u[4];
            total(t * kThinRows + 64 + c, u);
            if (a.save) {
                put(a.out[1], at(a.out[1]), valid, vec && valid == 4, x);
                put(a.out[2], at(a.out[2]), valid, vec && valid == 4, u);
            }
#pragma unroll
            for (int l = 0; l < 4; ++l) x[l] = activate<GELU>(x[l]) * u[l];
        }
        put(a.out[0], at(a.out[0]), valid, vec && valid == 4, x);
    }
    if (cs > 1) cluster_sync();  // the others have read this CTA's sums
}

// Of thin_kernel's size but for tensor memory; never launched (thin_clusters).
static __global__ void __launch_bounds__(kThinThreads) thin_room_kernel() {
    extern __shared__ unsigned char raw[];
    if (blockDim.x > kThinThreads) raw[threadIdx.x] = 0;
    dependent_launch_prologue();
}

// ------------------------------------------------------------------ operands laid out
// Rows that TMA cannot address (a row that does not start on 16 bytes, leading axes that do not fold into one), and
// weights that stand in the arena in 32 bits, are copied once, rounded to the type of the products.
struct LayMatrix {
    const void* from;
    void* to;  // [rows][pitch]
    long long so, si;
    unsigned rows, n_inner;
    int f32;  // rounded from 32 bits
};
struct LayArgs {
    LayMatrix m[3];  // of one width; those without rows are left out
    unsigned columns, pitch;
};
constexpr int kLayThreads = 256;
// kLayRows rows a thread, all on their way before the first is shifted and written.  (2 x 11007 x 4095 bf16, 361 MB read and
// written, beside 64 tokens' product: 105 us in all; 107 and 111 with one and four rows, 128 with a branch for each alignment.)
constexpr int kLayRows = 2;
template <typename T>
__global__ void __launch_bounds__(kLayThreads) lay_kernel(const __grid_constant__ LayArgs a) {
    dependent_launch_prologue();
    const unsigned col = (blockIdx.y * blockDim.x + threadIdx.x) * 8, step = gridDim.x * blockDim.y, rows = a.m[0].rows + a.m[1].rows + a.m[2].rows;
    if (col >= a.columns) return;
    const unsigned many = min(8u, a.columns - col);
    for (unsigned row = blockIdx.x * blockDim.y + threadIdx.y; row < rows; row += kLayRows * step) {
        uint4 u[kLayRows], v[kLayRows];
        unsigned shift[kLayRows];
        const float* slow[kLayRows];
        T* to[kLayRows];
#pragma unroll
        for (int i = 0; i < kLayRows; ++i) {
            unsigned r = min(row + i * step, rows - 1);  // (behind the last row: that again, not written)
            const int k = r < a.m[0].rows ? 0 : r - a.m[0].rows < a.m[1].rows ? 1 : 2;
            r -= (k > 0 ? a.m[0].rows : 0) + (k > 1 ? a.m[1].rows : 0);
            const LayMatrix& m = a.m[k];
            to[i] = static_cast<T*>(m.to) + (size_t)r * a.pitch + col;
            const long long at = (r / m.n_inner) * m.so + (r % m.n_inner) * m.si + col;
            const uintptr_t p = reinterpret_cast<uintptr_t>(m.from) + at * (m.f32 ? 4 : 2);
            const bool pieces = m.f32 && (many < 8 || (p & 15) != 0);  // element by element
            slow[i] = pieces ? reinterpret_cast<const float*>(p) : nullptr;
            shift[i] = m.f32 ? 16 : (unsigned)(p & 15);
            // the words that hold elements of these; none that holds none
            const uintptr_t first = pieces ? p & ~(uintptr_t)15 : p - (m.f32 ? 0 : shift[i]), end = p + many * (m.f32 ? 4 : 2);
            const uintptr_t second = first + 16 < end ? first + 16 : first;
            u[i] = *reinterpret_cast<const uint4*>(first);
            v[i] = *reinterpret_cast<const uint4*>(second);
        }
#pragma unroll
        for (int i = 0; i < kLayRows; ++i) {
            if (row + i * step >= rows) break;
            uint4 q;
            if (shift[i] < 16) {
                q = shifted(u[i], v[i], shift[i]);
            } else {
                float x[8] = {__uint_as_float(u[i].x), __uint_as_float(u[i].y), __uint_as_float(u[i].z), __uint_as_float(u[i].w),
                              __uint_as_float(v[i].x), __uint_as_float(v[i].y), __uint_as_float(v[i].z), __uint_as_float(v[i].w)};
                if (slow[i] != nullptr) {
#pragma unroll
                    for (int l = 0; l < 8; ++l) x[l] = l < (int)many ? slow[i][l] : 0.0f;
                }
                q = pack<T>(x);
            }
            *reinterpret_cast<uint4*>(to[i]) = q;
        }
    }
}

// ------------------------------------------------------------------ gradient of the two projections
// dg = dh up act'(gate), du = dh act(gate), rounded to 16 bits: they are operands of the products that follow.
struct SlopeArgs {
    RowsOut gate, up, dh;
    void* dg;
    void* du;  // [rows][pitch]
    unsigned rows, n_inner, columns, pitch;
    int vec;
};
template <typename T, bool GELU>
__global__ void __launch_bounds__(kLayThreads) slope_kernel(const __grid_constant__ SlopeArgs a) {
    dependent_launch_prologue();
    const unsigned col = (blockIdx.y * blockDim.x + threadIdx.x) * 8;
    if (col >= a.columns) return;
    for (unsigned row = blockIdx.x * blockDim.y + threadIdx.y; row < a.rows; row += gridDim.x * blockDim.y) {
        const unsigned o = row / a.n_inner, i = row % a.n_inner;
        const T* const pg = static_cast<const T*>(a.gate.p) + o * a.gate.so + i * a.gate.si + col;
        const T* const pu = static_cast<const T*>(a.up.p) + o * a.up.so + i * a.up.si + col;
        const T* const pd = static_cast<const T*>(a.dh.p) + o * a.dh.so + i * a.dh.si + col;
        float g[8] = {}, u[8] = {}, d[8] = {};
        if (a.vec && col + 8 <= a.columns) {
            unpack<T>(*reinterpret_cast<const uint4*>(pg), g);
            unpack<T>(*reinterpret_cast<const uint4*>(pu), u);
            unpack<T>(*reinterpret_cast<const uint4*>(pd), d);
        } else if (col + 8 <= a.columns) {
            unpack<T>(load_anywhere(pg), g);
            unpack<T>(load_anywhere(pu), u);
            unpack<T>(load_anywhere(pd), d);
        } else {
#pragma unroll
            for (int l = 0; l < 8; ++l) {
                if (col + l < a.columns) g[l] = to_f32<T>(pg[l]), u[l] = to_f32<T>(pu[l]), d[l] = to_f32<T>(pd[l]);
            }
        }
#pragma unroll
        for (int l = 0; l < 8; ++l) {
            const Activated act = activate_with_slope<GELU>(g[l]);
            g[l] = d[l] * u[l] * act.slope;
            u[l] = d[l] * act.value;
        }
        const size_t at = (size_t)row * a.pitch + col;
        *reinterpret_cast<uint4*>(static_cast<T*>(a.dg) + at) = pack<T>(g);
        *reinterpret_cast<uint4*>(static_cast<T*>(a.du) + at) = pack<T>(u);
    }
}

}  // namespace odsgd_lm
