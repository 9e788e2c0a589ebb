// Device code of the language-model operators around the update (sm_100a): token embedding and
// its gradient, token scores, the clipped policy loss with its gradient, gradient norm and clip.
//
// All of them are bound by memory traffic; each kernel's comment says how it keeps to one read of
// what it reads and one write of what it writes, and what was measured.  Times are of the kernels alone on
// one B200, whose copy rate is 6549 GB/s, in a CUDA graph of a few passes.  Passes that go on for longer
// run at the clock that the power limit leaves, which costs those with an exponential an element up to a
// sixth, the others a few per cent; calls that are shorter than some 10 us wait for the host.
// Every kernel waits (griddepcontrol.wait, dependent_launch_prologue) before it reads.
#pragma once

#include "odsgd_lm_softmax.cuh"

namespace odsgd_lm {

// ------------------------------------------------------------------ rows of logits
// A cluster of `cluster` CTAs takes a row; the row's 16-byte vectors are split evenly over it.
constexpr int kRowCluster = 8;  // most CTAs of a row (the portable limit)

struct VecView {
    const float* p;
    long long so, si;
};

struct RowArgs {
    const void* z;
    const void* labels;
    VecView old_logp, ref_logp, adv, weight;
    void* dz;
    float* logp;
    float* lse;
    float* terms;  // [3][rows]: w pg, w kl, w of clipped rows
    long long z_so, z_si, l_so, l_si, d_so, d_si;
    long long vocab;
    unsigned rows, n_inner;
    int wide_labels;
    int cluster;
    int hold;  // losses: batches of a row that a CTA holds in shared memory
    float inv_temp, clip_low, clip_high, kl_coef, grad_scale;
    float exp_temp;  // inv_temp as RowExp takes it
};

__device__ __forceinline__ void store_elements(float* p, const uint4& q) {
    p[0] = __uint_as_float(q.x);
    p[1] = __uint_as_float(q.y);
    p[2] = __uint_as_float(q.z);
    p[3] = __uint_as_float(q.w);
}
template <typename T>
__device__ __forceinline__ void store_elements(T* p, const uint4& q) {
    const uint32_t u[4] = {q.x, q.y, q.z, q.w};
    unsigned short* h = reinterpret_cast<unsigned short*>(p);
#pragma unroll
    for (int i = 0; i < 8; ++i) h[i] = (unsigned short)(u[i / 2] >> (i % 2 * 16));
}
// `aligned`: the gradient's row starts as far behind a 16-byte boundary as the logits' does.  Where it does not
// (a shifted view of an odd vocabulary, with a contiguous gradient) elements are stored one by one: 8184 rows of
// 50257 bf16 take 1084 us, of 50256 298.
template <typename T>
__device__ __forceinline__ void store_vector(T* p, const uint4& q, bool aligned) {
    if (aligned) __stcs(reinterpret_cast<uint4*>(p), q);
    else store_elements(p, q);
}

// A row's inputs besides its logits.
struct RowInputs {
    float old_logp = 0.0f, ref_logp = 0.0f, adv = 0.0f;
    __device__ __forceinline__ void load(const RowArgs& a, long long o, long long i) {
        old_logp = a.old_logp.p[o * a.old_logp.so + i * a.old_logp.si];
        if (a.ref_logp.p != nullptr) ref_logp = a.ref_logp.p[o * a.ref_logp.so + i * a.ref_logp.si];
        adv = a.adv.p[o * a.adv.so + i * a.adv.si];
    }
};
// What a row's statistics make of its loss, and the factor k of its gradient.
struct RowLoss {
    float k, pg, kl, clipped;
    __device__ __forceinline__ RowLoss(const RowArgs& a, const RowInputs& in, float logp, float w) {
        const float r = expf(logp - in.old_logp);
        const float bounded = fminf(fmaxf(r, 1.0f - a.clip_low), 1.0f + a.clip_high) * in.adv;
        const float free_term = r * in.adv;
        const bool cut = free_term > bounded;
        // NaN stays: a comparison with it is false, and r itself is NaN
        pg = -w * (cut ? bounded : free_term);
        clipped = cut ? w : 0.0f;
        float g = cut ? 0.0f : -free_term;
        kl = 0.0f;
        if (a.ref_logp.p != nullptr) {
            const float d = in.ref_logp - logp;
            const float em = expm1f(d);  // exp(d) - 1 without its cancellation near d = 0
            kl = w * (em - d);
            if (a.kl_coef != 0.0f) g -= a.kl_coef * em;  // (0 times an em that overflows would be NaN)
        }
        k = w * g * a.inv_temp * a.grad_scale;
    }
    __device__ __forceinline__ void store(const RowArgs& a, unsigned row, float logp) const {
        a.logp[row] = logp;
        a.terms[row] = pg;
        a.terms[a.rows + row] = kl;
        a.terms[2 * (size_t)a.rows + row] = clipped;
    }
};

// dz_j = k ([j == y] - exp(c (z_j - m)) / s): of a vector's elements as if none were the label, and
// of one element.
template <typename T>
struct RowGradient {
    RowExp<T> e;
    float neg;  // -k / s
    __device__ __forceinline__ RowGradient(float exp_temp, float m, float neg_) : e(exp_temp, m), neg(neg_) {}
    __device__ __forceinline__ uint4 operator()(const uint4& q) const {
        constexpr int L = kLanes<T>;
        float p[L];
        unpack<T>(q, p);
#pragma unroll
        for (int l = 0; l < L; l += 2) split(e(p[l], p[l + 1]) * f2(neg, neg), p[l], p[l + 1]);
        return pack<T>(p);
    }
    __device__ __forceinline__ T element(float z, float k) const {
        float p0, p1;
        split(e(z, z) * f2(neg, neg), p0, p1);
        return from_f32<T>(p0 + k);
    }
};

// Scores, and the loss with its gradient.  One CTA takes a row (a cluster shares it where rows are
// few, or so long that the rows in flight would not stay in the L2) and goes over it twice: maximum
// and sum, then the gradient.  The second reading finds the row's first batches in the CTA's shared
// memory, its last in registers and the rest in the L2; DRAM sees about one read and one write (8192
// rows of 131072 bf16: 0.62 ms against 0.55 for those bytes at the copy rate; 0.66 with the whole
// second reading from the L2, which by then has lost a sixth of it).
// Scores: 8184 rows of 50021 bf16 126 us, 0.97 of the copy rate, in 128-thread CTAs, twelve an SM
// (182 in 512-thread ones: the more rows in flight, the less the latency of label, row and join
// shows).  Losses: 256 threads, five an SM, and for rows the L2 holds fewer of 512, two an SM.
// Four vectors a thread in flight rather than eight: 881 -> 681 us for the wide loss, by the warps
// that fit.
// Measured slower: the row held in registers, or in shared memory with the next rows on their way by
// asynchronous copies, across a cluster of 4 or 8 CTAs (716-990 us: the cluster's sums are waited for,
// and clusters of eight leave 16 SMs empty); a quarter or half of the exponentials by a polynomial on
// the multiply-add units (2 % and 9 % slower: issue slots, not the special-function units, run out).
template <typename T, bool LOSS, int THREADS, int CTAS>
__global__ void __launch_bounds__(THREADS, CTAS) row_kernel(const __grid_constant__ RowArgs a) {
    constexpr int L = kLanes<T>;
    __shared__ MaxSum warp_part[THREADS / 32];
    __shared__ MaxSum cta_part[kRowCluster];
    extern __shared__ uint4 held[];  // [a.hold][kRowVectors][threads]: each thread's vectors of the first batches
    dependent_launch_prologue();
    const unsigned cs = (unsigned)a.cluster;
    const unsigned row = blockIdx.x / cs, rank = blockIdx.x % cs;
    const int tid = (int)threadIdx.x, threads = (int)blockDim.x;
    const long long o = row / a.n_inner, i = row % a.n_inner;
    const T* zrow = static_cast<const T*>(a.z) + o * a.z_so + i * a.z_si;
    T* drow = LOSS ? static_cast<T*>(a.dz) + o * a.d_so + i * a.d_si : nullptr;
    const bool aligned = ((reinterpret_cast<uintptr_t>(drow) ^ reinterpret_cast<uintptr_t>(zrow)) & 15) == 0;
    const long long y = load_token(a.labels, a.wide_labels != 0, o * a.l_so + i * a.l_si);
    const float w = LOSS ? a.weight.p[o * a.weight.so + i * a.weight.si] : 1.0f;
    const RowParts<T> parts(zrow, (int)a.vocab);
    const int per = (parts.vectors + (int)cs - 1) / (int)cs;
    const int v0 = min((int)rank * per, parts.vectors), n = min(per, parts.vectors - v0);
    const uint4* zv = reinterpret_cast<const uint4*>(zrow + parts.head) + v0;  // the CTA's n vectors
    T* dv = drow + parts.head + v0 * L;
    const int edge = rank == 0 ? parts.edge(tid) : -1;
    const bool first = rank == 0 && tid == 0;

    if (w == 0.0f || y < 0 || y >= a.vocab) {  // the whole cluster leaves here together
        if (first) {
            a.logp[row] = 0.0f;
            if (LOSS) a.terms[row] = a.terms[a.rows + row] = a.terms[2 * (size_t)a.rows + row] = 0.0f;
            else if (a.lse != nullptr) a.lse[row] = 0.0f;
        }
        if (LOSS) {
            for (int v = tid; v < n; v += threads) store_vector(dv + v * L, make_uint4(0, 0, 0, 0), aligned);
            if (edge >= 0) drow[edge] = from_f32<T>(0.0f);
        }
        return;
    }
    if (cs > 1) cluster_arrive();  // this CTA runs: its shared memory may be written (waited for below)
    const float zy = to_f32(zrow[y]);
    const float ze = edge >= 0 ? to_f32(zrow[edge]) : -CUDART_INF_F;

    MaxSum x = single(ze);
    const int step = threads * kRowVectors;
    uint4 q[kRowVectors];
    int b = 0;
    const int kept = LOSS ? a.hold * step : 0;  // vectors before this one are held
    for (; b + step <= n; b += step) {
        if (LOSS && b >= kept) {
#pragma unroll
            for (int k = 0; k < kRowVectors; ++k) q[k] = zv[b + k * threads + tid];
        } else {
#pragma unroll
            for (int k = 0; k < kRowVectors; ++k) q[k] = __ldcs(zv + b + k * threads + tid);
        }
        if (LOSS && b < kept) {
#pragma unroll
            for (int k = 0; k < kRowVectors; ++k) held[b + k * threads + tid] = q[k];
        }
        x = add_vectors<T>(x, q, a.inv_temp, a.exp_temp);
    }
    if (b < n) {
#pragma unroll
        for (int k = 0; k < kRowVectors; ++k) q[k] = b + k * threads + tid < n ? __ldcs(zv + b + k * threads + tid) : neg_inf_vector<T>();
        x = add_vectors<T>(x, q, a.inv_temp, a.exp_temp);
    } else {
        b -= step;  // the batch that q holds
    }
    RowInputs in;
    if (LOSS) in.load(a, o, i);
    x = warp_join(x, a.inv_temp);
    const int lane = tid & 31, warps = threads >> 5;
    if (warps > 1) {
        if (lane == 0) warp_part[tid >> 5] = x;
        __syncthreads();
        x = lane < warps ? warp_part[lane] : MaxSum{-CUDART_INF_F, 0.0f};
        x = warp_join(x, a.inv_temp);
    }
    if (cs > 1) {
        cluster_wait();
        if (threadIdx.x < cs) {
            const uint32_t at = cluster_address(&cta_part[rank], threadIdx.x);
            cluster_store(at, x.m);
            cluster_store(at + 4, x.s);
        }
        // also orders every CTA's reads of z[y] ahead of every CTA's writes, for dz == z
        cluster_sync();
        x = lane < (int)cs ? cta_part[lane] : MaxSum{-CUDART_INF_F, 0.0f};
        x = warp_join(x, a.inv_temp);
    } else if (LOSS) {
        __syncthreads();  // every thread has read z[y] before one of them may write there
    }
    const float log_s = logf(x.s);
    const float logp = (zy - x.m) * a.inv_temp - log_s;
    if (!LOSS) {
        if (first) {
            a.logp[row] = logp;
            if (a.lse != nullptr) a.lse[row] = x.m * a.inv_temp + log_s;
        }
        return;
    }
    const RowLoss loss(a, in, logp, w);
    if (first) loss.store(a, row, logp);
    const RowGradient<T> grad(a.exp_temp, x.m, -loss.k / x.s);
    if (aligned) {
        uint4* to = reinterpret_cast<uint4*>(dv);
#pragma unroll
        for (int k = 0; k < kRowVectors; ++k) {
            const int v = b + k * threads + tid;
            if (v >= 0 && v < n) __stcs(to + v, grad(q[k]));
        }
        for (b -= step; b >= 0; b -= step) {
            if (b < kept) {
#pragma unroll
                for (int k = 0; k < kRowVectors; ++k) q[k] = held[b + k * threads + tid];
            } else {
#pragma unroll
                for (int k = 0; k < kRowVectors; ++k) q[k] = __ldcs(zv + b + k * threads + tid);
            }
#pragma unroll
            for (int k = 0; k < kRowVectors; ++k) __stcs(to + b + k * threads + tid, grad(q[k]));
        }
    } else {
        for (int v = tid; v < n; v += threads) store_elements(dv + v * L, grad(zv[v]));
    }
    // the label's element again, by the thread that has written its vector
    const int at = (int)y - parts.head - v0 * L;
    if (at >= 0 && at / L < n && at / L % threads == tid) dv[at] = grad.element(zy, loss.k);
    if (edge >= 0) drow[edge] = grad.element(ze, edge == (int)y ? loss.k : 0.0f);
}

// Sums the rows' terms in a fixed order, in 64 bits: one CTA.
struct StatsArgs {
    const float* terms;
    float* stats;
    unsigned rows;
    float kl_coef;
};
constexpr int kStatsThreads = 1024;

template <int N, int THREADS>
__device__ __forceinline__ void block_sum(double (&x)[N], double* smem) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) x[n] += __shfl_down_sync(0xffffffffu, x[n], d);
        if (lane == 0) smem[n * (THREADS / 32) + warp] = x[n];
    }
    __syncthreads();
    if (warp == 0) {
#pragma unroll
        for (int n = 0; n < N; ++n) {
            x[n] = lane < THREADS / 32 ? smem[n * (THREADS / 32) + lane] : 0.0;
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) x[n] += __shfl_down_sync(0xffffffffu, x[n], d);
        }
    }
}

__global__ void __launch_bounds__(kStatsThreads) stats_kernel(const __grid_constant__ StatsArgs a) {
    __shared__ double part[3 * kStatsThreads / 32];
    dependent_launch_prologue();
    double x[3] = {0.0, 0.0, 0.0};
    for (unsigned r = threadIdx.x; r < a.rows; r += kStatsThreads) {
#pragma unroll
        for (int n = 0; n < 3; ++n) x[n] += a.terms[(size_t)n * a.rows + r];
    }
    block_sum<3, kStatsThreads>(x, part);
    if (threadIdx.x == 0) {
        a.stats[0] = (float)(a.kl_coef != 0.0f ? x[0] + (double)a.kl_coef * x[1] : x[0]);
        a.stats[1] = (float)x[0];
        a.stats[2] = (float)x[1];
        a.stats[3] = (float)x[2];
    }
}

// ------------------------------------------------------------------ embedding lookup
struct LookupArgs {
    const void* tokens;
    const void* table;
    void* act;
    long long t_so, t_si, a_so, a_si, stride, vocab, dim;
    unsigned rows, n_inner;
    int wide_tokens;
    int per;  // rows of a thread
    float scale;
};
constexpr int kLookupThreads = 256;
constexpr int kLookupRows = 64;  // most rows of a CTA
template <typename TT, typename TA, bool VEC>
constexpr int kLookupColumns = VEC ? (kLanes<TT> < kLanes<TA> ? kLanes<TT> : kLanes<TA>) : 4;  // of a thread

// A thread's W columns of a row, from column `col` on.  VEC: next to one another, as many as 16 bytes of
// the wider type hold: that side moves 16 bytes a thread, the other 8 or 16, and both without
// gaps between the threads.  Otherwise (rows that are not aligned): blockDim.x apart, up to dim.
template <typename T, bool VEC, int W>
__device__ __forceinline__ void load_columns(const T* row, long long col, long long dim, float (&x)[W]) {
    const T* p = row + col;
    if constexpr (!VEC) {
#pragma unroll
        for (int l = 0; l < W; ++l)
            if (col + l * (int)blockDim.x < dim) x[l] = to_f32(p[l * (int)blockDim.x]);
    } else if constexpr (W == kLanes<T>) {
        unpack<T>(*reinterpret_cast<const uint4*>(p), x);
    } else {
        float y[8];
        const uint2 q = *reinterpret_cast<const uint2*>(p);
        unpack<T>(make_uint4(q.x, q.y, 0, 0), y);
#pragma unroll
        for (int l = 0; l < W; ++l) x[l] = y[l];
    }
}
template <typename T, bool VEC, int W>
__device__ __forceinline__ void store_columns(T* row, long long col, long long dim, const float (&x)[W]) {
    T* p = row + col;
    if constexpr (!VEC) {
#pragma unroll
        for (int l = 0; l < W; ++l)
            if (col + l * (int)blockDim.x < dim) p[l * (int)blockDim.x] = from_f32<T>(x[l]);
    } else if constexpr (W == kLanes<T>) {
        *reinterpret_cast<uint4*>(p) = pack<T>(x);
    } else {
        const float y[8] = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
        const uint4 q = pack<T>(y);
        *reinterpret_cast<uint2*>(p) = make_uint2(q.x, q.y);
    }
}

// blockDim = (columns, rows); the CTA's rows, a.per for each of its thread rows, are looked up once, by as many
// threads, and four rows a thread are in flight.  32760 tokens, 4096 columns, fp32 -> bf16: 74 us, 0.90
// of the copy rate for one read of the rows that occur and one write (every thread looking its
// rows up by itself 83 us; one row a thread 166).
template <typename TT, typename TA, bool VEC>
__global__ void __launch_bounds__(kLookupThreads) lookup_kernel(const __grid_constant__ LookupArgs a) {
    constexpr int W = kLookupColumns<TT, TA, VEC>;
    constexpr int B = 4;
    __shared__ const TT* from[kLookupRows];
    __shared__ TA* to[kLookupRows];
    dependent_launch_prologue();
    const unsigned rows = blockDim.y * a.per, r0 = blockIdx.x * rows, n = min(rows, a.rows - r0);
    for (unsigned r = threadIdx.y * blockDim.x + threadIdx.x; r < n; r += blockDim.x * blockDim.y) {
        const unsigned o = (r0 + r) / a.n_inner, i = (r0 + r) % a.n_inner;
        const long long t = load_token(a.tokens, a.wide_tokens != 0, o * a.t_so + i * a.t_si);
        from[r] = t >= 0 && t < a.vocab ? static_cast<const TT*>(a.table) + t * a.stride : nullptr;
        to[r] = static_cast<TA*>(a.act) + o * a.a_so + i * a.a_si;
    }
    __syncthreads();
    const long long col = (long long)blockIdx.y * blockDim.x * W + threadIdx.x * (VEC ? W : 1);
    if (col >= a.dim) return;
    for (unsigned r = threadIdx.y; r < n; r += B * blockDim.y) {
        float x[B][W];
#pragma unroll
        for (int k = 0; k < B; ++k) {
#pragma unroll
            for (int l = 0; l < W; ++l) x[k][l] = 0.0f;
            const unsigned j = r + k * blockDim.y;
            if (j < n && from[j] != nullptr) load_columns<TT, VEC>(from[j], col, a.dim, x[k]);
        }
#pragma unroll
        for (int k = 0; k < B; ++k) {
            const unsigned j = r + k * blockDim.y;
            if (j >= n) break;
            if (from[j] != nullptr) {  // (zeros stay zeros whatever the scale)
#pragma unroll
                for (int l = 0; l < W; ++l) x[k][l] *= a.scale;
            }
            store_columns<TA, VEC>(to[j], col, a.dim, x[k]);
        }
    }
}

// ------------------------------------------------------------------ embedding gradient
// Three launches.
//   sort_kernel  One cluster sorts the tokens' positions by token, stably (up to 8192 by a bitonic
//                network in each CTA and a merge: 2040 tokens 18.5 -> 13.6 us in all; more, least significant
//                digit first, up to 9 bits a pass), marks the tokens that occur, and lists those whose run crosses a
//                block boundary.  The other CTAs of the grid meanwhile write zeros to the first
//                `early` rows of the table, as many as the sort takes time for, named or not.
//   sum_kernel   A CTA takes `block` consecutive sorted positions and a slab of columns, and adds
//                runs of equal tokens in 32 bits.  A run inside the block is written to the table,
//                the part of one that crosses a boundary to the workspace.  Work is split by
//                position, so that a token that fills half the batch holds up no CTA here; its parts, one a
//                block, are left to the join.
//                Further CTAs, spread among these, write zeros to the other rows that no token names.
//   join_kernel  Adds the parts of the runs that cross boundaries, in an order that the sizes fix: a CTA takes a run and a
//                slab of columns, so one very long run is added by few.
// The order of every sum depends on sizes and tokens alone.
// 32760 tokens, 2048 bf16 columns, a table of 50021 rows (544 MB): 109 us, 0.76 of the copy rate: 25 us of
// zeros beside the sort (of which the sort takes 20), 75 for sums and the other zeros, 8 for the join.
// Rows kept packed until they are added, so that eight rows a thread and eight CTAs an SM are in flight:
// sums 77 -> 36 us.
constexpr int kSortCluster = 8;
constexpr int kSortThreads = 1024;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortBits = 9;
constexpr int kSortRadix = 1 << kSortBits;
constexpr int kSortSmem = (kSortWarps * kSortRadix + 2 * kSortRadix + kSortWarps) * 4;
static_assert(kSortSmem >= (kSortCluster * 4 + 2 * 8) * kSortThreads, "the parts and buffers of sort_some_tokens");
constexpr int kFillClusters = 1000;  // most clusters that write zeros beside the sort, ...
constexpr int kFillBytes = 1 << 18;  // ... each at least so many of the table
constexpr int kFillRows = 32;        // rows of a CTA that writes zeros beside the sums: one word of marks

struct SpanRun {
    unsigned token, first, last;  // blocks [first, last]
};

struct EmbedGradArgs {
    const void* tokens;
    const void* act;
    float* table;
    long long t_so, t_si, a_so, a_si, stride, vocab, dim, padding;
    unsigned n, n_inner;
    int wide_tokens, accumulate;
    int flat;  // token t lies at t * t_si
    float scale;
    // workspace
    unsigned* key[2];
    unsigned* pos[2];
    unsigned* counts;  // [0] spanning runs
    unsigned* named;   // a bit for each row from `early` on: some token names it
    unsigned early;    // a multiple of kFillRows, or vocab
    unsigned fills;    // CTAs of sum_kernel that write zeros
    SpanRun* runs;
    float* head;  // [blocks][pitch]: part of the run that began in an earlier block
    float* tail;  // [blocks][pitch]: first part of a run that goes on in the next block
    long long pitch;
    unsigned block;  // positions of a block
    int passes, bits;
};

// Tokens t, t + step, ... as sort keys; those that do not count, and places beyond n, as `vocab`.
constexpr int kKeyBatch = 4;
__device__ __forceinline__ void token_keys(const EmbedGradArgs& a, unsigned t, unsigned step, unsigned (&key)[kKeyBatch]) {
    long long x[kKeyBatch];
#pragma unroll
    for (int k = 0; k < kKeyBatch; ++k) {
        const unsigned j = t + k * step;
        x[k] = -1;
        if (j < a.n) x[k] = load_token(a.tokens, a.wide_tokens != 0, a.flat ? j * a.t_si : j / a.n_inner * a.t_so + j % a.n_inner * a.t_si);
    }
#pragma unroll
    for (int k = 0; k < kKeyBatch; ++k) key[k] = x[k] >= 0 && x[k] < a.vocab && x[k] != a.padding ? (unsigned)x[k] : (unsigned)a.vocab;
}

__device__ __forceinline__ void clear_marks(const EmbedGradArgs& a, unsigned thread, unsigned threads) {
    if (a.fills == 0) return;
    const unsigned words = ((unsigned)a.vocab - a.early + 31) / 32;
    for (unsigned i = thread; i < words; i += threads) a.named[i] = 0;
}

// Of the sorted tokens: marks the rows that are named, and lists the runs that cross a block
// boundary (the first boundary inside the run does, with the block its last position lies in),
// counting them at `count`.
template <typename Key>
__device__ __forceinline__ void list_runs(const EmbedGradArgs& a, unsigned thread, unsigned threads, unsigned* count, Key key) {
    if (a.fills > 0) {
#pragma unroll 4
        for (unsigned t = thread; t < a.n; t += threads) {
            const unsigned k = key(t), row = k - a.early;
            if (k >= a.early && k < (unsigned)a.vocab && (t == 0 || key(t - 1) != k)) atomicOr(a.named + row / 32, 1u << row % 32);
        }
    }
    for (unsigned t = (thread + 1) * a.block; t < a.n; t += threads * a.block) {
        const unsigned k = key(t), before = key(t - 1), earlier = key(t - min(t, a.block + 1));
        if (k == (unsigned)a.vocab || before != k || (t != a.block && earlier == k)) continue;
        // The block of the run's end: eight places are looked at together, 1, 2, 4, ... blocks on (most
        // runs cross one boundary), then at the eighths of what is left.
        unsigned last = t / a.block, up = (a.n - 1) / a.block;  // key(last * block) == k
        for (bool grown = false; last < up; grown = true) {
            const unsigned left = up - last, eighth = (left + 7) / 8;
            unsigned same = 0;  // of the places, the first so many are in the run
#pragma unroll
            for (unsigned j = 0; j < 8; ++j) {
                const unsigned d = grown ? (j + 1) * eighth : 1u << j;
                same += key((last + min(d, left)) * a.block) == k && d <= left;
            }
            if (same < 8) up = min(up, last + (grown ? (same + 1) * eighth : 1u << same) - 1);
            if (same > 0) last += grown ? same * eighth : 1u << (same - 1);
        }
        a.runs[atomicAdd(count, 1u)] = SpanRun{k, t / a.block - 1, last};
    }
}

__device__ __forceinline__ void sort_tokens(const EmbedGradArgs& a, unsigned* smem) {
    unsigned* cnt = smem;                           // [warps][radix]
    unsigned* tot = cnt + kSortWarps * kSortRadix;  // [radix], read by the other CTAs
    unsigned* base = tot + kSortRadix;              // [radix]
    unsigned* wsum = base + kSortRadix;             // [warps]
    const unsigned rank = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned radix = 1u << a.bits;
    // each warp of the cluster owns a contiguous range, so that warp order is position order
    unsigned per = (a.n + kSortCluster * kSortWarps - 1) / (kSortCluster * kSortWarps);
    per = (per + 31) / 32 * 32;
    const unsigned lo = min(a.n, (rank * kSortWarps + warp) * per), hi = min(a.n, lo + per);
    if (rank == 0 && tid == 0) a.counts[0] = 0;
    clear_marks(a, rank * kSortThreads + tid, kSortCluster * kSortThreads);
    for (int pass = 0; pass < a.passes; ++pass) {
        const unsigned* kin = a.key[pass & 1];
        const unsigned* pin = a.pos[pass & 1];
        unsigned* kout = a.key[(pass & 1) ^ 1];
        unsigned* pout = a.pos[(pass & 1) ^ 1];
        const int shift = pass * a.bits;
        for (unsigned d = tid; d < kSortWarps * radix; d += kSortThreads) cnt[d] = 0;
        __syncthreads();
        unsigned* mine = cnt + warp * radix;
        unsigned key[kKeyBatch], pos[kKeyBatch];
        const auto load = [&](unsigned t) {
            if (pass == 0) {
                token_keys(a, t, 32, key);
#pragma unroll
                for (int k = 0; k < kKeyBatch; ++k) pos[k] = t + 32 * k;
            } else {
#pragma unroll
                for (int k = 0; k < kKeyBatch; ++k) {
                    key[k] = t + 32 * k < hi ? __ldcg(kin + t + 32 * k) : 0;
                    pos[k] = t + 32 * k < hi ? __ldcg(pin + t + 32 * k) : 0;
                }
            }
        };
        for (unsigned t = lo + lane; t < hi; t += 32 * kKeyBatch) {
            load(t);
#pragma unroll
            for (int k = 0; k < kKeyBatch; ++k)
                if (t + 32 * k < hi) atomicAdd(mine + ((key[k] >> shift) & (radix - 1)), 1u);
        }
        __syncthreads();
        if (tid < radix) {  // exclusive scan over the warps, digit by digit
            unsigned run = 0;
#pragma unroll 1
            for (int v0 = 0; v0 < kSortWarps; v0 += 8) {
                unsigned c[8];
#pragma unroll
                for (int v = 0; v < 8; ++v) c[v] = cnt[(v0 + v) * radix + tid];
#pragma unroll
                for (int v = 0; v < 8; ++v) {
                    cnt[(v0 + v) * radix + tid] = run;
                    run += c[v];
                }
            }
            tot[tid] = run;
        }
        cluster_sync();
        // place of each digit: all smaller digits, then this digit in the CTAs before this one
        unsigned all = 0, before = 0;
        if (tid < radix) {
            for (unsigned c = 0; c < kSortCluster; ++c) {
                const unsigned x = cluster_load(cluster_address(tot + tid, c));
                before += c < rank ? x : 0;
                all += x;
            }
        }
        unsigned scan = all;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const unsigned y = __shfl_up_sync(0xffffffffu, scan, d);
            if (lane >= (unsigned)d) scan += y;
        }
        if (lane == 31) wsum[warp] = scan;
        __syncthreads();
        unsigned below = lane < warp ? wsum[lane] : 0;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) below += __shfl_xor_sync(0xffffffffu, below, d);
        if (tid < radix) base[tid] = below + scan - all + before;
        __syncthreads();
        for (unsigned t0 = lo; t0 < hi; t0 += 32 * kKeyBatch) {
            if (per > 32 * kKeyBatch) load(t0 + lane);  // else all are in registers still
#pragma unroll
            for (int k = 0; k < kKeyBatch; ++k) {
                const bool in = t0 + 32 * k + lane < hi;
                const unsigned act = __ballot_sync(0xffffffffu, in);
                if (in) {
                    const unsigned d = (key[k] >> shift) & (radix - 1);
                    const unsigned peers = __match_any_sync(act, d);
                    const unsigned at = base[d] + mine[d] + __popc(peers & ((1u << lane) - 1));
                    __syncwarp(act);
                    if ((peers >> lane) == 1) mine[d] += __popc(peers);  // the last of the equal lanes
                    kout[at] = key[k];
                    pout[at] = pos[k];
                }
                __syncwarp();
            }
        }
        cluster_sync();  // the pass is complete, in memory, for all CTAs of the cluster
    }
    const unsigned* sorted = a.key[a.passes & 1];
    list_runs(a, rank * kSortThreads + tid, kSortCluster * kSortThreads, a.counts, [&](unsigned t) { return __ldcg(sorted + t); });
}

// A token and its place in the CTA (10 bits) in one number: 32 bits where the vocabulary leaves them
// (sorting 1020 tokens takes 2.4 us so, 3.6 with 64), else 64.
template <typename N>
constexpr int kPlaceBits = sizeof(N) == 4 ? 10 : 32;
constexpr long long kNarrowVocab = (1ll << 22) - 1;  // below: no number is ~0

// Sorts the numbers that a CTA's threads hold by a bitonic network, the exchanges inside a warp by
// shuffles, the others through two buffers in turn.  Those of the threads from n on are the largest.
template <typename N>
__device__ __forceinline__ N sort_across(N x, unsigned n, N* smem) {
    const unsigned tid = threadIdx.x;
    unsigned turn = 0;
#pragma unroll
    for (unsigned size = 2; size <= kSortThreads; size *= 2) {
        if (size > 32 && size / 2 >= n) break;  // what lies beyond n is in its place already
        const bool up = (tid & size) == 0;
#pragma unroll
        for (unsigned d = size / 2; d > 0; d /= 2) {
            N y;
            if (d >= 32) {
                N* buffer = smem + turn * kSortThreads;
                turn ^= 1;
                buffer[tid] = x;
                __syncthreads();
                y = buffer[tid ^ d];
            } else {
                y = __shfl_xor_sync(0xffffffffu, x, d);
            }
            const bool lower = (tid & d) == 0;
            x = lower == up ? min(x, y) : max(x, y);
        }
    }
    return x;
}

// At most one position a thread of one CTA.
template <typename N>
__device__ __forceinline__ void sort_few_tokens(const EmbedGradArgs& a, void* smem) {
    __shared__ unsigned count;
    const unsigned tid = threadIdx.x;
    unsigned* sorted = static_cast<unsigned*>(smem);
    unsigned key[kKeyBatch];
    token_keys(a, tid, a.n, key);  // the first of the batch; the others lie beyond n
    if (tid == 0) count = 0;
    clear_marks(a, tid, kSortThreads);
    const N x = sort_across<N>((N)key[0] << kPlaceBits<N> | tid, a.n, reinterpret_cast<N*>(sorted + kSortThreads));
    key[0] = (unsigned)(x >> kPlaceBits<N>);
    if (tid < a.n) {
        a.key[a.passes & 1][tid] = key[0];
        a.pos[a.passes & 1][tid] = (unsigned)x % kSortThreads;
    }
    sorted[tid] = key[0];
    __syncthreads();
    list_runs(a, tid, kSortThreads, &count, [&](unsigned t) { return sorted[t]; });
    __syncthreads();
    if (tid == 0) a.counts[0] = count;
}

// At most one position a thread of the cluster: each CTA sorts its part, and finds for each of its
// tokens how many of every other part come before it (equal ones do from the parts before its own).
template <typename N>
__device__ __forceinline__ void sort_some_tokens(const EmbedGradArgs& a, void* smem) {
    const unsigned rank = blockIdx.x, tid = threadIdx.x;
    const unsigned per = (a.n + kSortCluster - 1) / kSortCluster, t = rank * per + tid;
    unsigned* parts = static_cast<unsigned*>(smem);  // [cluster][threads]
    unsigned* mine = parts + rank * kSortThreads;
    const bool in = tid < per && t < a.n;
    unsigned key[kKeyBatch];
    token_keys(a, in ? t : a.n, a.n, key);
    if (rank == 0 && tid == 0) a.counts[0] = 0;
    clear_marks(a, rank * kSortThreads + tid, kSortCluster * kSortThreads);
    const N none = ~(N)0;
    const N x = sort_across<N>(in ? (N)key[0] << kPlaceBits<N> | tid : none, per, reinterpret_cast<N*>(parts + kSortCluster * kSortThreads));
    const unsigned k = x == none ? ~0u : (unsigned)(x >> kPlaceBits<N>);
    mine[tid] = k;
    cluster_sync();
    unsigned size = 32;  // of the parts, in whole steps of the search
    while (size < per) size *= 2;
    unsigned got[kSortCluster - 1];
    if (tid < size) {
#pragma unroll
        for (unsigned c = 0; c < kSortCluster - 1; ++c) {
            const unsigned other = (rank + 1 + c) % kSortCluster;
            got[c] = cluster_load(cluster_address(parts + other * kSortThreads + tid, other));
        }
#pragma unroll
        for (unsigned c = 0; c < kSortCluster - 1; ++c) parts[(rank + 1 + c) % kSortCluster * kSortThreads + tid] = got[c];
    }
    __syncthreads();
    if (x != none) {
        // neighbours in a warp are neighbours in order: their searches take nearly one path
        unsigned to[kSortCluster - 1];
#pragma unroll
        for (unsigned c = 0; c < kSortCluster - 1; ++c) to[c] = (rank + 1 + c) % kSortCluster * kSortThreads;
        const auto smaller = [&](unsigned c, unsigned i) { return parts[i] < k + (rank + 1 + c >= kSortCluster ? 1 : 0); };
        for (unsigned step = size / 2; step > 0; step /= 2) {
#pragma unroll
            for (unsigned c = 0; c < kSortCluster - 1; ++c)
                if (smaller(c, to[c] + step - 1)) to[c] += step;
        }
        unsigned at = tid;
#pragma unroll
        for (unsigned c = 0; c < kSortCluster - 1; ++c) at += to[c] % kSortThreads + (smaller(c, to[c]) ? 1 : 0);
        a.key[a.passes & 1][at] = k;
        a.pos[a.passes & 1][at] = rank * per + (unsigned)x % kSortThreads;
    }
    cluster_sync();  // in memory, for all CTAs of the cluster; and no part is read any more
    const unsigned* sorted = a.key[a.passes & 1];
    list_runs(a, rank * kSortThreads + tid, kSortCluster * kSortThreads, a.counts, [&](unsigned t) { return __ldcg(sorted + t); });
}

// DIGITS: more tokens than the cluster has threads.  CTAS: of an SM.  What writes zeros needs two (32760
// tokens, 205 MB of zeros: 66 us, with one 92), for which a thread has 32 registers; the digit
// passes alone are faster with more (131072 tokens, 13 MB of zeros: 84 us, else 89).
template <bool DIGITS, int CTAS>
__global__ void __launch_bounds__(kSortThreads, CTAS) __cluster_dims__(kSortCluster, 1, 1)
    sort_kernel(const __grid_constant__ EmbedGradArgs a) {
    extern __shared__ __align__(8) unsigned smem[];
    dependent_launch_prologue();
    if (blockIdx.x < kSortCluster) {
        const bool narrow = a.vocab < kNarrowVocab;
        if constexpr (DIGITS) {
            sort_tokens(a, smem);
        } else if (a.n > kSortThreads) {
            if (narrow) sort_some_tokens<unsigned>(a, smem);
            else sort_some_tokens<unsigned long long>(a, smem);
        } else if (blockIdx.x == 0) {
            if (narrow) sort_few_tokens<unsigned>(a, smem);
            else sort_few_tokens<unsigned long long>(a, smem);
        }
        return;
    }
    const unsigned ctas = gridDim.x - kSortCluster, me = blockIdx.x - kSortCluster;
    const unsigned per = (a.early + ctas - 1) / ctas, lo = min(a.early, me * per), hi = min(a.early, lo + per);
    const bool vec = (reinterpret_cast<uintptr_t>(a.table) & 15) == 0 && a.stride % 4 == 0;
    if (vec && a.stride == a.dim) {  // one piece of memory
        float4* p = reinterpret_cast<float4*>(a.table + lo * a.dim);
        const long long n4 = (long long)(hi - lo) * a.dim / 4;
#pragma unroll 4
        for (long long j = threadIdx.x; j < n4; j += kSortThreads) __stcs(p + j, make_float4(0, 0, 0, 0));
        return;
    }
    const unsigned lane = threadIdx.x & 31;
    for (unsigned r = lo + (threadIdx.x >> 5); r < hi; r += kSortWarps) {
        float* row = a.table + r * a.stride;
        const long long n4 = vec ? a.dim / 4 : 0;
        for (long long j = lane; j < n4; j += 32) __stcs(reinterpret_cast<float4*>(row) + j, make_float4(0, 0, 0, 0));
        for (long long j = n4 * 4 + lane; j < a.dim; j += 32) __stcs(row + j, 0.0f);
    }
}

constexpr int kSumThreads = 128;
constexpr int kSumCtas = 8;
constexpr int kSumBatch = 8;       // rows a thread has in flight
constexpr int kSumMaxBlock = 64;   // most positions of a block: 16, 32 or 64

// A thread's columns of a row: a vector of T, or (rows that are not aligned) T's blockDim.x apart, of
// which `left` columns remain.
template <typename T, bool VEC>
struct Piece;
template <typename T>
struct Piece<T, true> {
    static constexpr int W = kLanes<T>;
    uint4 q;
    __device__ __forceinline__ void load(const T* p, long long) { q = __ldcs(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void add_to(float (&acc)[W]) const {
        float x[W];
        unpack<T>(q, x);
#pragma unroll
        for (int l = 0; l < W; ++l) acc[l] += x[l];
    }
};
template <typename T>
struct Piece<T, false> {
    static constexpr int W = 4;
    T x[W];
    __device__ __forceinline__ void load(const T* p, long long left) {
#pragma unroll
        for (int l = 0; l < W; ++l) x[l] = l * (int)blockDim.x < left ? p[l * (int)blockDim.x] : from_f32<T>(0.0f);
    }
    __device__ __forceinline__ void add_to(float (&acc)[W]) const {
#pragma unroll
        for (int l = 0; l < W; ++l) acc[l] += to_f32(x[l]);
    }
};

template <typename T, bool VEC>
__global__ void __launch_bounds__(kSumThreads, kSumCtas) sum_kernel(const __grid_constant__ EmbedGradArgs a) {
    constexpr int W = Piece<T, VEC>::W;
    __shared__ unsigned key[kSumMaxBlock + 2];   // of the positions, and one on either side
    __shared__ const T* row[kSumMaxBlock];
    dependent_launch_prologue();
    const long long col = (long long)blockIdx.y * blockDim.x * W + threadIdx.x * (VEC ? W : 1), left = a.dim - col;
    // CTA x writes zeros if the number of those before it grows behind it: they are spread evenly
    const unsigned fill = (unsigned)((unsigned long long)blockIdx.x * a.fills / gridDim.x);
    if ((unsigned)((blockIdx.x + 1ull) * a.fills / gridDim.x) != fill) {
        if (left <= 0) return;
        const unsigned r0 = a.early + fill * kFillRows, rows = min((unsigned)a.vocab - r0, (unsigned)kFillRows);
        const unsigned named = a.named[fill];
        for (unsigned r = 0; r < rows; ++r) {
            if ((named >> r) & 1) continue;
            float* p = a.table + (r0 + r) * a.stride + col;
            const float zero[8] = {};
            if constexpr (VEC) {
                if (W == 8 && aligned32(p)) {
                    store_eight(p, zero);
                } else {
#pragma unroll
                    for (int l = 0; l < W; l += 4) __stcs(reinterpret_cast<float4*>(p + l), make_float4(0, 0, 0, 0));
                }
            } else {
#pragma unroll
                for (int l = 0; l < W; ++l)
                    if (l * (int)blockDim.x < left) p[l * (int)blockDim.x] = 0.0f;
            }
        }
        return;
    }
    const unsigned me = blockIdx.x - fill, i0 = me * a.block, n = min(a.block, a.n - i0);
    const unsigned none = (unsigned)a.vocab;
    for (unsigned i = threadIdx.x; i < n + 2; i += blockDim.x) {
        const unsigned t = i0 + i - 1;  // wraps to a large number before the first
        key[i] = t < a.n ? a.key[a.passes & 1][t] : none;
        if (i >= 1 && i <= n) {
            const unsigned p = a.pos[a.passes & 1][t];
            row[i - 1] = static_cast<const T*>(a.act) + p / a.n_inner * a.a_so + p % a.n_inner * a.a_si;
        }
    }
    __syncthreads();
    if (left <= 0) return;
    float acc[W];
#pragma unroll
    for (int l = 0; l < W; ++l) acc[l] = 0.0f;
    bool crossed = key[0] == key[1];  // the run began in an earlier block
    for (unsigned b = 0; b < n && key[b + 1] != none; b += kSumBatch) {
        Piece<T, VEC> x[kSumBatch];
#pragma unroll
        for (int k = 0; k < kSumBatch; ++k)
            if (b + k < n && key[b + k + 1] != none) x[k].load(row[b + k] + col, left);
#pragma unroll
        for (int k = 0; k < kSumBatch; ++k) {
            if (b + k >= n) continue;
            const unsigned here = key[b + k + 1], next = key[b + k + 2];
            if (here == none) continue;
            x[k].add_to(acc);
            const bool last = b + k + 1 == n;
            if (next == here && !last) continue;
            // the run ends, or the block does
            float* dst;
            if (crossed) {
                dst = a.head + me * a.pitch + col;
            } else if (next == here) {
                dst = a.tail + me * a.pitch + col;
            } else {
                dst = a.table + here * a.stride + col;
#pragma unroll
                for (int l = 0; l < W; ++l) acc[l] *= a.scale;
                if (a.accumulate) {
#pragma unroll
                    for (int l = 0; l < W; ++l) {
                        const int j = VEC ? l : l * (int)blockDim.x;
                        if (VEC || j < left) acc[l] += dst[j];
                    }
                }
            }
            if constexpr (VEC) {
                // every place by its own address: the table's rows, and the parts in the workspace, need only
                // start on 16 bytes
                const bool wide = W == 8 && aligned32(dst);
                if constexpr (W == 8) {
                    if (wide) store_eight(dst, acc);
                }
#pragma unroll
                for (int l = 0; l < W && !wide; l += 4)
                    *reinterpret_cast<float4*>(dst + l) = make_float4(acc[l], acc[l + 1], acc[l + 2], acc[l + 3]);
            } else {
#pragma unroll
                for (int l = 0; l < W; ++l)
                    if (l * (int)blockDim.x < left) dst[l * (int)blockDim.x] = acc[l];
            }
#pragma unroll
            for (int l = 0; l < W; ++l) acc[l] = 0.0f;
            crossed = false;
        }
    }
}

// A CTA takes a run and a slab of columns; four warps share its parts, and the warps' sums are
// added in warp order.
constexpr int kJoinWarps = 4;
constexpr int kJoinGrid = 148;
constexpr int kJoinColumns = 128;  // four a lane
__global__ void __launch_bounds__(32 * kJoinWarps) join_kernel(const __grid_constant__ EmbedGradArgs a) {
    __shared__ float4 part[kJoinWarps][32];
    dependent_launch_prologue();
    const unsigned runs = a.counts[0];
    SpanRun run = a.runs[blockIdx.x];  // not after the count is known (there is room for a run a block)
    const unsigned lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long col = (long long)blockIdx.y * kJoinColumns + 4 * lane;  // the parts' pitch is a multiple of four
    for (unsigned r = blockIdx.x; r < runs; r += gridDim.x) {
        if (r != blockIdx.x) run = a.runs[r];
        float4 s = make_float4(0, 0, 0, 0);
        if (col < a.dim) {
#pragma unroll 4
            for (unsigned b = run.first + warp; b <= run.last; b += kJoinWarps) {
                const float4 x = *reinterpret_cast<const float4*>((b == run.first ? a.tail : a.head) + b * a.pitch + col);
                s.x += x.x;
                s.y += x.y;
                s.z += x.z;
                s.w += x.w;
            }
        }
        part[warp][lane] = s;
        __syncthreads();
        {  // a column a thread
            const long long c = (long long)blockIdx.y * kJoinColumns + threadIdx.x;
            const float* p = reinterpret_cast<const float*>(part);
            float t = p[threadIdx.x];
#pragma unroll
            for (int v = 1; v < kJoinWarps; ++v) t += p[v * kJoinColumns + threadIdx.x];
            t *= a.scale;
            if (c < a.dim) {
                float* dst = a.table + run.token * a.stride + c;
                *dst = a.accumulate ? *dst + t : t;
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ gradient norm and clip
// Three launches.  norm_kernel, a CTA a chunk, adds the chunk's squares and leaves one partial;
// finish_kernel, a CTA a group, adds the group's partials in chunk order and stores norm and factor
// (4 % of the whole faster than the last CTA of a group doing it, and no atomics); clip_kernel walks the
// chunks backwards, as the ones read last are still in the L2, and reads and writes past it (with
// cached reads it took 17 % longer).  A persistent grid with the next chunk on its way in registers
// took 957 us where this takes 860: eight workers' 61 M 32-bit gradients.
constexpr int kClipThreads = 256;
constexpr int kClipVectors = 8;  // a thread has in flight

struct GradChunk {
    const void* src;
    float* dst;      // place in the arena, or nullptr: in place
    unsigned n;      // elements
    unsigned short type_vec;  // type | (both places 16-byte aligned) << 8
    unsigned short group;
};
struct GradGroup {
    unsigned first_chunk, n_chunks;
    float factor;
};
struct GradArgs {
    const GradChunk* chunks;
    double* partial;  // of each chunk
    GradGroup* groups;
    float* norms;
    unsigned n_chunks;
    int n_groups;
    float max_norm;
};

__device__ __forceinline__ float clip_factor(double norm, float max_norm) {
    return norm > (double)max_norm ? (float)((double)max_norm / norm) : 1.0f;
}

__device__ __forceinline__ bool chunk_vec(const GradChunk& c) { return (c.type_vec >> 8) != 0; }

// Sum of the squares of a vector.  In 32 bits where that neither overflows nor loses small squares
// (conversions to 64 bits, one an element, would take longer than the loads); else in 64.
template <typename T>
__device__ __forceinline__ double vector_squares(const uint4& q) {
    constexpr int L = kLanes<T>;
    float x[L];
    unpack<T>(q, x);
    float s = x[0] * x[0];
#pragma unroll
    for (int l = 1; l < L; ++l) s = fmaf(x[l], x[l], s);
    // squares below 2^-100 lose bits; a vector of zeros has none to lose
    if ((s > 7.9e-31f && s < 3e38f) || (q.x | q.y | q.z | q.w) == 0) return (double)s;
    double d = 0.0;
#pragma unroll
    for (int l = 0; l < L; ++l) d = fma((double)x[l], (double)x[l], d);
    return d;
}
template <typename T>
__device__ __forceinline__ double chunk_squares(const GradChunk& c) {
    constexpr int L = kLanes<T>;
    const T* p = static_cast<const T*>(c.src);
    double s = 0.0;
    unsigned done = 0;
    if (chunk_vec(c)) {
        const unsigned nv = c.n / L;
        for (unsigned b = 0; b < nv; b += kClipVectors * kClipThreads) {
            uint4 q[kClipVectors];
#pragma unroll
            for (int k = 0; k < kClipVectors; ++k) {
                const unsigned v = b + k * kClipThreads + threadIdx.x;
                q[k] = v < nv ? reinterpret_cast<const uint4*>(p)[v] : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < kClipVectors; ++k) s += vector_squares<T>(q[k]);
        }
        done = nv * L;
    }
    for (unsigned j = done + threadIdx.x; j < c.n; j += kClipThreads) {
        const double x = to_f32(p[j]);
        s = fma(x, x, s);
    }
    return s;
}

__global__ void __launch_bounds__(kClipThreads) norm_kernel(const __grid_constant__ GradArgs a) {
    __shared__ double part[kClipThreads / 32];
    dependent_launch_prologue();
    const GradChunk c = a.chunks[blockIdx.x];
    const int type = c.type_vec & 0xff;
    double s[1];
    s[0] = type == ODSGD_F32 ? chunk_squares<float>(c) : type == ODSGD_BF16 ? chunk_squares<bf16>(c) : chunk_squares<f16>(c);
    block_sum<1, kClipThreads>(s, part);
    if (threadIdx.x == 0) a.partial[blockIdx.x] = s[0];
}

// The norm of a group from its chunks' partials, by thread 0 of a CTA.
template <int THREADS>
__device__ __forceinline__ double group_norm(const GradArgs& a, const GradGroup& g, double* smem) {
    double t[1] = {0.0};
#pragma unroll 4
    for (unsigned j = threadIdx.x; j < g.n_chunks; j += THREADS) t[0] += a.partial[g.first_chunk + j];
    block_sum<1, THREADS>(t, smem);
    return sqrt(t[0]);
}

// A CTA a group.
constexpr int kFinishThreads = 512;
__global__ void __launch_bounds__(kFinishThreads) finish_kernel(const __grid_constant__ GradArgs a) {
    __shared__ double part[kFinishThreads / 32];
    dependent_launch_prologue();
    GradGroup* g = a.groups + blockIdx.x;
    const double norm = group_norm<kFinishThreads>(a, *g, part);
    if (threadIdx.x == 0) {
        g->factor = clip_factor(norm, a.max_norm);
        if (a.norms != nullptr) a.norms[blockIdx.x] = (float)norm;
    }
}

// A chunk times f, to D: the arena's float or the tensor's own type.
template <typename T, typename D>
__device__ __forceinline__ void chunk_scale(const GradChunk& c, D* d, float f) {
    constexpr int L = kLanes<T>;
    const T* p = static_cast<const T*>(c.src);
    const bool wide = aligned32(d);
    unsigned done = 0;
    if (chunk_vec(c)) {
        const unsigned nv = c.n / L;
        for (unsigned b = 0; b < nv; b += kClipVectors * kClipThreads) {
            uint4 q[kClipVectors];
#pragma unroll
            for (int k = 0; k < kClipVectors; ++k) {
                const unsigned v = b + k * kClipThreads + threadIdx.x;
                if (v < nv) q[k] = __ldcs(reinterpret_cast<const uint4*>(p) + v);
            }
#pragma unroll
            for (int k = 0; k < kClipVectors; ++k) {
                const unsigned v = b + k * kClipThreads + threadIdx.x;
                if (v >= nv) continue;
                float x[L];
                unpack<T>(q[k], x);
#pragma unroll
                for (int l = 0; l < L; ++l) x[l] *= f;
                if constexpr (sizeof(T) == sizeof(D)) {
                    __stcs(reinterpret_cast<uint4*>(d) + v, pack<T>(x));
                } else if (wide) {
                    store_eight(d + (size_t)v * L, x);
                } else {
#pragma unroll
                    for (int l = 0; l < L; l += 4)
                        __stcs(reinterpret_cast<float4*>(d + (size_t)v * L + l), make_float4(x[l], x[l + 1], x[l + 2], x[l + 3]));
                }
            }
        }
        done = nv * L;
    }
    for (unsigned j = done + threadIdx.x; j < c.n; j += kClipThreads) d[j] = from_f32<D>(to_f32(p[j]) * f);
}

template <typename T>
__device__ __forceinline__ void scale_chunk(const GradChunk& c, float f) {
    if (c.dst != nullptr) chunk_scale<T, float>(c, c.dst, f);
    else if (f != 1.0f) chunk_scale<T, T>(c, static_cast<T*>(const_cast<void*>(c.src)), f);  // else every bit stays
}

// JOIN: each CTA adds its group's partials itself, which saves a launch where they are few.
constexpr unsigned kJoinChunks = 1024;
template <bool JOIN>
__global__ void __launch_bounds__(kClipThreads) clip_kernel(const __grid_constant__ GradArgs a) {
    __shared__ double part[kClipThreads / 32];
    __shared__ float factor;
    dependent_launch_prologue();
    const unsigned i = a.n_chunks - 1 - blockIdx.x;
    const GradChunk c = a.chunks[i];
    float f;
    if (JOIN) {
        const GradGroup g = a.groups[c.group];
        const double norm = group_norm<kClipThreads>(a, g, part);
        if (threadIdx.x == 0) {
            factor = clip_factor(norm, a.max_norm);
            if (i == g.first_chunk && a.norms != nullptr) a.norms[c.group] = (float)norm;
        }
        if (blockIdx.x == 0 && threadIdx.x < a.n_groups && a.groups[threadIdx.x].n_chunks == 0 && a.norms != nullptr)
            a.norms[threadIdx.x] = 0.0f;
        __syncthreads();
        f = factor;
    } else {
        f = a.groups[c.group].factor;
    }
    const int type = c.type_vec & 0xff;
    if (type == ODSGD_F32) scale_chunk<float>(c, f);
    else if (type == ODSGD_BF16) scale_chunk<bf16>(c, f);
    else scale_chunk<f16>(c, f);
}

}  // namespace odsgd_lm
