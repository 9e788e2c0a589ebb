// Device code of the verification of drafted tokens (sm_100a).
//
// Two launches.  The first reads every row of logits once and leaves maximum and sum of exponentials of its parts, in
// 32 bits.  The second takes a sequence by a cluster: it decides its drafts in order, and draws one token from what the target has
// beyond the draft (or, behind the last draft, from the target), for which two rows are read again in 64 bits:
// where the running sum passes a random number is a matter of its last bits.
#pragma once

#include "odsgd_lm_softmax.cuh"

namespace odsgd_lm {

constexpr int kVerifyDrafts = 255;
constexpr int kPartThreads = 256;
constexpr int kDrawThreads = 512;
constexpr int kDrawWarps = kDrawThreads / 32;
constexpr int kDrawCluster = 8;

struct VerifyArgs {
    const void* target;  // [batch][drafts + 1][vocab]
    const void* draft;   // [batch][drafts][vocab] or nullptr: each draft has all of its distribution
    const void* tokens;
    const float* uniforms;
    void* out_tokens;
    int* accepted;
    float* logp;
    MaxSum* parts;  // [rows][chunks], the target's rows first
    long long t_sb, t_sr, d_sb, d_sr, k_sb, k_sr, u_sb, u_sr;
    unsigned batch, drafts, target_rows, chunks;
    int vocab, wide_tokens, cluster;
    float inv_temp, draft_temp;  // of target and draft
    float exp_temp, draft_exp;   // the same as RowExp takes them
};

// Part `chunk` of row `row`.
template <typename T>
__global__ void __launch_bounds__(kPartThreads) parts_kernel(const __grid_constant__ VerifyArgs a) {
    __shared__ MaxSum warp_part[kPartThreads / 32];
    dependent_launch_prologue();
    const unsigned row = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const bool second = row >= a.target_rows;
    const unsigned r = second ? row - a.target_rows : row, many = second ? a.drafts : a.drafts + 1;
    const T* const z = second ? static_cast<const T*>(a.draft) + (r / many) * a.d_sb + (r % many) * a.d_sr
                              : static_cast<const T*>(a.target) + (r / many) * a.t_sb + (r % many) * a.t_sr;
    const float temp = second ? a.draft_temp : a.inv_temp, exp_temp = second ? a.draft_exp : a.exp_temp;
    const RowParts<T> parts(z, a.vocab);
    const int per = (parts.vectors + (int)a.chunks - 1) / (int)a.chunks;
    const int v0 = min((int)chunk * per, parts.vectors), n = min(per, parts.vectors - v0);
    const uint4* const v = reinterpret_cast<const uint4*>(z + parts.head) + v0;
    const int tid = (int)threadIdx.x, edge = chunk == 0 ? parts.edge(tid) : -1;
    MaxSum x = single(edge >= 0 ? to_f32(z[edge]) : -CUDART_INF_F);
    uint4 q[kRowVectors];
    for (int b = 0; b < n; b += kPartThreads * kRowVectors) {
#pragma unroll
        for (int k = 0; k < kRowVectors; ++k) q[k] = b + k * kPartThreads + tid < n ? v[b + k * kPartThreads + tid] : neg_inf_vector<T>();
        x = add_vectors<T>(x, q, temp, exp_temp);
    }
    x = warp_join(x, temp);
    if (tid % 32 == 0) warp_part[tid / 32] = x;
    __syncthreads();
    if (tid < 32) {
        x = tid < kPartThreads / 32 ? warp_part[tid] : MaxSum{-CUDART_INF_F, 0.0f};
        x = warp_join(x, temp);
        if (tid == 0) a.parts[blockIdx.x] = x;
    }
}

__device__ __forceinline__ double cluster_load_f64(uint32_t addr) {
    double x;
    asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(x) : "r"(addr) : "memory");
    return x;
}
__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}

enum Decision { kRefused, kAccepted, kNear, kEnds };

struct DrawState {
    double warp_part[2][kDrawWarps];
    double cta_part[2];  // read by the other CTAs
    unsigned char decision[kVerifyDrafts + 1];
    float logp[kVerifyDrafts + 1];
    float maxima[kVerifyDrafts + 1], draft_maxima[kVerifyDrafts + 1];
};

// 2^y in 64 bits, within 3e-14: the nearest whole number goes into the exponent, the rest, at most a half, through 1 + f r(f),
// r being the polynomial that meets (2^f - 1) / f at the nine Chebyshev points of [-1/2, 1/2].  1 at 0, 0 below 2^-1000;
// for y <= 1 or NaN.
__device__ __forceinline__ double power_of_two(double y) {
    const double whole = y + 6755399441055744.0;  // 1.5 * 2^52: the last bits are the whole number
    const double f = y - (whole - 6755399441055744.0);
    double r = 1.0203121063391729e-07;
    r = fma(r, f, 1.3255224878668817e-06);
    r = fma(r, f, 1.525268684626772e-05);
    r = fma(r, f, 0.00015403455852453838);
    r = fma(r, f, 0.0013333558179043112);
    r = fma(r, f, 0.009618129159402558);
    r = fma(r, f, 0.055504108664760424);
    r = fma(r, f, 0.2402265069581299);
    r = fma(r, f, 0.6931471805599453);
    r = fma(r, f, 1.0);
    r = __hiloint2double(__double2hiint(r) + (__double2loint(whole) << 20), __double2loint(r));
    return y < -1000.0 ? 0.0 : r;
}

// One of the target's rows and the draft's beside it, element by element in 64 bits.
template <typename T>
struct RowPair {
    const T* p;
    const T* q;     // nullptr: only `hot` has a probability
    long long hot;  // -1: no draft to take off
    double mp, mq, cp, cq;  // maxima, temperatures times log2 e
    int vocab;
    __device__ __forceinline__ static double one(float z, double m, double c) { return power_of_two(((double)z - m) * c); }
    __device__ __forceinline__ double target(int j) const { return one(to_f32(p[j]), mp, cp); }
    __device__ __forceinline__ double draft(int j) const { return one(to_f32(q[j]), mq, cq); }
    // Elements j to j + 7 of a row; -inf behind its end.
    __device__ __forceinline__ void load(const T* row, int j, float (&z)[8]) const {
        if (j + 8 <= vocab && (reinterpret_cast<uintptr_t>(row + j) & 15) == 0) {
#pragma unroll
            for (int h = 0; h < 8; h += kLanes<T>) {
                float y[kLanes<T>];
                unpack<T>(*reinterpret_cast<const uint4*>(row + j + h), y);
#pragma unroll
                for (int l = 0; l < kLanes<T>; ++l) z[h + l] = y[l];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = j + i < vocab ? to_f32(row[j + i]) : -CUDART_INF_F;
        }
    }
    __device__ __forceinline__ void target(int j, double (&e)[8]) const {
        float z[8];
        load(p, j, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = one(z[i], mp, cp);
    }
    __device__ __forceinline__ void draft(int j, double (&e)[8]) const {
        float z[8];
        load(q, j, z);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = one(z[i], mq, cq);
    }
};
__device__ __forceinline__ double sum_of(const double (&x)[8]) { return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7])); }

// Sums of two values over the cluster, in the same order in every CTA.
__device__ __forceinline__ void cluster_sums(DrawState& s, unsigned cs, double x, double y, double& all_x, double& all_y) {
    const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    x = warp_sum(x);
    y = warp_sum(y);
    if (lane == 0) s.warp_part[0][warp] = x, s.warp_part[1][warp] = y;
    __syncthreads();
    if (threadIdx.x == 0) {
        double sx = 0.0, sy = 0.0;
        for (int w = 0; w < kDrawWarps; ++w) sx += s.warp_part[0][w], sy += s.warp_part[1][w];
        s.cta_part[0] = sx, s.cta_part[1] = sy;
    }
    if (cs > 1) cluster_sync();
    else __syncthreads();
    all_x = all_y = 0.0;
    for (unsigned c = 0; c < cs; ++c) {
        all_x += cs > 1 ? cluster_load_f64(cluster_address(&s.cta_part[0], c)) : s.cta_part[0];
        all_y += cs > 1 ? cluster_load_f64(cluster_address(&s.cta_part[1], c)) : s.cta_part[1];
    }
    if (cs > 1) cluster_sync();  // (before the parts are written again)
    else __syncthreads();
}

__device__ __forceinline__ void store_token(const VerifyArgs& a, unsigned seq, unsigned i, long long t) {
    const size_t at = (size_t)seq * (a.drafts + 1) + i;
    if (a.wide_tokens) static_cast<long long*>(a.out_tokens)[at] = t;
    else static_cast<int*>(a.out_tokens)[at] = (int)t;
}

template <typename T>
__global__ void __launch_bounds__(kDrawThreads) draw_kernel(const __grid_constant__ VerifyArgs a) {
    __shared__ DrawState s;
    dependent_launch_prologue();
    const unsigned cs = (unsigned)a.cluster, seq = blockIdx.x / cs, rank = blockIdx.x % cs;
    const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const T* const target = static_cast<const T*>(a.target) + seq * a.t_sb;
    const T* const draft = a.draft ? static_cast<const T*>(a.draft) + seq * a.d_sb : nullptr;
    const float* const u = a.uniforms + seq * a.u_sb;
    const auto token = [&](unsigned i) { return load_token(a.tokens, a.wide_tokens != 0, seq * a.k_sb + i * a.k_sr); };
    const auto known = [&](long long t) { return t >= 0 && t < a.vocab; };

    // Every CTA decides every draft by the rows' sums in 32 bits; those next to the border are left open.
    for (unsigned i = warp; i <= a.drafts; i += kDrawWarps) {
        const auto row_sum = [&](const MaxSum* parts, float c) {
            MaxSum x = {-CUDART_INF_F, 0.0f};
            for (unsigned k = lane; k < a.chunks; k += 32) x = join(x, parts[k], c);
            return warp_join(x, c);
        };
        const MaxSum t = row_sum(a.parts + (size_t)(seq * (a.drafts + 1) + i) * a.chunks, a.inv_temp);
        MaxSum d = {0.0f, 1.0f};
        if (draft && i < a.drafts) d = row_sum(a.parts + (size_t)(a.target_rows + seq * a.drafts + i) * a.chunks, a.draft_temp);
        if (lane == 0) {
            s.maxima[i] = t.m;
            s.draft_maxima[i] = d.m;
            const long long x = i < a.drafts ? token(i) : -1;
            int what = kEnds;
            if (known(x)) {
                const float lp = (to_f32(target[i * a.t_sr + x]) - t.m) * a.inv_temp - logf(t.s);
                const float lq = draft ? (to_f32(draft[i * a.d_sr + x]) - d.m) * a.draft_temp - logf(d.s) : 0.0f;
                const float over = lp - lq - logf(u[i * a.u_sr]);
                s.logp[i] = lp;
                // 32 bits leave `over` uncertain by some 1e-6; infinities and NaN are left to the exact comparison too
                what = over > 1e-4f + 4e-6f * (fabsf(lp) + fabsf(lq)) ? kAccepted : over < -1e-4f - 4e-6f * (fabsf(lp) + fabsf(lq)) ? kRefused : kNear;
            }
            s.decision[i] = (unsigned char)what;
        }
    }
    __syncthreads();

    // this warp's part of the vocabulary: whole steps of eight elements a lane
    const int per_warp = ((a.vocab + (int)(cs * kDrawWarps) - 1) / (int)(cs * kDrawWarps) + 255) / 256 * 256;
    const int lo = (int)min((long long)a.vocab, (long long)(rank * kDrawWarps + warp) * per_warp), hi = min(a.vocab, lo + per_warp);
    const int own = lo + 8 * (int)lane;

    // The first draft that is not accepted; the sums of its two rows in 64 bits.
    RowPair<T> row;
    double sum_p = 0.0, sum_q = 0.0;
    unsigned n = 0;
    bool refused = false;
    for (;; ++n) {
        while (s.decision[n] == kAccepted) ++n;  // (behind the last draft it is kEnds)
        const bool ends = s.decision[n] == kEnds;
        const long long x = ends ? -1 : token(n);
        row = RowPair<T>{target + n * a.t_sr, draft && !ends ? draft + n * a.d_sr : nullptr, x, s.maxima[n], s.draft_maxima[n],
                         a.inv_temp * 1.4426950408889634, a.draft_temp * 1.4426950408889634, a.vocab};
        double p = 0.0, q = 0.0;
        for (int j = own; j < hi; j += 256) {
            double e[8];
            row.target(j, e);
            p += sum_of(e);
            if (row.q) {
                row.draft(j, e);
                q += sum_of(e);
            }
        }
        cluster_sums(s, cs, p, q, sum_p, sum_q);
        if (ends) break;
        refused = !((double)u[n * a.u_sr] * (row.q ? row.draft((int)x) / sum_q : 1.0) < row.target((int)x) / sum_p);
        if (refused) break;
    }

    // What is left of the target (times sum_p), and its sum in every warp's part.
    const double ratio = row.q ? sum_p / sum_q : 0.0;
    const auto left = [&](int j, double (&e)[8]) {
        row.target(j, e);
        if (!refused) return;
        if (row.q) {
            double f[8];
            row.draft(j, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double r = fma(-ratio, f[i], e[i]);
                e[i] = r < 0.0 ? 0.0 : r;  // (NaN stays)
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = j + i == row.hot ? 0.0 : e[i];
        }
    };
    double all = 0.0;
    for (;;) {
        double mine = 0.0, none;
        for (int j = own; j < hi; j += 256) {
            double e[8];
            left(j, e);
            mine += sum_of(e);
        }
        cluster_sums(s, cs, mine, 0.0, all, none);
        if (!refused || all != 0.0) break;
        refused = false;  // nothing is left (a draft that neither gives a probability): the whole target
    }
    const bool drawn = all > 0.0 && all < CUDART_INF;  // not where a row holds NaN, +inf or nothing but -inf
    const double bound = (double)u[a.drafts * a.u_sr] * all;

    // The CTA, and in it the warp, in whose part the running sum passes the bound: the last that begins no higher, of
    // those that have anything.
    const auto last_begin = [&](unsigned many, double before, auto part, double& begin) {
        int at = -1;
        for (unsigned i = 0; i < many; ++i) {
            const double x = part(i);
            if (x > 0.0 && (at < 0 || before <= bound)) at = (int)i, begin = before;
            before += x;
        }
        return at;
    };
    double begin = 0.0;
    const int cta = last_begin(cs, 0.0, [&](unsigned c) { return cs > 1 ? cluster_load_f64(cluster_address(&s.cta_part[0], c)) : s.cta_part[0]; }, begin);
    if (drawn && cta == (int)rank) {
        const int at = last_begin(kDrawWarps, begin, [&](unsigned w) { return s.warp_part[0][w]; }, begin);
        if (at == (int)warp) {
            int found = -1, last = -1;
            for (int j0 = lo; j0 < hi && found < 0; j0 += 256) {
                const int j = j0 + 8 * (int)lane;
                double e[8] = {};
                if (j < hi) left(j, e);
#pragma unroll
                for (int i = 1; i < 8; ++i) e[i] += e[i - 1];
                double run = e[7];
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const double t = __shfl_up_sync(~0u, run, d);
                    if ((int)lane >= d) run += t;
                }
                double before = __shfl_up_sync(~0u, run, 1);
                before = begin + (lane == 0 ? 0.0 : before);
                int at_over = 8, at_last = -1;
#pragma unroll
                for (int i = 7; i >= 0; --i) {
                    const bool some = e[i] > (i > 0 ? e[i - 1] : 0.0);
                    if (some && before + e[i] > bound) at_over = i;
                    if (some && at_last < 0) at_last = i;
                }
                const unsigned over = __ballot_sync(~0u, at_over < 8), some = __ballot_sync(~0u, at_last >= 0);
                if (over != 0) {
                    const int l = __ffs((int)over) - 1;
                    found = j0 + 8 * l + __shfl_sync(~0u, at_over, l);
                }
                if (some != 0) {
                    const int l = 31 - __clz((int)some);
                    last = j0 + 8 * l + __shfl_sync(~0u, at_last, l);
                }
                begin += __shfl_sync(~0u, run, 31);
            }
            if (found < 0) found = last;  // (the bound is the whole sum, but for a rounding)
            if (lane == 0) {
                store_token(a, seq, n, found);
                a.logp[(size_t)seq * (a.drafts + 1) + n] = (float)(((double)to_f32(row.p[found]) - row.mp) * a.inv_temp - log(sum_p));
            }
        }
    }
    if (rank == 0) {
        if (threadIdx.x == 0) a.accepted[seq] = (int)n;
        for (unsigned i = threadIdx.x; i <= a.drafts; i += kDrawThreads) {
            if (i == n && drawn) continue;
            store_token(a, seq, i, i < n ? token(i) : -1);
            a.logp[(size_t)seq * (a.drafts + 1) + i] = i < n ? s.logp[i] : i > n ? 0.0f : CUDART_NAN_F;
        }
    }
    if (cs > 1) cluster_sync();  // the others have read this CTA's sums
}

}  // namespace odsgd_lm
