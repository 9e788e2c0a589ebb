// Device code of the verification of drafted tokens (sm_100a).
//
// Two launches.  The first reads every row of logits once and leaves maximum and sum of exponentials of its parts, in
// 32 bits.  The second takes a sequence by a cluster: it decides its drafts in order, and draws one token from what the target has
// beyond the draft (or, behind the last draft, from the target), for which two rows are read again in 64 bits:
// where the running sum passes a random number is a matter of its last bits.
#pragma once

#include <limits.h>

#include "odsgd_lm_softmax.cuh"

namespace odsgd_lm {

constexpr int kVerifyDrafts = 255;
constexpr int kPartThreads = 256;
constexpr int kDrawWarps = 16;  // most of a CTA that draws
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

__device__ __forceinline__ void cluster_store_f64(uint32_t addr, double x) {
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(x) : "memory");
}
__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}

enum Decision { kRefused, kAccepted, kNear, kEnds };

constexpr int kDrawSums = 5;
struct DrawState {
    double warp_part[kDrawSums][kDrawWarps];
    double cta_part[2][kDrawSums][kDrawCluster];  // of every CTA, written by it; two sets in turn
    unsigned char decision[kVerifyDrafts + 1];
    float logp[kVerifyDrafts + 1];
    int found, last;
    float maxima[kVerifyDrafts + 1], draft_maxima[kVerifyDrafts + 1], sums[kVerifyDrafts + 1], draft_sums[kVerifyDrafts + 1];
};

// 2^(d c) in 64 bits, within 4e-14: the nearest whole number goes into the exponent, the rest f, at most a half, through 1 + f r(f),
// r being the polynomial that meets (2^f - 1) / f at the nine Chebyshev points of [-1/2, 1/2].  1 at 0, 0 below 2^-1000 and
// at -inf; for d c <= 1 or NaN.
__device__ __forceinline__ double power_of_two(double d, double c) {
    const double w = fma(d, c, 6755399441055744.0);  // 1.5 * 2^52: the lower half is the whole number
    const double f = fma(d, c, 6755399441055744.0 - w);
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
    // (a number below -2^31 leaves another upper half)
    const bool none = __double2hiint(w) < 0x4337ffff || __double2loint(w) < -1000;
    return __hiloint2double(none ? 0 : __double2hiint(r) + (__double2loint(w) << 20), none ? 0 : __double2loint(r));
}

// One of the target's rows and the draft's beside it, element by element in 64 bits.
template <typename T>
struct RowPair {
    const T* p;
    const T* q;     // nullptr: only `hot` has a probability
    long long hot;  // -1: no draft to take off
    double mp, mq, cp, cq;  // maxima, temperatures times log2 e
    int vocab;
    __device__ __forceinline__ double target(int j) const { return power_of_two((double)to_f32(p[j]) - mp, cp); }
    __device__ __forceinline__ double draft(int j) const { return power_of_two((double)to_f32(q[j]) - mq, cq); }
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
    __device__ __forceinline__ void target(const float (&z)[8], double (&e)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = power_of_two((double)z[i] - mp, cp);
    }
    __device__ __forceinline__ void draft(const float (&z)[8], double (&e)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = power_of_two((double)z[i] - mq, cq);
    }
    // f(j, logits of the target, of the draft) for each eight from `from` on, a warp's width apart; the next are loaded ahead.
    template <typename F>
    __device__ __forceinline__ void each(int from, int hi, F f) const {
        float z[8], y[8] = {}, next_z[8], next_y[8] = {};
        if (from < hi) {
            load(p, from, z);
            if (q) load(q, from, y);
        }
#pragma unroll 1
        for (int j = from; j < hi; j += 256) {
            if (j + 256 < hi) {
                load(p, j + 256, next_z);
                if (q) load(q, j + 256, next_y);
            }
            f(j, z, y);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = next_z[i], y[i] = next_y[i];
        }
    }
};
__device__ __forceinline__ double sum_of(const double (&x)[8]) { return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7])); }

// Sums over the cluster, in the same order in every CTA; set `turn` of the parts holds those of the CTAs
// afterwards, warp_part those of this CTA's warps.  Turns alternate: who writes a set again has been through the
// barrier of the other, and with it everybody who reads it.
template <int WARPS>
__device__ __forceinline__ void cluster_sums(DrawState& s, unsigned cs, unsigned rank, unsigned turn, double (&x)[kDrawSums]) {
    const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 0; k < kDrawSums; ++k) {
        x[k] = warp_sum(x[k]);
        if (lane == 0) s.warp_part[k][warp] = x[k];
    }
    __syncthreads();
    if (warp < kDrawSums) {
        const double sum = warp_sum(lane < WARPS ? s.warp_part[warp][lane] : 0.0);
        if (lane < cs) cluster_store_f64(cluster_address(&s.cta_part[turn][warp][rank], lane), sum);
    }
    if (cs > 1) cluster_sync();
    else __syncthreads();
#pragma unroll
    for (int k = 0; k < kDrawSums; ++k) {
        x[k] = 0.0;
        for (unsigned c = 0; c < cs; ++c) x[k] += s.cta_part[turn][k][c];
    }
}

__device__ __forceinline__ void store_token(const VerifyArgs& a, unsigned seq, unsigned i, long long t) {
    const size_t at = (size_t)seq * (a.drafts + 1) + i;
    if (a.wide_tokens) static_cast<long long*>(a.out_tokens)[at] = t;
    else static_cast<int*>(a.out_tokens)[at] = (int)t;
}

template <typename T, int WARPS>
__global__ void __launch_bounds__(WARPS * 32) draw_kernel(const __grid_constant__ VerifyArgs a) {
    __shared__ DrawState s;
    dependent_launch_prologue();
    const unsigned cs = (unsigned)a.cluster, seq = blockIdx.x / cs, rank = blockIdx.x % cs;
    const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const T* const target = static_cast<const T*>(a.target) + seq * a.t_sb;
    const T* const draft = a.draft ? static_cast<const T*>(a.draft) + seq * a.d_sb : nullptr;
    const float* const u = a.uniforms + seq * a.u_sb;
    const auto token = [&](unsigned i) { return load_token(a.tokens, a.wide_tokens != 0, seq * a.k_sb + i * a.k_sr); };
    const auto known = [&](long long t) { return t >= 0 && t < a.vocab; };
    if (cs > 1) cluster_arrive();  // this CTA runs: its shared memory may be written (waited for below)

    // Every CTA decides every draft by the rows' sums in 32 bits; those next to the border are left open.
    for (unsigned i = warp; i <= a.drafts; i += WARPS) {
        const long long x = i < a.drafts ? token(i) : -1;
        const float zt = known(x) ? to_f32(target[i * a.t_sr + x]) : 0.0f;
        const float zd = known(x) && draft ? to_f32(draft[i * a.d_sr + x]) : 0.0f;
        const float random = u[i * a.u_sr];
        const auto row_sum = [&](const MaxSum* parts, float c) {
            MaxSum v = {-CUDART_INF_F, 0.0f};
            for (unsigned k = lane; k < a.chunks; k += 32) v = join(v, parts[k], c);
            return warp_join(v, c);
        };
        const MaxSum t = row_sum(a.parts + (size_t)(seq * (a.drafts + 1) + i) * a.chunks, a.inv_temp);
        MaxSum d = {0.0f, 1.0f};
        if (draft && i < a.drafts) d = row_sum(a.parts + (size_t)(a.target_rows + seq * a.drafts + i) * a.chunks, a.draft_temp);
        if (lane == 0) {
            s.maxima[i] = t.m;
            s.draft_maxima[i] = d.m;
            s.sums[i] = t.s;
            s.draft_sums[i] = d.s;
            int what = kEnds;
            if (known(x)) {
                const float lp = (zt - t.m) * a.inv_temp - logf(t.s);
                const float lq = draft ? (zd - d.m) * a.draft_temp - logf(d.s) : 0.0f;
                const float over = lp - lq - logf(random);
                s.logp[i] = lp;
                // 32 bits leave `over` uncertain by some 1e-6; infinities and NaN are left to the exact comparison too
                const float margin = 1e-4f + 4e-6f * (fabsf(lp) + fabsf(lq));
                what = over > margin ? kAccepted : over < -margin ? kRefused : kNear;
            }
            s.decision[i] = (unsigned char)what;
        }
    }
    if (threadIdx.x == 0) s.found = INT_MAX, s.last = -1;
    if (cs > 1) cluster_wait();
    __syncthreads();

    // this warp's part of the vocabulary: whole steps of eight elements a lane
    const int per_warp = ((a.vocab + (int)(cs * WARPS) - 1) / (int)(cs * WARPS) + 255) / 256 * 256;
    const int lo = (int)min((long long)a.vocab, (long long)(rank * WARPS + warp) * per_warp), hi = min(a.vocab, lo + per_warp);
    const int own = lo + 8 * (int)lane;

    // The first draft that is not accepted.  One pass over its two rows gives, in 64 bits, the sums P and Q of the target's
    // and the draft's exponentials (relative to their maxima), and with a ratio k near P / Q, for the target
    // beyond the draft (times P),
    //     R = sum of max(0, p - k q)    D = sum of q where p > k q    N = sum of p where p is within 2^-18 of k q
    // The ratio comes from the sums in 32 bits, some 1e-7 off.  With the right one, P / Q, R is R - (P / Q - k) D, but for the
    // elements that change sides, which N bounds: where it does not bound them well enough (distributions that are equal on much
    // of their mass) the pass is made again with the right ratio.
    RowPair<T> row;
    double x[kDrawSums];  // P, Q, R, D, N
    double ratio = 0.0, off = 0.0;
    unsigned n = 0, turn = 0;
    bool refused = false;
    for (bool again = false;; turn ^= 1) {
        if (!again)
            while (s.decision[n] == kAccepted) ++n;  // (behind the last draft it is kEnds)
        const bool ends = s.decision[n] == kEnds;
        const long long t = ends ? -1 : token(n);
        row = RowPair<T>{target + n * a.t_sr, draft && !ends ? draft + n * a.d_sr : nullptr, t, s.maxima[n], s.draft_maxima[n],
                         a.inv_temp * 1.4426950408889634, a.draft_temp * 1.4426950408889634, a.vocab};
        if (row.q && !again) ratio = (double)s.sums[n] / (double)s.draft_sums[n];
#pragma unroll
        for (int k = 0; k < kDrawSums; ++k) x[k] = 0.0;
        row.each(own, hi, [&](int j, const float (&z)[8], const float (&y)[8]) {
            double e[8];
            row.target(z, e);
            x[0] += sum_of(e);
            if (row.q) {
                double f[8];
                row.draft(y, f);
                x[1] += sum_of(f);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const double r = fma(-ratio, f[i], e[i]);
                    const int high = __double2hiint(r), whole = __double2hiint(e[i]);
                    if ((high & 0x7fffffff) < whole - (18 << 20)) x[4] += e[i];
                    e[i] = high < 0 && r == r ? 0.0 : r;  // (NaN stays)
                    f[i] = high < 0 ? 0.0 : f[i];
                }
                x[2] += sum_of(e);
                x[3] += sum_of(f);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) e[i] = j + i == row.hot ? 0.0 : e[i];
                x[2] += sum_of(e);
            }
        });
        cluster_sums<WARPS>(s, cs, rank, turn, x);
        if (ends) break;
        if (!again) {
            refused = s.decision[n] == kRefused ||
                      !((double)u[n * a.u_sr] * (row.q ? row.draft((int)t) / x[1] : 1.0) < row.target((int)t) / x[0]);
            if (!refused) {
                ++n;
                continue;
            }
        }
        if (!row.q) break;
        off = x[0] / x[1] - ratio;
        // (what is not finite is not mended by another pass)
        if (again || !(fabs(off) > 0x1p-19 * ratio || x[4] * fabs(off) > 1e-11 * ratio * x[2])) break;
        ratio += off;
        again = true;
    }
    // Where nothing is left (a draft that neither gives a probability, equal distributions): the whole target.
    double all = x[2] - off * x[3];
    if (refused && !(all > 0.0) && all == all) refused = false;
    if (!refused) all = x[0], row.q = nullptr, row.hot = -1;
    ratio += off;
    const auto part_left = [&](double p, double r, double d) { return refused ? fmax(0.0, r - off * d) : p; };
    const auto left = [&](int j, const float (&z)[8], const float (&y)[8], double (&e)[8]) {
        row.target(z, e);
        if (row.q) {
            double f[8];
            row.draft(y, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = fmax(0.0, fma(-ratio, f[i], e[i]));
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = j + i == row.hot ? 0.0 : e[i];
        }
    };
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
    const int cta = last_begin(cs, 0.0, [&](unsigned c) { return part_left(s.cta_part[turn][0][c], s.cta_part[turn][2][c], s.cta_part[turn][3][c]); }, begin);
    if (drawn && cta == (int)rank) {
        const int at = last_begin(WARPS, begin, [&](unsigned w) { return part_left(s.warp_part[0][w], s.warp_part[2][w], s.warp_part[3][w]); }, begin);
        // its part again, 256 elements a warp, all warps of the CTA together
        const int from = min(a.vocab, (int)(rank * WARPS + at) * per_warp), to = min(a.vocab, from + per_warp);
        for (int j0 = from; j0 < to; j0 += 256 * WARPS) {
            const int j = j0 + 256 * (int)warp + 8 * (int)lane;
            double e[8] = {};
            if (j < to) {
                float z[8], y[8] = {};
                row.load(row.p, j, z);
                if (row.q) row.load(row.q, j, y);
                left(j, z, y, e);
            }
#pragma unroll
            for (int i = 1; i < 8; ++i) e[i] += e[i - 1];
            double run = e[7];
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const double v = __shfl_up_sync(~0u, run, d);
                if ((int)lane >= d) run += v;
            }
            double before = __shfl_up_sync(~0u, run, 1);
            if (lane == 0) before = 0.0;
            __syncthreads();  // (the parts of before have been read)
            if (lane == 31) s.warp_part[0][warp] = run;
            __syncthreads();
            for (int w = 0; w < WARPS; ++w) {
                if (w == (int)warp) before += begin;
                begin += s.warp_part[0][w];
            }
            int over = INT_MAX, some = -1;
#pragma unroll
            for (int i = 7; i >= 0; --i) {
                const bool any = e[i] > (i > 0 ? e[i - 1] : 0.0);
                if (any && before + e[i] > bound) over = j + i;
                if (any && some < 0) some = j + i;
            }
            over = __reduce_min_sync(~0u, over);
            some = __reduce_max_sync(~0u, some);
            if (lane == 0 && over != INT_MAX) atomicMin(&s.found, over);
            if (lane == 0 && some >= 0) atomicMax(&s.last, some);
            __syncthreads();
            if (s.found != INT_MAX) break;
        }
        if (threadIdx.x == 0) {
            const int found = s.found != INT_MAX ? s.found : s.last;  // (the bound is the whole sum, but for a rounding)
            store_token(a, seq, n, found);
            a.logp[(size_t)seq * (a.drafts + 1) + n] = (float)(((double)to_f32(row.p[found]) - row.mp) * a.inv_temp - log(x[0]));
        }
    }
    if (rank == 0) {
        if (threadIdx.x == 0) a.accepted[seq] = (int)n;
        for (unsigned i = threadIdx.x; i <= a.drafts; i += WARPS * 32) {
            if (i == n && drawn) continue;
            store_token(a, seq, i, i < n ? token(i) : -1);
            a.logp[(size_t)seq * (a.drafts + 1) + i] = i < n ? s.logp[i] : i > n ? 0.0f : CUDART_NAN_F;
        }
    }
}

}  // namespace odsgd_lm
