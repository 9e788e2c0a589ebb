// Device code of the verification of drafted tokens (sm_100a).
//
// Three launches, or, for small vocabularies, the last alone.  parts_kernel reads every row of logits once and leaves maximum and sum of exponentials of its parts, in 32
// bits.  pass_kernel decides a sequence's drafts in order by those, and goes over the two rows of the first that is not
// accepted again, in 64 bits: where the running sum of what is left passes a random number is a matter of its last bits.
// draw_kernel finds that place.
#pragma once

#include <limits.h>

#include "odsgd_lm_softmax.cuh"

namespace odsgd_lm {

constexpr int kVerifyDrafts = 255;
constexpr int kPartThreads = 128;
constexpr int kPartCtas = 12;  // an SM
constexpr int kPassWarps = 8;     // of a CTA of pass_kernel
constexpr int kDrawThreads = 512;  // of draw_kernel
constexpr int kDrawWarps = kDrawThreads / 32;
constexpr int kSegments = kDrawThreads;  // most parts of the vocabulary, each summed by a warp
constexpr int kDrawSums = 5;
constexpr float kHeld = -600.0f;           // log-probabilities above this are no matter of the range of 64 bits

constexpr double kLeast = -1020.0;         // the exponent below which an element is nothing

enum Decision { kRefused, kAccepted, kNear, kEnds };

// Place i of a sequence, by the rows' sums in 32 bits.
struct Position {
    float max, sum, draft_max, draft_sum;
    float logp;  // of the draft under the target
    int decision;
    int token;   // the draft; -1 where decision is kEnds
};

struct VerifyArgs {
    const void* target;  // [batch][drafts + 1][vocab]
    const void* draft;   // [batch][drafts][vocab] or nullptr: each draft has all of its distribution
    const void* tokens;
    const float* uniforms;
    void* out_tokens;
    int* accepted;
    float* logp;
    MaxSum* parts;        // [rows][chunks], the target's rows first
    Position* positions;  // [batch][drafts + 1]
    double* sums;         // [batch][kDrawSums][segments]
    long long t_sb, t_sr, d_sb, d_sr, k_sb, k_sr, u_sb, u_sr;
    unsigned batch, drafts, target_rows, chunks;
    int vocab, wide_tokens;
    int segments, segment;  // how many, and elements of each (a multiple of 256)
    int pass_ctas;          // of a sequence
    float inv_temp, draft_temp;  // of target and draft
    float exp_temp, draft_exp;   // the same as RowExp takes them
    double least, draft_least;   // kLeast in logits: kLeast / (temperature times log2 e)
};

// What THREADS threads, of which this is `tid`, find in part `chunk` of a row, each its own share.
template <typename T, int THREADS>
__device__ __forceinline__ MaxSum part_of_row(const T* z, int vocab, unsigned chunk, unsigned chunks, int tid, float temp, float exp_temp) {
    const RowParts<T> parts(z, vocab);
    const int per = (parts.vectors + (int)chunks - 1) / (int)chunks;
    const int v0 = min((int)chunk * per, parts.vectors), n = min(per, parts.vectors - v0);
    const uint4* const v = reinterpret_cast<const uint4*>(z + parts.head) + v0;
    const int edge = chunk == 0 ? parts.edge(tid) : -1;
    MaxSum x = single(edge >= 0 ? to_f32(z[edge]) : -CUDART_INF_F);
    uint4 q[kRowVectors];
    for (int b = 0; b < n; b += THREADS * kRowVectors) {
#pragma unroll
        for (int k = 0; k < kRowVectors; ++k) q[k] = b + k * THREADS + tid < n ? v[b + k * THREADS + tid] : neg_inf_vector<T>();
        x = add_vectors<T>(x, q, temp, exp_temp);
    }
    return x;
}

// Part `chunk` of row `row`.  Bound by memory traffic, as the scores are: small CTAs, twelve an SM, and three times as many
// parts as run at once (48 x 15 rows of 131072 bf16: 37 us in 256-thread CTAs of a row each, 30 so; the copy rate for
// their bytes is 29).
template <typename T>
__global__ void __launch_bounds__(kPartThreads, kPartCtas) parts_kernel(const __grid_constant__ VerifyArgs a) {
    __shared__ MaxSum warp_part[kPartThreads / 32];
    dependent_launch_prologue();
    const unsigned row = blockIdx.x / a.chunks, chunk = blockIdx.x % a.chunks;
    const bool second = row >= a.target_rows;
    const unsigned r = second ? row - a.target_rows : row, many = second ? a.drafts : a.drafts + 1;
    const T* const z = second ? static_cast<const T*>(a.draft) + (r / many) * a.d_sb + (r % many) * a.d_sr
                              : static_cast<const T*>(a.target) + (r / many) * a.t_sb + (r % many) * a.t_sr;
    const float temp = second ? a.draft_temp : a.inv_temp, exp_temp = second ? a.draft_exp : a.exp_temp;
    const int tid = (int)threadIdx.x;
    MaxSum x = part_of_row<T, kPartThreads>(z, a.vocab, chunk, a.chunks, tid, temp, exp_temp);
    x = warp_join(x, temp);
    if (tid % 32 == 0) warp_part[tid / 32] = x;
    __syncthreads();
    if (tid < 32) {
        x = tid < kPartThreads / 32 ? warp_part[tid] : MaxSum{-CUDART_INF_F, 0.0f};
        x = warp_join(x, temp);
        if (tid == 0) a.parts[blockIdx.x] = x;
    }
}

__device__ __forceinline__ double warp_sum(double x) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(~0u, x, d);
    return x;
}

// 2^(d c) in 64 bits, within 4e-14: the nearest whole number goes into the exponent, the rest f, at most a half, through 1 + f r(f),
// r being the polynomial that meets (2^f - 1) / f at the nine Chebyshev points of [-1/2, 1/2].  1 at 0; for kLeast <= d c <= 0.
// What is lower counts as nothing (is_nothing): a mask, or at that size no matter to any sum.
__device__ __forceinline__ bool is_nothing(double d, double c) { return d * c < kLeast; }
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
    return __hiloint2double(__double2hiint(r) + (__double2loint(w) << 20), __double2loint(r));
}

// One of the target's rows and the draft's beside it, element by element in 64 bits.
template <typename T>
struct RowPair {
    const T* p;
    const T* q;     // nullptr: only `hot` has a probability
    long long hot;  // -1: no draft to take off
    double mp, mq, cp, cq;  // maxima, temperatures times log2 e
    int vocab;
    float low_p, low_q;     // no element above these is nothing
    __device__ __forceinline__ static double one(float z, double m, double c) {
        const double d = (double)z - m;
        return is_nothing(d, c) ? 0.0 : power_of_two(d, c);
    }
    __device__ __forceinline__ double target(int j) const { return one(to_f32(p[j]), mp, cp); }
    __device__ __forceinline__ double draft(int j) const { return one(to_f32(q[j]), mq, cq); }
    // Elements j to j + 7 of a row, as the 16-byte words that hold them: loaded ahead, taken apart when they are needed.  No word
    // is read that has none of them.
    static constexpr int kWords = 8 * (int)sizeof(T) / 16 + 1;
    struct Raw {
        uint4 w[kWords];
    };
    __device__ __forceinline__ Raw fetch(const T* row, int j) const {
        const uintptr_t at = reinterpret_cast<uintptr_t>(row + j), from = at & ~(uintptr_t)15, end = reinterpret_cast<uintptr_t>(row + min(j + 8, vocab));
        Raw out;
#pragma unroll
        for (int k = 0; k < kWords; ++k) out.w[k] = from + 16 * k < end ? reinterpret_cast<const uint4*>(from)[k] : make_uint4(0, 0, 0, 0);
        return out;
    }
    // -inf behind the row's end
    __device__ __forceinline__ void take(const Raw& raw, const T* row, int j, float (&z)[8]) const {
        uint32_t x[4 * kWords];
#pragma unroll
        for (int k = 0; k < kWords; ++k) x[4 * k] = raw.w[k].x, x[4 * k + 1] = raw.w[k].y, x[4 * k + 2] = raw.w[k].z, x[4 * k + 3] = raw.w[k].w;
        const unsigned shift = (unsigned)(reinterpret_cast<uintptr_t>(row + j) & 15);  // the same for all of a row
        if (shift != 0) {
#pragma unroll
            for (int i = 0; i + 2 < 4 * kWords; ++i) x[i] = shift & 8 ? x[i + 2] : x[i];
#pragma unroll
            for (int i = 0; i + 1 < 4 * kWords; ++i) x[i] = shift & 4 ? x[i + 1] : x[i];
            if (sizeof(T) == 2) {
#pragma unroll
                for (int i = 0; i + 1 < 4 * kWords; ++i) x[i] = shift & 2 ? __funnelshift_r(x[i], x[i + 1], 16) : x[i];
            }
        }
#pragma unroll
        for (int h = 0; h < 8; h += kLanes<T>) {
            float y[kLanes<T>];
            const int k = h / kLanes<T> * 4;
            unpack<T>(make_uint4(x[k], x[k + 1], x[k + 2], x[k + 3]), y);
#pragma unroll
            for (int l = 0; l < kLanes<T>; ++l) z[h + l] = y[l];
        }
        if (j + 8 > vocab) {
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = j + i < vocab ? z[i] : -CUDART_INF_F;
        }
    }
    __device__ __forceinline__ void load(const T* row, int j, float (&z)[8]) const { take(fetch(row, j), row, j, z); }
    // Eight at a time; only where one may be nothing they are looked at one by one (asked of each it takes three instructions more,
    // 48 x 7 drafts at 131072: 73 us in all, 68 so).
    __device__ __forceinline__ static void eight(const float (&z)[8], double m, double c, float low, double (&e)[8]) {
        float least = z[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) least = fminf(least, z[i]);
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = power_of_two((double)z[i] - m, c);
        if (least <= low) {
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = is_nothing((double)z[i] - m, c) ? 0.0 : e[i];
        }
    }
    __device__ __forceinline__ void target(const float (&z)[8], double (&e)[8]) const { eight(z, mp, cp, low_p, e); }
    __device__ __forceinline__ void draft(const float (&z)[8], double (&e)[8]) const { eight(z, mq, cq, low_q, e); }
    // f(j, logits of the target, of the draft) for each eight from `from` on, a warp's width apart; the next are loaded ahead.
    template <typename F>
    __device__ __forceinline__ void each(int from, int hi, F f) const {
        Raw next_p = {}, next_q = {};
        if (from < hi) {
            next_p = fetch(p, from);
            if (q) next_q = fetch(q, from);
        }
#pragma unroll 1
        for (int j = from; j < hi; j += 256) {
            const Raw now_p = next_p, now_q = next_q;
            if (j + 256 < hi) {
                next_p = fetch(p, j + 256);
                if (q) next_q = fetch(q, j + 256);
            }
            float z[8], y[8] = {};
            take(now_p, p, j, z);
            if (q) take(now_q, q, j, y);
            f(j, z, y);
        }
    }
};
__device__ __forceinline__ double sum_of(const double (&x)[8]) { return ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7])); }

// A sequence's inputs.
template <typename T>
struct Sequence {
    const T* target;
    const T* draft;
    const float* u;
    const VerifyArgs& a;
    unsigned seq;
    __device__ __forceinline__ Sequence(const VerifyArgs& a_, unsigned seq_)
        : target(static_cast<const T*>(a_.target) + seq_ * a_.t_sb),
          draft(a_.draft ? static_cast<const T*>(a_.draft) + seq_ * a_.d_sb : nullptr),
          u(a_.uniforms + seq_ * a_.u_sb),
          a(a_),
          seq(seq_) {}
    __device__ __forceinline__ long long token(unsigned i) const { return load_token(a.tokens, a.wide_tokens != 0, seq * a.k_sb + i * a.k_sr); }
    // Place i, by a warp; `target_sum` and `draft_sum` give the sums of its rows to every lane.
    template <typename F, typename G>
    __device__ __forceinline__ Position decide(unsigned i, F target_sum, G draft_sum) const {
        const long long x = i < a.drafts ? token(i) : -1;
        const bool known = x >= 0 && x < a.vocab;
        const float zt = known ? to_f32(target[i * a.t_sr + x]) : 0.0f;
        const float zd = known && draft ? to_f32(draft[i * a.d_sr + x]) : 0.0f;
        const float random = u[i * a.u_sr];
        const MaxSum t = target_sum();
        MaxSum d = {0.0f, 1.0f};
        if (draft && i < a.drafts) d = draft_sum();
        Position p = {t.m, t.s, d.m, d.s, 0.0f, kEnds, -1};
        if (known) {
            p.token = (int)x;
            p.logp = (zt - t.m) * a.inv_temp - logf(t.s);
            const float lq = draft ? (zd - d.m) * a.draft_temp - logf(d.s) : 0.0f;
            const float over = p.logp - lq - logf(random);
            // 32 bits leave `over` uncertain by some 1e-6; infinities and NaN are left to the exact comparison too, and so is a draft to
            // which the target may give nothing that 64 bits hold (a masked token at u = 0, or masked in both rows)
            const float margin = 1e-4f + 4e-6f * (fabsf(p.logp) + fabsf(lq));
            p.decision = over > margin && p.logp > kHeld ? kAccepted : over < -margin ? kRefused : kNear;
        }
        return p;
    }
    // (rounded up, so that all above is above kLeast, however large the logits and the temperature are)
    __device__ __forceinline__ static float low(double m, double least) { return __double2float_ru(m + least); }
    __device__ __forceinline__ RowPair<T> row(unsigned n, const Position& p) const {
        const double cp = a.inv_temp * 1.4426950408889634, cq = a.draft_temp * 1.4426950408889634;
        return RowPair<T>{target + n * a.t_sr, draft && p.token >= 0 ? draft + n * a.d_sr : nullptr, p.token, p.max, p.draft_max, cp, cq, a.vocab,
                          low(p.max, a.least), low(p.draft_max, a.draft_least)};
    }
};
// A row that holds NaN or +inf has a sum that is NaN, one of nothing but -inf a sum of 0.
__device__ __forceinline__ bool is_void(const Position& p) { return !(p.sum > 0.0f && p.draft_sum > 0.0f); }
__device__ __forceinline__ double ratio_of(const Position& p) { return (double)p.sum / (double)p.draft_sum; }

// One pass over the two rows of a place gives, in 64 bits, the sums P and Q of the target's and the draft's exponentials
// (relative to their maxima), and with a ratio k near P / Q, for the target beyond the draft (times P),
//     R = sum of max(0, p - k q)    D = sum of q where p > k q    N = sum of p where p is within 2^-18 of k q
// The ratio comes from the sums in 32 bits, some 1e-7 off.  With the right one, P / Q, R is R - (P / Q - k) D, but for the
// elements that change sides, which N bounds: where it does not bound them well enough (distributions that are equal on much
// of their mass) the pass is made again with the right ratio.  So two exponentials an element are the rule, not four.
// Here: of one segment, by a warp.
template <typename T>
__device__ __forceinline__ void pass_segment(const RowPair<T>& row, double ratio, int lo, int hi, double (&x)[kDrawSums]) {
#pragma unroll
    for (int k = 0; k < kDrawSums; ++k) x[k] = 0.0;
    row.each(lo + 8 * (int)(threadIdx.x & 31), hi, [&](int j, const float (&z)[8], const float (&y)[8]) {
        double e[8];
        row.target(z, e);
        x[0] += sum_of(e);
        if (row.q) {
            double f[8], r[8];
            row.draft(y, f);
            x[1] += sum_of(f);
            int near = 0;  // the least of the exponents of |p - k q| less those of p
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                r[i] = fma(-ratio, f[i], e[i]);
                near = min(near, (__double2hiint(r[i]) & 0x7fffffff) - __double2hiint(e[i]));
            }
            if (near < -(18 << 20)) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if ((__double2hiint(r[i]) & 0x7fffffff) < __double2hiint(e[i]) - (18 << 20)) x[4] += e[i];
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {  // (rows with NaN do not count: is_void)
                const bool less = __double2hiint(r[i]) < 0;
                e[i] = less ? 0.0 : r[i];
                f[i] = less ? 0.0 : f[i];
            }
            x[2] += sum_of(e);
            x[3] += sum_of(f);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) e[i] = j + i == row.hot ? 0.0 : e[i];
            x[2] += sum_of(e);
        }
    });
#pragma unroll
    for (int k = 0; k < kDrawSums; ++k) x[k] = warp_sum(x[k]);
}

template <typename T>
__global__ void __launch_bounds__(kPassWarps * 32) pass_kernel(const __grid_constant__ VerifyArgs a) {
    __shared__ Position place[kVerifyDrafts + 1];
    dependent_launch_prologue();
    const unsigned seq = blockIdx.x / a.pass_ctas, rank = blockIdx.x % a.pass_ctas;
    const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const Sequence<T> in(a, seq);
    // Every CTA decides every draft by the rows' sums in 32 bits; those next to the border are left open.
    for (unsigned i = warp; i <= a.drafts; i += kPassWarps) {
        const auto row_sum = [&](const MaxSum* parts, float c) {
            MaxSum v = {-CUDART_INF_F, 0.0f};
            for (unsigned k = lane; k < a.chunks; k += 32) v = join(v, parts[k], c);
            return warp_join(v, c);
        };
        const Position p = in.decide(i, [&] { return row_sum(a.parts + (size_t)(seq * (a.drafts + 1) + i) * a.chunks, a.inv_temp); },
                                     [&] { return row_sum(a.parts + (size_t)(a.target_rows + seq * a.drafts + i) * a.chunks, a.draft_temp); });
        if (lane == 0) {
            place[i] = p;
            if (rank == 0) a.positions[(size_t)seq * (a.drafts + 1) + i] = p;
        }
    }
    __syncthreads();
    unsigned n = 0;
    while (place[n].decision == kAccepted) ++n;  // (behind the last draft it is kEnds)
    const RowPair<T> row = in.row(n, place[n]);
    const double ratio = ratio_of(place[n]);
    double* const sums = a.sums + (size_t)seq * kDrawSums * a.segments;
    for (int g = (int)(rank * kPassWarps + warp); g < a.segments; g += a.pass_ctas * kPassWarps) {
        double x[kDrawSums];
        pass_segment(row, ratio, g * a.segment, min(a.vocab, (g + 1) * a.segment), x);
#pragma unroll
        for (int k = 0; k < kDrawSums; ++k)
            if ((int)lane == k) sums[k * a.segments + g] = x[k];
    }
}

__device__ __forceinline__ void store_token(const VerifyArgs& a, unsigned seq, unsigned i, long long t) {
    const size_t at = (size_t)seq * (a.drafts + 1) + i;
    if (a.wide_tokens) static_cast<long long*>(a.out_tokens)[at] = t;
    else static_cast<int*>(a.out_tokens)[at] = (int)t;
}

struct DrawState {
    Position place[kVerifyDrafts + 1];
    double warp_part[kDrawSums][kDrawWarps];
    double segment[kDrawSums][kSegments];  // written again where the pass has to be repeated here
    int found, last, at;
    double begin;
};

// The token at which the running sum of what is left passes `bound`, to every thread: first the segment, by the sums `part` of
// its thread's, then the element.  Sums and elements come out of different roundings, so that a segment that is next to nothing
// can turn out to hold none; the whole row is then gone over.  -1 where that has nothing either.
template <typename T>
__device__ __forceinline__ int find_place(const RowPair<T>& row, double ratio, double part, double bound, int segment, DrawState& s) {
    const unsigned warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int mine = (int)threadIdx.x;
    // The segment in which the running sum passes the bound: the last that begins no higher, of those that have anything.
    double run = part;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const double v = __shfl_up_sync(~0u, run, d);
        if ((int)lane >= d) run += v;
    }
    __syncthreads();
    if (lane == 31) s.warp_part[0][warp] = run;
    if (threadIdx.x == 0) s.found = INT_MAX, s.last = -1, s.at = -1;
    __syncthreads();
    double begin = warp_sum(lane < warp ? s.warp_part[0][lane] : 0.0);
    const double before = __shfl_up_sync(~0u, run, 1);
    if (lane > 0) begin += before;
    // (a bound that is NaN or below 0 takes the first that has anything)
    const int candidate = __reduce_max_sync(~0u, part > 0.0 && begin <= bound ? mine : -1);
    const unsigned some_part = __ballot_sync(~0u, part > 0.0);
    if (lane == 0 && candidate >= 0) atomicMax(&s.at, candidate);
    if (lane == 0 && some_part != 0) atomicMin(&s.found, (int)warp * 32 + __ffs((int)some_part) - 1);
    __syncthreads();
    const int at = s.at >= 0 ? s.at : s.found;
    if (mine == at) s.begin = begin;
    __syncthreads();
    begin = s.begin;
    if (threadIdx.x == 0) s.found = INT_MAX;
    int from = 0, to = row.vocab;
    if (at != INT_MAX) from = at * segment, to = min(row.vocab, from + segment);
    else begin = 0.0;
    for (;;) {  // twice at most
        // its elements again, 256 a warp
        for (int j0 = from; j0 < to; j0 += 256 * kDrawWarps) {
            const int j = j0 + 256 * (int)warp + 8 * (int)lane;
            double e[8] = {};
            if (j < to) {
                float z[8];
                row.load(row.p, j, z);
                row.target(z, e);
                if (row.q) {
                    double f[8];
                    row.load(row.q, j, z);
                    row.draft(z, f);
#pragma unroll
                    for (int i = 0; i < 8; ++i) e[i] = fmax(0.0, fma(-ratio, f[i], e[i]));
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) e[i] = j + i == row.hot ? 0.0 : e[i];
                }
            }
#pragma unroll
            for (int i = 1; i < 8; ++i) e[i] += e[i - 1];
            run = e[7];
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) {
                const double v = __shfl_up_sync(~0u, run, d);
                if ((int)lane >= d) run += v;
            }
            __syncthreads();  // (the sums of before have been read)
            if (lane == 31) s.warp_part[0][warp] = run;
            __syncthreads();
            double ahead = begin + warp_sum(lane < warp ? s.warp_part[0][lane] : 0.0);
            begin += warp_sum(lane < kDrawWarps ? s.warp_part[0][lane] : 0.0);
            const double lower = __shfl_up_sync(~0u, run, 1);
            if (lane > 0) ahead += lower;
            int over = INT_MAX, some = -1;
#pragma unroll
            for (int i = 7; i >= 0; --i) {
                const bool any = e[i] > (i > 0 ? e[i - 1] : 0.0);
                if (any && ahead + e[i] > bound) over = j + i;
                if (any && some < 0) some = j + i;
            }
            over = __reduce_min_sync(~0u, over);
            some = __reduce_max_sync(~0u, some);
            if (lane == 0 && over != INT_MAX) atomicMin(&s.found, over);
            if (lane == 0 && some >= 0) atomicMax(&s.last, some);
            __syncthreads();
            if (s.found != INT_MAX) break;
        }
        if (s.last >= 0 || (from == 0 && to == row.vocab)) break;
        from = 0, to = row.vocab, begin = 0.0;
    }
    return s.found != INT_MAX ? s.found : s.last;  // (the bound is the whole sum, but for a rounding)
}

// A CTA a sequence, a thread a segment.  ALONE: the CTA also does what the other kernels do ahead of it, a warp a row and a
// segment.  That pays up to some 2000 tokens: 8 x 3 drafts, bf16, of 200 / 2000 / 4000 take 11.3 / 12.3 / 15.4 us so, 13.8 / 14.3 / 14.3
// by three launches, which cost the host 5 us more.
template <typename T, bool ALONE>
__global__ void __launch_bounds__(kDrawThreads) draw_kernel(const __grid_constant__ VerifyArgs a) {
    __shared__ DrawState s;
    dependent_launch_prologue();
    const unsigned seq = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int mine = (int)threadIdx.x;
    const Sequence<T> in(a, seq);
    const double last_random = (double)in.u[a.drafts * a.u_sr];
    double x[kDrawSums];  // of the thread's segment, then P, Q, R, D, N
    if constexpr (ALONE) {
        for (unsigned i = warp; i <= a.drafts; i += kDrawWarps) {
            const auto row_sum = [&](const T* z, float c, float exp_temp) { return warp_join(part_of_row<T, 32>(z, a.vocab, 0, 1, (int)lane, c, exp_temp), c); };
            const Position p = in.decide(i, [&] { return row_sum(in.target + i * a.t_sr, a.inv_temp, a.exp_temp); },
                                         [&] { return row_sum(in.draft + i * a.d_sr, a.draft_temp, a.draft_exp); });
            if (lane == 0) s.place[i] = p;
        }
    } else {
#pragma unroll
        for (int k = 0; k < kDrawSums; ++k) x[k] = mine < a.segments ? a.sums[((size_t)seq * kDrawSums + k) * a.segments + mine] : 0.0;
        if (threadIdx.x <= a.drafts) s.place[threadIdx.x] = a.positions[(size_t)seq * (a.drafts + 1) + threadIdx.x];
    }
    __syncthreads();
    unsigned n = 0;
    while (s.place[n].decision == kAccepted) ++n;
    RowPair<T> row = in.row(n, s.place[n]);
    double ratio = ratio_of(s.place[n]), off = 0.0, part_p, part_r, part_d;
    bool refused = false;
    for (bool again = false, here = ALONE;; here = true) {
        if (here) {  // the pass over this place, by this CTA: not behind pass_kernel, but for the rare cases below
            __syncthreads();
            for (int g = (int)warp; g < a.segments; g += kDrawWarps) {
                pass_segment(row, ratio, g * a.segment, min(a.vocab, (g + 1) * a.segment), x);
#pragma unroll
                for (int k = 0; k < kDrawSums; ++k)
                    if ((int)lane == k) s.segment[k][g] = x[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < kDrawSums; ++k) x[k] = mine < a.segments ? s.segment[k][mine] : 0.0;
        }
        part_p = x[0], part_r = x[2], part_d = x[3];
#pragma unroll
        for (int k = 0; k < kDrawSums; ++k) {
            x[k] = warp_sum(x[k]);
            if (lane == 0) s.warp_part[k][warp] = x[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kDrawSums; ++k) x[k] = warp_sum(lane < kDrawWarps ? s.warp_part[k][lane] : 0.0);
        if (s.place[n].decision == kEnds || is_void(s.place[n])) break;
        bool next = false;
        if (!again) {
            const int t = (int)row.hot;
            refused = s.place[n].decision == kRefused || !((double)in.u[n * a.u_sr] * (row.q ? row.draft(t) / x[1] : 1.0) < row.target(t) / x[0]);
            next = !refused;
        }
        if (!next) {
            if (!row.q) break;
            off = x[0] / x[1] - ratio;
            // (what is not finite is not mended by another pass)
            if (again || !(fabs(off) > 0x1p-19 * ratio || x[4] * fabs(off) > 1e-11 * ratio * x[2])) break;
            ratio += off;
            again = true;
        } else {
            do ++n;
            while (s.place[n].decision == kAccepted);
            row = in.row(n, s.place[n]);
            ratio = ratio_of(s.place[n]);
        }
    }
    // Where nothing is left (a draft that neither gives a probability, equal distributions, by the sums or by the elements): the
    // whole target.
    ratio += off;
    if (refused && x[2] - off * x[3] <= 0.0) refused = false;
    if (threadIdx.x == 0) a.accepted[seq] = (int)n;
    for (unsigned i = threadIdx.x; i <= a.drafts; i += kDrawThreads) {
        if (i == n) continue;
        store_token(a, seq, i, i < n ? s.place[i].token : -1);
        a.logp[(size_t)seq * (a.drafts + 1) + i] = i < n ? s.place[i].logp : 0.0f;
    }
    int found = -1;
    while (!is_void(s.place[n])) {  // twice at most
        if (!refused) row.q = nullptr, row.hot = -1;
        const double all = refused ? x[2] - off * x[3] : x[0];
        found = find_place(row, ratio, refused ? fmax(0.0, part_r - off * part_d) : part_p, last_random * all, a.segment, s);
        if (found >= 0 || !refused) break;
        refused = false;
    }
    if (threadIdx.x == 0) {
        store_token(a, seq, n, found);
        a.logp[(size_t)seq * (a.drafts + 1) + n] =
            found >= 0 ? (float)(((double)to_f32(row.p[found]) - row.mp) * a.inv_temp - log(x[0])) : CUDART_NAN_F;
    }
}

}  // namespace odsgd_lm
