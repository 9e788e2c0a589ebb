// Host side of the language-model operators around the update: checks of arguments, choice of
// launch shapes, launches.  No allocation (but for the table of a gradient set), no
// synchronisation, nothing thrown across the boundary.
#include <cuda_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <new>
#include <string>
#include <vector>

#include "odsgd.h"
#include "odsgd_lm_kernels.cuh"

using namespace odsgd_lm;

namespace odsgd {
void set_thread_error(const std::string& msg);  // text of odsgd_last_error(NULL)
}

namespace {

using wide = __int128;

int fail(int code, const std::string& msg) {
    odsgd::set_thread_error(msg);
    return code;
}

// Nothing may be thrown across the C boundary.  What the bodies can throw is that host memory has run out (a set's
// tables, an error text).
template <typename F>
int guarded(F body) noexcept {
    try {
        return body();
    } catch (...) {
        try {
            return fail(ODSGD_ERR_ARG, "out of host memory");
        } catch (...) {
            return ODSGD_ERR_ARG;  // not even for the text
        }
    }
}

int size_of(int type) {
    switch (type) {
        case ODSGD_F32: return 4;
        case ODSGD_BF16: return 2;
        case ODSGD_F16: return 2;
        case ODSGD_I32: return 4;
        case ODSGD_I64: return 8;
        default: return 0;
    }
}
bool is_float_type(int t) { return t == ODSGD_F32 || t == ODSGD_BF16 || t == ODSGD_F16; }
bool is_token_type(int t) { return t == ODSGD_I32 || t == ODSGD_I64; }

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// One buffer of a call: [n_outer][n_inner] rows of `len` elements.
struct Buf {
    const char* name;
    const void* p;
    int elem;
    int64_t so, si, len;
    bool written;
};

struct Range {
    uintptr_t lo, hi;
};

bool range_of(const Buf& b, int64_t n_outer, int64_t n_inner, Range* r) {
    const wide n = ((wide)(n_outer - 1) * b.so + (wide)(n_inner - 1) * b.si + b.len) * b.elem;
    const wide end = (wide) reinterpret_cast<uintptr_t>(b.p) + n;
    if (n > ((wide)1 << 62) || end > (wide)UINTPTR_MAX) return false;
    *r = Range{reinterpret_cast<uintptr_t>(b.p), (uintptr_t)end};
    return true;
}

// Pointers, alignments, strides, and that nothing written overlaps anything else of the call.
// `same_ok`: index of a written buffer that may be exactly the buffer 0 (gradient in place).
int check_buffers(const Buf* bufs, int n, int64_t n_outer, int64_t n_inner, int same_ok) {
    Range r[16];
    for (int i = 0; i < n; ++i) {
        const Buf& b = bufs[i];
        if (b.so < 0 || b.si < 0) return fail(ODSGD_ERR_ARG, std::string(b.name) + ": negative stride");
        if (n_outer == 0 || n_inner == 0) continue;
        if (!b.p) return fail(ODSGD_ERR_ARG, std::string(b.name) + " is NULL");
        if (reinterpret_cast<uintptr_t>(b.p) % b.elem != 0)
            return fail(ODSGD_ERR_ALIGN, std::string(b.name) + " is not aligned to its element type");
        if (!range_of(b, n_outer, n_inner, &r[i])) return fail(ODSGD_ERR_UNSUPPORTED, std::string(b.name) + " is beyond the address range");
        if (b.written) {
            const wide so = b.so, si = b.si, len = b.len;
            const bool nested = (n_inner == 1 || si >= len) && (n_outer == 1 || so >= (n_inner - 1) * si + len);
            const bool swapped = (n_outer == 1 || so >= len) && (n_inner == 1 || si >= (n_outer - 1) * so + len);
            if (!nested && !swapped) return fail(ODSGD_ERR_OVERLAP, std::string(b.name) + ": its rows overlap one another");
        }
    }
    if (n_outer == 0 || n_inner == 0) return ODSGD_OK;
    for (int i = 0; i < n; ++i) {
        for (int j = 0; j < n; ++j) {
            if (i == j || !bufs[i].written || (bufs[j].written && j < i)) continue;
            if (i == same_ok && j == 0 && bufs[i].p == bufs[0].p && (n_outer == 1 || bufs[i].so == bufs[0].so) &&
                (n_inner == 1 || bufs[i].si == bufs[0].si))
                continue;
            if (r[i].lo < r[j].hi && r[j].lo < r[i].hi)
                return fail(ODSGD_ERR_OVERLAP, std::string(bufs[i].name) + " overlaps " + bufs[j].name);
        }
    }
    return ODSGD_OK;
}

// A written buffer of `bytes` bytes without rows (sums, workspace) against the others of a call.
int check_outside(const char* name, const void* p, size_t bytes, const Buf* bufs, int n, int64_t n_outer, int64_t n_inner) {
    if (n_outer == 0 || n_inner == 0) return ODSGD_OK;
    const uintptr_t lo = reinterpret_cast<uintptr_t>(p);
    for (int i = 0; i < n; ++i) {
        Range r;
        if (range_of(bufs[i], n_outer, n_inner, &r) && lo < r.hi && r.lo < lo + bytes)
            return fail(ODSGD_ERR_OVERLAP, std::string(name) + " overlaps " + bufs[i].name);
    }
    return ODSGD_OK;
}

int check_workspace(const void* ws, size_t have, size_t need) {
    if (!ws) return fail(ODSGD_ERR_ARG, "workspace is NULL");
    if (!aligned16(ws)) return fail(ODSGD_ERR_ALIGN, "workspace is not 16-byte aligned");
    if (have < need) return fail(ODSGD_ERR_ARG, "workspace has " + std::to_string(have) + " bytes, " + std::to_string(need) + " are needed");
    return ODSGD_OK;
}

int cuda_fail(const char* what, cudaError_t e) {
    cudaGetLastError();
    return fail(ODSGD_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

// One launch on `st`, allowed to be scheduled while the kernel ahead of it drains.
template <typename Args>
int launch(const char* what, void (*kernel)(const Args), dim3 grid, dim3 block, size_t smem, int cluster, void* st, const Args& a) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(st);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, a);
    return e == cudaSuccess ? ODSGD_OK : cuda_fail(what, e);
}

constexpr int kMaxDevices = 64;

int current_device(int* dev) {
    const cudaError_t e = cudaGetDevice(dev);
    if (e != cudaSuccess) return cuda_fail("cudaGetDevice", e);
    return ODSGD_OK;
}

int sm_count(int* out) {
    static std::atomic<int> known[kMaxDevices] = {};
    int dev = 0;
    const int rc = current_device(&dev);
    if (rc != ODSGD_OK) return rc;
    int n = dev < kMaxDevices ? known[dev].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        const cudaError_t e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return cuda_fail("cudaDeviceGetAttribute", e);
        if (dev < kMaxDevices) known[dev].store(n, std::memory_order_relaxed);
    }
    *out = n;
    return ODSGD_OK;
}

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ------------------------------------------------------------------ embedding
constexpr int64_t kMaxDim = 1 << 20;  // column slabs of every kernel stay below the grid's limit in y

// The lookup writes act, the gradient writes the table.
int check_embed(const odsgd_embed_desc* d, bool lookup, const void* ws = nullptr, size_t ws_bytes = 0) {
    if (!d) return fail(ODSGD_ERR_ARG, "desc is NULL");
    if (!is_token_type(d->token_type)) return fail(ODSGD_ERR_ARG, "token_type must be ODSGD_I32 or ODSGD_I64");
    if (!is_float_type(d->act_type)) return fail(ODSGD_ERR_ARG, "act_type must be ODSGD_F32, ODSGD_BF16 or ODSGD_F16");
    if (!is_float_type(d->table_type)) return fail(ODSGD_ERR_ARG, "table_type must be ODSGD_F32, ODSGD_BF16 or ODSGD_F16");
    if (!lookup && d->table_type != ODSGD_F32) return fail(ODSGD_ERR_ARG, "the gradient's table must be ODSGD_F32");
    if (d->n_outer < 0 || d->n_inner < 0) return fail(ODSGD_ERR_ARG, "n_outer / n_inner is negative");
    if ((wide)d->n_outer * d->n_inner > ODSGD_MAX_TOKENS)
        return fail(ODSGD_ERR_UNSUPPORTED, "more than ODSGD_MAX_TOKENS tokens in one call");
    if (d->vocab < 1 || d->dim < 1) return fail(ODSGD_ERR_ARG, "vocab and dim must be at least 1");
    if (d->vocab >= INT32_MAX || d->dim > kMaxDim) return fail(ODSGD_ERR_UNSUPPORTED, "vocab or dim beyond the limits");
    if (d->table_stride < d->dim) return fail(ODSGD_ERR_ARG, "table_stride is smaller than dim");
    if (!std::isfinite(d->scale)) return fail(ODSGD_ERR_ARG, "scale is not finite");
    if (!d->table) return fail(ODSGD_ERR_ARG, "table is NULL");
    if (reinterpret_cast<uintptr_t>(d->table) % size_of(d->table_type) != 0)
        return fail(ODSGD_ERR_ALIGN, "table is not aligned to its element type");
    const Buf bufs[2] = {
        {"act", d->act, size_of(d->act_type), d->act_stride_outer, d->act_stride_inner, d->dim, lookup},
        {"tokens", d->tokens, size_of(d->token_type), d->token_stride_outer, d->token_stride_inner, 1, false},
    };
    const int rc = check_buffers(bufs, 2, d->n_outer, d->n_inner, -1);
    if (rc != ODSGD_OK) return rc;
    const Buf table = {"table", d->table, size_of(d->table_type), 0, d->table_stride, d->dim, !lookup};
    Range t, r;
    if (!range_of(table, 1, d->vocab, &t)) return fail(ODSGD_ERR_UNSUPPORTED, "table is beyond the address range");
    if (ws) {
        int rc_ws = check_outside("workspace", ws, ws_bytes, &table, 1, 1, d->vocab);
        if (rc_ws == ODSGD_OK) rc_ws = check_outside("workspace", ws, ws_bytes, bufs, 2, d->n_outer, d->n_inner);
        if (rc_ws != ODSGD_OK) return rc_ws;
    }
    if (d->n_outer == 0 || d->n_inner == 0) return ODSGD_OK;
    for (int i = 0; i < 2; ++i) {
        if (lookup && i == 1) continue;  // two inputs
        range_of(bufs[i], d->n_outer, d->n_inner, &r);
        if (r.lo < t.hi && t.lo < r.hi) return fail(ODSGD_ERR_OVERLAP, std::string("table overlaps ") + bufs[i].name);
    }
    return ODSGD_OK;
}

// Whether all rows of a strided buffer start on 16 bytes.
bool rows_aligned(const void* p, int elem, int64_t so, int64_t si, int64_t n_outer, int64_t n_inner) {
    return aligned16(p) && (n_outer <= 1 || so * elem % 16 == 0) && (n_inner <= 1 || si * elem % 16 == 0);
}

template <typename TT, typename TA>
int launch_lookup(LookupArgs a, bool vec_ok, void* stream) {
    const bool vec = vec_ok && a.dim % kLookupColumns<TT, TA, true> == 0;
    const int64_t cols = ceil_div(a.dim, vec ? kLookupColumns<TT, TA, true> : kLookupColumns<TT, TA, false>);
    // as many threads along the row as it has pieces, the rest along the rows
    const int slabs = (int)ceil_div(cols, kLookupThreads);
    const int bx = (int)ceil_div(ceil_div(cols, slabs), 32) * 32;
    const int by = std::max(1, kLookupThreads / bx);
    // eight rows a thread where that still gives every SM several CTAs, down to one where it does not
    a.per = 8;
    while (a.per > 1 && ceil_div(a.rows, (int64_t)by * a.per) * slabs < 148 * 8) a.per /= 2;
    const dim3 grid((unsigned)ceil_div(a.rows, (int64_t)by * a.per), (unsigned)slabs);
    const dim3 block((unsigned)bx, (unsigned)by);
    return vec ? launch("lookup kernel", lookup_kernel<TT, TA, true>, grid, block, 0, 1, stream, a)
               : launch("lookup kernel", lookup_kernel<TT, TA, false>, grid, block, 0, 1, stream, a);
}

template <typename TT>
int launch_lookup_t(const LookupArgs& a, int act_type, bool vec, void* stream) {
    switch (act_type) {
        case ODSGD_F32: return launch_lookup<TT, float>(a, vec, stream);
        case ODSGD_BF16: return launch_lookup<TT, bf16>(a, vec, stream);
        default: return launch_lookup<TT, f16>(a, vec, stream);
    }
}

// Launch shape and workspace of the embedding gradient: functions of sizes and types alone.
struct GradShape {
    unsigned n, blocks, block;
    int64_t pitch;
    int bits, passes;
    size_t at_key[2], at_pos[2], at_counts, at_named, at_runs, at_head, at_tail, bytes;
};

GradShape grad_shape(const odsgd_embed_desc* d) {
    GradShape s = {};
    s.n = (unsigned)(d->n_outer * d->n_inner);
    int need = 1;
    while (((int64_t)1 << need) <= d->vocab) ++need;  // keys 0 .. vocab
    s.passes = (need + kSortBits - 1) / kSortBits;
    s.bits = (need + s.passes - 1) / s.passes;
    // positions of a block: enough CTAs to fill the machine several times over before blocks grow
    const int64_t slabs = ceil_div(d->dim, (int64_t)kSumThreads * (16 / size_of(d->act_type)));
    s.block = 16;
    while (s.block < (unsigned)kSumMaxBlock && (int64_t)(s.n / s.block) * slabs > 148 * 16) s.block *= 2;
    s.blocks = (unsigned)ceil_div(s.n, s.block);
    s.pitch = ceil_div(d->dim, 8) * 8;
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    for (int i = 0; i < 2; ++i) {
        s.at_key[i] = take(4 * (size_t)s.n);
        s.at_pos[i] = take(4 * (size_t)s.n);
    }
    s.at_counts = take(8);
    s.at_named = take((size_t)ceil_div(d->vocab, 32) * 4);
    s.at_runs = take(sizeof(SpanRun) * (size_t)s.blocks);
    s.at_head = take(4 * (size_t)s.blocks * s.pitch);
    s.at_tail = take(4 * (size_t)s.blocks * s.pitch);
    s.bytes = at;
    return s;
}

template <typename T>
int launch_sum(const EmbedGradArgs& a, const GradShape& s, bool vec_ok, void* stream) {
    const bool vec = vec_ok && a.dim % kLanes<T> == 0;
    const int64_t cols = ceil_div(a.dim, vec ? Piece<T, true>::W : Piece<T, false>::W);
    const int64_t slabs = ceil_div(cols, kSumThreads);
    const unsigned threads = (unsigned)(ceil_div(ceil_div(cols, slabs), 32) * 32);
    const dim3 grid(s.blocks + a.fills, (unsigned)slabs);
    return vec ? launch("embedding gradient kernel", sum_kernel<T, true>, grid, dim3(threads), 0, 1, stream, a)
               : launch("embedding gradient kernel", sum_kernel<T, false>, grid, dim3(threads), 0, 1, stream, a);
}

int allow_sort_smem() {
    static std::atomic<bool> done[kMaxDevices] = {};
    int dev = 0;
    const int rc = current_device(&dev);
    if (rc != ODSGD_OK) return rc;
    if (dev < kMaxDevices && done[dev].load(std::memory_order_relaxed)) return ODSGD_OK;
    cudaError_t e = cudaSuccess;
    for (auto kernel : {sort_kernel<false, 2>, sort_kernel<true, 1>, sort_kernel<true, 2>})
        if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSortSmem);
    if (e != cudaSuccess) return cuda_fail("cudaFuncSetAttribute", e);
    if (dev < kMaxDevices) done[dev].store(true, std::memory_order_relaxed);
    return ODSGD_OK;
}

// ------------------------------------------------------------------ rows of logits
int check_policy(const odsgd_policy_desc* d, bool loss, const void* ws = nullptr, size_t ws_bytes = 0) {
    if (!d) return fail(ODSGD_ERR_ARG, "desc is NULL");
    if (!is_float_type(d->type)) return fail(ODSGD_ERR_ARG, "type must be ODSGD_F32, ODSGD_BF16 or ODSGD_F16");
    if (!is_token_type(d->label_type)) return fail(ODSGD_ERR_ARG, "label_type must be ODSGD_I32 or ODSGD_I64");
    if (d->n_outer < 0 || d->n_inner < 0) return fail(ODSGD_ERR_ARG, "n_outer / n_inner is negative");
    if ((wide)d->n_outer * d->n_inner >= (1 << 27)) return fail(ODSGD_ERR_UNSUPPORTED, "too many rows in one call");
    if (d->vocab < 1) return fail(ODSGD_ERR_ARG, "vocab must be at least 1");
    if (d->vocab > (1 << 30)) return fail(ODSGD_ERR_UNSUPPORTED, "vocab beyond 2^30");
    if (!(d->inv_temp > 0.0f) || !std::isfinite(d->inv_temp)) return fail(ODSGD_ERR_ARG, "inv_temp must be positive and finite");
    const int es = size_of(d->type);
    const int64_t ni = d->n_inner;
    Buf bufs[12];
    int n = 0, same_ok = -1;
    bufs[n++] = {"logits", d->logits, es, d->logits_stride_outer, d->logits_stride_inner, d->vocab, false};
    bufs[n++] = {"labels", d->labels, size_of(d->label_type), d->label_stride_outer, d->label_stride_inner, 1, false};
    bufs[n++] = {"logp", d->logp, 4, ni, 1, 1, true};
    if (!loss) {
        if (d->lse) bufs[n++] = {"lse", d->lse, 4, ni, 1, 1, true};
        return check_buffers(bufs, n, d->n_outer, ni, -1);
    }
    if (!(d->clip_low >= 0.0f) || !(d->clip_high >= 0.0f)) return fail(ODSGD_ERR_ARG, "clip_low and clip_high must not be negative");
    if (!std::isfinite(d->kl_coef) || !std::isfinite(d->grad_scale)) return fail(ODSGD_ERR_ARG, "kl_coef and grad_scale must be finite");
    if (!d->stats) return fail(ODSGD_ERR_ARG, "stats is NULL");
    if (reinterpret_cast<uintptr_t>(d->stats) % 4 != 0) return fail(ODSGD_ERR_ALIGN, "stats is not 4-byte aligned");
    if (!d->ref_logp && d->kl_coef != 0.0f && d->n_outer > 0 && ni > 0) return fail(ODSGD_ERR_ARG, "kl_coef needs ref_logp");
    bufs[n++] = {"old_logp", d->old_logp, 4, d->old_stride_outer, d->old_stride_inner, 1, false};
    if (d->ref_logp) bufs[n++] = {"ref_logp", d->ref_logp, 4, d->ref_stride_outer, d->ref_stride_inner, 1, false};
    bufs[n++] = {"advantages", d->advantages, 4, d->adv_stride_outer, d->adv_stride_inner, 1, false};
    bufs[n++] = {"weights", d->weights, 4, d->weight_stride_outer, d->weight_stride_inner, 1, false};
    same_ok = n;
    bufs[n++] = {"dlogits", d->dlogits, es, d->dlogits_stride_outer, d->dlogits_stride_inner, d->vocab, true};
    int rc = check_buffers(bufs, n, d->n_outer, ni, same_ok);
    if (rc == ODSGD_OK) rc = check_outside("stats", d->stats, 16, bufs, n, d->n_outer, ni);
    if (rc != ODSGD_OK || !ws) return rc;
    const uintptr_t w = reinterpret_cast<uintptr_t>(ws), st = reinterpret_cast<uintptr_t>(d->stats);
    if (w < st + 16 && st < w + ws_bytes) return fail(ODSGD_ERR_OVERLAP, "workspace overlaps stats");
    return check_outside("workspace", ws, ws_bytes, bufs, n, d->n_outer, ni);
}

// How a call cuts its rows: CTAs of a row, threads of a CTA, and which build of the kernel.
struct RowShape {
    int cluster, threads;
    bool wide;  // loss: 512-thread CTAs, two an SM, instead of 256-thread ones, five an SM
};

constexpr int kScoreThreads = 128, kScoreCtas = 12;
constexpr int kNarrowThreads = 256, kNarrowCtas = 5;
constexpr int kWideThreads = 512, kWideCtas = 2;
constexpr int kHoldNarrow = 40 << 10, kHoldWide = 108 << 10;  // shared memory of a full CTA: an SM's, over its CTAs
// What the rows in flight do not hold on the chip is read again from the L2 (126 MB), while their
// gradients pass through it.
constexpr int64_t kRowsInFlightBytes = 80 << 20;

RowShape row_shape(int64_t rows, int64_t vocab, int elem, bool loss, int sms) {
    RowShape s;
    const int64_t vectors = std::max<int64_t>(1, vocab / (16 / elem));
    s.wide = loss && (vectors * 16 - kHoldNarrow) * kNarrowCtas * sms > kRowsInFlightBytes;
    s.cluster = 1;
    if (loss)
        while (s.cluster < kRowCluster && (vectors * 16 / s.cluster - kHoldWide) * kWideCtas * sms > kRowsInFlightBytes) s.cluster *= 2;
    while (s.cluster < kRowCluster && rows * s.cluster < sms && vectors > (int64_t)s.cluster * 256) s.cluster *= 2;
    const int64_t part = ceil_div(vectors, s.cluster);
    // four batches of vectors a thread when there are rows enough to fill the GPU (4096 rows of 4000
    // 32-bit logits: 26 us where one batch takes 36), one vector when there are not
    const int64_t each = rows * s.cluster >= 2 * (int64_t)sms ? 4 * kRowVectors : 1;
    const int64_t most = !loss ? kScoreThreads : s.wide ? kWideThreads : kNarrowThreads;
    s.threads = (int)std::min(most, std::max<int64_t>(32, ceil_div(ceil_div(part, each), 32) * 32));
    return s;
}

template <typename T, int THREADS, int CTAS>
int launch_loss(RowArgs a, const RowShape& s, int hold_bytes, void* stream) {
    static std::atomic<bool> done[kMaxDevices] = {};
    int dev = 0;
    const int rc = current_device(&dev);
    if (rc != ODSGD_OK) return rc;
    if (dev >= kMaxDevices || !done[dev].load(std::memory_order_relaxed)) {
        const cudaError_t e = cudaFuncSetAttribute(row_kernel<T, true, THREADS, CTAS>, cudaFuncAttributeMaxDynamicSharedMemorySize, hold_bytes);
        if (e != cudaSuccess) return cuda_fail("cudaFuncSetAttribute", e);
        if (dev < kMaxDevices) done[dev].store(true, std::memory_order_relaxed);
    }
    // as many whole batches as fit (smaller CTAs, of which an SM takes more, have less room each), but
    // for the row's last, which stays in registers; nothing of short rows, which gain nothing by it
    // (16 KB: 27 us against 26; 48 KB: 72 against 77)
    const int64_t batch = (int64_t)s.threads * kRowVectors * 16;
    const int64_t part = ceil_div(a.vocab / kLanes<T>, s.cluster) * 16, batches = ceil_div(part, batch);
    a.hold = part < 32 << 10 ? 0 : (int)std::max<int64_t>(0, std::min((int64_t)hold_bytes * s.threads / THREADS / batch, batches - 1));
    return launch("policy loss kernel", row_kernel<T, true, THREADS, CTAS>, dim3(a.rows * (unsigned)s.cluster), dim3((unsigned)s.threads),
                  (size_t)(a.hold * batch), s.cluster, stream, a);
}

template <typename T>
int launch_rows_t(RowArgs a, const RowShape& s, bool loss, void* stream) {
    a.exp_temp = RowExp<T>::bounded(a.inv_temp);
    if (!loss)
        return launch("score kernel", row_kernel<T, false, kScoreThreads, kScoreCtas>, dim3(a.rows * (unsigned)s.cluster),
                      dim3((unsigned)s.threads), 0, s.cluster, stream, a);
    return s.wide ? launch_loss<T, kWideThreads, kWideCtas>(a, s, kHoldWide, stream)
                  : launch_loss<T, kNarrowThreads, kNarrowCtas>(a, s, kHoldNarrow, stream);
}

int launch_rows(const odsgd_policy_desc* d, bool loss, float* terms, void* stream) {
    int sms = 0;
    const int rc = sm_count(&sms);
    if (rc != ODSGD_OK) return rc;
    RowArgs a = {};
    a.z = d->logits;
    a.labels = d->labels;
    a.z_so = d->logits_stride_outer;
    a.z_si = d->logits_stride_inner;
    a.l_so = d->label_stride_outer;
    a.l_si = d->label_stride_inner;
    a.vocab = d->vocab;
    a.rows = (unsigned)(d->n_outer * d->n_inner);
    a.n_inner = (unsigned)d->n_inner;
    a.wide_labels = d->label_type == ODSGD_I64;
    a.inv_temp = d->inv_temp;
    a.logp = d->logp;
    if (loss) {
        a.old_logp = {d->old_logp, d->old_stride_outer, d->old_stride_inner};
        a.ref_logp = {d->ref_logp, d->ref_stride_outer, d->ref_stride_inner};
        a.adv = {d->advantages, d->adv_stride_outer, d->adv_stride_inner};
        a.weight = {d->weights, d->weight_stride_outer, d->weight_stride_inner};
        a.dz = d->dlogits;
        a.d_so = d->dlogits_stride_outer;
        a.d_si = d->dlogits_stride_inner;
        a.terms = terms;
        a.clip_low = d->clip_low;
        a.clip_high = d->clip_high;
        a.kl_coef = d->kl_coef;
        a.grad_scale = d->grad_scale;
    } else {
        a.lse = d->lse;
    }
    const RowShape s = row_shape(a.rows, a.vocab, size_of(d->type), loss, sms);
    a.cluster = s.cluster;
    switch (d->type) {
        case ODSGD_F32: return launch_rows_t<float>(a, s, loss, stream);
        case ODSGD_BF16: return launch_rows_t<bf16>(a, s, loss, stream);
        default: return launch_rows_t<f16>(a, s, loss, stream);
    }
}

size_t policy_bytes(const odsgd_policy_desc* d) { return std::max<size_t>(16, (size_t)(d->n_outer * d->n_inner) * 12); }

}  // namespace

namespace {
// Memory that a gradient set reads (kind 0) or writes (1).
struct Span {
    uintptr_t lo, hi;
    int kind;
};

// Lets this thread allocate and free while a stream that is not the call's is being captured: both would
// otherwise fail, and end that capture.
struct BesideCapture {
    cudaStreamCaptureMode mode = cudaStreamCaptureModeRelaxed;
    BesideCapture() { swap(); }
    ~BesideCapture() { swap(); }
    BesideCapture(const BesideCapture&) = delete;
    BesideCapture& operator=(const BesideCapture&) = delete;

private:
    void swap() {
        if (cudaThreadExchangeStreamCaptureMode(&mode) != cudaSuccess) cudaGetLastError();
    }
};
}  // namespace

struct odsgd_grad_set {
    std::vector<Span> spans;  // in ascending order; `norms` may lie in none of them
    int device = 0;
    int n_groups = 0;
    unsigned n_chunks = 0, most_chunks = 0;  // in all, and of a group
    void* table = nullptr;
    std::vector<unsigned char> host;  // what the table was filled from
    const GradChunk* chunks = nullptr;
    double* partial = nullptr;
    GradGroup* groups = nullptr;
    ~odsgd_grad_set() {
        if (!table) return;
        const BesideCapture beside;
        if (cudaFree(table) != cudaSuccess) cudaGetLastError();  // not left for the caller's next check
    }
};

namespace {

int make_set(odsgd_grad_set* s, const odsgd_grad_tensor* t, size_t n, int n_groups, float* const* arenas, size_t arena_len,
             cudaStream_t stream) {
    std::vector<size_t> order;
    std::vector<Span> spans;
    size_t total = 0;
    for (size_t k = 0; k < n; ++k) {
        const std::string name = "tensors[" + std::to_string(k) + "]";
        if (!is_float_type(t[k].type)) return fail(ODSGD_ERR_ARG, name + ": type must be ODSGD_F32, ODSGD_BF16 or ODSGD_F16");
        if (t[k].group < 0 || t[k].group >= n_groups) return fail(ODSGD_ERR_ARG, name + ": group out of range");
        if (arenas && (t[k].offset > arena_len || t[k].numel > arena_len - t[k].offset))
            return fail(ODSGD_ERR_ARG, name + " reaches beyond its arena");
        if (t[k].numel == 0) continue;
        if (!t[k].data) return fail(ODSGD_ERR_ARG, name + ": data is NULL");
        const uintptr_t at = reinterpret_cast<uintptr_t>(t[k].data);
        const uintptr_t es = (uintptr_t)size_of(t[k].type);
        if (at % es != 0) return fail(ODSGD_ERR_ALIGN, name + " is not aligned to its element type");
        if (t[k].numel > (UINTPTR_MAX - at) / es || t[k].numel > (size_t)1 << 48) return fail(ODSGD_ERR_ARG, name + " is beyond the address range");
        spans.push_back({at, at + t[k].numel * es, arenas ? 0 : 1});
        if (arenas) {
            const uintptr_t d = reinterpret_cast<uintptr_t>(arenas[t[k].group]) + t[k].offset * 4;
            spans.push_back({d, d + t[k].numel * 4, 1});
        }
        total += t[k].numel;
        order.push_back(k);
    }
    std::sort(spans.begin(), spans.end(), [](const Span& a, const Span& b) { return a.lo < b.lo; });
    // sources may share memory with one another; nothing may share it with a written range
    uintptr_t end_any = 0, end_written = 0;
    for (const Span& p : spans) {
        if (p.lo < end_written || (p.kind == 1 && p.lo < end_any))
            return fail(ODSGD_ERR_OVERLAP, arenas ? "a tensor's place in an arena overlaps another place or a gradient tensor"
                                                  : "gradient tensors that are scaled in place overlap");
        end_any = std::max(end_any, p.hi);
        if (p.kind == 1) end_written = std::max(end_written, p.hi);
    }
    // for the check of `norms`: where spans nest, the end of those so far
    for (size_t i = 1; i < spans.size(); ++i) spans[i].hi = std::max(spans[i].hi, spans[i - 1].hi);
    s->spans = spans;
    std::stable_sort(order.begin(), order.end(), [&](size_t a, size_t b) { return t[a].group < t[b].group; });
    // chunks of 16384 elements; of 4096 where those would leave SMs without work
    const size_t most = total / 16384 < 148 * 4 ? 4096 : 16384;
    std::vector<GradChunk> chunks;
    std::vector<GradGroup> groups((size_t)n_groups, GradGroup{0, 0, 1.0f});
    for (size_t k : order) {
        const size_t es = (size_t)size_of(t[k].type);
        const size_t count = (t[k].numel + most - 1) / most;
        if (chunks.size() + count >= (size_t)INT32_MAX / 4) return fail(ODSGD_ERR_UNSUPPORTED, "too many elements in one gradient set");
        float* dst = arenas ? arenas[t[k].group] + t[k].offset : nullptr;
        const bool vec = aligned16(t[k].data) && aligned16(dst);
        GradGroup& g = groups[(size_t)t[k].group];
        if (g.n_chunks == 0) g.first_chunk = (unsigned)chunks.size();
        g.n_chunks += (unsigned)count;
        for (size_t at = 0; at < t[k].numel; at += most) {
            GradChunk c = {};
            c.src = static_cast<const char*>(t[k].data) + at * es;
            c.dst = dst ? dst + at : nullptr;
            c.n = (unsigned)std::min(most, t[k].numel - at);
            c.type_vec = (unsigned short)(t[k].type | (vec ? 1 << 8 : 0));
            c.group = (unsigned short)t[k].group;
            chunks.push_back(c);
        }
    }
    s->n_chunks = (unsigned)chunks.size();
    s->n_groups = n_groups;
    for (const GradGroup& g : groups) s->most_chunks = std::max(s->most_chunks, g.n_chunks);
    const size_t at_groups = chunks.size() * sizeof(GradChunk);
    const size_t filled = (at_groups + groups.size() * sizeof(GradGroup) + 15) / 16 * 16;
    s->host.resize(filled);
    if (!chunks.empty()) memcpy(s->host.data(), chunks.data(), at_groups);
    memcpy(s->host.data() + at_groups, groups.data(), groups.size() * sizeof(GradGroup));
    cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
    cudaError_t e = cudaStreamIsCapturing(stream, &cap);
    if (e != cudaSuccess) return cuda_fail("cudaStreamIsCapturing", e);
    if (cap != cudaStreamCaptureStatusNone) return fail(ODSGD_ERR_STATE, "odsgd_grad_set_create cannot be recorded into a stream capture");
    const int rc = current_device(&s->device);
    if (rc != ODSGD_OK) return rc;
    const BesideCapture beside;
    e = cudaMalloc(&s->table, filled + (size_t)s->n_chunks * 8);
    if (e != cudaSuccess) {
        s->table = nullptr;
        return cuda_fail("gradient set table allocation", e);
    }
    unsigned char* base = static_cast<unsigned char*>(s->table);
    s->chunks = reinterpret_cast<const GradChunk*>(base);
    s->groups = reinterpret_cast<GradGroup*>(base + at_groups);
    s->partial = reinterpret_cast<double*>(base + filled);
    e = cudaMemcpyAsync(s->table, s->host.data(), filled, cudaMemcpyHostToDevice, stream);
    if (e != cudaSuccess) return cuda_fail("gradient set table upload", e);
    return ODSGD_OK;
}

int run_set(odsgd_grad_set* s, bool clip, float max_norm, float* norms, void* stream) {
    if (!s) return fail(ODSGD_ERR_ARG, "set is NULL");
    if (!clip && !norms) return fail(ODSGD_ERR_ARG, "norms is NULL");
    if (clip && !(max_norm >= 0.0f)) return fail(ODSGD_ERR_ARG, "max_norm is negative or NaN");
    if (reinterpret_cast<uintptr_t>(norms) % 4 != 0) return fail(ODSGD_ERR_ALIGN, "norms is not 4-byte aligned");
    if (norms) {
        // of the spans that begin below the end of norms, does one reach into it?
        const uintptr_t lo = reinterpret_cast<uintptr_t>(norms), hi = lo + 4 * (size_t)s->n_groups;
        const auto it = std::lower_bound(s->spans.begin(), s->spans.end(), hi, [](const Span& a, uintptr_t x) { return a.lo < x; });
        if (it != s->spans.begin() && (it - 1)->hi > lo) return fail(ODSGD_ERR_OVERLAP, "norms overlaps a gradient tensor or its place in an arena");
    }
    int dev = 0;
    int rc = current_device(&dev);
    if (rc != ODSGD_OK) return rc;
    if (dev != s->device) return fail(ODSGD_ERR_STATE, "the gradient set belongs to another device than the current one");
    GradArgs a = {};
    a.chunks = s->chunks;
    a.partial = s->partial;
    a.groups = s->groups;
    a.norms = norms;
    a.n_chunks = s->n_chunks;
    a.n_groups = s->n_groups;
    a.max_norm = max_norm;
    const dim3 chunks(s->n_chunks), block(kClipThreads);
    if (s->n_chunks > 0) rc = launch("gradient norm kernel", norm_kernel, chunks, block, 0, 1, stream, a);
    if (rc != ODSGD_OK) return rc;
    if (clip && s->n_chunks > 0 && s->most_chunks <= kJoinChunks)
        return launch("gradient clip kernel", clip_kernel<true>, chunks, block, 0, 1, stream, a);
    rc = launch("gradient norm sum kernel", finish_kernel, dim3((unsigned)s->n_groups), dim3(kFinishThreads), 0, 1, stream, a);
    if (rc != ODSGD_OK || !clip || s->n_chunks == 0) return rc;
    return launch("gradient clip kernel", clip_kernel<false>, chunks, block, 0, 1, stream, a);
}

}  // namespace

extern "C" {

int odsgd_embed_lookup(const odsgd_embed_desc* d, void* stream) {
    return guarded([&] {
        const int rc = check_embed(d, true);
        if (rc != ODSGD_OK) return rc;
        LookupArgs a = {};
        a.rows = (unsigned)(d->n_outer * d->n_inner);
        if (a.rows == 0) return ODSGD_OK;
        a.tokens = d->tokens;
        a.table = d->table;
        a.act = d->act;
        a.t_so = d->token_stride_outer;
        a.t_si = d->token_stride_inner;
        a.a_so = d->act_stride_outer;
        a.a_si = d->act_stride_inner;
        a.stride = d->table_stride;
        a.vocab = d->vocab;
        a.dim = d->dim;
        a.n_inner = (unsigned)d->n_inner;
        a.wide_tokens = d->token_type == ODSGD_I64;
        a.scale = d->scale;
        const bool vec = rows_aligned(d->table, size_of(d->table_type), 0, a.stride, 1, a.vocab) &&
                         rows_aligned(d->act, size_of(d->act_type), a.a_so, a.a_si, d->n_outer, d->n_inner);
        switch (d->table_type) {
            case ODSGD_F32: return launch_lookup_t<float>(a, d->act_type, vec, stream);
            case ODSGD_BF16: return launch_lookup_t<bf16>(a, d->act_type, vec, stream);
            default: return launch_lookup_t<f16>(a, d->act_type, vec, stream);
        }
    });
}

int odsgd_embed_grad_workspace(const odsgd_embed_desc* d, size_t* bytes) {
    return guarded([&] {
        if (!d || !bytes) return fail(ODSGD_ERR_ARG, "desc / bytes is NULL");
        *bytes = 0;
        if (!is_float_type(d->act_type)) return fail(ODSGD_ERR_ARG, "act_type must be ODSGD_F32, ODSGD_BF16 or ODSGD_F16");
        if (d->n_outer < 0 || d->n_inner < 0 || d->vocab < 1 || d->dim < 1) return fail(ODSGD_ERR_ARG, "sizes out of range");
        if ((wide)d->n_outer * d->n_inner > ODSGD_MAX_TOKENS || d->vocab >= INT32_MAX || d->dim > kMaxDim)
            return fail(ODSGD_ERR_UNSUPPORTED, "sizes beyond the limits");
        *bytes = grad_shape(d).bytes;
        return ODSGD_OK;
    });
}

int odsgd_embed_grad(const odsgd_embed_desc* d, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&] {
        int rc = check_embed(d, false);
        if (rc != ODSGD_OK) return rc;
        const GradShape s = grad_shape(d);
        rc = check_workspace(workspace, workspace_bytes, s.bytes);
        if (rc == ODSGD_OK) rc = check_embed(d, false, workspace, s.bytes);
        if (rc != ODSGD_OK) return rc;
        rc = allow_sort_smem();
        if (rc != ODSGD_OK) return rc;
        if (s.n == 0 && d->accumulate) return ODSGD_OK;
        unsigned char* ws = static_cast<unsigned char*>(workspace);
        EmbedGradArgs a = {};
        a.tokens = d->tokens;
        a.act = d->act;
        a.table = static_cast<float*>(d->table);
        a.t_so = d->token_stride_outer;
        a.t_si = d->token_stride_inner;
        a.a_so = d->act_stride_outer;
        a.a_si = d->act_stride_inner;
        a.stride = d->table_stride;
        a.vocab = d->vocab;
        a.dim = d->dim;
        a.padding = d->padding_token;
        a.n = s.n;
        a.n_inner = (unsigned)std::max<int64_t>(1, d->n_inner);
        a.wide_tokens = d->token_type == ODSGD_I64;
        a.flat = d->n_outer == 1 || a.t_so == d->n_inner * a.t_si;
        a.accumulate = d->accumulate != 0;
        a.scale = d->scale;
        for (int i = 0; i < 2; ++i) {
            a.key[i] = reinterpret_cast<unsigned*>(ws + s.at_key[i]);
            a.pos[i] = reinterpret_cast<unsigned*>(ws + s.at_pos[i]);
        }
        a.counts = reinterpret_cast<unsigned*>(ws + s.at_counts);
        a.runs = reinterpret_cast<SpanRun*>(ws + s.at_runs);
        a.head = reinterpret_cast<float*>(ws + s.at_head);
        a.tail = reinterpret_cast<float*>(ws + s.at_tail);
        a.pitch = s.pitch;
        a.block = s.block;
        a.passes = s.passes;
        a.bits = s.bits;
        // Zeros beside the sort: for few tokens 128 MB (all of 65 MB beside 500 tokens: 21 us, 24 MB of it
        // 27), else as many as the digit passes take time for, some 10 us and 0.8 us per thousand tokens
        // (131072 tokens, 537 MB: 199 us at 4000 bytes a token, 216 at 2000).
        int64_t early = 0;
        if (!a.accumulate) {
            const int64_t bytes = s.n <= (unsigned)kSortThreads ? 128 << 20 : (50 << 20) + (int64_t)s.n * 4000;
            early = std::min<int64_t>(a.vocab, ceil_div(bytes / (a.dim * 4), kFillRows) * kFillRows);
            if (s.n == 0) early = a.vocab;
            a.fills = (unsigned)ceil_div(a.vocab - early, kFillRows);
        }
        a.early = (unsigned)early;
        a.named = reinterpret_cast<unsigned*>(ws + s.at_named);
        const unsigned fill = (unsigned)std::min<int64_t>(kFillClusters, ceil_div(early * a.dim * 4, kFillBytes));
        // one CTA an SM where it still writes the zeros within the digit passes' time (32760 tokens, 51 MB: 39 us
        // with one, 41 with two; 102 MB: 57, 49; 131072 tokens, 102 MB: 101, 105; 205 MB: 150, 148)
        const bool few_zeros = early * a.dim * 4 <= (45 << 20) + (int64_t)s.n * 500;
        const auto sort = s.n <= (unsigned)(kSortCluster * kSortThreads) ? sort_kernel<false, 2> : few_zeros ? sort_kernel<true, 1> : sort_kernel<true, 2>;
        rc = launch("token sort kernel", sort, dim3((1 + fill) * kSortCluster), dim3(kSortThreads), kSortSmem, 1, stream, a);
        if (rc != ODSGD_OK || s.n == 0) return rc;
        const bool vec = aligned16(a.table) && a.stride % 4 == 0 &&
                         rows_aligned(d->act, size_of(d->act_type), a.a_so, a.a_si, d->n_outer, d->n_inner);
        switch (d->act_type) {
            case ODSGD_F32: rc = launch_sum<float>(a, s, vec, stream); break;
            case ODSGD_BF16: rc = launch_sum<bf16>(a, s, vec, stream); break;
            default: rc = launch_sum<f16>(a, s, vec, stream); break;
        }
        if (rc != ODSGD_OK || s.blocks < 2) return rc;
        const dim3 grid(std::min<unsigned>(s.blocks - 1, kJoinGrid), (unsigned)ceil_div(a.dim, kJoinColumns));
        return launch("embedding gradient join kernel", join_kernel, grid, dim3(32 * kJoinWarps), 0, 1, stream, a);
    });
}

int odsgd_token_logprob(const odsgd_policy_desc* d, void* stream) {
    return guarded([&] {
        const int rc = check_policy(d, false);
        if (rc != ODSGD_OK || d->n_outer == 0 || d->n_inner == 0) return rc;
        return launch_rows(d, false, nullptr, stream);
    });
}

int odsgd_policy_loss_workspace(const odsgd_policy_desc* d, size_t* bytes) {
    return guarded([&] {
        if (!d || !bytes) return fail(ODSGD_ERR_ARG, "desc / bytes is NULL");
        *bytes = 0;
        if (d->n_outer < 0 || d->n_inner < 0) return fail(ODSGD_ERR_ARG, "n_outer / n_inner is negative");
        if ((wide)d->n_outer * d->n_inner >= (1 << 27)) return fail(ODSGD_ERR_UNSUPPORTED, "too many rows in one call");
        *bytes = policy_bytes(d);
        return ODSGD_OK;
    });
}

int odsgd_policy_loss(const odsgd_policy_desc* d, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&] {
        int rc = check_policy(d, true);
        if (rc != ODSGD_OK) return rc;
        rc = check_workspace(workspace, workspace_bytes, policy_bytes(d));
        if (rc == ODSGD_OK) rc = check_policy(d, true, workspace, policy_bytes(d));
        if (rc != ODSGD_OK) return rc;
        StatsArgs st = {};
        st.terms = static_cast<const float*>(workspace);
        st.stats = d->stats;
        st.rows = (unsigned)(d->n_outer * d->n_inner);
        st.kl_coef = d->kl_coef;
        if (st.rows > 0) rc = launch_rows(d, true, static_cast<float*>(workspace), stream);
        if (rc != ODSGD_OK) return rc;
        return launch("policy loss sum kernel", stats_kernel, dim3(1), dim3(kStatsThreads), 0, 1, stream, st);
    });
}

int odsgd_grad_set_create(odsgd_grad_set** out, const odsgd_grad_tensor* tensors, size_t n_tensors, int n_groups,
                          float* const* arenas, size_t arena_len, void* stream) {
    return guarded([&] {
        if (!out) return fail(ODSGD_ERR_ARG, "out is NULL");
        *out = nullptr;
        if (n_groups < 1 || n_groups > ODSGD_MAX_WORKERS)
            return fail(ODSGD_ERR_ARG, "n_groups must be in 1.." + std::to_string(ODSGD_MAX_WORKERS));
        if (n_tensors > 0 && !tensors) return fail(ODSGD_ERR_ARG, "tensors is NULL");
        if (arenas)
            for (int g = 0; g < n_groups; ++g) {
                const std::string name = "arenas[" + std::to_string(g) + "]";
                if (!arenas[g]) return fail(ODSGD_ERR_ARG, name + " is NULL");
                if (reinterpret_cast<uintptr_t>(arenas[g]) % 4 != 0) return fail(ODSGD_ERR_ALIGN, name + " is not 4-byte aligned");
                if (arena_len > (UINTPTR_MAX - reinterpret_cast<uintptr_t>(arenas[g])) / 4)
                    return fail(ODSGD_ERR_ARG, name + " is beyond the address range");
            }
        odsgd_grad_set* s = new odsgd_grad_set;
        int rc;
        try {
            rc = make_set(s, tensors, n_tensors, n_groups, arenas, arena_len, static_cast<cudaStream_t>(stream));
        } catch (...) {
            delete s;
            throw;
        }
        if (rc != ODSGD_OK) {
            delete s;
            return rc;
        }
        *out = s;
        return ODSGD_OK;
    });
}

int odsgd_grad_set_norm(odsgd_grad_set* set, float* norms, void* stream) {
    return guarded([&] { return run_set(set, false, HUGE_VALF, norms, stream); });
}

int odsgd_grad_set_clip(odsgd_grad_set* set, float max_norm, float* norms, void* stream) {
    return guarded([&] { return run_set(set, true, max_norm, norms, stream); });
}

int odsgd_grad_set_destroy(odsgd_grad_set* set) {
    if (!set) return ODSGD_ERR_ARG;
    delete set;
    return ODSGD_OK;
}

}  // extern "C"
