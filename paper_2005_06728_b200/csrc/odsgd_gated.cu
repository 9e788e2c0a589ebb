// Host side of the gated feed-forward block: checks of arguments, operands that have to be laid out, tensor maps,
// launches.  No allocation, no synchronisation (but in odsgd_stalled_waits), nothing thrown across the boundary.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "odsgd.h"
#include "odsgd_lm_host.h"
#include "odsgd_gated_kernels.cuh"

using namespace odsgd_lm;

namespace {

constexpr int64_t kMaxGatedDim = 1 << 20;

bool is_half_type(int t) { return t == ODSGD_BF16 || t == ODSGD_F16; }

// A matrix as TMA takes it: 16-bit elements, rows that start on 16 bytes.
struct Matrix {
    const void* p = nullptr;
    int64_t rows = 0, columns = 0, stride = 0;
};

// What a call lays out in the workspace, and where.
struct GatedPlan {
    bool lay_x = false, lay_w[2] = {false, false};
    int64_t tokens = 0, dim_pitch = 0, width_pitch = 0;
    size_t x = 0, w[2] = {0, 0}, dg = 0, du = 0, bytes = 0;
};

// `line`: bytes that every row has to start on.
bool tma_rows(const void* p, int64_t rows, int64_t columns, int64_t stride, int64_t line = 16) {
    if (reinterpret_cast<uintptr_t>(p) % line != 0 || (rows > 1 && stride * 2 % line != 0)) return false;
    return aligned16(p) && (rows <= 1 || (stride % 8 == 0 && stride >= columns && stride < (int64_t)1 << 38));
}

// Rows of two levels as rows of one; false if they are not evenly spaced.
bool one_level(int64_t n_outer, int64_t n_inner, int64_t so, int64_t si, int64_t* stride) {
    *stride = n_inner > 1 ? si : so;
    return n_outer <= 1 || n_inner <= 1 || so == n_inner * si;
}

GatedPlan gated_plan(const odsgd_gated_desc* d, bool backward) {
    GatedPlan p;
    p.tokens = d->n_outer * d->n_inner;
    // whole lines of 128 bytes: a box's rows then are one line each
    p.dim_pitch = ceil_div(d->dim, 64) * 64;
    p.width_pitch = ceil_div(d->width, 64) * 64;
    const auto take = [&](int64_t rows, int64_t pitch) {
        const size_t at = p.bytes;
        p.bytes += (size_t)ceil_div(rows * pitch * 2, 128) * 128;
        return at;
    };
    // A box of rows that start on 16 bytes but not on 64 crosses twice the lines: the forward pass then takes a quarter longer, which
    // pays for laying operands out where the product is large against them (8192 tokens of 4088 x 11008 1178 us as they are,
    // of 4095 1031, laid out; 2044 of 2040 x 5440 75, of 2047 88).  The backward products lose less by it.  The rule: a quarter of the
    // products' time at 1.6 PFLOP/s against the launch and the bytes of the layout at 5 TB/s.
    const double n = (double)p.tokens, dim = (double)d->dim, width = (double)d->width;
    const bool large = !backward && 0.25 * 4.0 * n * dim * width / 1.6e15 > 4e-6 + 4.0 * dim * (n + 2.0 * width) / 5e12;
    const int64_t line = large ? 64 : 16;
    int64_t stride = 0;
    p.lay_x = !one_level(d->n_outer, d->n_inner, d->x_stride_outer, d->x_stride_inner, &stride) || !tma_rows(d->x, p.tokens, d->dim, stride, line);
    if (backward && !d->dw_gate) p.lay_x = false;
    if (p.lay_x) p.x = take(p.tokens, p.dim_pitch);
    const bool weights = !backward || d->dx;
    p.lay_w[0] = weights && (d->weight_type == ODSGD_F32 || !tma_rows(d->w_gate, d->width, d->dim, d->w_gate_stride, line));
    p.lay_w[1] = weights && (d->weight_type == ODSGD_F32 || !tma_rows(d->w_up, d->width, d->dim, d->w_up_stride, line));
    for (int i = 0; i < 2; ++i)
        if (p.lay_w[i]) p.w[i] = take(d->width, p.dim_pitch);
    if (backward) {
        p.dg = take(p.tokens, p.width_pitch);
        p.du = take(p.tokens, p.width_pitch);
    }
    return p;
}

int check_gated(const odsgd_gated_desc* d, bool backward) {
    if (!d) return fail(ODSGD_ERR_ARG, "desc is NULL");
    if (!is_half_type(d->type)) return fail(ODSGD_ERR_ARG, "type must be ODSGD_BF16 or ODSGD_F16");
    if (d->weight_type != d->type && d->weight_type != ODSGD_F32) return fail(ODSGD_ERR_ARG, "weight_type must be ODSGD_F32 or the type of x");
    if (d->activation != ODSGD_SILU && d->activation != ODSGD_GELU) return fail(ODSGD_ERR_ARG, "activation must be ODSGD_SILU or ODSGD_GELU");
    if (d->n_outer < 0 || d->n_inner < 0) return fail(ODSGD_ERR_ARG, "n_outer / n_inner is negative");
    if ((wide)d->n_outer * d->n_inner > ODSGD_MAX_TOKENS) return fail(ODSGD_ERR_UNSUPPORTED, "more than ODSGD_MAX_TOKENS tokens in one call");
    if (d->dim < 1 || d->width < 1) return fail(ODSGD_ERR_ARG, "dim and width must be at least 1");
    if (d->dim > kMaxGatedDim || d->width > kMaxGatedDim) return fail(ODSGD_ERR_UNSUPPORTED, "dim or width beyond the limits");
    if (d->w_gate_stride < d->dim || d->w_up_stride < d->dim) return fail(ODSGD_ERR_ARG, "a weight stride is smaller than dim");
    if ((d->gate == nullptr) != (d->up == nullptr)) return fail(ODSGD_ERR_ARG, "gate and up go together");
    if (backward) {
        if (!d->dx && !d->dw_gate) return fail(ODSGD_ERR_ARG, "neither dx nor dw_gate / dw_up is wanted");
        if ((d->dw_gate == nullptr) != (d->dw_up == nullptr)) return fail(ODSGD_ERR_ARG, "dw_gate and dw_up go together");
        if (d->dw_gate) {
            if (d->dw_type != d->type && d->dw_type != ODSGD_F32) return fail(ODSGD_ERR_ARG, "dw_type must be ODSGD_F32 or the type of x");
            if (d->accumulate && d->dw_type != ODSGD_F32) return fail(ODSGD_ERR_ARG, "only ODSGD_F32 gradients are added to");
            if (d->dw_gate_stride < d->dim || d->dw_up_stride < d->dim) return fail(ODSGD_ERR_ARG, "a gradient stride is smaller than dim");
        }
    }
    const int es = size_of(d->type), we = size_of(d->weight_type), ge = d->dw_gate ? size_of(d->dw_type) : 4;
    // buffers of rows of tokens
    Buf rows[8];
    int n = 0;
    rows[n++] = {"x", d->x, es, d->x_stride_outer, d->x_stride_inner, d->dim, false};
    rows[n++] = {backward ? "dh" : "h", d->h, es, d->h_stride_outer, d->h_stride_inner, d->width, !backward};
    if (d->gate || backward) {
        rows[n++] = {"gate", d->gate, es, d->gate_stride_outer, d->gate_stride_inner, d->width, !backward};
        rows[n++] = {"up", d->up, es, d->up_stride_outer, d->up_stride_inner, d->width, !backward};
    }
    if (backward && d->dx) rows[n++] = {"dx", d->dx, es, d->dx_stride_outer, d->dx_stride_inner, d->dim, true};
    int rc = check_buffers(rows, n, d->n_outer, d->n_inner, -1);
    if (rc != ODSGD_OK) return rc;
    // buffers of rows of weights
    Buf mats[4];
    int m = 0;
    mats[m++] = {"w_gate", d->w_gate, we, 0, d->w_gate_stride, d->dim, false};
    mats[m++] = {"w_up", d->w_up, we, 0, d->w_up_stride, d->dim, false};
    if (backward && d->dw_gate) {
        mats[m++] = {"dw_gate", d->dw_gate, ge, 0, d->dw_gate_stride, d->dim, true};
        mats[m++] = {"dw_up", d->dw_up, ge, 0, d->dw_up_stride, d->dim, true};
    }
    rc = check_buffers(mats, m, 1, d->width, -1);
    if (rc != ODSGD_OK || d->n_outer == 0 || d->n_inner == 0) return rc;
    for (int i = 0; i < n; ++i) {
        for (int j = 0; j < m; ++j) {
            Range a, b;
            range_of(rows[i], d->n_outer, d->n_inner, &a);
            range_of(mats[j], 1, d->width, &b);
            if ((rows[i].written || mats[j].written) && a.lo < b.hi && b.lo < a.hi)
                return fail(ODSGD_ERR_OVERLAP, std::string(mats[j].name) + " overlaps " + rows[i].name);
        }
    }
    return ODSGD_OK;
}

// The workspace against all buffers of a checked call.
int check_gated_workspace(const odsgd_gated_desc* d, bool backward, const void* ws, size_t have, size_t need) {
    if (need == 0) return ODSGD_OK;
    int rc = check_workspace(ws, have, need);
    if (rc != ODSGD_OK) return rc;
    const int es = size_of(d->type);
    const Buf rows[5] = {{"x", d->x, es, d->x_stride_outer, d->x_stride_inner, d->dim, false},
                         {"h", d->h, es, d->h_stride_outer, d->h_stride_inner, d->width, false},
                         {"gate", d->gate, es, d->gate_stride_outer, d->gate_stride_inner, d->width, false},
                         {"up", d->up, es, d->up_stride_outer, d->up_stride_inner, d->width, false},
                         {"dx", d->dx, es, d->dx_stride_outer, d->dx_stride_inner, d->dim, false}};
    for (int i = 0; i < (backward ? 5 : 4) && rc == ODSGD_OK; ++i)
        if (rows[i].p) rc = check_outside("workspace", ws, need, &rows[i], 1, d->n_outer, d->n_inner);
    const Buf mats[4] = {{"w_gate", d->w_gate, size_of(d->weight_type), 0, d->w_gate_stride, d->dim, false},
                         {"w_up", d->w_up, size_of(d->weight_type), 0, d->w_up_stride, d->dim, false},
                         {"dw_gate", d->dw_gate, d->dw_gate ? size_of(d->dw_type) : 4, 0, d->dw_gate_stride, d->dim, false},
                         {"dw_up", d->dw_up, d->dw_gate ? size_of(d->dw_type) : 4, 0, d->dw_up_stride, d->dim, false}};
    for (int i = 0; i < (backward ? 4 : 2) && rc == ODSGD_OK; ++i)
        if (mats[i].p) rc = check_outside("workspace", ws, need, &mats[i], 1, 1, d->width);
    return rc;
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*,
                                 const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

int encode_function(EncodeTiled* out) {
    static std::atomic<EncodeTiled> known{nullptr};
    EncodeTiled f = known.load(std::memory_order_relaxed);
    if (!f) {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
        const cudaError_t e = cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found);
        if (e != cudaSuccess) return cuda_fail("cudaGetDriverEntryPointByVersion", e);
        if (found != cudaDriverEntryPointSuccess || !p) return fail(ODSGD_ERR_CUDA, "the driver has no cuTensorMapEncodeTiled");
        f = reinterpret_cast<EncodeTiled>(p);
        known.store(f, std::memory_order_relaxed);
    }
    *out = f;
    return ODSGD_OK;
}

// Boxes of 64 columns and `box_rows` rows; zeros beyond the matrix.
int encode(CUtensorMap* map, const Matrix& m, int type, int box_rows) {
    EncodeTiled f = nullptr;
    const int rc = encode_function(&f);
    if (rc != ODSGD_OK) return rc;
    const cuuint64_t sizes[2] = {(cuuint64_t)m.columns, (cuuint64_t)m.rows};
    const int64_t stride = m.rows > 1 ? m.stride : ceil_div(m.columns, 8) * 8;  // (of a single row it is not used)
    const cuuint64_t strides[1] = {(cuuint64_t)stride * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, steps[2] = {1, 1};
    const CUresult r = f(map, type == ODSGD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, const_cast<void*>(m.p), sizes,
                         strides, box, steps, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                         CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? ODSGD_OK : fail(ODSGD_ERR_CUDA, "cuTensorMapEncodeTiled: error " + std::to_string((int)r));
}

// The largest dynamic shared memory of a kernel, set once a device.
int allow_smem(const void* kernel, int bytes, std::atomic<bool>* done) {
    int dev = 0;
    const int rc = current_device(&dev);
    if (rc != ODSGD_OK) return rc;
    if (dev < kMaxDevices && done[dev].load(std::memory_order_relaxed)) return ODSGD_OK;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e != cudaSuccess) return cuda_fail("cudaFuncSetAttribute", e);
    if (dev < kMaxDevices) done[dev].store(true, std::memory_order_relaxed);
    return ODSGD_OK;
}

template <int KIND, typename T, bool GELU = false>
int launch_gated(const GatedArgs& a, void* stream) {
    static std::atomic<bool> done[kMaxDevices] = {};
    int sms = 0;
    int rc = sm_count(&sms);
    if (rc == ODSGD_OK) rc = allow_smem((const void*)gated_kernel<KIND, T, GELU>, kGatedSmem, done);
    if (rc != ODSGD_OK) return rc;
    const int64_t columns = KIND == kForward ? kTileColumns / 2 : kTileColumns;
    const int64_t tiles = ceil_div(a.rows, kTileRows) * ceil_div(a.columns, columns) * (KIND == kGradW ? 2 : 1);
    const unsigned pairs = (unsigned)std::min<int64_t>(tiles, sms / 2);
    return launch(KIND == kForward ? "gated forward kernel" : KIND == kGradX ? "gated gradient kernel (x)" : "gated gradient kernel (weights)",
                  gated_kernel<KIND, T, GELU>, dim3(2 * pairs), dim3(kGatedThreads), kGatedSmem, 1, stream, a);
}

// dynamic shared memory of a CTA of thin_kernel, one and two an SM
constexpr int kThinSmem[2] = {226 * 1024, 110 * 1024};

// How many clusters of `cluster` CTAs of thin_kernel run at once, one or two CTAs an SM: what the GPU's clusters of SMs leave
// room for, asked once a device.  The question is put for a kernel without tensor memory: for one that has some the answer
// is one CTA an SM, though two of thin_kernel do run (their times and SMs were recorded).
int thin_clusters(int dev, int per_sm, int cluster, int* out) {
    static std::atomic<int> known[kMaxDevices][2][kThinCluster + 1] = {};
    static std::atomic<bool> done[kMaxDevices] = {};
    int n = dev < kMaxDevices ? known[dev][per_sm - 1][cluster].load(std::memory_order_relaxed) : 0;
    if (n == 0) {
        const int rc = allow_smem((const void*)thin_room_kernel, kThinSmem[0], done);
        if (rc != ODSGD_OK) return rc;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)cluster);
        cfg.blockDim = dim3(kThinThreads);
        cfg.dynamicSmemBytes = (size_t)kThinSmem[per_sm - 1];
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)cluster;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        const cudaError_t e = cudaOccupancyMaxActiveClusters(&n, thin_room_kernel, &cfg);
        if (e != cudaSuccess) return cuda_fail("cudaOccupancyMaxActiveClusters", e);
        n = std::max(n, 1);
        if (dev < kMaxDevices) known[dev][per_sm - 1][cluster].store(n, std::memory_order_relaxed);
    }
    *out = n;
    return ODSGD_OK;
}

// Whether a product of `tokens` goes to thin_kernel, and how: its tokens in chunks of up to 256, each CTA of a cluster with four
// blocks of the long axis at least, as many CTAs to a cluster as leave all clusters running at once.
struct ThinShape {
    int64_t chunk = 0;  // 0: gated_kernel
    int cluster = 1, per_sm = 1;
};
// Both kernels' cycles, from runs of (dim, width) (256, 700) to (4096, 11000) with 1 to 3000 tokens, burst, forward and gradient
// of x: a block of the long axis takes gated_kernel some 520 where tiles are few and operands come from memory; thin_kernel
// takes it at 60 bytes a cycle and SM, and finishes at 65 cycles a token; 12500 and 7600 pass beside that.  For example
// (2048, 5440), forward: 64 tokens 11.0 us thin and 16.2 not, 128 14.1 and 16.7, 200 18.8 and 16.7; gradient of x: 256 tokens
// 22 and 58, 1024 58 and 66, 1536 79 and 71; (512, 1400), forward, 768 tokens 8.9 and 9.6, 1024 10.4 and 10.1.
template <int KIND>
int thin_shape(int64_t tokens, int64_t columns, int64_t depth, int sms, ThinShape* out) {
    const int64_t blocks = ceil_div(depth, kBlockK) * (KIND == kGradX ? 2 : 1), tiles = ceil_div(columns, KIND == kForward ? 64 : 128);
    const int64_t wide = ceil_div(tokens, kTileRows) * ceil_div(columns, KIND == kForward ? kTileColumns / 2 : kTileColumns);
    double least = 12500.0 + 520.0 * (double)ceil_div(wide, sms / 2) * (double)blocks;
    *out = ThinShape{};
    if (tokens > 8192) return ODSGD_OK;
    int dev = 0;
    const int rc = current_device(&dev);
    if (rc != ODSGD_OK) return rc;
    for (int64_t most : {64, 96, 128, 192, 256}) {
        const int64_t chunks = ceil_div(tokens, most), chunk = ceil_div(ceil_div(tokens, chunks), 16) * 16;
        const int64_t stage = kThinRows * kBlockK * 2 + chunk * kBlockK * 2, sums = chunk * kThinRows * 4;
        const int per_sm = std::max(3 * stage, sums) <= kThinSmem[1] - 1024 ? 2 : 1;
        int cluster = 1;
        for (int c = 2; c <= kThinCluster && blocks >= 4 * c; ++c) {
            int room = 0;
            const int asked = thin_clusters(dev, per_sm, c, &room);
            if (asked != ODSGD_OK) return asked;
            if (tiles * chunks <= room) cluster = c;
        }
        const double ctas = (double)(tiles * chunks * cluster), waves = std::ceil(ctas / (per_sm * sms));
        const double an_sm = std::max(1.0, std::min((double)per_sm, ctas / sms));
        const double cycles = 7600.0 + waves * ((double)ceil_div(blocks, cluster) * an_sm * (double)stage / 60.0 + 65.0 * (double)chunk);
        if (cycles < least) least = cycles, *out = ThinShape{chunk, cluster, per_sm};
        if (chunks == 1) break;  // (the wider ones are the same)
    }
    return ODSGD_OK;
}

template <int KIND, typename T, bool GELU = false>
int launch_thin(const GatedArgs& g, unsigned tokens, const ThinShape& s, void* stream) {
    static std::atomic<bool> done[kMaxDevices] = {};
    const int rc = allow_smem((const void*)thin_kernel<KIND, T, GELU>, kThinSmem[0], done);
    if (rc != ODSGD_OK) return rc;
    ThinArgs a;
    for (int i = 0; i < 2; ++i) a.a[i] = g.b[i], a.b[i] = g.a[KIND == kForward ? 0 : i];
    for (int i = 0; i < 3; ++i) a.out[i] = g.out[i];
    a.tokens = tokens, a.n_inner = g.n_inner, a.columns = g.columns, a.depth = g.depth, a.is_bf16 = g.is_bf16, a.save = g.save;
    a.chunk = (unsigned)s.chunk, a.cluster = (unsigned)s.cluster;
    a.tensor_columns = 32;
    while (a.tensor_columns < a.chunk) a.tensor_columns *= 2;
    const int64_t stage = kThinRows * kBlockK * 2 + s.chunk * kBlockK * 2, sums = s.chunk * kThinRows * 4;
    a.stages = (unsigned)std::min<int64_t>(kThinStages, (kThinSmem[s.per_sm - 1] - 1024) / stage);
    const size_t smem = 1024 + (size_t)std::max(a.stages * stage, sums);
    const int64_t tiles = ceil_div(a.columns, KIND == kForward ? 64 : 128);
    return launch("gated kernel for few tokens", thin_kernel<KIND, T, GELU>, dim3((unsigned)tiles * a.cluster, (unsigned)ceil_div(tokens, s.chunk)),
                  dim3(kThinThreads), smem, s.cluster, stream, a);
}

// Blocks of rows: threads along a row, eight columns each, and the rest of a CTA's across rows.
void row_blocks(int64_t rows, int64_t columns, int rows_a_thread, dim3* grid, dim3* block) {
    const int64_t cols = ceil_div(columns, 8), slabs = ceil_div(cols, kLayThreads);
    const int64_t x = ceil_div(ceil_div(cols, slabs), 32) * 32, y = kLayThreads / x;
    *block = dim3((unsigned)x, (unsigned)y);
    *grid = dim3((unsigned)std::min<int64_t>(ceil_div(rows, y * rows_a_thread), 1 << 20), (unsigned)slabs);
}

template <typename T>
int run_gated(const odsgd_gated_desc* d, bool backward, const GatedPlan& p, char* ws, void* stream) {
    const int64_t n = p.tokens;
    Matrix x, w[2];
    int rc = ODSGD_OK;
    x.rows = n, x.columns = d->dim;
    LayArgs lay = {};
    lay.columns = (unsigned)d->dim, lay.pitch = (unsigned)p.dim_pitch;
    int64_t lay_rows = 0;
    if (p.lay_x) {
        lay.m[0] = {d->x, ws + p.x, d->x_stride_outer, d->x_stride_inner, (unsigned)n, (unsigned)d->n_inner, 0};
        lay_rows += n;
        x.p = ws + p.x, x.stride = p.dim_pitch;
    } else {
        one_level(d->n_outer, d->n_inner, d->x_stride_outer, d->x_stride_inner, &x.stride);
        x.p = d->x;
    }
    const void* const wp[2] = {d->w_gate, d->w_up};
    const int64_t wst[2] = {d->w_gate_stride, d->w_up_stride};
    for (int i = 0; i < 2; ++i) {
        w[i].rows = d->width, w[i].columns = d->dim;
        if (p.lay_w[i]) {
            lay.m[1 + i] = {wp[i], ws + p.w[i], 0, wst[i], (unsigned)d->width, (unsigned)d->width, d->weight_type == ODSGD_F32};
            lay_rows += d->width;
            w[i].p = ws + p.w[i], w[i].stride = p.dim_pitch;
        } else {
            w[i].p = wp[i], w[i].stride = wst[i];
        }
    }
    dim3 grid, block;
    if (lay_rows > 0) {
        for (LayMatrix& m : lay.m) m.n_inner = std::max(m.n_inner, 1u);
        row_blocks(lay_rows, d->dim, kLayRows, &grid, &block);
        rc = launch("operand layout kernel", lay_kernel<T>, grid, block, 0, 1, stream, lay);
        if (rc != ODSGD_OK) return rc;
    }
    int sms = 0;
    rc = sm_count(&sms);
    if (rc != ODSGD_OK) return rc;
    ThinShape shape;
    GatedArgs a = {};
    a.is_bf16 = d->type == ODSGD_BF16;
    const bool gelu = d->activation == ODSGD_GELU;
    a.n_inner = (unsigned)d->n_inner;
    if (!backward) {
        rc = thin_shape<kForward>(n, d->width, d->dim, sms, &shape);
        if (rc != ODSGD_OK) return rc;
        const bool thin = shape.chunk > 0;
        rc = encode(&a.a[0], x, d->type, thin ? (int)shape.chunk : 128);
        for (int i = 0; i < 2 && rc == ODSGD_OK; ++i) rc = encode(&a.b[i], w[i], d->type, thin ? 64 : 128);
        if (rc != ODSGD_OK) return rc;
        a.out[0] = {d->h, d->h_stride_outer, d->h_stride_inner};
        a.out[1] = {d->gate, d->gate_stride_outer, d->gate_stride_inner};
        a.out[2] = {d->up, d->up_stride_outer, d->up_stride_inner};
        a.rows = (unsigned)n, a.columns = (unsigned)d->width, a.depth = (unsigned)d->dim;
        a.save = d->gate != nullptr;
        if (thin) return gelu ? launch_thin<kForward, T, true>(a, (unsigned)n, shape, stream) : launch_thin<kForward, T, false>(a, (unsigned)n, shape, stream);
        return gelu ? launch_gated<kForward, T, true>(a, stream) : launch_gated<kForward, T, false>(a, stream);
    }
    SlopeArgs s = {};
    s.gate = {d->gate, d->gate_stride_outer, d->gate_stride_inner};
    s.up = {d->up, d->up_stride_outer, d->up_stride_inner};
    s.dh = {d->h, d->h_stride_outer, d->h_stride_inner};
    s.dg = ws + p.dg, s.du = ws + p.du;
    s.rows = (unsigned)n, s.n_inner = (unsigned)d->n_inner, s.columns = (unsigned)d->width, s.pitch = (unsigned)p.width_pitch;
    s.vec = rows_aligned(d->gate, 2, s.gate.so, s.gate.si, d->n_outer, d->n_inner) && rows_aligned(d->up, 2, s.up.so, s.up.si, d->n_outer, d->n_inner) &&
            rows_aligned(d->h, 2, s.dh.so, s.dh.si, d->n_outer, d->n_inner);
    row_blocks(n, d->width, 1, &grid, &block);
    rc = gelu ? launch("gated slope kernel", slope_kernel<T, true>, grid, block, 0, 1, stream, s)
              : launch("gated slope kernel", slope_kernel<T, false>, grid, block, 0, 1, stream, s);
    if (rc != ODSGD_OK) return rc;
    Matrix g[2];
    for (int i = 0; i < 2; ++i) g[i].p = ws + (i ? p.du : p.dg), g[i].rows = n, g[i].columns = d->width, g[i].stride = p.width_pitch;
    if (d->dx) {
        rc = thin_shape<kGradX>(n, d->dim, d->width, sms, &shape);
        const bool thin = shape.chunk > 0;
        for (int i = 0; i < 2 && rc == ODSGD_OK; ++i) rc = encode(&a.a[i], g[i], d->type, thin ? (int)shape.chunk : 128);
        for (int i = 0; i < 2 && rc == ODSGD_OK; ++i) rc = encode(&a.b[i], w[i], d->type, kBlockK);
        if (rc != ODSGD_OK) return rc;
        a.out[0] = {d->dx, d->dx_stride_outer, d->dx_stride_inner};
        a.rows = (unsigned)n, a.columns = (unsigned)d->dim, a.depth = (unsigned)d->width;
        rc = thin ? launch_thin<kGradX, T>(a, (unsigned)n, shape, stream) : launch_gated<kGradX, T>(a, stream);
        if (rc != ODSGD_OK) return rc;
    }
    if (d->dw_gate) {
        for (int i = 0; i < 2 && rc == ODSGD_OK; ++i) rc = encode(&a.a[i], g[i], d->type, kBlockK);
        if (rc == ODSGD_OK) rc = encode(&a.b[0], x, d->type, kBlockK);
        if (rc != ODSGD_OK) return rc;
        a.out[0] = {d->dw_gate, 0, d->dw_gate_stride};
        a.out[1] = {d->dw_up, 0, d->dw_up_stride};
        a.rows = (unsigned)d->width, a.columns = (unsigned)d->dim, a.depth = (unsigned)n, a.n_inner = (unsigned)d->width;
        a.out_f32 = d->dw_type == ODSGD_F32;
        a.accumulate = d->accumulate != 0;
        rc = launch_gated<kGradW, T>(a, stream);
    }
    return rc;
}

// Without tokens there is nothing but gradients of zeros.
int no_tokens(const odsgd_gated_desc* d, bool backward, void* stream) {
    if (!backward || !d->dw_gate || d->accumulate) return ODSGD_OK;
    const size_t es = (size_t)size_of(d->dw_type);
    void* const to[2] = {d->dw_gate, d->dw_up};
    const int64_t st[2] = {d->dw_gate_stride, d->dw_up_stride};
    for (int i = 0; i < 2; ++i) {
        const cudaError_t e = cudaMemset2DAsync(to[i], (size_t)st[i] * es, 0, (size_t)d->dim * es, (size_t)d->width, static_cast<cudaStream_t>(stream));
        if (e != cudaSuccess) return cuda_fail("cudaMemset2DAsync", e);
    }
    return ODSGD_OK;
}

int gated(const odsgd_gated_desc* d, bool backward, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_gated(d, backward);
    if (rc != ODSGD_OK) return rc;
    const GatedPlan p = gated_plan(d, backward);
    rc = check_gated_workspace(d, backward, workspace, workspace_bytes, p.bytes);
    if (rc != ODSGD_OK) return rc;
    if (p.tokens == 0) return no_tokens(d, backward, stream);
    char* const ws = static_cast<char*>(workspace);
    return d->type == ODSGD_BF16 ? run_gated<bf16>(d, backward, p, ws, stream) : run_gated<f16>(d, backward, p, ws, stream);
}

}  // namespace

extern "C" {

int odsgd_gated_workspace(const odsgd_gated_desc* desc, int backward, size_t* bytes) {
    return guarded([&] {
        if (!bytes) return fail(ODSGD_ERR_ARG, "bytes is NULL");
        const int rc = check_gated(desc, backward != 0);
        if (rc != ODSGD_OK) return rc;
        *bytes = gated_plan(desc, backward != 0).bytes;
        return (int)ODSGD_OK;
    });
}

int odsgd_gated_forward(const odsgd_gated_desc* desc, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&] { return gated(desc, false, workspace, workspace_bytes, stream); });
}

int odsgd_gated_backward(const odsgd_gated_desc* desc, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&] { return gated(desc, true, workspace, workspace_bytes, stream); });
}

int odsgd_stalled_waits(unsigned int* count) {
    return guarded([&] {
        if (!count) return fail(ODSGD_ERR_ARG, "count is NULL");
        cudaError_t e = cudaDeviceSynchronize();  // (the copy by itself waits for no stream that was made non-blocking)
        if (e != cudaSuccess) return cuda_fail("cudaDeviceSynchronize", e);
        e = cudaMemcpyFromSymbol(count, stalled_waits, sizeof(*count));
        return e == cudaSuccess ? (int)ODSGD_OK : cuda_fail("cudaMemcpyFromSymbol", e);
    });
}

}  // extern "C"
