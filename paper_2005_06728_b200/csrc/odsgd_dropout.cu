// Host side of dropout: checks of arguments and the launch.  No allocation, no synchronisation, nothing thrown
// across the boundary.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "odsgd.h"
#include "odsgd_lm_host.h"
#include "odsgd_dropout_kernels.cuh"

using namespace odsgd_lm;

namespace {

constexpr int64_t kMaxDropoutDim = 1 << 20;

int check_dropout(const odsgd_dropout_desc* d) {
    if (!d) return fail(ODSGD_ERR_ARG, "desc is NULL");
    if (!is_float_type(d->type)) return fail(ODSGD_ERR_ARG, "type must be ODSGD_F32, ODSGD_BF16 or ODSGD_F16");
    if (!is_float_type(d->out_type)) return fail(ODSGD_ERR_ARG, "out_type must be ODSGD_F32, ODSGD_BF16 or ODSGD_F16");
    if (d->n_outer < 0 || d->n_inner < 0) return fail(ODSGD_ERR_ARG, "n_outer / n_inner is negative");
    if ((wide)d->n_outer * d->n_inner > ODSGD_MAX_TOKENS) return fail(ODSGD_ERR_UNSUPPORTED, "more than ODSGD_MAX_TOKENS rows in one call");
    if (d->dim < 1) return fail(ODSGD_ERR_ARG, "dim must be at least 1");
    if (d->dim > kMaxDropoutDim) return fail(ODSGD_ERR_UNSUPPORTED, "dim beyond the limits");
    if (!(d->p >= 0.0) || std::nearbyint(d->p * 65536.0) > 65535.0) return fail(ODSGD_ERR_ARG, "p must be in [0, 65535.5 / 65536)");
    if (d->counter && reinterpret_cast<uintptr_t>(d->counter) % 8 != 0) return fail(ODSGD_ERR_ALIGN, "counter is not aligned to its element type");
    const Buf x = {"x", d->x, size_of(d->type), d->x_stride_outer, d->x_stride_inner, d->dim, false};
    const Buf r = {"residual", d->residual, size_of(d->out_type), d->residual_stride_outer, d->residual_stride_inner, d->dim, false};
    const Buf out = {"out", d->out, size_of(d->out_type), d->out_stride_outer, d->out_stride_inner, d->dim, true};
    // in place, on x or on the residual: an element is read by the thread that writes it
    const Buf pair[2] = {x, out};
    int rc = check_buffers(pair, 2, d->n_outer, d->n_inner, d->type == d->out_type ? 1 : -1);
    if (rc == ODSGD_OK && d->residual) {
        const Buf other[2] = {r, out};
        rc = check_buffers(other, 2, d->n_outer, d->n_inner, 1);
    }
    if (rc == ODSGD_OK && d->counter) rc = check_outside("counter", d->counter, 8, &out, 1, d->n_outer, d->n_inner);
    return rc;
}

// Rows that follow one another without a gap.
bool flat(int64_t so, int64_t si, const odsgd_dropout_desc* d) {
    return (d->n_inner <= 1 || si == d->dim) && (d->n_outer <= 1 || so == d->n_inner * d->dim);
}

template <typename TX, typename TO>
int launch_dropout(DropoutArgs a, bool vec, int sms, void* stream) {
    const int64_t most = (int64_t)sms * 64;
    if (vec) {
        const int64_t blocks = a.n / 8;
        const dim3 grid((unsigned)std::min<int64_t>(ceil_div(blocks, kDropoutThreads), most));
        const int rc = blocks > 0 ? launch("dropout kernel", dropout_kernel<TX, TO>, grid, dim3(kDropoutThreads), 0, 1, stream, a) : (int)ODSGD_OK;
        if (rc != ODSGD_OK || a.n % 8 == 0) return rc;
        a.first = blocks;  // fewer than eight elements are left
    }
    const int64_t rows = a.n / a.dim, blocks = a.first > 0 ? 1 : a.dim / 8 + 2;
    const int64_t x = std::min<int64_t>(kDropoutThreads, ceil_div(blocks, 32) * 32), y = kDropoutThreads / x;
    const dim3 grid((unsigned)std::min<int64_t>(ceil_div(rows, y), most), (unsigned)std::min<int64_t>(ceil_div(blocks, x), 4096));
    return launch("dropout kernel (rows)", row_dropout_kernel<TX, TO>, grid, dim3((unsigned)x, (unsigned)y), 0, 1, stream, a);
}

template <typename TX>
int launch_dropout_t(const DropoutArgs& a, int out_type, bool vec, int sms, void* stream) {
    switch (out_type) {
        case ODSGD_F32: return launch_dropout<TX, float>(a, vec, sms, stream);
        case ODSGD_BF16: return launch_dropout<TX, bf16>(a, vec, sms, stream);
        default: return launch_dropout<TX, f16>(a, vec, sms, stream);
    }
}

int dropout(const odsgd_dropout_desc* d, void* stream) {
    int sms = 0;
    int rc = check_dropout(d);
    if (rc != ODSGD_OK || d->n_outer == 0 || d->n_inner == 0) return rc;
    rc = sm_count(&sms);
    if (rc != ODSGD_OK) return rc;
    DropoutArgs a = {};
    a.x = d->x, a.residual = d->residual, a.out = d->out;
    a.x_so = d->x_stride_outer, a.x_si = d->x_stride_inner;
    a.r_so = d->residual_stride_outer, a.r_si = d->residual_stride_inner;
    a.o_so = d->out_stride_outer, a.o_si = d->out_stride_inner;
    a.n = d->n_outer * d->n_inner * d->dim;
    a.dim = d->dim, a.n_inner = d->n_inner;
    a.seed = d->seed, a.offset = d->offset, a.counter = d->counter;
    a.threshold = (unsigned)std::nearbyint(d->p * 65536.0);
    a.scale = (float)(65536.0 / (65536.0 - a.threshold));
    bool vec;
    if (flat(a.x_so, a.x_si, d) && flat(a.o_so, a.o_si, d) && (!d->residual || flat(a.r_so, a.r_si, d))) {
        a.dim = a.n, a.n_inner = 1;  // one row
        vec = aligned16(d->x) && aligned16(d->out) && aligned16(d->residual);
    } else {
        vec = d->dim % 8 == 0 && rows_aligned(d->x, size_of(d->type), a.x_so, a.x_si, d->n_outer, d->n_inner) &&
              rows_aligned(d->out, size_of(d->out_type), a.o_so, a.o_si, d->n_outer, d->n_inner) &&
              (!d->residual || rows_aligned(d->residual, size_of(d->out_type), a.r_so, a.r_si, d->n_outer, d->n_inner));
    }
    switch (d->type) {
        case ODSGD_F32: return launch_dropout_t<float>(a, d->out_type, vec, sms, stream);
        case ODSGD_BF16: return launch_dropout_t<bf16>(a, d->out_type, vec, sms, stream);
        default: return launch_dropout_t<f16>(a, d->out_type, vec, sms, stream);
    }
}

}  // namespace

extern "C" int odsgd_dropout(const odsgd_dropout_desc* desc, void* stream) {
    return guarded([&] { return dropout(desc, stream); });
}
