// Host side of the verification of drafted tokens: checks of arguments and launches.  No allocation, no
// synchronisation, nothing thrown across the boundary.
#include <cuda_runtime.h>

#include <algorithm>
#include <cmath>

#include "odsgd.h"
#include "odsgd_lm_host.h"
#include "odsgd_verify_kernels.cuh"

using namespace odsgd_lm;

namespace {

static_assert(kVerifyDrafts == ODSGD_MAX_DRAFTS, "the shared arrays of the kernels");

int check_verify(const odsgd_verify_desc* d, const void* ws, size_t have) {
    if (!d) return fail(ODSGD_ERR_ARG, "desc is NULL");
    if (!is_float_type(d->type)) return fail(ODSGD_ERR_ARG, "type must be ODSGD_F32, ODSGD_BF16 or ODSGD_F16");
    if (!is_token_type(d->token_type)) return fail(ODSGD_ERR_ARG, "token_type must be ODSGD_I32 or ODSGD_I64");
    if (d->batch < 0 || d->drafts < 0) return fail(ODSGD_ERR_ARG, "batch / drafts is negative");
    if (d->vocab < 1) return fail(ODSGD_ERR_ARG, "vocab must be at least 1");
    if (d->drafts > ODSGD_MAX_DRAFTS || d->batch > 1 << 16 || d->vocab > 1 << 30)
        return fail(ODSGD_ERR_UNSUPPORTED, "batch, drafts or vocab beyond the limits");
    if (!(d->inv_temp >= 1e-30f && d->inv_temp <= 1e30f && d->draft_inv_temp >= 1e-30f && d->draft_inv_temp <= 1e30f))
        return fail(ODSGD_ERR_ARG, "inv_temp and draft_inv_temp must be in [1e-30, 1e30]");
    const int es = size_of(d->type), ts = size_of(d->token_type);
    const int64_t many = d->drafts + 1;
    const Buf rows[6] = {{"target", d->target, es, d->target_stride_batch, d->target_stride_row, d->vocab, false},
                         {"uniforms", d->uniforms, 4, d->uniform_stride_batch, d->uniform_stride_row, 1, false},
                         {"out_tokens", d->out_tokens, ts, many, 1, 1, true},
                         {"logp", d->logp, 4, many, 1, 1, true},
                         {"draft", d->draft, es, d->draft_stride_batch, d->draft_stride_row, d->vocab, false},
                         {"tokens", d->tokens, ts, d->token_stride_batch, d->token_stride_row, 1, false}};
    const Buf accepted = {"accepted", d->accepted, 4, 1, 0, 1, true};
    int rc = check_buffers(rows, 4, d->batch, many, -1);
    if (rc == ODSGD_OK) rc = check_buffers(rows + (d->draft ? 4 : 5), d->draft ? 2 : 1, d->batch, d->drafts, -1);
    if (rc == ODSGD_OK) rc = check_buffers(&accepted, 1, d->batch, 1, -1);
    if (rc != ODSGD_OK || d->batch == 0) return rc;
    // what is written against everything else
    struct Out {
        const char* name;
        const void* p;
        size_t bytes;
    };
    const size_t n = (size_t)(d->batch * many);
    const Out out[4] = {{"accepted", d->accepted, (size_t)d->batch * 4}, {"out_tokens", d->out_tokens, n * ts}, {"logp", d->logp, n * 4}, {"workspace", ws, have}};
    for (int i = 0; i < (ws ? 4 : 3) && rc == ODSGD_OK; ++i) {
        rc = check_outside(out[i].name, out[i].p, out[i].bytes, rows, 2, d->batch, many);
        if (rc == ODSGD_OK) rc = check_outside(out[i].name, out[i].p, out[i].bytes, rows + 5, 1, d->batch, d->drafts);
        if (rc == ODSGD_OK && d->draft) rc = check_outside(out[i].name, out[i].p, out[i].bytes, rows + 4, 1, d->batch, d->drafts);
        for (int j = 0; j < i && rc == ODSGD_OK; ++j) {
            const uintptr_t a = reinterpret_cast<uintptr_t>(out[i].p), b = reinterpret_cast<uintptr_t>(out[j].p);
            if (a < b + out[j].bytes && b < a + out[i].bytes) return fail(ODSGD_ERR_OVERLAP, std::string(out[i].name) + " overlaps " + out[j].name);
        }
    }
    return rc;
}

// Up to so many tokens a CTA does a sequence's whole work.
constexpr int64_t kAloneVocab = 2048;
// SMs that the shapes are made for: a B200's.  Not asked of the device, so that the workspace stays a function of sizes alone; on
// another number the same results would come out in more or fewer waves.
constexpr int64_t kVerifySms = 148;

// Launch shapes and workspace: functions of sizes alone.
struct VerifyShape {
    int64_t rows, chunks;  // all rows, parts of each
    int64_t pass_ctas;     // of a sequence
    int64_t segments, segment;
    size_t positions, sums, bytes;
};
VerifyShape verify_shape(const odsgd_verify_desc* d) {
    VerifyShape s;
    s.rows = d->batch * (2 * d->drafts + 1);
    // parts of at least 4096 elements, as many as fill every SM three times; each of whole steps of its CTA, so that none goes round
    // again for a few elements (16 x 11 rows of 50021 bf16: 7.3 us in 12 parts a row, 6.1 in 13)
    const int64_t step = (int64_t)kPartThreads * kRowVectors * 16 / size_of(d->type);
    const int64_t wanted = std::max<int64_t>(1, std::min(ceil_div(kVerifySms * kPartCtas * 3, std::max<int64_t>(s.rows, 1)), d->vocab / 4096));
    s.chunks = ceil_div(d->vocab, step * std::max<int64_t>(1, d->vocab / (step * wanted)));
    // CTAs of 2048 elements and more, as many as run at once, two an SM
    s.pass_ctas = std::max<int64_t>(1, std::min(2 * kVerifySms / std::max<int64_t>(d->batch, 1), ceil_div(d->vocab, 2048)));
    // a warp's share, in pieces that draw_kernel goes over in one step, but no more of them than it has threads
    const int64_t share = ceil_div(d->vocab, s.pass_ctas * kPassWarps);
    const int64_t piece = std::max(ceil_div(share, ceil_div(share, 256 * kDrawWarps)), ceil_div(d->vocab, kSegments));
    s.segment = ceil_div(piece, 256) * 256;
    if (d->vocab <= kAloneVocab) s.segment = 256;
    s.segments = ceil_div(d->vocab, s.segment);
    s.positions = (size_t)ceil_div(s.rows * s.chunks * (int64_t)sizeof(MaxSum), 16) * 16;
    s.sums = s.positions + (size_t)ceil_div(d->batch * (d->drafts + 1) * (int64_t)sizeof(Position), 16) * 16;
    s.bytes = std::max<size_t>(16, s.sums + (size_t)(d->batch * kDrawSums * s.segments) * sizeof(double));
    return s;
}

template <typename T>
int launch_verify(VerifyArgs a, bool alone, void* stream) {
    a.exp_temp = RowExp<T>::bounded(a.inv_temp);
    a.draft_exp = RowExp<T>::bounded(a.draft_temp);
    const unsigned rows = a.target_rows + (a.draft ? a.batch * a.drafts : 0);
    if (alone) return launch("verification kernel (alone)", draw_kernel<T, true>, dim3(a.batch), dim3(kDrawThreads), 0, 1, stream, a);
    int rc = launch("verification kernel (rows)", parts_kernel<T>, dim3(rows * a.chunks), dim3(kPartThreads), 0, 1, stream, a);
    if (rc == ODSGD_OK) rc = launch("verification kernel (pass)", pass_kernel<T>, dim3(a.batch * (unsigned)a.pass_ctas), dim3(kPassWarps * 32), 0, 1, stream, a);
    if (rc == ODSGD_OK) rc = launch("verification kernel (draw)", draw_kernel<T, false>, dim3(a.batch), dim3(kDrawThreads), 0, 1, stream, a);
    return rc;
}

int verify(const odsgd_verify_desc* d, void* ws, size_t ws_bytes, void* stream) {
    int rc = check_verify(d, nullptr, 0);
    if (rc != ODSGD_OK) return rc;
    const VerifyShape s = verify_shape(d);
    rc = check_workspace(ws, ws_bytes, s.bytes);
    if (rc == ODSGD_OK) rc = check_verify(d, ws, s.bytes);
    if (rc != ODSGD_OK || d->batch == 0) return rc;
    VerifyArgs a = {};
    a.target = d->target, a.draft = d->drafts > 0 ? d->draft : nullptr, a.tokens = d->tokens, a.uniforms = d->uniforms;
    a.out_tokens = d->out_tokens, a.accepted = d->accepted, a.logp = d->logp;
    char* const at = static_cast<char*>(ws);
    a.parts = reinterpret_cast<MaxSum*>(at);
    a.positions = reinterpret_cast<Position*>(at + s.positions);
    a.sums = reinterpret_cast<double*>(at + s.sums);
    a.t_sb = d->target_stride_batch, a.t_sr = d->target_stride_row;
    a.d_sb = d->draft_stride_batch, a.d_sr = d->draft_stride_row;
    a.k_sb = d->token_stride_batch, a.k_sr = d->token_stride_row;
    a.u_sb = d->uniform_stride_batch, a.u_sr = d->uniform_stride_row;
    a.batch = (unsigned)d->batch, a.drafts = (unsigned)d->drafts, a.target_rows = (unsigned)(d->batch * (d->drafts + 1));
    a.chunks = (unsigned)s.chunks;
    a.pass_ctas = (int)s.pass_ctas, a.segments = (int)s.segments, a.segment = (int)s.segment;
    a.vocab = (int)d->vocab;
    a.wide_tokens = d->token_type == ODSGD_I64;
    a.inv_temp = d->inv_temp, a.draft_temp = d->draft_inv_temp;
    a.least = kLeast / (d->inv_temp * 1.4426950408889634), a.draft_least = kLeast / (d->draft_inv_temp * 1.4426950408889634);
    const bool alone = d->vocab <= kAloneVocab;
    switch (d->type) {
        case ODSGD_F32: return launch_verify<float>(a, alone, stream);
        case ODSGD_BF16: return launch_verify<bf16>(a, alone, stream);
        default: return launch_verify<f16>(a, alone, stream);
    }
}

}  // namespace

extern "C" {

int odsgd_verify_workspace(const odsgd_verify_desc* desc, size_t* bytes) {
    return guarded([&] {
        if (!desc || !bytes) return fail(ODSGD_ERR_ARG, "desc / bytes is NULL");
        *bytes = 0;
        if (!is_float_type(desc->type)) return fail(ODSGD_ERR_ARG, "type must be ODSGD_F32, ODSGD_BF16 or ODSGD_F16");
        if (desc->batch < 0 || desc->drafts < 0 || desc->vocab < 1) return fail(ODSGD_ERR_ARG, "sizes out of range");
        if (desc->drafts > ODSGD_MAX_DRAFTS || desc->batch > 1 << 16 || desc->vocab > 1 << 30)
            return fail(ODSGD_ERR_UNSUPPORTED, "batch, drafts or vocab beyond the limits");
        *bytes = verify_shape(desc).bytes;
        return (int)ODSGD_OK;
    });
}

int odsgd_verify_draft(const odsgd_verify_desc* desc, void* workspace, size_t workspace_bytes, void* stream) {
    return guarded([&] { return verify(desc, workspace, workspace_bytes, stream); });
}

}  // extern "C"
