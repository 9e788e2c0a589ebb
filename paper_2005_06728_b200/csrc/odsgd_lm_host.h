// Host-side helpers that the language-model calls share: error texts, checks of buffers and workspaces, launches.
// Internal: included by the sources of the library alone.
#pragma once

#include <cuda_runtime.h>

#include <atomic>
#include <cstring>
#include <string>

#include "odsgd.h"

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

// Whether all rows of a strided buffer start on 16 bytes.
bool rows_aligned(const void* p, int elem, int64_t so, int64_t si, int64_t n_outer, int64_t n_inner) {
    return aligned16(p) && (n_outer <= 1 || so * elem % 16 == 0) && (n_inner <= 1 || si * elem % 16 == 0);
}

}  // namespace
