// What the layers on rows of channels (layer norm, linear) share on the host side: matrices of evenly spaced rows, and their checks.
#pragma once
#include "abi.h"

#define ESC_TRY(call)                    \
    do {                                 \
        const int rc__ = (call);         \
        if (rc__ != ESC_OK) return rc__; \
    } while (0)

namespace esc { namespace rows {

inline bool known(int dtype) { return dtype == ESC_F32 || dtype == ESC_BF16; }

inline int launched() {
    ESC_ABI_CUDA(cudaGetLastError());
    abi::launched();
    return ESC_OK;
}

// A kernel that may start while the one before it in the stream ends, and waits for that itself (griddepcontrol.wait).
template <typename... P, typename... A> int launch_behind(void (*kernel)(P...), unsigned blocks, int threads, cudaStream_t st, size_t smem, A... args) {
    cudaLaunchAttribute attr{};
    attr.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(blocks); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = st; cfg.attrs = &attr; cfg.numAttrs = 1;
    ESC_ABI_CUDA(cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...));
    return launched();
}

// A matrix in memory: `rows` runs of `width` values, `stride` values apart.
struct Matrix {
    const void* p;
    long long rows, stride, width;
    size_t es;
    size_t bytes() const { return p && rows > 0 ? ((size_t)(rows - 1) * stride + width) * es : 0; }
};
// Whether two of them share memory; slices side by side of one wider tensor do not.
inline bool touch(const Matrix& a, const Matrix& b) {
    if (!a.bytes() || !b.bytes() || !abi::overlap(a.p, a.bytes(), b.p, b.bytes())) return false;
    const size_t step = (size_t)a.stride * a.es;
    if (step != (size_t)b.stride * b.es || a.rows == 1 || b.rows == 1) return true;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
    const size_t far = (x > y ? x - y : y - x) % step;
    const size_t ahead = x > y ? step - far : far;                 // from a run of a to the next run of b
    return far == 0 || ahead < (size_t)a.width * a.es || step - ahead < (size_t)b.width * b.es;
}
inline Matrix flat(const void* p, long long count, size_t es) { return Matrix{p, p ? 1 : 0, count, count, es}; }

inline int check_rows(long long rows, long long width, long long stride) {
    if (rows < 0 || width <= 0 || stride < width) return ESC_ERR_SHAPE;
    return (long double)rows * stride > 4.0e15L ? ESC_ERR_SHAPE : ESC_OK;
}
inline int zero(void* p, size_t bytes, cudaStream_t st) {
    if (p) ESC_ABI_CUDA(cudaMemsetAsync(p, 0, bytes, st));
    return ESC_OK;
}

}}  // namespace esc::rows
