// What the translation units of the library share on the host side.  The thread-local state behind it lives in
// esc_convattn.cu.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/esc_convattn.h"

namespace esc { namespace abi {

int cuda_fail(cudaError_t e, const char* what);   // records the text for esc_last_error(), returns ESC_ERR_CUDA
void launches_reset();                            // a call that launches kernels starts
void launched();                                  // one more kernel of this call

inline size_t elem_size(int dtype) { return dtype == ESC_BF16 ? 2 : 4; }
inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }
inline size_t round_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
inline bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + b_bytes && y < x + a_bytes;
}

// SM count of the current device; a B200's 148 where no device can be asked (size queries on a machine without a GPU).
inline int sm_count() {
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return 148;
    }
    return n > 0 ? n : 148;
}

}}  // namespace esc::abi

#define ESC_ABI_CUDA(call)                                              \
    do {                                                                \
        cudaError_t e__ = (call);                                       \
        if (e__ != cudaSuccess) return esc::abi::cuda_fail(e__, #call); \
    } while (0)
