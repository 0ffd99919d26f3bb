// C ABI of the optimiser's step: argument checks, the plan of a list of tensors, launches.
#include "abi.h"

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "adamw.cuh"

namespace {

using esc::adamw::Chunk;
using esc::adamw::kChunk;
using esc::adamw::kQuant;

long long count_chunks(int n_tensors, const long long* sizes) {   // -1: a size is negative or the list is too long
    long long n = 0;
    for (int i = 0; i < n_tensors; ++i) {
        if (sizes[i] < 0 || sizes[i] > (1LL << 50)) return -1;
        n += (sizes[i] + kChunk - 1) / kChunk;
    }
    return n <= 0x7fffffffLL ? n : -1;
}

// The memory that a step touches.  Every value is read, changed and written by one thread, in no order: what is written has to be nobody else's.
struct Range { uintptr_t from, to; bool written; };
bool shared(std::vector<Range>& ranges) {
    std::sort(ranges.begin(), ranges.end(), [](const Range& a, const Range& b) { return a.from < b.from; });
    uintptr_t end = 0, end_written = 0;             // of those that start earlier
    for (const Range& r : ranges) {
        if (r.from < (r.written ? end : end_written)) return true;
        end = std::max(end, r.to);
        if (r.written) end_written = std::max(end_written, r.to);
    }
    return false;
}

template <typename P, typename G>
int launch(const Chunk* chunks, unsigned blocks, const esc::adamw::Hyper& h, const float* scalars, const int* skip, int states, cudaStream_t st) {
    if (states == ESC_STATES_F32) esc::adamw::step<P, G, float><<<blocks, esc::adamw::kThreads, 0, st>>>(chunks, h, scalars, skip);
    else esc::adamw::step<P, G, __nv_fp8_e4m3><<<blocks, esc::adamw::kThreads, 0, st>>>(chunks, h, scalars, skip);
    ESC_ABI_CUDA(cudaGetLastError());
    esc::abi::launched();
    return ESC_OK;
}

bool known(int dtype) { return dtype == ESC_F32 || dtype == ESC_BF16; }

}  // namespace

extern "C" {

size_t esc_adamw_plan_bytes(int n_tensors, const long long* sizes) {
    if (n_tensors <= 0 || !sizes) return 0;
    const long long n = count_chunks(n_tensors, sizes);
    return n < 0 ? 0 : esc::abi::round_up((size_t)(n > 0 ? n : 1) * sizeof(Chunk), 256);
}

int esc_adamw_plan_init(int n_tensors, const long long* sizes, void* const* params, const void* const* grads, void* const* exp_avgs,
                        void* const* exp_avg_sqs, float* const* avg_scales, float* const* sq_scales, void* const* copies,
                        int param_dtype, int grad_dtype, int states, void* plan, size_t plan_bytes, long long* n_chunks, void* stream) {
    if (n_tensors <= 0) return ESC_ERR_SHAPE;
    if (!sizes || !params || !grads || !exp_avgs || !exp_avg_sqs || !n_chunks) return ESC_ERR_NULL;
    if (!known(param_dtype) || !known(grad_dtype) || (states != ESC_STATES_F32 && states != ESC_STATES_E4M3)) return ESC_ERR_UNSUPPORTED;
    const bool eight = states == ESC_STATES_E4M3;
    if (eight && (!avg_scales || !sq_scales)) return ESC_ERR_NULL;
    const long long n = count_chunks(n_tensors, sizes);
    if (n < 0) return ESC_ERR_SHAPE;
    if (!plan || !esc::abi::aligned(plan, 256) || plan_bytes < esc_adamw_plan_bytes(n_tensors, sizes)) return ESC_ERR_WORKSPACE;
    const size_t ps = esc::abi::elem_size(param_dtype), gs = esc::abi::elem_size(grad_dtype), ss = eight ? 1 : 4;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    try {
        std::vector<Chunk> chunks;
        chunks.reserve((size_t)n);
        std::vector<Range> ranges;
        ranges.reserve((size_t)n_tensors * 7 + 1);
        auto touch = [&](const void* p, size_t bytes, bool written) {
            if (p) ranges.push_back({reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p) + bytes, written});
        };
        touch(plan, esc_adamw_plan_bytes(n_tensors, sizes), false);
        for (int i = 0; i < n_tensors; ++i) {
            if (sizes[i] == 0) continue;
            if (!params[i] || !grads[i] || !exp_avgs[i] || !exp_avg_sqs[i]) return ESC_ERR_NULL;
            if (eight && (!avg_scales[i] || !sq_scales[i])) return ESC_ERR_NULL;
            void* copy = copies ? copies[i] : nullptr;
            if (!esc::abi::aligned(params[i], ps) || !esc::abi::aligned(grads[i], gs) || !esc::abi::aligned(exp_avgs[i], ss) ||
                !esc::abi::aligned(exp_avg_sqs[i], ss) || !esc::abi::aligned(copy, 2)) return ESC_ERR_ALIGN;
            if (eight && (!esc::abi::aligned(avg_scales[i], 4) || !esc::abi::aligned(sq_scales[i], 4))) return ESC_ERR_ALIGN;
            const bool wide = esc::abi::aligned(params[i], 4 * ps) && esc::abi::aligned(grads[i], 4 * gs) && esc::abi::aligned(exp_avgs[i], 4 * ss) &&
                              esc::abi::aligned(exp_avg_sqs[i], 4 * ss) && esc::abi::aligned(copy, 8);
            const size_t count = (size_t)sizes[i], scales = (count + kQuant - 1) / kQuant * sizeof(float);
            touch(params[i], count * ps, true);
            touch(grads[i], count * gs, false);
            touch(exp_avgs[i], count * ss, true);
            touch(exp_avg_sqs[i], count * ss, true);
            touch(copy, count * 2, true);
            if (eight) { touch(avg_scales[i], scales, true); touch(sq_scales[i], scales, true); }
            for (long long at = 0; at < sizes[i]; at += kChunk) {
                Chunk c;
                c.p = static_cast<char*>(params[i]) + at * ps;
                c.g = static_cast<const char*>(grads[i]) + at * gs;
                c.m = static_cast<char*>(exp_avgs[i]) + at * ss;
                c.v = static_cast<char*>(exp_avg_sqs[i]) + at * ss;
                c.m_scale = eight ? avg_scales[i] + at / kQuant : nullptr;
                c.v_scale = eight ? sq_scales[i] + at / kQuant : nullptr;
                c.copy = copy ? static_cast<__nv_bfloat16*>(copy) + at : nullptr;
                c.n = (int)(sizes[i] - at < kChunk ? sizes[i] - at : kChunk);
                c.wide = wide;
                chunks.push_back(c);
            }
        }
        if (shared(ranges)) return ESC_ERR_ALIAS;
        // the copy comes from this function's own memory, so it has to be over before the function is
        cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
        ESC_ABI_CUDA(cudaStreamIsCapturing(st, &capture));
        if (capture != cudaStreamCaptureStatusNone) return ESC_ERR_UNSUPPORTED;
        if (!chunks.empty()) {
            ESC_ABI_CUDA(cudaMemcpyAsync(plan, chunks.data(), chunks.size() * sizeof(Chunk), cudaMemcpyHostToDevice, st));
            ESC_ABI_CUDA(cudaStreamSynchronize(st));
        }
    } catch (const std::bad_alloc&) {
        return ESC_ERR_SHAPE;
    }
    *n_chunks = n;
    return ESC_OK;
}

int esc_adamw_scalars(long long step, double lr, double beta1, double beta2, double weight_decay, double grad_scale, float* scalars_host) {
    if (!scalars_host) return ESC_ERR_NULL;
    if (step < 1 || !(lr >= 0) || !(beta1 >= 0 && beta1 < 1) || !(beta2 >= 0 && beta2 < 1) || !(weight_decay >= 0)) return ESC_ERR_SHAPE;
    scalars_host[0] = (float)(1.0 - lr * weight_decay);
    scalars_host[1] = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
    scalars_host[2] = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    scalars_host[3] = (float)grad_scale;
    return ESC_OK;
}

int esc_adamw_step(const void* plan, long long n_chunks, int param_dtype, int grad_dtype, int states, long long step, double lr, double beta1,
                   double beta2, double eps, double weight_decay, double grad_scale, const float* scalars, const int* skip, void* stream) {
    esc::abi::launches_reset();
    if (!plan) return ESC_ERR_NULL;
    if (!esc::abi::aligned(plan, 256)) return ESC_ERR_WORKSPACE;
    if (n_chunks < 0 || n_chunks > 0x7fffffffLL || !(eps >= 0)) return ESC_ERR_SHAPE;
    if (!known(param_dtype) || !known(grad_dtype) || (states != ESC_STATES_F32 && states != ESC_STATES_E4M3)) return ESC_ERR_UNSUPPORTED;
    if (!esc::abi::aligned(scalars, 4) || !esc::abi::aligned(skip, 4)) return ESC_ERR_ALIGN;
    float s[4];
    const int rc = esc_adamw_scalars(step, lr, beta1, beta2, weight_decay, grad_scale, s);
    if (rc != ESC_OK) return rc;
    if (n_chunks == 0) return ESC_OK;
    const esc::adamw::Hyper h{(float)beta1, (float)(1.0 - beta1), (float)beta2, (float)(1.0 - beta2), (float)eps, s[0], s[1], s[2], s[3]};
    const Chunk* chunks = static_cast<const Chunk*>(plan);
    const unsigned blocks = (unsigned)n_chunks;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (param_dtype == ESC_F32)
        return grad_dtype == ESC_F32 ? launch<float, float>(chunks, blocks, h, scalars, skip, states, st)
                                     : launch<float, __nv_bfloat16>(chunks, blocks, h, scalars, skip, states, st);
    return grad_dtype == ESC_F32 ? launch<__nv_bfloat16, float>(chunks, blocks, h, scalars, skip, states, st)
                                 : launch<__nv_bfloat16, __nv_bfloat16>(chunks, blocks, h, scalars, skip, states, st);
}

}  // extern "C"
