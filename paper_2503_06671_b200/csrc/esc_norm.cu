// C ABI of the layer norm: argument checks, kernel selection and launches.
#include "rows.h"

#include <algorithm>
#include <cmath>
#include <iterator>

#include "layer_norm.cuh"

namespace {

namespace abi = esc::abi;
namespace ln = esc::norm;
using namespace esc::rows;
using bf16 = __nv_bfloat16;

// How a row is spread: vectors of `vec` values, `nv` of them to each of `g` threads; nv = 0: too long for a block's registers.
struct Spread { int vec, nv, g; };
template <typename T> Spread spread(int C, bool sixteen, bool pairs) {
    constexpr int V = esc::Elem<T>::kVec;
    const int vec = sixteen ? V : pairs ? 2 : 1, items = C / vec;
    if (sixteen && C <= 512) {
        if (items <= 4) return {vec, 1, items == 3 ? 4 : items};
        // as few idle lanes as possible, then few vectors to a thread
        int best = 1 << 30;
        Spread s{vec, 0, 0};
        for (int g = 32; g >= 4; g /= 2) {
            const int nv = (items + g - 1) / g;
            if (nv <= 4 && g * nv < best) { best = g * nv; s = Spread{vec, nv, g}; }
        }
        return s;
    }
    const int most = sixteen ? 4 : 8;
    for (int g : {32, ln::kThreads}) {
        if (g == 32 && C > 512) continue;
        const int nv = (items + g - 1) / g;
        if (nv <= most) return {vec, nv <= 1 ? 1 : nv <= 2 ? 2 : nv <= 4 ? 4 : 8, g};
    }
    return {vec, 0, 0};
}

template <typename T, int VEC, int NV, int G, bool BACK> int launch_norm(const ln::Rows<T>& p, int blocks, cudaStream_t st) {
    if constexpr (BACK) ln::backward<T, VEC, NV, G><<<blocks, ln::kThreads, G <= 32 && p.part ? (size_t)(ln::kThreads / 32) * 2 * p.C * sizeof(float) : 0, st>>>(p);
    else ln::forward<T, VEC, NV, G><<<blocks, ln::kThreads, 0, st>>>(p);
    return launched();
}
template <typename T, int VEC, int G, bool BACK> int launch_norm_nv(const Spread& s, const ln::Rows<T>& p, int blocks, cudaStream_t st) {
    constexpr bool wide = VEC == esc::Elem<T>::kVec;
    switch (s.nv) {
        case 1: return launch_norm<T, VEC, 1, G, BACK>(p, blocks, st);
        case 2: return launch_norm<T, VEC, 2, G, BACK>(p, blocks, st);
        case 3: return launch_norm<T, VEC, wide ? 3 : 4, G, BACK>(p, blocks, st);
        case 4: return launch_norm<T, VEC, 4, G, BACK>(p, blocks, st);
        default: return launch_norm<T, VEC, wide ? 4 : 8, G, BACK>(p, blocks, st);
    }
}
template <typename T, bool BACK> int launch_norm_any(const Spread& s, const ln::Rows<T>& p, int blocks, cudaStream_t st) {
    constexpr int V = esc::Elem<T>::kVec;
    if (s.vec == V) {
        switch (s.g) {
            case 1: return launch_norm<T, V, 1, 1, BACK>(p, blocks, st);
            case 2: return launch_norm<T, V, 1, 2, BACK>(p, blocks, st);
            case 4: return launch_norm_nv<T, V, 4, BACK>(s, p, blocks, st);
            case 8: return launch_norm_nv<T, V, 8, BACK>(s, p, blocks, st);
            case 16: return launch_norm_nv<T, V, 16, BACK>(s, p, blocks, st);
            case 32: return launch_norm_nv<T, V, 32, BACK>(s, p, blocks, st);
            default: return launch_norm_nv<T, V, ln::kThreads, BACK>(s, p, blocks, st);
        }
    }
    if constexpr (V == 8)
        if (s.vec == 2) return s.g == 32 ? launch_norm_nv<T, 2, 32, BACK>(s, p, blocks, st) : launch_norm_nv<T, 2, ln::kThreads, BACK>(s, p, blocks, st);
    return s.g == 32 ? launch_norm_nv<T, 1, 32, BACK>(s, p, blocks, st) : launch_norm_nv<T, 1, ln::kThreads, BACK>(s, p, blocks, st);
}

// Blocks of the backward pass at most: each leaves a partial sum of every column.
int norm_parts(long long rows, int per_sm = 4) { return (int)std::max(1LL, std::min<long long>(rows, (long long)per_sm * abi::sm_count())); }
// Of the wide kernels: the blocks that share a column's rows, one where there are more columns than SMs could have blocks for.
int wide_across(int C) { return (C + ln::kThreads - 1) / ln::kThreads; }
int wide_parts(long long rows, int C) { return std::max(1, norm_parts(rows) / wide_across(C)); }
bool long_row(int C) { return C > ln::kThreads * 8; }       // may need the wide kernels: C odd
bool longest_row(int C) { return C > ln::kThreads * 4 * esc::Elem<bf16>::kVec; }   // always does, whatever its type and alignment
size_t norm_stats_offset(long long rows, int C) {
    const size_t parts = longest_row(C) ? wide_parts(rows, C) : norm_parts(rows);
    return abi::round_up(parts * 2 * C * sizeof(float), 256);
}
size_t norm_ws_bytes(long long rows, int C) { return norm_stats_offset(rows, C) + (long_row(C) ? abi::round_up((size_t)rows * (sizeof(float2) + sizeof(float)), 256) : 0); }

template <typename T> bool all_aligned(const ln::Rows<T>& p, size_t bytes) {
    const void* pointers[] = {p.x, p.weight, p.bias, p.y, p.gy, p.skip, p.gx};
    const long long strides[] = {p.x_stride, p.y_stride, p.C};
    return std::all_of(std::begin(pointers), std::end(pointers), [&](const void* q) { return abi::aligned(q, bytes); }) &&
           std::all_of(std::begin(strides), std::end(strides), [&](long long s) { return (size_t)s * sizeof(T) % bytes == 0; });
}

template <typename T> int norm_forward_t(const ln::Rows<T>& p, cudaStream_t st) {
    const Spread s = spread<T>(p.C, all_aligned(p, 16), sizeof(T) == 2 && all_aligned(p, 4));
    const long long most = 8LL * abi::sm_count();
    if (s.nv == 0) {
        ln::forward_wide<T><<<(unsigned)std::min(p.rows, most), ln::kThreads, 0, st>>>(p);
        return launched();
    }
    const long long per = ln::kThreads / s.g;
    return launch_norm_any<T, false>(s, p, (int)std::min((p.rows + per - 1) / per, most), st);
}

int launch_sum_columns(const float* part, int parts, int C, int grad_dtype, void* gw, void* gb, cudaStream_t st) {
    const unsigned blocks = (unsigned)((2LL * C + 31) / 32);
    if (grad_dtype == ESC_F32) return launch_behind(ln::sum_columns<float>, blocks, esc::kSumThreads, st, 0, part, parts, C, static_cast<float*>(gw), static_cast<float*>(gb));
    return launch_behind(ln::sum_columns<bf16>, blocks, esc::kSumThreads, st, 0, part, parts, C, static_cast<bf16*>(gw), static_cast<bf16*>(gb));
}

template <typename T> int norm_backward_t(ln::Rows<T> p, bool columns, int grad_dtype, void* gw, void* gb, char* ws, cudaStream_t st) {
    const Spread s = spread<T>(p.C, all_aligned(p, 16), sizeof(T) == 2 && all_aligned(p, 4));
    const int most = norm_parts(p.rows);
    p.part = columns ? reinterpret_cast<float*>(ws) : nullptr;
    int parts;
    if (s.nv == 0) {
        float2* stats = reinterpret_cast<float2*>(ws + norm_stats_offset(p.rows, p.C));
        float* from = reinterpret_cast<float*>(stats + p.rows);
        ln::backward_wide<T><<<most, ln::kThreads, 0, st>>>(p, stats, from);
        ESC_TRY(launched());
        parts = wide_parts(p.rows, p.C);
        if (columns) {
            ln::columns_wide<T><<<dim3(wide_across(p.C), parts), ln::kThreads, 0, st>>>(p, stats, from);
            ESC_TRY(launched());
        }
    } else {
        const long long per = ln::kThreads / s.g;
        parts = (int)std::min<long long>((p.rows + per - 1) / per, norm_parts(p.rows, ln::back_blocks(s.vec * s.nv)));
        ESC_TRY((launch_norm_any<T, true>(s, p, parts, st)));
    }
    return columns ? launch_sum_columns(p.part, parts, p.C, grad_dtype, gw, gb, st) : ESC_OK;
}

int check_norm(const void* x, long long x_stride, const void* weight, const void* bias, float eps, long long rows, int C, int dtype) {
    ESC_TRY(check_rows(rows, C, x_stride));
    if (C > ln::kMaxChannels || !known(dtype) || !(eps >= 0.f) || std::isinf(eps)) return ESC_ERR_UNSUPPORTED;
    if (!x && rows > 0) return ESC_ERR_NULL;
    for (const void* p : {x, weight, bias})
        if (!abi::aligned(p, abi::elem_size(dtype))) return ESC_ERR_ALIGN;
    return ESC_OK;
}

}  // namespace

extern "C" {

int esc_layer_norm_forward(const void* x, long long x_stride, const void* weight, const void* bias, float eps, void* y, long long y_stride,
                           long long rows, int C, int dtype, void* stream) {
    abi::launches_reset();
    ESC_TRY(check_norm(x, x_stride, weight, bias, eps, rows, C, dtype));
    ESC_TRY(check_rows(rows, C, y_stride));
    const size_t es = abi::elem_size(dtype);
    if (!y && rows > 0) return ESC_ERR_NULL;
    if (!abi::aligned(y, es)) return ESC_ERR_ALIGN;
    const Matrix out{y, rows, y_stride, C, es};
    if (touch(out, Matrix{x, rows, x_stride, C, es}) || touch(out, flat(weight, C, es)) || touch(out, flat(bias, C, es))) return ESC_ERR_ALIAS;
    if (rows == 0) return ESC_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto go = [&](auto zero_value) {
        using T = decltype(zero_value);
        ln::Rows<T> p{};
        p.x = static_cast<const T*>(x); p.x_stride = x_stride; p.rows = rows; p.C = C; p.eps = eps;
        p.weight = static_cast<const T*>(weight); p.bias = static_cast<const T*>(bias);
        p.y = static_cast<T*>(y); p.y_stride = y_stride;
        return norm_forward_t<T>(p, st);
    };
    return dtype == ESC_F32 ? go(float{}) : go(bf16{});
}

size_t esc_layer_norm_backward_workspace_bytes(long long rows, int C) {
    if (check_rows(rows, C, C) != ESC_OK || C > ln::kMaxChannels) return 0;
    return norm_ws_bytes(rows, C);
}

int esc_layer_norm_backward(const void* x, long long x_stride, const void* weight, float eps, const void* grad_y, const void* grad_skip, void* grad_x,
                            void* grad_weight, void* grad_bias, long long rows, int C, int dtype, int grad_dtype, void* workspace,
                            size_t workspace_bytes, void* stream) {
    abi::launches_reset();
    ESC_TRY(check_norm(x, x_stride, weight, nullptr, eps, rows, C, dtype));
    if (!known(grad_dtype)) return ESC_ERR_UNSUPPORTED;
    if (((!grad_y || !grad_x) && rows > 0) || (grad_weight && !weight)) return ESC_ERR_NULL;
    const size_t es = abi::elem_size(dtype), gs = abi::elem_size(grad_dtype);
    for (const void* p : {grad_y, grad_skip, static_cast<const void*>(grad_x)})
        if (!abi::aligned(p, es)) return ESC_ERR_ALIGN;
    if (!abi::aligned(grad_weight, gs) || !abi::aligned(grad_bias, gs)) return ESC_ERR_ALIGN;
    const Matrix written[] = {Matrix{grad_x, rows, C, C, es}, flat(grad_weight, C, gs), flat(grad_bias, C, gs)};
    const Matrix read[] = {Matrix{x, rows, x_stride, C, es}, flat(weight, C, es), Matrix{grad_y, rows, C, C, es}, Matrix{grad_skip, rows, C, C, es}};
    for (const Matrix& o : written)
        for (const Matrix& i : read)
            if (touch(o, i)) return ESC_ERR_ALIAS;
    if (touch(written[0], written[1]) || touch(written[0], written[2]) || touch(written[1], written[2])) return ESC_ERR_ALIAS;
    if (!workspace || !abi::aligned(workspace, 256) || workspace_bytes < norm_ws_bytes(rows, C)) return ESC_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0) {
        ESC_TRY(zero(grad_weight, C * gs, st));
        return zero(grad_bias, C * gs, st);
    }
    auto go = [&](auto zero_value) {
        using T = decltype(zero_value);
        ln::Rows<T> p{};
        p.x = static_cast<const T*>(x); p.x_stride = x_stride; p.rows = rows; p.C = C; p.eps = eps; p.y_stride = C;
        p.weight = static_cast<const T*>(weight);
        p.gy = static_cast<const T*>(grad_y); p.skip = static_cast<const T*>(grad_skip); p.gx = static_cast<T*>(grad_x);
        return norm_backward_t<T>(p, grad_weight || grad_bias, grad_dtype, grad_weight, grad_bias, static_cast<char*>(workspace), st);
    };
    return dtype == ESC_F32 ? go(float{}) : go(bf16{});
}

}  // extern "C"
