// C ABI of the linear layers: argument checks, kernel selection and launches.
#include "rows.h"

#include <algorithm>

#include "linear.cuh"

namespace {

namespace abi = esc::abi;
namespace lin = esc::linear;
using namespace esc::rows;
using bf16 = __nv_bfloat16;

struct Call {
    const void* x;
    long long x_stride;
    const void* w;
    long long rows;
    int K, N, act, dtype;
    size_t es() const { return abi::elem_size(dtype); }
    Matrix mx() const { return Matrix{x, rows, x_stride, K, es()}; }
    Matrix mw() const { return flat(w, (long long)N * K, es()); }
    Matrix out(const void* p, long long width) const { return Matrix{p, rows, width, width, es()}; }
};

constexpr int kMaxWidth = 1 << 20;

int check_sizes(long long rows, int K, int N, int act, int dtype) {
    if (rows < 0 || K <= 0 || N <= 0) return ESC_ERR_SHAPE;
    if (!known(dtype) || act < ESC_ACT_NONE || act > ESC_ACT_GELU) return ESC_ERR_UNSUPPORTED;
    if (K > kMaxWidth || N > kMaxWidth || rows > 0x7fffffffLL - 4096) return ESC_ERR_UNSUPPORTED;
    return ESC_OK;
}
int check_call(const Call& c) {
    ESC_TRY(check_sizes(c.rows, c.K, c.N, c.act, c.dtype));
    ESC_TRY(check_rows(c.rows, c.K, c.x_stride));
    if (!c.w || (!c.x && c.rows > 0)) return ESC_ERR_NULL;
    for (const void* p : {c.x, c.w})
        if (!abi::aligned(p, c.es())) return ESC_ERR_ALIGN;
    return ESC_OK;
}

template <typename T> lin::Layer<T> layer_of(const Call& c) {
    lin::Layer<T> p{};
    p.x = static_cast<const T*>(c.x); p.w = static_cast<const T*>(c.w);
    p.x_stride = c.x_stride; p.rows = c.rows; p.K = c.K; p.N = c.N; p.act = c.act;
    return p;
}
unsigned tiles(long long n) { return (unsigned)((n + lin::kTile - 1) / lin::kTile); }

// The weights' gradient is summed over as many runs of rows as fill the SMs twice, of 256 rows or more.
int grad_splits(const Call& c) {
    const long long blocks = (long long)tiles(c.N) * tiles(c.K);
    return (int)std::max(1LL, std::min((2LL * abi::sm_count() + blocks - 1) / blocks, (c.rows + 255) / 256));
}
int bias_parts(const Call& c) {
    const long long across = (c.N + 31) / 32;
    return (int)std::max(1LL, std::min((8LL * abi::sm_count() + across - 1) / across, (c.rows + 63) / 64));
}
struct LinearWs { float *part, *bias; size_t bytes; };
LinearWs carve(void* ws, const Call& c) {
    LinearWs w;
    char* base = static_cast<char*>(ws);
    size_t off = 0;
    auto take = [&](size_t bytes) { char* p = base + off; off += abi::round_up(bytes, 256); return p; };
    w.part = reinterpret_cast<float*>(take((size_t)grad_splits(c) * c.N * c.K * sizeof(float)));
    w.bias = reinterpret_cast<float*>(take((size_t)bias_parts(c) * c.N * sizeof(float)));
    w.bytes = off;
    return w;
}

template <typename T> int linear_forward_t(const lin::Layer<T>& p, cudaStream_t st) {
    lin::product<T, lin::kForward><<<dim3(tiles(p.rows), tiles(p.N)), 256, 0, st>>>(p);
    return launched();
}

template <typename G> int launch_sum_parts(const float* part, int parts, long long count, void* out, cudaStream_t st) {
    lin::sum_parts<G><<<(unsigned)std::min<long long>((count + 255) / 256, 8LL * abi::sm_count()), 256, 0, st>>>(part, parts, count, static_cast<G*>(out));
    return launched();
}
int sum_to(const float* part, int parts, long long count, void* out, int grad_dtype, cudaStream_t st) {
    return grad_dtype == ESC_F32 ? launch_sum_parts<float>(part, parts, count, out, st) : launch_sum_parts<bf16>(part, parts, count, out, st);
}

template <typename T> int linear_backward_t(const Call& c, lin::Layer<T> p, void* gw, void* gb, int grad_dtype, const LinearWs& w, cudaStream_t st) {
    if (p.gx) {
        lin::product<T, lin::kGradX><<<dim3(tiles(p.rows), tiles(p.K)), 256, 0, st>>>(p);
        ESC_TRY(launched());
    }
    if (gw) {
        const int splits = grad_splits(c);
        p.part = w.part;
        lin::product<T, lin::kGradW><<<dim3(tiles(p.N), tiles(p.K), splits), 256, 0, st>>>(p);
        ESC_TRY(launched());
        ESC_TRY(sum_to(w.part, splits, (long long)p.N * p.K, gw, grad_dtype, st));
    }
    if (gb) {
        const int parts = bias_parts(c);
        lin::grad_bias_parts<T><<<dim3((p.N + 31) / 32, parts), 256, 0, st>>>(p, w.bias);
        ESC_TRY(launched());
        ESC_TRY(sum_to(w.bias, parts, p.N, gb, grad_dtype, st));
    }
    return ESC_OK;
}

}  // namespace

extern "C" {

int esc_linear_forward(const void* x, long long x_stride, const void* weight, const void* bias, int activation, const void* residual, void* out, void* z,
                       long long rows, int K, int N, int dtype, void* stream) {
    abi::launches_reset();
    const Call c{x, x_stride, weight, rows, K, N, activation, dtype};
    ESC_TRY(check_call(c));
    if (!out && rows > 0) return ESC_ERR_NULL;
    for (const void* p : {bias, residual, static_cast<const void*>(out), static_cast<const void*>(z)})
        if (!abi::aligned(p, c.es())) return ESC_ERR_ALIGN;
    const Matrix read[] = {c.mx(), c.mw(), flat(bias, N, c.es()), c.out(residual, N)};
    for (const Matrix& i : read)
        if (touch(c.out(out, N), i) || touch(c.out(z, N), i)) return ESC_ERR_ALIAS;
    if (touch(c.out(out, N), c.out(z, N))) return ESC_ERR_ALIAS;
    if (rows == 0) return ESC_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto go = [&](auto zero_value) {
        using T = decltype(zero_value);
        lin::Layer<T> p = layer_of<T>(c);
        p.b = static_cast<const T*>(bias); p.residual = static_cast<const T*>(residual);
        p.out = static_cast<T*>(out); p.z = static_cast<T*>(z);
        return linear_forward_t<T>(p, st);
    };
    return dtype == ESC_F32 ? go(float{}) : go(bf16{});
}

size_t esc_linear_backward_workspace_bytes(long long rows, int K, int N, int activation, int dtype) {
    if (check_sizes(rows, K, N, activation, dtype) != ESC_OK) return 0;
    return carve(nullptr, Call{nullptr, K, nullptr, rows, K, N, activation, dtype}).bytes;
}

int esc_linear_backward(const void* x, long long x_stride, const void* weight, const void* z, int activation, const void* grad_out, void* grad_x,
                        void* grad_weight, void* grad_bias, long long rows, int K, int N, int dtype, int grad_dtype, void* workspace,
                        size_t workspace_bytes, void* stream) {
    abi::launches_reset();
    const Call c{x, x_stride, weight, rows, K, N, activation, dtype};
    ESC_TRY(check_call(c));
    if (!known(grad_dtype)) return ESC_ERR_UNSUPPORTED;
    if (rows > 0 && (!grad_out || (activation != ESC_ACT_NONE && !z))) return ESC_ERR_NULL;
    const size_t gs = abi::elem_size(grad_dtype);
    for (const void* p : {z, grad_out, static_cast<const void*>(grad_x)})
        if (!abi::aligned(p, c.es())) return ESC_ERR_ALIGN;
    if (!abi::aligned(grad_weight, gs) || !abi::aligned(grad_bias, gs)) return ESC_ERR_ALIGN;
    const Matrix written[] = {c.out(grad_x, K), flat(grad_weight, (long long)N * K, gs), flat(grad_bias, N, gs)};
    const Matrix read[] = {c.mx(), c.mw(), c.out(activation != ESC_ACT_NONE ? z : nullptr, N), c.out(grad_out, N)};
    for (const Matrix& o : written)
        for (const Matrix& i : read)
            if (touch(o, i)) return ESC_ERR_ALIAS;
    if (touch(written[0], written[1]) || touch(written[0], written[2]) || touch(written[1], written[2])) return ESC_ERR_ALIAS;
    const LinearWs w = carve(workspace, c);
    if (!workspace || !abi::aligned(workspace, 256) || workspace_bytes < w.bytes) return ESC_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0) {
        ESC_TRY(zero(grad_weight, (size_t)N * K * gs, st));
        return zero(grad_bias, N * gs, st);
    }
    auto go = [&](auto zero_value) {
        using T = decltype(zero_value);
        lin::Layer<T> p = layer_of<T>(c);
        p.go = static_cast<const T*>(grad_out); p.kept = static_cast<const T*>(z); p.gx = static_cast<T*>(grad_x);
        return linear_backward_t<T>(c, p, grad_weight, grad_bias, grad_dtype, w, st);
    };
    return dtype == ESC_F32 ? go(float{}) : go(bf16{});
}

}  // extern "C"
