// Linear layers of rows: z = x w^T + b, out = act(z) + residual, and their gradients g = grad_out act'(z), gx = g w, gw = g^T x,
// gb = sum of g.  Here: the activations, the sums over rows, and products on the FP32 pipe for operands of any alignment.
#pragma once
#include "common.cuh"

namespace esc { namespace linear {

constexpr int kActNone = 0, kActRelu = 1, kActGelu = 2;

// With x = |z|, e = exp(-z^2 / 2) and Q(x) = Phi(-x) / e, which falls smoothly from 1/2:
//
//   GELU      z Phi(z) = max(z, 0) - x e Q(x)
//   its slope Phi(z) + z phi(z) = [z >= 0] + sign(z) e (x / sqrt(2 pi) - Q(x))
//
// Q is a polynomial in t = 1 / (1 + p x) without a constant term (the form that Hastings gave the error function), fitted here by least
// squares with Lawson's weights to erfcx(x / sqrt 2) / 2 on [0, 15]: nine terms, 2.6e-8 relative at most, in the left tail too.  One 2^x and
// one reciprocal a value: against erfcf and expf a third of the instructions (320x180 from 192 to 384 channels and the gradients of
// 64 x 64x64 were bound by those, 86 us each).  GELU that is rounded to bf16 takes six terms: 1e-5 relative at most, less than the 2^-16 by
// which half a step of bf16 above a power of two falls short of 2^-8.
__device__ __forceinline__ float pow2(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float inverse(float v) { float r; asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float min_nan(float a, float b) { float r; asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }

struct Gauss { float x, e, q; };
template <bool NINE> __device__ __forceinline__ Gauss gauss(float z) {
    Gauss g;
    g.x = min_nan(fabsf(z), 30.f);                                 // beyond, e is zero in fp32: 0 times infinity does not come up
    g.e = pow2(g.x * g.x * -0.72134752044f);
    const float t = inverse(fmaf(g.x, NINE ? 0.345f : 0.31f, 1.f));
    float q;
    if (NINE) {
        q = fmaf(-0.0279335122f, t, 0.143238278f);
        q = fmaf(q, t, -0.267236026f);
        q = fmaf(q, t, 0.183022695f);
        q = fmaf(q, t, -0.0349471461f);
        q = fmaf(q, t, 0.110766168f);
        q = fmaf(q, t, 0.117478006f);
        q = fmaf(q, t, 0.137990677f);
        q = fmaf(q, t, 0.137620871f);
    } else {
        q = fmaf(-0.073929169f, t, 0.180450428f);
        q = fmaf(q, t, 0.0157446193f);
        q = fmaf(q, t, 0.133429833f);
        q = fmaf(q, t, 0.120441264f);
        q = fmaf(q, t, 0.123860703f);
    }
    g.q = q * t;
    return g;
}
// GELU for results of type T.
template <typename T> __device__ __forceinline__ float gelu(float z) {
    const Gauss g = gauss<sizeof(T) == 4>(z);
    return fmaf(-g.x, g.e * g.q, max_nan(z, 0.f));
}
__device__ __forceinline__ float gelu_slope(float z) {
    const Gauss g = gauss<true>(z);
    const float h = g.e * fmaf(g.x, 0.39894228040f, -g.q);
    return z >= 0.f ? 1.f + h : -h;
}
__device__ __forceinline__ float act_slope(int act, float z) { return act == kActGelu ? gelu_slope(z) : act == kActRelu ? (z > 0.f ? 1.f : 0.f) : 1.f; }

template <typename T> struct Layer {
    const T *x, *w, *b;                 // [rows, K], [N, K], [N] or null
    long long x_stride, rows;
    int K, N, act;
    const T* residual;                  // [rows, N] or null
    T *out, *z;                         // [rows, N]; z may be null
    const T *go, *kept;                 // backward: [rows, N]; kept: z of the forward pass (null without an activation)
    T* gx;
};

enum Role { kForward, kGradX, kGradW };

// g = go act'(z) and its column sums, as far as they are asked for: g [rows, g_ld] of the type (rounded: the operand that two products
// read), part [gridDim.y][N] fp32 sums of the unrounded g.  A thread has V neighbouring columns and every so many rows; a block has
// min(N / V, 32) such pieces of a row.  V > 1: rows are whole aligned pieces.
template <typename T, int V> __device__ __forceinline__ void load_values(const T* p, float* f) {
    if constexpr (V == 1) f[0] = Elem<T>::to_f32(*p);
    else unpack16<T>(*reinterpret_cast<const uint4*>(p), f);
}
template <typename T, int V> __global__ void __launch_bounds__(256) grad_z_sums(const Layer<T> p, T* g, long long g_ld, float* part)
{
    __shared__ float acc[256 * V];
    const int all = p.N / V, across = all < 32 ? all : 32, down = 256 / across;
    const int col = threadIdx.x % across, v = blockIdx.x * across + col, r = threadIdx.x / across;
    float sum[V] = {};
    if (r < down && v < all) {
        const long long step = (long long)gridDim.y * down;
#pragma unroll 2
        for (long long row = (long long)blockIdx.y * down + r; row < p.rows; row += step) {
            const long long at = row * p.N + v * V;
            float f[V];
            load_values<T, V>(p.go + at, f);
            if (p.act != kActNone) {
                float z[V];
                load_values<T, V>(p.kept + at, z);
#pragma unroll
                for (int e = 0; e < V; ++e) f[e] *= act_slope(p.act, z[e]);
            }
            if (g) {
                T* to = g + row * g_ld + v * V;
                if constexpr (V == 1) *to = Elem<T>::from_f32(f[0]);
                else if constexpr (sizeof(T) == 4) *reinterpret_cast<float4*>(to) = make_float4(f[0], f[1], f[2], f[3]);
                else {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
                        w[e] = *reinterpret_cast<const uint32_t*>(&h);
                    }
                    *reinterpret_cast<uint4*>(to) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] += f[e];
        }
    }
    if (!part) return;
#pragma unroll
    for (int e = 0; e < V; ++e) acc[e * 256 + threadIdx.x] = sum[e];
    __syncthreads();
    for (int c = threadIdx.x; c < across * V; c += 256) {
        const int n = blockIdx.x * across * V + c;
        if (n >= p.N) break;
        float s = 0.f;
        for (int q = 0; q < down; ++q) s += acc[c % V * 256 + q * across + c / V];
        part[(size_t)blockIdx.y * p.N + n] = s;
    }
}

// Partial sums [parts][count], to be added up: the weights' and the bias' gradients in one launch, either may be empty.
struct Parts { const float* p; int parts; long long count; };

// Many parts: 32 sums to a block, a warp takes every eighth part, the warps are added in order.  Up to kFewParts: a thread has four sums.
constexpr int kFewParts = 8;
inline __host__ __device__ long long sum_blocks(const Parts& t) { return t.parts <= kFewParts ? (t.count + 1023) / 1024 : (t.count + 31) / 32; }
template <typename G> __global__ void __launch_bounds__(256) sum_parts(const Parts w, const Parts b, G* gw, G* gb)
{
    __shared__ float acc[8][32];
    const long long ours = sum_blocks(w);
    const bool of_b = blockIdx.x >= ours;
    const Parts t = of_b ? b : w;
    const long long block = blockIdx.x - (of_b ? ours : 0);
    G* out = of_b ? gb : gw;
    if (t.parts <= kFewParts) {
        const long long e = block * 1024 + threadIdx.x * 4;
        float s[4] = {};
        for (int i = 0; i < t.parts; ++i) {
            const float* at = t.p + (size_t)i * t.count + e;
            if (t.count % 4 == 0 && e < t.count) {
                const float4 v = __ldcg(reinterpret_cast<const float4*>(at));
                s[0] += v.x; s[1] += v.y; s[2] += v.z; s[3] += v.w;
            } else {
                for (int u = 0; u < 4 && e + u < t.count; ++u) s[u] += __ldcg(at + u);
            }
        }
        for (int u = 0; u < 4 && e + u < t.count; ++u) out[e + u] = Elem<G>::from_f32(s[u]);
        return;
    }
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const long long e = block * 32 + lane;
    float s = 0.f;
    if (e < t.count) {
#pragma unroll 8
        for (int i = warp; i < t.parts; i += 8) s += __ldcg(t.p + (size_t)i * t.count + e);
    }
    acc[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || e >= t.count) return;
#pragma unroll
    for (int v = 1; v < 8; ++v) s += acc[v][lane];
    out[e] = Elem<G>::from_f32(s);
}

}}  // namespace esc::linear
