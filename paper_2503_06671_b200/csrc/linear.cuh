// Linear layers of rows: z = x w^T + b, out = act(z) + residual, and their gradients g = grad_out act'(z), gx = g w, gw = g^T x,
// gb = sum of g.  Here: the activations, the sums over rows, and products on the FP32 pipe for operands of any alignment.
#pragma once
#include "common.cuh"

namespace esc { namespace linear {

constexpr int kActNone = 0, kActRelu = 1, kActGelu = 2;

// GELU with the exact normal distribution function; erfc keeps its left tail.
__device__ __forceinline__ float normal_cdf(float z) { return 0.5f * erfcf(z * -0.70710678118654752f); }
__device__ __forceinline__ float act_of(int act, float z) {
    return act == kActGelu ? z * normal_cdf(z) : act == kActRelu ? fmaxf(z, 0.f) : z;
}
__device__ __forceinline__ float act_slope(int act, float z) {
    if (act == kActGelu) return normal_cdf(z) + z * expf(-0.5f * z * z) * 0.39894228040143268f;
    return act == kActRelu ? (z > 0.f ? 1.f : 0.f) : 1.f;
}

template <typename T> struct Layer {
    const T *x, *w, *b;                 // [rows, K], [N, K], [N] or null
    long long x_stride, rows;
    int K, N, act;
    const T* residual;                  // [rows, N] or null
    T *out, *z;                         // [rows, N]; z may be null
    const T *go, *kept;                 // backward: [rows, N]; kept: z of the forward pass (null without an activation)
    T* gx;
    float* part;                        // [splits][N][K]
};

template <typename T> __device__ __forceinline__ float grad_z(const Layer<T>& p, long long row, int n) {
    const float g = Elem<T>::to_f32(p.go[row * p.N + n]);
    return p.act == kActNone ? g : g * act_slope(p.act, Elem<T>::to_f32(p.kept[row * p.N + n]));
}

enum Role { kForward, kGradX, kGradW };

// D[i][j] = sum over c of A(i, c) B(j, c): 64 x 64 of D to a block, 4 x 4 to a thread.  kGradW splits the rows over blockIdx.z.
constexpr int kTile = 64, kDepth = 16;
template <typename T, Role ROLE> __global__ void __launch_bounds__(256) product(const Layer<T> p)
{
    __shared__ float as[kDepth][kTile + 4], bs[kDepth][kTile + 4];
    const long long I = ROLE == kGradW ? p.N : p.rows, c_all = ROLE == kForward ? p.K : ROLE == kGradX ? p.N : p.rows;
    const int J = ROLE == kForward ? p.N : p.K;
    const long long i0 = (long long)blockIdx.x * kTile;
    const int j0 = blockIdx.y * kTile, tid = threadIdx.x, ti = tid / 16, tj = tid % 16;
    const long long c_begin = c_all * blockIdx.z / gridDim.z, c_end = c_all * (blockIdx.z + 1) / gridDim.z;
    float acc[4][4] = {};
    for (long long c0 = c_begin; c0 < c_end; c0 += kDepth) {
        for (int e = tid; e < kTile * kDepth; e += 256) {
            // neighbouring threads read neighbouring values
            const int i = ROLE == kGradW ? e % kTile : e / kDepth, ca = ROLE == kGradW ? e / kTile : e % kDepth;
            const int j = ROLE == kForward ? e / kDepth : e % kTile, cb = ROLE == kForward ? e % kDepth : e / kTile;
            float a = 0.f, b = 0.f;
            if (i0 + i < I && c0 + ca < c_end) {
                if (ROLE == kForward) a = Elem<T>::to_f32(p.x[(i0 + i) * p.x_stride + c0 + ca]);
                else a = ROLE == kGradX ? grad_z(p, i0 + i, (int)(c0 + ca)) : grad_z(p, c0 + ca, (int)(i0 + i));
            }
            if (j0 + j < J && c0 + cb < c_end) {
                if (ROLE == kGradW) b = Elem<T>::to_f32(p.x[(c0 + cb) * p.x_stride + j0 + j]);
                else b = Elem<T>::to_f32(ROLE == kForward ? p.w[(long long)(j0 + j) * p.K + c0 + cb] : p.w[(c0 + cb) * p.K + j0 + j]);
            }
            as[ca][i] = a;
            bs[cb][j] = b;
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < kDepth; ++c) {
            float a[4], b[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) { a[u] = as[c][ti * 4 + u]; b[u] = bs[c][tj * 4 + u]; }
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[u][v] += a[u] * b[v];
        }
        __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const long long i = i0 + ti * 4 + u;
        if (i >= I) break;
        for (int v = 0; v < 4; ++v) {
            const int j = j0 + tj * 4 + v;
            if (j >= J) break;
            float d = acc[u][v];
            if (ROLE == kGradW) p.part[((long long)blockIdx.z * p.N + i) * p.K + j] = d;
            else if (ROLE == kGradX) p.gx[i * p.K + j] = Elem<T>::from_f32(d);
            else {
                if (p.b) d += Elem<T>::to_f32(p.b[j]);
                if (p.z) p.z[i * p.N + j] = Elem<T>::from_f32(d);
                d = act_of(p.act, d);
                if (p.residual) d += Elem<T>::to_f32(p.residual[i * p.N + j]);
                p.out[i * p.N + j] = Elem<T>::from_f32(d);
            }
        }
    }
}

// Column sums of g: a block has 32 columns and every gridDim.y-th run of eight rows; part [gridDim.y][N].
template <typename T> __global__ void __launch_bounds__(256) grad_bias_parts(const Layer<T> p, float* part)
{
    __shared__ float acc[8][32];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, n = blockIdx.x * 32 + lane;
    float s = 0.f;
    if (n < p.N)
        for (long long row = (long long)blockIdx.y * 8 + warp; row < p.rows; row += (long long)gridDim.y * 8) s += grad_z(p, row, n);
    acc[warp][lane] = s;
    __syncthreads();
    if (warp != 0 || n >= p.N) return;
#pragma unroll
    for (int v = 1; v < 8; ++v) s += acc[v][lane];
    part[(size_t)blockIdx.y * p.N + n] = s;
}

// out[e] = sum over `parts` of part[.][e], in order.
template <typename G> __global__ void __launch_bounds__(256) sum_parts(const float* part, int parts, long long count, G* out)
{
    for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < count; e += (long long)gridDim.x * 256) {
        float s = 0.f;
#pragma unroll 8
        for (int i = 0; i < parts; ++i) s += __ldcg(part + (size_t)i * count + e);
        out[e] = Elem<G>::from_f32(s);
    }
}

}}  // namespace esc::linear
