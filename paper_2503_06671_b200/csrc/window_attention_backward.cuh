// Backward pass of the window self-attention (window_attention.cuh).  With go = dL/dout and p recomputed from lse:
//
//   D[i]     = go[i] . out[i]                      dp[i,j] = go[i] . v[j]
//   ds[i,j]  = p[i,j] (dp[i,j] - D[i])             (dL/ds; the bias enters s directly)
//   g_q[i]   = scale sum_j ds[i,j] k[j]            g_k[j]  = scale sum_i ds[i,j] q[i]
//   g_v[j]   = sum_i p[i,j] go[i]                  g_table[b,h] = sum of ds over all windows' pairs of bucket b
//
// Every sum has a fixed order.  A query without keys (lse = -inf) has p = 0 and so takes and gives nothing.
#pragma once
#include "window_attention.cuh"

namespace esc { namespace winatt { namespace bwd {

// D, in [B][heads][H][W] like lse.  Bound: HBM, go and out are read once.
constexpr int kDotThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kDotThreads)
row_dots(const T* __restrict__ go, const T* __restrict__ out, long long pixels, long long hw, int heads, int d, float* __restrict__ dots) {
    constexpr int V = Elem<T>::kVec;
    const bool wide = d % V == 0;
    for (long long e = (long long)blockIdx.x * kDotThreads + threadIdx.x; e < pixels * heads; e += (long long)gridDim.x * kDotThreads) {
        const long long pixel = e / heads;
        const int head = (int)(e - pixel * heads);
        const T *a = go + e * d, *b = out + e * d;
        float sum = 0.0f;
        if (wide) {
            for (int c = 0; c < d; c += V) {
                float x[V], y[V];
                unpack16<T>(*reinterpret_cast<const uint4*>(a + c), x);
                unpack16<T>(*reinterpret_cast<const uint4*>(b + c), y);
#pragma unroll
                for (int i = 0; i < V; ++i) sum = fmaf(x[i], y[i], sum);
            }
        } else {
            for (int c = 0; c < d; ++c) sum = fmaf(Elem<T>::to_f32(a[c]), Elem<T>::to_f32(b[c]), sum);
        }
        const long long image = pixel / hw;
        dots[(image * heads + head) * hw + pixel - image * hw] = sum;
    }
}

// What the backward kernels need beyond Maps.
template <typename T> struct Grads {
    const T* go;                                   // dense
    const float *lse, *dots;
    T *g_q, *g_k, *g_v;                            // pixels `stride` values apart
    float* part;                                   // [groups][heads][offsets] sums of ds, or null
    int windows, groups;
};
template <typename T> __device__ __forceinline__ long long row_of(const Maps<T>& m, const Window& w, int head, long long pixel) {
    const long long hw = (long long)m.H * m.W;
    return ((long long)w.b * m.heads + head) * hw + pixel - w.b * hw;
}
// 2^(c s' - this) is p; +inf where the row has no keys.
__device__ __forceinline__ float base_of(float lse) { return lse == -INFINITY ? INFINITY : lse * kLog2e; }

// ---- fp32: CUDA cores -----------------------------------------------------------------------------------------------------
// Two kernels, so that every gradient is a sum in one thread's registers: in the first a thread has a key (k, v and their gradients
// in registers) and the queries pass by, in the second it has a query.  A row of 64 channels is shared by two neighbouring lanes.
// Bound: the FP32 pipe, 7 D multiply-adds per pair.
namespace f32 {
using winatt::f32::kThreads;
using winatt::f32::stage_rows;
constexpr int kRows = winatt::f32::kKeys;
__host__ __device__ constexpr int lanes_of(int D) { return D > 32 ? 2 : 1; }

template <int D> struct Lane {                     // a thread's share of a row
    static constexpr int S = lanes_of(D), N = D / S;
    static __device__ __forceinline__ int row() { return threadIdx.x / S; }
    static __device__ __forceinline__ int first() { return threadIdx.x % S * N; }
    static __device__ __forceinline__ int rows() { return blockDim.x / S; }
    static __device__ __forceinline__ void load(const float* __restrict__ src, int d, float* f) {
#pragma unroll
        for (int c = 0; c < N; ++c) f[c] = first() + c < d ? src[first() + c] : 0.0f;
    }
    static __device__ __forceinline__ void store(float* __restrict__ dst, int d, const float* f, float by) {
#pragma unroll
        for (int c = 0; c < N; ++c)
            if (first() + c < d) dst[first() + c] = f[c] * by;
    }
    static __device__ __forceinline__ float dot(const float* f, const float* row, float sum) {
        const float4* r = reinterpret_cast<const float4*>(row + first());
#pragma unroll
        for (int c = 0; c < N / 4; ++c) {
            const float4 v = r[c];
            sum = fmaf(f[4 * c], v.x, sum); sum = fmaf(f[4 * c + 1], v.y, sum);
            sum = fmaf(f[4 * c + 2], v.z, sum); sum = fmaf(f[4 * c + 3], v.w, sum);
        }
        if (S == 2) sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        return sum;
    }
    static __device__ __forceinline__ void add(float* f, const float* row, float by) {
        const float4* r = reinterpret_cast<const float4*>(row + first());
#pragma unroll
        for (int c = 0; c < N / 4; ++c) {
            const float4 v = r[c];
            f[4 * c] = fmaf(by, v.x, f[4 * c]); f[4 * c + 1] = fmaf(by, v.y, f[4 * c + 1]);
            f[4 * c + 2] = fmaf(by, v.z, f[4 * c + 2]); f[4 * c + 3] = fmaf(by, v.w, f[4 * c + 3]);
        }
    }
};

template <int D>
__global__ void __launch_bounds__(kThreads)
grad_kv(Maps<float> m, Grads<float> g, int tiles) {
    using L = Lane<D>;
    extern __shared__ __align__(16) float smem[];
    float *qs = smem, *gs = qs + kRows * D, *base = gs + kRows * D, *dots = base + kRows;
    int* as = reinterpret_cast<int*>(dots + kRows);
    float* table = reinterpret_cast<float*>(as + kRows);
    int id = blockIdx.x;
    const int tile = id % tiles; id /= tiles;
    const int head = id % m.heads;
    const Window w = window_at(m, id / m.heads);
    const int n = w.tokens(), pitch = 2 * m.ww - 1, first = tile * L::rows();
    if (first >= n) return;
    stage_table(m, head, table);
    const float c = m.scale * kLog2e;
    const int j = min(first + L::row(), n - 1);
    const long long pixel = pixel_of(m, w, j), at = pixel * m.stride + (long long)head * m.d;
    const int b = j / w.w * pitch + j % w.w;
    float k[L::N], v[L::N], gk[L::N], gv[L::N];
    L::load(m.k + at, m.d, k);
    L::load(m.v + at, m.d, v);
#pragma unroll
    for (int x = 0; x < L::N; ++x) gk[x] = gv[x] = 0.0f;
    for (int row = 0; row < n; row += kRows) {
        __syncthreads();
        stage_rows<D>(m, m.q, m.stride, w, head, row, qs);
        stage_rows<D>(m, g.go, (long long)m.heads * m.d, w, head, row, gs);
        for (int r = threadIdx.x; r < kRows; r += blockDim.x) {
            const int i = row + r, y = i / w.w;
            const long long p = i < n ? row_of(m, w, head, pixel_of(m, w, i)) : 0;
            as[r] = i < n ? (y + m.wh - 1) * pitch + i - y * w.w + m.ww - 1 : (m.wh - 1) * pitch + m.ww - 1;
            base[r] = i < n ? base_of(g.lse[p]) : INFINITY;
            dots[r] = i < n ? g.dots[p] : 0.0f;
        }
        __syncthreads();
        const int rows = min(kRows, n - row);
        for (int r = 0; r < rows; ++r) {
            const float s = L::dot(k, qs + r * D, 0.0f) + table[as[r] - b];
            const float p = ex2(fmaf(s, c, -base[r])), dp = L::dot(v, gs + r * D, 0.0f);
            L::add(gv, gs + r * D, p);
            L::add(gk, qs + r * D, p * (dp - dots[r]));
        }
    }
    if (first + L::row() < n) {
        L::store(g.g_k + at, m.d, gk, m.scale);
        L::store(g.g_v + at, m.d, gv, 1.0f);
    }
}

// Also the sums for the table's gradient: a block keeps one copy of the head's offsets for each warp over all tiles of queries that
// it takes.  At one step the lanes of a warp have different queries and one key, so all their offsets differ.
template <int D>
__global__ void __launch_bounds__(kThreads)
grad_q(Maps<float> m, Grads<float> g, int tiles) {
    using L = Lane<D>;
    extern __shared__ __align__(16) float smem[];
    float *ks = smem, *vs = ks + kRows * D;
    int* bs = reinterpret_cast<int*>(vs + kRows * D);
    float* table = reinterpret_cast<float*>(bs + kRows);
    const int pitch = 2 * m.ww - 1, offsets = (2 * m.wh - 1) * pitch, warps = blockDim.x / 32;
    float *sums = table + offsets, *mine = sums + threadIdx.x / 32 * offsets;
    const int head = blockIdx.x % m.heads, group = blockIdx.x / m.heads;
    stage_table(m, head, table);
    if (g.part)
        for (int o = threadIdx.x; o < offsets * warps; o += blockDim.x) sums[o] = 0.0f;
    const float c = m.scale * kLog2e;
    for (int unit = group; unit < g.windows * tiles; unit += g.groups) {
        const Window w = window_at(m, unit / tiles);
        const int n = w.tokens(), first = unit % tiles * L::rows();
        if (first >= n) continue;
        const bool own = first + L::row() < n;
        const int i = min(first + L::row(), n - 1);
        const long long pixel = pixel_of(m, w, i), at = pixel * m.stride + (long long)head * m.d, row = row_of(m, w, head, pixel);
        const int a = (i / w.w + m.wh - 1) * pitch + i % w.w + m.ww - 1;
        const float base = own ? base_of(g.lse[row]) : INFINITY, dot = own ? g.dots[row] : 0.0f;
        float q[L::N], go[L::N], gq[L::N];
        L::load(m.q + at, m.d, q);
        L::load(g.go + (pixel * m.heads + head) * m.d, m.d, go);
#pragma unroll
        for (int x = 0; x < L::N; ++x) gq[x] = 0.0f;
        for (int key = 0; key < n; key += kRows) {
            __syncthreads();
            stage_rows<D>(m, m.k, m.stride, w, head, key, ks);
            stage_rows<D>(m, m.v, m.stride, w, head, key, vs);
            for (int r = threadIdx.x; r < kRows; r += blockDim.x) {
                const int j = key + r, y = j / w.w;
                bs[r] = j < n ? y * pitch + j - y * w.w : 0;
            }
            __syncthreads();
            const int rows = min(kRows, n - key);
            for (int r = 0; r < rows; ++r) {
                const int o = a - bs[r];
                const float s = L::dot(q, ks + r * D, 0.0f) + table[o];
                const float p = ex2(fmaf(s, c, -base)), ds = p * (L::dot(go, vs + r * D, 0.0f) - dot);
                L::add(gq, ks + r * D, ds);
                if (g.part && own && L::first() == 0) mine[o] += ds;
                __syncwarp();                      // the next key's offsets are the neighbours'
            }
        }
        if (own) L::store(g.g_q + at, m.d, gq, m.scale);
    }
    if (!g.part) return;
    __syncthreads();
    for (int o = threadIdx.x; o < offsets; o += blockDim.x) {
        float sum = 0.0f;
        for (int x = 0; x < warps; ++x) sum += sums[x * offsets + o];
        g.part[((size_t)group * m.heads + head) * offsets + o] = sum;
    }
}

}  // namespace f32
}}}  // namespace esc::winatt::bwd
