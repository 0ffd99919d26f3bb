// Self-attention over non-overlapping windows with a learned relative position bias (ESC paper, Section 3.3: the block's
// one self-attention; relpos_bias.cuh has the bias).  Per image, head and window of wh x ww pixels -- those at the right and lower border
// hold the pixels that the map has there --, with i, j over the window's pixels and d channels per head:
//
//   s[i,j] = scale q[i] . k[j] + bias[i,j]      lse[i] = log sum_j exp s[i,j]      p[i,j] = exp(s[i,j] - lse[i])
//   out[i] = sum_j p[i,j] v[j]
//
// A table's entry of kMasked or less counts as -inf, and a query that all keys are masked for gets out = 0 and lse = -inf: the backward
// pass has p from s - lse alone, which holds nothing more of s where all of a row is that far from zero.
//
// The running maximum and sum of a row stay in registers while the keys pass by (one pass, nothing of s is stored).  The table
// of one head is expanded once per block into shared memory, divided by the scale: it is then where the sum q . k starts from, and
// p = 2^(c s' - c m') with c = scale log2(e) is one multiply-add and one exponential.
#pragma once
#include "common.cuh"
#include "relpos_bias.cuh"

namespace esc { namespace winatt {

constexpr int kMaxHeadDim = 64;
constexpr float kMasked = -9984.0f;          // -10000 as bf16 rounds it
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// What every kernel of the attention needs to know.  q, k, v and their gradients have pixels `stride` values apart; out and its
// gradient are dense; lse and the rows' dot products are [B][heads][H][W].
template <typename T> struct Maps {
    const T *q, *k, *v;
    long long stride;
    int B, heads, d, H, W, wh, ww, ny, nx;         // ny x nx windows per image
    const T* table;
    const int* bucket;
    int n_buckets;
    float scale, inv_scale;
};

// One window of one image: its first pixel and its size inside the map.
struct Window {
    long long pixel;                               // index of its first pixel in [B][H][W]
    int h, w, y0, x0, b;
    __device__ __forceinline__ int tokens() const { return h * w; }
};
template <typename T> __device__ __forceinline__ Window window_at(const Maps<T>& m, int id) {
    Window r;
    const int wx = id % m.nx, t = id / m.nx, wy = t % m.ny;
    r.b = t / m.ny;
    r.y0 = wy * m.wh; r.x0 = wx * m.ww;
    r.h = min(m.wh, m.H - r.y0); r.w = min(m.ww, m.W - r.x0);
    r.pixel = ((long long)r.b * m.H + r.y0) * m.W + r.x0;
    return r;
}
template <typename T> __device__ __forceinline__ long long pixel_of(const Maps<T>& m, const Window& w, int token) {
    const int y = token / w.w;
    return w.pixel + (long long)y * m.W + (token - y * w.w);
}

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The head's table into shared memory, divided by the scale.
template <typename T> __device__ __forceinline__ void stage_table(const Maps<T>& m, int head, float* dst) {
    const int offsets = (2 * m.wh - 1) * (2 * m.ww - 1);
    for (int o = threadIdx.x; o < offsets; o += blockDim.x) {
        const float t = relpos::table_at(m.table, m.bucket, m.n_buckets, m.heads, head, o);
        dst[o] = t <= kMasked ? -INFINITY : t * m.inv_scale;
    }
}

// ---- fp32: CUDA cores -----------------------------------------------------------------------------------------------------
// A thread has Q queries (their channels, accumulators, running maxima and sums in registers); the block's keys and values are
// staged kKeys at a time as rows of D channels, which all threads read at the same address.  D: d rounded up, the rest is zero.
// Bound: the FP32 pipe, 2 D multiply-adds per pair of query and key next to about 10 other instructions.
namespace f32 {
constexpr int kThreads = 128, kKeys = 32, kStep = 8;

__host__ __device__ constexpr int queries_of(int D) { return D <= 16 ? 2 : 1; }

template <int D> __device__ __forceinline__ void load_row(const float* __restrict__ src, int d, float* f) {
#pragma unroll
    for (int c = 0; c < D; ++c) f[c] = c < d ? src[c] : 0.0f;
}

// kKeys rows of D channels of `src`, of the tokens from `first` on; rows behind the window's last are zero.
template <int D>
__device__ __forceinline__ void stage_rows(const Maps<float>& m, const float* __restrict__ src, long long stride, const Window& w, int head, int first, float* dst) {
    constexpr int kPer = D / 4;                    // pieces of four channels
    const bool wide = m.d % 4 == 0 && stride % 4 == 0 && (reinterpret_cast<uintptr_t>(src) & 15) == 0;
    for (int e = threadIdx.x; e < kKeys * kPer; e += blockDim.x) {
        const int r = e / kPer, c = e % kPer * 4, token = first + r;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (token < w.tokens() && c < m.d) {
            const float* p = src + pixel_of(m, w, token) * stride + (long long)head * m.d + c;
            if (wide) v = *reinterpret_cast<const float4*>(p);
            else {
                v.x = p[0];
                if (c + 1 < m.d) v.y = p[1];
                if (c + 2 < m.d) v.z = p[2];
                if (c + 3 < m.d) v.w = p[3];
            }
        }
        *reinterpret_cast<float4*>(dst + r * D + c) = v;
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads)
forward(Maps<float> m, int tiles, float* __restrict__ out, float* __restrict__ lse) {
    constexpr int Q = queries_of(D);
    extern __shared__ __align__(16) float smem[];
    float *ks = smem, *vs = ks + kKeys * D;
    int* bs = reinterpret_cast<int*>(vs + kKeys * D);
    float* table = reinterpret_cast<float*>(bs + kKeys);
    int id = blockIdx.x;
    const int tile = id % tiles; id /= tiles;
    const int head = id % m.heads;
    const Window w = window_at(m, id / m.heads);
    const int n = w.tokens(), pitch = 2 * m.ww - 1, first = tile * blockDim.x * Q;
    if (first >= n) return;
    stage_table(m, head, table);
    const float c = m.scale * kLog2e;
    float q[Q][D], acc[Q][D], top[Q], sum[Q];
    int at[Q];                                     // A(i): offset of key j is A(i) - B(j)
#pragma unroll
    for (int a = 0; a < Q; ++a) {
        const int i = min(first + a * (int)blockDim.x + (int)threadIdx.x, n - 1);   // spare threads repeat the last query
        load_row<D>(m.q + pixel_of(m, w, i) * m.stride + (long long)head * m.d, m.d, q[a]);
        const int y = i / w.w;
        at[a] = (y + m.wh - 1) * pitch + i - y * w.w + m.ww - 1;
        top[a] = -INFINITY; sum[a] = 0.0f;
#pragma unroll
        for (int x = 0; x < D; ++x) acc[a][x] = 0.0f;
    }
    for (int key = 0; key < n; key += kKeys) {
        __syncthreads();
        stage_rows<D>(m, m.k, m.stride, w, head, key, ks);
        stage_rows<D>(m, m.v, m.stride, w, head, key, vs);
        for (int r = threadIdx.x; r < kKeys; r += blockDim.x) {
            const int j = key + r, y = j / w.w;
            bs[r] = j < n ? y * pitch + j - y * w.w : 0;
        }
        __syncthreads();
        const int keys = min(kKeys, n - key);
        for (int r = 0; r < keys; r += kStep) {
            float s[Q][kStep];
#pragma unroll
            for (int u = 0; u < kStep; ++u) {
                const int b = bs[r + u];
                const float4* kr = reinterpret_cast<const float4*>(ks + (r + u) * D);
#pragma unroll
                for (int a = 0; a < Q; ++a) s[a][u] = table[at[a] - b];
#pragma unroll
                for (int x = 0; x < D / 4; ++x) {
                    const float4 k4 = kr[x];
#pragma unroll
                    for (int a = 0; a < Q; ++a) {
                        s[a][u] = fmaf(q[a][4 * x], k4.x, s[a][u]);
                        s[a][u] = fmaf(q[a][4 * x + 1], k4.y, s[a][u]);
                        s[a][u] = fmaf(q[a][4 * x + 2], k4.z, s[a][u]);
                        s[a][u] = fmaf(q[a][4 * x + 3], k4.w, s[a][u]);
                    }
                }
                if (r + u >= keys)
#pragma unroll
                    for (int a = 0; a < Q; ++a) s[a][u] = -INFINITY;
            }
#pragma unroll
            for (int a = 0; a < Q; ++a) {
                float t = top[a];
#pragma unroll
                for (int u = 0; u < kStep; ++u) t = fmaxf(t, s[a][u]);
                const float base = t == -INFINITY ? 0.0f : t * c, old = ex2(fmaf(top[a], c, -base));   // first step: 2^-inf = 0
                top[a] = t;
                sum[a] *= old;
#pragma unroll
                for (int x = 0; x < D; ++x) acc[a][x] *= old;
#pragma unroll
                for (int u = 0; u < kStep; ++u) {
                    s[a][u] = ex2(fmaf(s[a][u], c, -base));
                    sum[a] += s[a][u];
                }
            }
#pragma unroll
            for (int u = 0; u < kStep; ++u) {
                const float4* vr = reinterpret_cast<const float4*>(vs + (r + u) * D);
#pragma unroll
                for (int x = 0; x < D / 4; ++x) {
                    const float4 v4 = vr[x];
#pragma unroll
                    for (int a = 0; a < Q; ++a) {
                        acc[a][4 * x] = fmaf(s[a][u], v4.x, acc[a][4 * x]);
                        acc[a][4 * x + 1] = fmaf(s[a][u], v4.y, acc[a][4 * x + 1]);
                        acc[a][4 * x + 2] = fmaf(s[a][u], v4.z, acc[a][4 * x + 2]);
                        acc[a][4 * x + 3] = fmaf(s[a][u], v4.w, acc[a][4 * x + 3]);
                    }
                }
            }
        }
    }
#pragma unroll
    for (int a = 0; a < Q; ++a) {
        const int i = first + a * (int)blockDim.x + (int)threadIdx.x;
        if (i >= n) continue;
        const long long pixel = pixel_of(m, w, i);
        const float inv = sum[a] == 0.0f ? 0.0f : 1.0f / sum[a];
        float* o = out + (pixel * m.heads + head) * m.d;
        const bool wide = m.d % 4 == 0;
        if (wide) {
#pragma unroll
            for (int x = 0; x < D; x += 4)
                if (x < m.d) *reinterpret_cast<float4*>(o + x) = make_float4(acc[a][x] * inv, acc[a][x + 1] * inv, acc[a][x + 2] * inv, acc[a][x + 3] * inv);
        } else {
#pragma unroll
            for (int x = 0; x < D; ++x)
                if (x < m.d) o[x] = acc[a][x] * inv;
        }
        if (lse) {
            const long long hw = (long long)m.H * m.W;
            lse[((long long)w.b * m.heads + head) * hw + pixel - w.b * hw] = sum[a] == 0.0f ? -INFINITY : fmaf(top[a], m.scale, logf(sum[a]));
        }
    }
}

}  // namespace f32
}}  // namespace esc::winatt
