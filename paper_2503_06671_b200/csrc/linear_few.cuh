// Linear layers of a few rows (at most kMostRows), on the CUDA cores: bound by the bytes of the weights and by latency, where a tile of 128 rows
// on the tensor cores would be nearly empty and one block would walk the whole contraction.
//
// Forward: a warp has two or four outputs of all rows and a slice of the inputs, its lanes neighbouring pieces of w's rows; x comes from L1.  The
// lanes' sums are added by halving (each lane ends with its share of the sums), the slices of a block in order through shared memory.
// Backward: a warp has a stretch of outputs n and 32 V neighbouring inputs k.  It works g out for 32 outputs at a time into shared memory, reads
// w[n, k] once for gx and, with x in registers, writes gw[n, k] = sum over rows of g x as it passes; gx is left as a partial sum per stretch.
// 6 x 1782 to 192 in fp32: 70 -> 9 us; backward, 1 x 1024 to 4096 in fp32 132 -> 16 us, in bf16 38 -> 17.
#pragma once
#include "linear.cuh"

namespace esc { namespace linear { namespace few {

constexpr int kMostRows = 16, kWarps = 8;

// R: rows, rounded up to 1, 2, 4, 8 or 16.  C: outputs of a warp.  Rows beyond the last are read as the last and dropped.
template <typename T, int V, int R, int C> __global__ void __launch_bounds__(32 * kWarps) forward(const Layer<T> p, int slices)
{
    constexpr int S = C * R;                                // sums of a lane
    __shared__ float part[kWarps][S];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, slice = warp % slices, groups = kWarps / slices;
    const int n0 = (blockIdx.x * groups + warp / slices) * C, rows = (int)p.rows;
    float acc[S];
#pragma unroll
    for (int s = 0; s < S; ++s) acc[s] = 0.f;
    const T* w[C];
#pragma unroll
    for (int c = 0; c < C; ++c) w[c] = p.w + (long long)min(n0 + c, p.N - 1) * p.K;
    for (int k = (slice * 32 + lane) * V; k < p.K; k += slices * 32 * V) {
        float wf[C][V];
#pragma unroll
        for (int c = 0; c < C; ++c) load_values<T, V>(w[c] + k, wf[c]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float x[V];
            load_values<T, V>(p.x + (long long)min(r, rows - 1) * p.x_stride + k, x);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int v = 0; v < V; ++v) acc[c * R + r] = fmaf(wf[c][v], x[v], acc[c * R + r]);
        }
    }
    // halving: after a step a lane has the sums of half as many outputs, over twice as many lanes
    int mine = 0;                                                  // this lane's first sum
#pragma unroll
    for (int o = 16, count = S; o > 0; o >>= 1) {
        if (count > 1) {
            count /= 2;
            const bool upper = lane & o;
            mine += upper ? count : 0;
#pragma unroll
            for (int s = 0; s < count; ++s) {
                const float keep = upper ? acc[s + count] : acc[s], give = upper ? acc[s] : acc[s + count];
                acc[s] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
        } else {
            acc[0] += __shfl_xor_sync(0xffffffffu, acc[0], o);
        }
    }
    constexpr int left = S > 32 ? S / 32 : 1;
    const bool first = S >= 32 || lane % (32 / (S < 32 ? S : 32)) == 0;
    if (first)
#pragma unroll
        for (int s = 0; s < left; ++s) part[warp][mine + s] = acc[s];
    __syncthreads();
    for (int e = threadIdx.x; e < groups * S; e += 32 * kWarps) {
        const int group = e / S, c = e % S / R, r = e % R, n = (blockIdx.x * groups + group) * C + c;
        if (n >= p.N || r >= rows) continue;
        float f = 0.f;
        for (int s = 0; s < slices; ++s) f += part[group * slices + s][e % S];
        const long long at = (long long)r * p.N + n;
        if (p.b) f += Elem<T>::to_f32(p.b[n]);
        if (p.z) p.z[at] = Elem<T>::from_f32(f);
        if (p.act == kActGelu) f = gelu<T>(f);
        if (p.act == kActRelu) f = max_nan(f, 0.f);
        if (p.residual) f += Elem<T>::to_f32(p.residual[at]);
        p.out[at] = Elem<T>::from_f32(f);
    }
}

// Warp (tile of k, stretch of n): `across` tiles; stretch s has outputs [N s / stretches, N (s + 1) / stretches).
template <typename T, typename G, int V, int R> __global__ void __launch_bounds__(128) backward(const Layer<T> p, int across, int stretches, float* part_x, G* gw, G* gb)
{
    __shared__ __align__(16) float gs[4][32][R];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, rows = (int)p.rows;
    const int unit = blockIdx.x * 4 + warp;
    pdl_launch_dependents();
    if (unit >= across * stretches) return;
    const int tile = unit % across, stretch = unit / across, k = (tile * 32 + lane) * V;
    const int first = (int)((long long)p.N * stretch / stretches), last = (int)((long long)p.N * (stretch + 1) / stretches);
    const bool in = k < p.K;
    const GaussConst gc;
    float x[R][V], gx[R][V];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (in && gw) load_values<T, V>(p.x + (long long)min(r, rows - 1) * p.x_stride + k, x[r]);
#pragma unroll
        for (int v = 0; v < V; ++v) gx[r][v] = 0.f;
    }
    for (int n0 = first; n0 < last; n0 += 32) {
        const int n = n0 + lane;
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float g = 0.f;
            if (n < last && r < rows) {
                const long long at = (long long)r * p.N + n;
                g = Elem<T>::to_f32(p.go[at]);
                if (p.act != kActNone) {
                    float z[1] = {Elem<T>::to_f32(p.kept[at])}, f[1] = {g};
                    times_slope<1>(p.act, gc, f, z);
                    g = f[0];
                }
            }
            gs[warp][lane][r] = g;
            sum += g;
        }
        if (gb && tile == 0 && n < last) gb[n] = Elem<G>::from_f32(sum);
        __syncwarp();
        const int count = min(32, last - n0);
        if (in)
#pragma unroll 2
            for (int i = 0; i < count; ++i) {
                const float* g = gs[warp][i];
                if (p.gx) {
                    float w[V];
                    load_values<T, V>(p.w + (long long)(n0 + i) * p.K + k, w);
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int v = 0; v < V; ++v) gx[r][v] = fmaf(g[r], w[v], gx[r][v]);
                }
                if (gw) {
                    float f[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) f[v] = 0.f;
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int v = 0; v < V; ++v) f[v] = fmaf(g[r], r < rows ? x[r][v] : 0.f, f[v]);
                    store_values<G, V>(gw + (long long)(n0 + i) * p.K + k, f);
                }
            }
        __syncwarp();
    }
    if (p.gx && in)
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (r < rows) store_values<float, V>(part_x + ((long long)stretch * rows + r) * p.K + k, gx[r]);
}

}}}  // namespace esc::linear::few
