// Layer norm of rows of C channels, forward and backward.
//
//   mu = p + sum (x - p) / C,  r = 1 / sqrt(sum (x - mu)^2 / C + eps),  xh = (x - mu) r
//   y  = xh w + b
//   a  = gy w;  gx = r (a - sum a / C - xh sum (a xh) / C) + skip;  gw = sum over rows of gy xh;  gb = of gy
//
// Bound by memory: a row is read once into registers, by G threads that hold NV vectors of VEC values each, and everything is worked
// out there.  The mean comes first and the squares are those of the differences, and all of a row is taken from p, one of its values: near p
// differences are exact, so a row far from zero loses nothing, and one of equal values has differences of zero.  (With the mean of x itself,
// a step of x off, such a row came out as large as that step by 1 / sqrt(eps): 61 values of 1000 gave 0.06.)  p is the middle one of three, as a
// channel may be far larger than the others: differences would be rounded at its size, and all of a row be off by some sqrt(C) steps.  (To look at
// mean and variance and take such a row again cost 57600 x 192 in fp32 18.7 -> 20.8 us, long rows a quarter.)  The backward pass works mean and r out
// anew from x, which it reads anyway: nothing is kept from the forward pass.
// G <= 32: 32 / G rows to a warp, so narrow rows (64 channels of bf16: eight threads, 16 bytes each) keep every lane loading and a
// sum over a row is log2 G shuffles; G = 256: a row to a block.  What no block holds in registers goes through `wide` kernels that read
// x again (from L2).
// gw and gb: a thread meets the same columns in all its rows and adds them up in registers, the threads of a block are added through
// shared memory, the blocks by `sum_columns`, all in a fixed order.
// 640x360 rows of 64 in bf16: 16.4 us (3.6 TB/s; a copy of these bytes takes 16); backward of 64 x 64x64 with skip 34.9 us (3.8 TB/s).
#pragma once
#include "sum_rows.cuh"

namespace esc { namespace norm {

constexpr int kThreads = 256;
constexpr int kMaxChannels = 1 << 20;
constexpr int back_blocks(int values) { return values <= 8 ? 3 : values <= 16 ? 2 : 1; }   // of an SM, by the values that a thread holds of a row: what registers allow

// VEC neighbouring values as one access of VEC * sizeof(T) bytes.
template <typename T, int VEC> struct Vec;
template <typename T> struct Vec<T, 1> {
    T v;
    __device__ __forceinline__ void load(const T* p) { v = *p; }
    __device__ __forceinline__ void get(float* f) const { f[0] = Elem<T>::to_f32(v); }
    static __device__ __forceinline__ void store(T* p, const float* f) { *p = Elem<T>::from_f32(f[0]); }
};
template <> struct Vec<__nv_bfloat16, 2> {
    __nv_bfloat162 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const __nv_bfloat162*>(p); }
    __device__ __forceinline__ void get(float* f) const { f[0] = __low2float(v); f[1] = __high2float(v); }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* f) { *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(f[0], f[1]); }
};
template <> struct Vec<__nv_bfloat16, 8> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void get(float* f) const { unpack16<__nv_bfloat16>(v, f); }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* f) {
        uint32_t u[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            u[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
    }
};
template <> struct Vec<float, 4> {
    float4 v;
    __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void get(float* f) const { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
    static __device__ __forceinline__ void store(float* p, const float* f) { *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]); }
};

template <typename T> struct Rows {
    const T* x;
    long long x_stride, rows;
    int C;
    float eps;
    const T *weight, *bias;             // either may be null
    T* y;                               // forward
    long long y_stride;
    const T *gy, *skip;                 // backward: dense; skip may be null
    T* gx;
    float* part;                        // [gridDim.x][2][C] or null
};

// Sums over the G threads of a row, to all of them.  G > 32: over the block, in the order of its warps; another call, or whatever else the block meets
// at, comes before these words of `scratch` are written again.
template <int G, int N> __device__ __forceinline__ void sum_row(float (&v)[N], float* scratch) {
#pragma unroll
    for (int o = (G < 32 ? G : 32) / 2; o > 0; o >>= 1)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] += __shfl_xor_sync(0xffffffffu, v[i], o);
    if (G > 32) {
        constexpr int warps = G / 32;
        const int warp = threadIdx.x / 32;
        if (threadIdx.x % 32 == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) scratch[i * warps + warp] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = 0.f;
#pragma unroll
            for (int w = 0; w < warps; ++w) s += scratch[i * warps + w];
            v[i] = s;
        }
    }
}

__device__ __forceinline__ float middle(float a, float b, float c) { return fmaxf(fminf(a, b), fminf(fmaxf(a, b), c)); }
// The values of a row, f, become what they are above the row's mean.  p is the middle one of three threads' first values, or of one thread's where it
// has all or half of the row.  Threads without a value, and rows without one, hold zeros.
// A row to a block: three meetings a row, here twice and once for the sums behind it, each over words of its own: who writes some has met the others
// twice since these were read.
constexpr int kScratch = 3 + kThreads / 32;                        // words of `scratch` that this takes; the others are its callers'
template <int G, int NV, int VEC> __device__ __forceinline__ void center(float (&f)[NV * VEC], const bool (&real)[NV], int C, float inv_c, float* scratch) {
    float p;
    if constexpr (G > 32) {
        if (threadIdx.x < 3) scratch[threadIdx.x] = f[0];
        __syncthreads();
        p = middle(scratch[0], scratch[1], scratch[2]);
    } else if constexpr (G < 4) {
        p = __shfl_sync(0xffffffffu, middle(f[0], f[VEC / 2], f[VEC - 1]), 0, G);
    } else {
        const int last = VEC > 2 ? 2 : C / VEC - 1;                // thread with a first value; of 16-byte pieces a row has three or more here
        p = middle(__shfl_sync(0xffffffffu, f[0], 0, G), __shfl_sync(0xffffffffu, f[0], min(1, last), G), __shfl_sync(0xffffffffu, f[0], min(2, last), G));
    }
    float s[1] = {0.f};
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (real[i])
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                f[i * VEC + j] -= p;
                s[0] += f[i * VEC + j];
            }
    sum_row<G>(s, scratch + 3);
    const float mean = s[0] * inv_c;
#pragma unroll
    for (int i = 0; i < NV; ++i)
        if (real[i])
#pragma unroll
            for (int j = 0; j < VEC; ++j) f[i * VEC + j] -= mean;
}

template <typename T, int VEC, int NV, int G>
__global__ void __launch_bounds__(kThreads) forward(const Rows<T> p)
{
    constexpr int per_block = kThreads / G, F = VEC * NV;
    __shared__ float scratch[G > 32 ? kScratch + kThreads / 32 : 1];
    const int in_row = threadIdx.x % G;
    const float inv_c = 1.f / (float)p.C;
    Vec<T, VEC> w[NV], b[NV];
    bool real[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * G + in_row) * VEC;
        real[i] = c < p.C;
        if (real[i] && p.weight) w[i].load(p.weight + c);
        if (real[i] && p.bias) b[i].load(p.bias + c);
    }
    // A warp's rows end together, so that all its lanes reach the shuffles.  The next row's values are under way while this one is worked on.
    const long long step = (long long)gridDim.x * per_block;
    long long row = (long long)blockIdx.x * per_block + threadIdx.x / G;
    Vec<T, VEC> x[NV], ahead[NV];
    auto load = [&](Vec<T, VEC> (&v)[NV], long long r) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (r < p.rows && real[i]) v[i].load(p.x + r * p.x_stride + (i * G + in_row) * VEC);
    };
    load(x, row);
    for (; row - threadIdx.x / G < p.rows; row += step) {
        load(ahead, row + step);
        const bool live = row < p.rows;
        float f[F];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (live && real[i]) x[i].get(f + i * VEC);
            else
#pragma unroll
                for (int j = 0; j < VEC; ++j) f[i * VEC + j] = 0.f;
        }
        center<G, NV, VEC>(f, real, p.C, inv_c, scratch);
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < F; ++i) s[0] += f[i] * f[i];
        sum_row<G>(s, scratch + kScratch);
        const float r = rsqrtf(s[0] * inv_c + p.eps);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!live || !real[i]) continue;
            float wf[VEC], bf[VEC], o[VEC];
            if (p.weight) w[i].get(wf);
            if (p.bias) b[i].get(bf);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                o[j] = f[i * VEC + j] * r;
                if (p.weight) o[j] *= wf[j];
                if (p.bias) o[j] += bf[j];
            }
            Vec<T, VEC>::store(p.y + row * p.y_stride + (i * G + in_row) * VEC, o);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = ahead[i];
    }
}

template <typename T, int VEC, int NV, int G>
__global__ void __launch_bounds__(kThreads, back_blocks(VEC * NV)) backward(const Rows<T> p)
{
    constexpr int per_block = kThreads / G, F = VEC * NV;
    __shared__ float scratch[G > 32 ? kScratch + 3 * (kThreads / 32) : 1];
    const int in_row = threadIdx.x % G;
    const float inv_c = 1.f / (float)p.C;
    Vec<T, VEC> w[NV];
    bool real[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = (i * G + in_row) * VEC;
        real[i] = c < p.C;
        if (real[i] && p.weight) w[i].load(p.weight + c);
    }
    float gw[F], gb[F];
#pragma unroll
    for (int i = 0; i < F; ++i) gw[i] = gb[i] = 0.f;
    // the next row's values are under way while this one is worked on, where registers allow that
    constexpr bool kAhead = F <= 8;
    const long long step = (long long)gridDim.x * per_block;
    long long row = (long long)blockIdx.x * per_block + threadIdx.x / G;
    struct Values { Vec<T, VEC> x[NV], g[NV], k[NV]; } at, ahead;
    auto load = [&](Values& v, long long r) {
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (r < p.rows && real[i]) {
                const int c = (i * G + in_row) * VEC;
                v.x[i].load(p.x + r * p.x_stride + c);
                v.g[i].load(p.gy + r * p.C + c);
                if (p.skip) v.k[i].load(p.skip + r * p.C + c);
            }
    };
    if (kAhead) load(at, row);
    for (; row - threadIdx.x / G < p.rows; row += step) {
        if (kAhead) load(ahead, row + step);
        else load(at, row);
        const bool live = row < p.rows;
        float f[F];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (live && real[i]) at.x[i].get(f + i * VEC);
            else
#pragma unroll
                for (int j = 0; j < VEC; ++j) f[i * VEC + j] = 0.f;
        }
        center<G, NV, VEC>(f, real, p.C, inv_c, scratch);
        float t[3] = {0.f, 0.f, 0.f};                              // sums of d^2, a and a d with d = x - mu
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!live || !real[i]) continue;
            float wf[VEC], gf[VEC];
            if (p.weight) w[i].get(wf);
            at.g[i].get(gf);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float d = f[i * VEC + j], a = p.weight ? gf[j] * wf[j] : gf[j];
                t[0] += d * d; t[1] += a; t[2] += a * d;
            }
        }
        sum_row<G>(t, scratch + kScratch);
        const float r = rsqrtf(t[0] * inv_c + p.eps), mean_a = t[1] * inv_c, along = t[2] * inv_c * r;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!live || !real[i]) continue;
            float wf[VEC], gf[VEC], kf[VEC], o[VEC];
            if (p.weight) w[i].get(wf);
            at.g[i].get(gf);
            if (p.skip) at.k[i].get(kf);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float xh = f[i * VEC + j] * r, a = p.weight ? gf[j] * wf[j] : gf[j];
                o[j] = r * (a - mean_a - xh * along);
                if (p.skip) o[j] += kf[j];
                gw[i * VEC + j] += gf[j] * xh;
                gb[i * VEC + j] += gf[j];
            }
            Vec<T, VEC>::store(p.gx + row * p.C + (i * G + in_row) * VEC, o);
        }
        if (kAhead) at = ahead;
    }
    pdl_launch_dependents();
    if (!p.part) return;
    float* out = p.part + (size_t)blockIdx.x * 2 * p.C;
    if constexpr (G > 32) {                                        // every column has one thread
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (real[i])
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    out[(i * G + in_row) * VEC + j] = gw[i * VEC + j];
                    out[p.C + (i * G + in_row) * VEC + j] = gb[i * VEC + j];
                }
    } else {
    // the rows of a warp, then the warps in order
    extern __shared__ float cols[];                                // [warps][2][C]
#pragma unroll
    for (int o = 16; o >= G; o >>= 1)
#pragma unroll
        for (int i = 0; i < F; ++i) {
            gw[i] += __shfl_xor_sync(0xffffffffu, gw[i], o);
            gb[i] += __shfl_xor_sync(0xffffffffu, gb[i], o);
        }
    float* mine = cols + (threadIdx.x / 32) * 2 * p.C;
    if (threadIdx.x % 32 < G)
#pragma unroll
        for (int i = 0; i < NV; ++i)
            if (real[i])
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    mine[(i * G + in_row) * VEC + j] = gw[i * VEC + j];
                    mine[p.C + (i * G + in_row) * VEC + j] = gb[i * VEC + j];
                }
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * p.C; c += kThreads) {
        float s = 0.f;
        for (int v = 0; v < kThreads / 32; ++v) s += cols[v * 2 * p.C + c];
        out[c] = s;
    }
    }
}

// Rows that no block holds in registers, three times over (backward five), eight values of a thread under way: 4096 rows of 5001 in bf16 42 us, 2048
// of 20000 in fp32 131; backward 126 and 368.
template <int N> __device__ __forceinline__ void sum_block(float (&v)[N], float* scratch) {
    sum_row<kThreads, N>(v, scratch);
    __syncthreads();
}

struct Stats { float p, mean, r; };                                // mean: of x - p
template <typename T> __device__ __forceinline__ float above(const Stats& st, T x) { return Elem<T>::to_f32(x) - st.p - st.mean; }
template <typename T> __device__ __forceinline__ Stats wide_stats(const T* x, int C, float eps, float* scratch) {
    // values of the lines that come first anyway; elsewhere in the row 20000 values in fp32 131 -> 144 us
    Stats st{middle(Elem<T>::to_f32(x[0]), Elem<T>::to_f32(x[kThreads]), Elem<T>::to_f32(x[2 * kThreads])), 0.f, 0.f};
    float s[1] = {0.f};
#pragma unroll 8
    for (int c = threadIdx.x; c < C; c += kThreads) s[0] += above(st, x[c]);
    sum_block(s, scratch);
    st.mean = s[0] / (float)C;
    s[0] = 0.f;
#pragma unroll 8
    for (int c = threadIdx.x; c < C; c += kThreads) {
        const float d = above(st, x[c]);
        s[0] += d * d;
    }
    sum_block(s, scratch);
    st.r = rsqrtf(s[0] / (float)C + eps);
    return st;
}

template <typename T> __global__ void __launch_bounds__(kThreads) forward_wide(const Rows<T> p)
{
    __shared__ float scratch[kThreads / 32];
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T* x = p.x + row * p.x_stride;
        const Stats st = wide_stats(x, p.C, p.eps, scratch);
#pragma unroll 8
        for (int c = threadIdx.x; c < p.C; c += kThreads) {
            float o = above(st, x[c]) * st.r;
            if (p.weight) o *= Elem<T>::to_f32(p.weight[c]);
            if (p.bias) o += Elem<T>::to_f32(p.bias[c]);
            p.y[row * p.y_stride + c] = Elem<T>::from_f32(o);
        }
    }
}

template <typename T> __global__ void __launch_bounds__(kThreads) backward_wide(const Rows<T> p, float2* stats, float* from)
{
    __shared__ float scratch[2 * (kThreads / 32)];
    for (long long row = blockIdx.x; row < p.rows; row += gridDim.x) {
        const T *x = p.x + row * p.x_stride, *gy = p.gy + row * p.C;
        const Stats st = wide_stats(x, p.C, p.eps, scratch);
        if (threadIdx.x == 0) { stats[row] = make_float2(st.mean, st.r); from[row] = st.p; }
        float t[2] = {0.f, 0.f};
        for (int c = threadIdx.x; c < p.C; c += kThreads) {
            const float a = Elem<T>::to_f32(gy[c]) * (p.weight ? Elem<T>::to_f32(p.weight[c]) : 1.f);
            t[0] += a;
            t[1] += a * above(st, x[c]);
        }
        sum_block(t, scratch);
        const float mean_a = t[0] / (float)p.C, along = t[1] / (float)p.C * st.r;
        for (int c = threadIdx.x; c < p.C; c += kThreads) {
            const float a = Elem<T>::to_f32(gy[c]) * (p.weight ? Elem<T>::to_f32(p.weight[c]) : 1.f);
            float o = st.r * (a - mean_a - above(st, x[c]) * st.r * along);
            if (p.skip) o += Elem<T>::to_f32(p.skip[row * p.C + c]);
            p.gx[row * p.C + c] = Elem<T>::from_f32(o);
        }
    }
}

// Their columns: block (x, y) has kThreads columns and the rows y, y + gridDim.y, ...
template <typename T> __global__ void __launch_bounds__(kThreads) columns_wide(const Rows<T> p, const float2* stats, const float* from)
{
    const int c = blockIdx.x * kThreads + threadIdx.x;
    if (c >= p.C) return;
    float gw = 0.f, gb = 0.f;
    for (long long row = blockIdx.y; row < p.rows; row += gridDim.y) {
        const T* x = p.x + row * p.x_stride;
        const Stats st{from[row], stats[row].x, stats[row].y};
        const float g = Elem<T>::to_f32(p.gy[row * p.C + c]);
        gw += g * (above(st, x[c]) * st.r);
        gb += g;
    }
    p.part[(size_t)blockIdx.y * 2 * p.C + c] = gw;
    p.part[(size_t)blockIdx.y * 2 * p.C + p.C + c] = gb;
}

// Column sums of `parts` partial sums [parts][2][C]: 32 columns to a block.
template <typename G> __global__ void __launch_bounds__(kSumThreads) sum_columns(const float* part, int parts, int C, G* gw, G* gb)
{
    const int c = blockIdx.x * 32 + threadIdx.x % 32;
    pdl_wait_primary();
    const float s = sum_rows(part + c, c < 2 * C, parts, (size_t)2 * C);
    if (threadIdx.x >= 32 || c >= 2 * C) return;
    G* out = c < C ? gw : gb;
    if (out) out[c < C ? c : c - C] = Elem<G>::from_f32(s);
}

}}  // namespace esc::norm
