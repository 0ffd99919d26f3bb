// Linear layers of rows: z = x w^T + b, out = act(z) + residual, and their gradients g = grad_out act'(z), gx = g w, gw = g^T x,
// gb = sum of g.  Here: the activations, g and its columns' sums, copies of ragged rows, and the sums of partial results.
#pragma once
#include "sum_rows.cuh"

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

// The slope two values at a time (packed fp32: half the instructions); who loops over values keeps the constants in registers, as a packed
// instruction takes none from its own words.
typedef unsigned long long F2;
__device__ __forceinline__ F2 f2(float lo, float hi) { F2 v; asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(lo), "f"(hi)); return v; }
__device__ __forceinline__ F2 held(float v) { F2 d; asm volatile("mov.b64 %0, {%1, %1};" : "=l"(d) : "f"(v)); return d; }
__device__ __forceinline__ void un2(F2 v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ F2 fma2(F2 a, F2 b, F2 c) { F2 d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
__device__ __forceinline__ F2 mul2(F2 a, F2 b) { F2 d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ F2 add2(F2 a, F2 b) { F2 d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }

constexpr float kLn = -0.72134752044f, kDensity = 0.39894228040f, kP9 = 0.345f, kP6 = 0.31f;
struct GaussConst {
    F2 ln, p, one, density, q[9];                                  // q: of -Q
    __device__ __forceinline__ GaussConst() {
        ln = held(kLn); p = held(kP9); one = held(1.f); density = held(kDensity);
        q[0] = held(-0.137620871f); q[1] = held(-0.137990677f); q[2] = held(-0.117478006f); q[3] = held(-0.110766168f); q[4] = held(0.0349471461f);
        q[5] = held(-0.183022695f); q[6] = held(0.267236026f); q[7] = held(-0.143238278f); q[8] = held(0.0279335122f);
    }
};
__device__ __forceinline__ void gelu_slope_pair(const GaussConst& k, float& a, float& b) {
    const F2 x = f2(min_nan(fabsf(a), 30.f), min_nan(fabsf(b), 30.f));   // beyond, e is zero in fp32: 0 times infinity does not come up
    float lo, hi;
    un2(mul2(mul2(x, x), k.ln), lo, hi);
    const F2 e = f2(pow2(lo), pow2(hi));
    un2(fma2(x, k.p, k.one), lo, hi);
    const F2 t = f2(inverse(lo), inverse(hi));
    F2 q = k.q[8];
#pragma unroll
    for (int i = 7; i >= 0; --i) q = fma2(q, t, k.q[i]);
    un2(mul2(e, fma2(x, k.density, mul2(q, t))), lo, hi);
    a = a >= 0.f ? 1.f + lo : -lo;
    b = b >= 0.f ? 1.f + hi : -hi;
}
// GELU for results of type T, one value at a time (in the products' epilogue registers are scarcer than instructions).
template <typename T> __device__ __forceinline__ float gelu(float z) {
    const float x = min_nan(fabsf(z), 30.f), e = pow2(x * x * kLn), t = inverse(fmaf(x, sizeof(T) == 4 ? kP9 : kP6, 1.f));
    float q;
    if (sizeof(T) == 4) {
        q = fmaf(0.0279335122f, t, -0.143238278f);
        q = fmaf(q, t, 0.267236026f);
        q = fmaf(q, t, -0.183022695f);
        q = fmaf(q, t, 0.0349471461f);
        q = fmaf(q, t, -0.110766168f);
        q = fmaf(q, t, -0.117478006f);
        q = fmaf(q, t, -0.137990677f);
        q = fmaf(q, t, -0.137620871f);
    } else {
        q = fmaf(0.073929169f, t, -0.180450428f);
        q = fmaf(q, t, -0.0157446193f);
        q = fmaf(q, t, -0.133429833f);
        q = fmaf(q, t, -0.120441264f);
        q = fmaf(q, t, -0.123860703f);
    }
    return fmaf(x, e * (q * t), max_nan(z, 0.f));
}
// f *= act'(z) for V values.
template <int V> __device__ __forceinline__ void times_slope(int act, const GaussConst& k, float* f, float* z) {
    if (act == kActGelu) {
        if constexpr (V == 1) {
            float other = z[0];
            gelu_slope_pair(k, z[0], other);
            f[0] *= z[0];
        } else {
#pragma unroll
            for (int e = 0; e < V; e += 2) {
                gelu_slope_pair(k, z[e], z[e + 1]);
                un2(mul2(f2(f[e], f[e + 1]), f2(z[e], z[e + 1])), f[e], f[e + 1]);
            }
        }
    } else if (act == kActRelu) {
#pragma unroll
        for (int e = 0; e < V; ++e) f[e] = z[e] > 0.f ? f[e] : 0.f;   // nothing passes where the slope is zero, an infinity neither
    }
}

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

constexpr int kSumBlocks = 4;                                      // of grad_z_sums, of an SM

// g = go act'(z) and its column sums, as far as they are asked for: g [rows, g_ld] of the type, part [gridDim.y][N] fp32 sums of the unrounded g.  A
// thread has V neighbouring columns and every so many rows; a block has `across` such pieces of a row; they divide the rows and their alignment.
//
// g of bf16 tensors is rounded to bf16: the operand of two products on the tensor cores, which take both operands in one type.  With GELU (ReLU's g needs
// no rounding) gradients are 2.3e-3 from exact in norm, 1.7e-3 with an unrounded g, which their own rounding leaves.  g in two bf16 parts would
// double both products (16384 x 1024 to 4096: 127 and 149 us) and the bytes of g; in the one-pass kernel (linear_backward_small.cuh), which has
// room for a second part where z was, it measured 51 -> 56 us (262144 x 64 to 128).
template <typename T, int V> __device__ __forceinline__ void load_values(const T* p, float* f) {
    constexpr int words = V * sizeof(T) / 4;
    if constexpr (words == 0) {
        f[0] = __uint_as_float((unsigned)*reinterpret_cast<const unsigned short*>(p) << 16);
    } else {
        unsigned w[words];
        if constexpr (words == 4) { const uint4 q = *reinterpret_cast<const uint4*>(p); w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w; }
        else if constexpr (words == 2) { const uint2 q = *reinterpret_cast<const uint2*>(p); w[0] = q.x; w[1] = q.y; }
        else w[0] = *reinterpret_cast<const unsigned*>(p);
#pragma unroll
        for (int i = 0; i < words; ++i) {
            if constexpr (sizeof(T) == 4) f[i] = __uint_as_float(w[i]);
            else { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
        }
    }
}
template <typename T, int V> __device__ __forceinline__ void store_values(T* p, const float* f) {
    constexpr int words = V * sizeof(T) / 4;
    if constexpr (words == 0) {
        *p = Elem<T>::from_f32(f[0]);
    } else {
        unsigned w[words];
#pragma unroll
        for (int i = 0; i < words; ++i) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(f[i]);
            else { const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]); w[i] = *reinterpret_cast<const unsigned*>(&h); }
        }
        if constexpr (words == 4) *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        else if constexpr (words == 2) *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<unsigned*>(p) = w[0];
    }
}
template <typename T, int V> __global__ void __launch_bounds__(256, kSumBlocks) grad_z_sums(const Layer<T> p, T* g, long long g_ld, float* part, int across)
{
    __shared__ float acc[256 * V];
    pdl_launch_dependents();                                       // products of a g that is not written here need not wait
    const int all = p.N / V, down = 256 / across;
    const int col = threadIdx.x % across, v = blockIdx.x * across + col, r = threadIdx.x / across;
    float sum[V] = {};
    const GaussConst k;
    if (r < down && v < all) {
        // several rows' loads before the first store
        constexpr int kBatch = V >= 8 ? 2 : V >= 4 ? 4 : 8;
        const long long step = down;
        for (long long row = (long long)blockIdx.y * down * kBatch + r; row < p.rows; row += step * kBatch * gridDim.y) {
            float f[kBatch][V], z[kBatch][V];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const long long at = (row + u * step < p.rows ? row + u * step : row) * p.N + v * V;
                load_values<T, V>(p.go + at, f[u]);
                if (p.act != kActNone) load_values<T, V>(p.kept + at, z[u]);
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                if (row + u * step >= p.rows) break;
                if (p.act != kActNone) times_slope<V>(p.act, k, f[u], z[u]);
                if (g) store_values<T, V>(g + (row + u * step) * g_ld + v * V, f[u]);
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] += f[u][e];
            }
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

// Rows that are not whole 16-byte pieces, copied to rows that are: 64 units of one or two bf16 values to a warp.
template <typename U> __global__ void __launch_bounds__(256) copy_rows(const U* in, long long in_ld, long long rows, int width, U* out, long long ld)
{
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, col = blockIdx.x * 64 + lane;
    const bool left = col < width, right = col + 32 < width;
    constexpr int kBatch = 8;
    for (long long row = ((long long)blockIdx.y * 8 + warp) * kBatch; row < rows; row += (long long)gridDim.y * 8 * kBatch) {
        U a[kBatch], b[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const U* p = in + (row + u < rows ? row + u : row) * in_ld;
            a[u] = p[left ? col : 0];
            b[u] = p[right ? col + 32 : 0];
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (row + u < rows && left) out[(row + u) * ld + col] = a[u];
            if (row + u < rows && right) out[(row + u) * ld + col + 32] = b[u];
        }
    }
}

// Partial sums [parts][count], to be added up: the weights' and the bias' gradients in one launch, either may be empty.
struct Parts { const float* p; int parts; long long count; };

// Many parts: 32 sums to a block.  Up to kFewParts: a thread has four sums.
constexpr int kFewParts = 8;
inline __host__ __device__ long long sum_blocks(const Parts& t) { return t.parts <= kFewParts ? (t.count + 4 * kSumThreads - 1) / (4 * kSumThreads) : (t.count + 31) / 32; }
template <typename G> __global__ void __launch_bounds__(kSumThreads) sum_parts(const Parts w, const Parts b, G* gw, G* gb)
{
    pdl_wait_primary();
    const long long ours = sum_blocks(w);
    const bool of_b = blockIdx.x >= ours;
    const Parts t = of_b ? b : w;
    const long long block = blockIdx.x - (of_b ? ours : 0);
    G* out = of_b ? gb : gw;
    if (t.parts <= kFewParts) {
        const long long e = block * (4 * kSumThreads) + threadIdx.x * 4;
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
    const long long e = block * 32 + threadIdx.x % 32;
    const float s = sum_rows(t.p + e, e < t.count, t.parts, (size_t)t.count);
    if (threadIdx.x >= 32 || e >= t.count) return;
    out[e] = Elem<G>::from_f32(s);
}

}}  // namespace esc::linear
