// AdamW (decoupled weight decay) over many tensors in one launch.  Per value, with t the step's number:
//
//   g = grad_scale * grad
//   m = beta1 m + (1 - beta1) g          v = beta2 v + (1 - beta2) g^2
//   p = (1 - lr wd) p - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// All arithmetic is fp32, every operation of the two moments rounded as written (no contraction).  States in fp32, or in 8 bits:
// m and r = sqrt(v) as e4m3 values times an fp32 scale for each kQuant values of a tensor, scale = largest magnitude * (1 / 448),
// values = x * (448 * (1 / largest)), each operation rounded.  The
// root, because e4m3 reaches from 448 down to 2^-9: 2^18 in r is 2^36 in v.  A root that is not zero is never stored as
// zero (2^-9 of the scale instead): a zero would divide the next update by eps alone.  Rounding is to nearest, a value off by at most
// 2^-4 of itself.  The update of p is made from the moments before they are rounded.
//
// Bound: HBM.  Bytes per value: fp32 states 28 (p, m, v read and written, g read), 8 bits 16 (12 + 4, and 16/256 of scales).  100 million
// values in 300 tensors: 412 us (6.8 TB/s) and 278 (5.8 TB/s; 500 with exact quotients and every value's place looked at).
#pragma once
#include <cuda_fp8.h>
#include "common.cuh"

namespace esc { namespace adamw {

constexpr int kQuant = 256;              // values that share a scale: what a warp holds, 8 to a lane
constexpr int kThreads = 256;
constexpr int kChunk = kQuant * kThreads / 32;
constexpr float kE4m3Max = 448.0f, kE4m3Least = 0.001953125f, kTiny = 1e-30f;

// A run of at most kChunk values of one tensor; the pointers are at its first value.  One of these is all that a block
// reads before its data.
struct Chunk {
    void* p;
    const void* g;
    void* m;
    void* v;                             // v, or the e4m3 roots
    float* m_scale;                      // null: fp32 states
    float* v_scale;
    __nv_bfloat16* copy;                 // p rounded to bf16, or null
    int n;
    int wide;                            // every pointer suits accesses of four values
};
static_assert(sizeof(Chunk) == 64, "one chunk is four 16-byte loads");

struct Hyper {
    float beta1, one1, beta2, one2, eps;
    float keep, size, root, grad_scale;  // 1 - lr wd, lr / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
};

template <typename T> struct Four;       // four neighbouring values
template <> struct Four<float> {
    static __device__ __forceinline__ void load(const float* p, float* f) {
        const float4 v = __ldcs(reinterpret_cast<const float4*>(p));
        f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w;
    }
    static __device__ __forceinline__ void store(float* p, const float* f) {
        __stcs(reinterpret_cast<float4*>(p), make_float4(f[0], f[1], f[2], f[3]));
    }
};
template <> struct Four<__nv_bfloat16> {
    static __device__ __forceinline__ void load(const __nv_bfloat16* p, float* f) {
        const uint2 v = __ldcs(reinterpret_cast<const uint2*>(p));
        f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xffff0000u);
        f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xffff0000u);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16* p, const float* f) {
        const __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
        uint2 v;
        v.x = *reinterpret_cast<const uint32_t*>(&a); v.y = *reinterpret_cast<const uint32_t*>(&b);
        __stcs(reinterpret_cast<uint2*>(p), v);
    }
};
template <> struct Four<__nv_fp8_e4m3> {
    static __device__ __forceinline__ void load(const __nv_fp8_e4m3* p, float* f) {
        const uint32_t v = __ldcs(reinterpret_cast<const uint32_t*>(p));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const __half2 h = __half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(v >> (16 * i)), __NV_E4M3));
            const float2 x = __half22float2(h);
            f[2 * i] = x.x; f[2 * i + 1] = x.y;
        }
    }
    static __device__ __forceinline__ void store(__nv_fp8_e4m3* p, const float* f) {
        const uint32_t a = __nv_cvt_float2_to_fp8x2(make_float2(f[0], f[1]), __NV_SATFINITE, __NV_E4M3);
        const uint32_t b = __nv_cvt_float2_to_fp8x2(make_float2(f[2], f[3]), __NV_SATFINITE, __NV_E4M3);
        __stcs(reinterpret_cast<uint32_t*>(p), a | b << 16);
    }
};
template <typename T> __device__ __forceinline__ float one_in(const T* p) { return Elem<T>::to_f32(*p); }
template <> __device__ __forceinline__ float one_in<__nv_fp8_e4m3>(const __nv_fp8_e4m3* p) { return float(*p); }
template <typename T> __device__ __forceinline__ void one_out(T* p, float f) { *p = Elem<T>::from_f32(f); }
template <> __device__ __forceinline__ void one_out<__nv_fp8_e4m3>(__nv_fp8_e4m3* p, float f) { *p = __nv_fp8_e4m3(f); }   // to nearest, saturating

// A lane's values of its warp's run: four at 4 lane and four at 128 + 4 lane, so that every access of a warp is one piece.  WHOLE: the run has
// all its values and its pointers suit accesses of four; nothing is looked at per value then.
template <bool WHOLE, typename T> __device__ __forceinline__ void in(const T* base, int n, int lane, float* f) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int at = 128 * h + 4 * lane;
        if (WHOLE) Four<T>::load(base + at, f + 4 * h);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) f[4 * h + i] = at + i < n ? one_in<T>(base + at + i) : 0.0f;
    }
}
template <bool WHOLE, typename T> __device__ __forceinline__ void out(T* base, int n, int lane, const float* f) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const int at = 128 * h + 4 * lane;
        if (WHOLE) Four<T>::store(base + at, f + 4 * h);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (at + i < n) one_out<T>(base + at + i, f[4 * h + i]);
    }
}

// The largest magnitude of a warp's values.  Infinities do not count (they are stored as the largest value; as NaN where the run's scale is
// zero), nor does NaN, which stays.
__device__ __forceinline__ float largest(const float* x, bool finite_only) {
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, !finite_only || fabsf(x[i]) <= 3.0e38f ? fabsf(x[i]) : 0.0f);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    return top;
}
// The scale of a warp's values x, which become the values to store.
template <bool ROOT> __device__ __forceinline__ float scale_values(float* x) {
    float top = largest(x, false);
    if (top > 3.0e38f) top = largest(x, true);
    const bool some = top >= kTiny;
    const float inverse = some ? __fmul_rn(kE4m3Max, __frcp_rn(top)) : 0.0f, least = some ? kE4m3Least : 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y = __fmul_rn(x[i], inverse);
        x[i] = ROOT && x[i] > 0.0f && y < least ? least : y;
    }
    return some ? __fmul_rn(top, 1.0f / kE4m3Max) : 0.0f;
}

// One run of a warp.
template <bool WHOLE, typename P, typename G, typename S>
__device__ __forceinline__ void step_run(const Chunk& c, const Hyper& h, int warp, int lane, int n) {
    constexpr bool kEight = sizeof(S) == 1;
    const int first = warp * kQuant;
    P* cp = static_cast<P*>(c.p) + first;
    S *cm = static_cast<S*>(c.m) + first, *cv = static_cast<S*>(c.v) + first;
    float p[8], g[8], m[8], v[8], ms = 0.0f, vs = 0.0f;
    in<WHOLE, G>(static_cast<const G*>(c.g) + first, n, lane, g);
    in<WHOLE, S>(cm, n, lane, m);
    in<WHOLE, S>(cv, n, lane, v);
    if (kEight) { ms = c.m_scale[warp]; vs = c.v_scale[warp]; }
    in<WHOLE, P>(cp, n, lane, p);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float gi = __fmul_rn(g[i], h.grad_scale);
        if (kEight) {
            m[i] = __fmul_rn(m[i], ms);
            v[i] = __fmul_rn(v[i], vs);
            v[i] = __fmul_rn(v[i], v[i]);
        }
        m[i] = __fadd_rn(__fmul_rn(m[i], h.beta1), __fmul_rn(gi, h.one1));
        v[i] = __fadd_rn(__fmul_rn(v[i], h.beta2), __fmul_rn(__fmul_rn(gi, gi), h.one2));
        const float r = __fsqrt_rn(v[i]);
        // the quotient to 2 ulp (an exact one is half of the update's instructions); nothing that is stored in 8 bits comes from it
        p[i] = __fsub_rn(__fmul_rn(p[i], h.keep), __fmul_rn(__fdividef(m[i], __fadd_rn(__fmul_rn(r, h.root), h.eps)), h.size));
        if (kEight) v[i] = r;
    }
    out<WHOLE, P>(cp, n, lane, p);
    if (c.copy) out<WHOLE, __nv_bfloat16>(c.copy + first, n, lane, p);
    if (kEight) {
        ms = scale_values<false>(m);
        vs = scale_values<true>(v);
        if (lane == 0) { c.m_scale[warp] = ms; c.v_scale[warp] = vs; }
    }
    out<WHOLE, S>(cm, n, lane, m);
    out<WHOLE, S>(cv, n, lane, v);
}

// P, G: types of the parameters and the gradients; S: float or __nv_fp8_e4m3 for the states.
// scalars (device, may be null) replaces keep, size, root and grad_scale, so that a captured graph can be replayed with other
// steps and rates; skip (device, may be null): nothing is done where it is not zero.
template <typename P, typename G, typename S>
__global__ void __launch_bounds__(kThreads)
step(const Chunk* __restrict__ chunks, Hyper h, const float* __restrict__ scalars, const int* __restrict__ skip) {
    if (skip && *skip != 0) return;
    const Chunk c = chunks[blockIdx.x];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = min(c.n - warp * kQuant, kQuant);
    if (n <= 0) return;
    if (scalars) { h.keep = scalars[0]; h.size = scalars[1]; h.root = scalars[2]; h.grad_scale = scalars[3]; }
    if (c.wide && n == kQuant) step_run<true, P, G, S>(c, h, warp, lane, n);
    else step_run<false, P, G, S>(c, h, warp, lane, n);
}

}}  // namespace esc::adamw
