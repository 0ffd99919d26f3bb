// Self-attention over non-overlapping windows with a learned relative position bias (ESC paper, Section 3.3: the block's
// one self-attention; relpos_bias.cuh has the bias).  Per image, head and window of wh x ww pixels -- those at the right and lower border
// hold the pixels that the map has there --, with i, j over the window's pixels and d channels per head:
//
//   s[i,j] = scale q[i] . k[j] + bias[i,j]      lse[i] = log sum_j exp s[i,j]      p[i,j] = exp(s[i,j] - lse[i])
//   out[i] = sum_j p[i,j] v[j]
//
// A table's entry of kMasked or less counts as -inf, and a query that all keys are masked for gets out = 0 and lse = -inf: the masks that
// programs write (-inf, -10000, a type's lowest value) mean one thing, also where a row has nothing else.  That is an agreement, not
// arithmetic: softmax of a row of -10000 alone would be a distribution, and the entries above kMasked are taken as the numbers that they
// are (fp32 is 2^-10 apart at 10^4, so p there is good to about 1e-3, forward and backward).
//
// The running maximum and sum of a row stay in registers while the keys pass by (one pass, nothing of s is stored).  The table
// of one head is expanded once per block into shared memory, divided by the scale: it is then where the sum q . k starts from, and
// p = 2^(c s' - c m') with c = scale log2(e) is one multiply-add and one exponential.
#pragma once
#include "common.cuh"
#include "relpos_bias.cuh"
#include "warp_mma.cuh"

namespace esc { namespace winatt {

constexpr int kMaxHeadDim = 64;
constexpr float kMasked = -9984.0f;          // -10000 as bf16 rounds it
// A row's powers are 2^(c s - base).  The base is the row's first maximum and moves only when one is kSlack above it (p is then at
// most 2^8, which costs nothing in a floating format), so that most steps only look whether it has to.
constexpr float kSlack = 8.0f;
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

__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
// Two fp32 values in one register pair, and arithmetic on both at a time.
using Two = unsigned long long;
__device__ __forceinline__ Two two(float x, float y) {
    Two d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(x), "f"(y));
    return d;
}
__device__ __forceinline__ void apart(Two v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ Two fma2(Two a, Two b, Two c) {
    Two d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ Two mul2(Two a, Two b) {
    Two d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ float2 lds2(uint32_t addr) {
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr));
    return v;
}
__device__ __forceinline__ float lds1(uint32_t addr) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(addr));
    return v;
}

// An offset's bias, divided by the scale.
template <typename T> __device__ __forceinline__ float bias_of(const Maps<T>& m, int head, int o) {
    const float v = relpos::table_at(m.table, m.bucket, m.n_buckets, m.heads, head, o);
    return v <= kMasked ? -INFINITY : v * m.inv_scale;
}
// The head's into shared memory.
template <typename T> __device__ __forceinline__ void stage_table(const Maps<T>& m, int head, float* dst) {
    const int offsets = (2 * m.wh - 1) * (2 * m.ww - 1);
    for (int o = threadIdx.x; o < offsets; o += blockDim.x) dst[o] = bias_of(m, head, o);
}

// ---- fp32: CUDA cores -----------------------------------------------------------------------------------------------------
// A thread has Q queries (their channels, accumulators, running maxima and sums in registers); the block's keys and values are
// staged kKeys at a time as rows of D channels, which all threads read at the same address.  D: d rounded up, the rest is zero.
// Bound: the FP32 pipe, 2 D multiply-adds per pair of query and key (two at a time: they issue in half the slots, at the same rate)
// next to about 10 other instructions.  427x240, windows of 24, 4 heads of 16: 596 us, 0.34 of that pipe, for 12 warps an SM and sums that wait
// on one another.  Steps of 4 keys or 8: 593, 606; 64 threads a block instead of 128: 652.
namespace f32 {
constexpr int kThreads = 128, kKeys = 32, kStep = 4;


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

template <int D, int Q>
__global__ void __launch_bounds__(kThreads)
forward(Maps<float> m, int tiles, float* __restrict__ out, float* __restrict__ lse) {
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
    const float slack = kSlack / c;
    Two q[Q][D / 2], acc[Q][D / 2];                // pairs of channels
    float limit[Q], off[Q], sum[Q];                // p = 2^(c s + off); the row's base moves where a score is above the limit
    int at[Q];                                     // A(i): offset of key j is A(i) - B(j)
#pragma unroll
    for (int a = 0; a < Q; ++a) {
        const int i = min(first + a * (int)blockDim.x + (int)threadIdx.x, n - 1);   // spare threads repeat the last query
        float row[D];
        load_row<D>(m.q + pixel_of(m, w, i) * m.stride + (long long)head * m.d, m.d, row);
        const int y = i / w.w;
        at[a] = (y + m.wh - 1) * pitch + i - y * w.w + m.ww - 1;
        limit[a] = -INFINITY; sum[a] = off[a] = 0.0f;
#pragma unroll
        for (int x = 0; x < D / 2; ++x) { q[a][x] = two(row[2 * x], row[2 * x + 1]); acc[a][x] = two(0.0f, 0.0f); }
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
                const ulonglong2* kr = reinterpret_cast<const ulonglong2*>(ks + (r + u) * D);
                Two d[Q];
#pragma unroll
                for (int a = 0; a < Q; ++a) d[a] = two(table[at[a] - b], 0.0f);
#pragma unroll
                for (int x = 0; x < D / 4; ++x) {
                    const ulonglong2 k4 = kr[x];
#pragma unroll
                    for (int a = 0; a < Q; ++a) { d[a] = fma2(q[a][2 * x], k4.x, d[a]); d[a] = fma2(q[a][2 * x + 1], k4.y, d[a]); }
                }
#pragma unroll
                for (int a = 0; a < Q; ++a) {
                    float x, y;
                    apart(d[a], x, y);
                    s[a][u] = r + u < keys ? x + y : -INFINITY;
                }
            }
#pragma unroll
            for (int a = 0; a < Q; ++a) {
                float high = s[a][0];
#pragma unroll
                for (int u = 1; u < kStep; ++u) high = fmaxf(high, s[a][u]);
                if (high > limit[a]) {
                    const float top = limit[a] - slack, to = -high * c, old = top == -INFINITY ? 0.0f : ex2(to - off[a]);
                    limit[a] = high + slack;
                    off[a] = to;
                    sum[a] *= old;
#pragma unroll
                    for (int x = 0; x < D / 2; ++x) acc[a][x] = mul2(acc[a][x], two(old, old));
                }
                float part = 0.0f;
#pragma unroll
                for (int u = 0; u < kStep; ++u) {
                    s[a][u] = ex2(fmaf(s[a][u], c, off[a]));
                    part += s[a][u];
                }
                sum[a] += part;
            }
#pragma unroll
            for (int u = 0; u < kStep; ++u) {
                const ulonglong2* vr = reinterpret_cast<const ulonglong2*>(vs + (r + u) * D);
                Two p[Q];
#pragma unroll
                for (int a = 0; a < Q; ++a) p[a] = two(s[a][u], s[a][u]);
#pragma unroll
                for (int x = 0; x < D / 4; ++x) {
                    const ulonglong2 v4 = vr[x];
#pragma unroll
                    for (int a = 0; a < Q; ++a) { acc[a][2 * x] = fma2(p[a], v4.x, acc[a][2 * x]); acc[a][2 * x + 1] = fma2(p[a], v4.y, acc[a][2 * x + 1]); }
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
#pragma unroll
        for (int x = 0; x < D; x += 4) {
            float4 v;
            apart(acc[a][x / 2], v.x, v.y);
            apart(acc[a][x / 2 + 1], v.z, v.w);
            v.x *= inv; v.y *= inv; v.z *= inv; v.w *= inv;
            if (wide) {
                if (x < m.d) *reinterpret_cast<float4*>(o + x) = v;
            } else {
                if (x < m.d) o[x] = v.x;
                if (x + 1 < m.d) o[x + 1] = v.y;
                if (x + 2 < m.d) o[x + 2] = v.z;
                if (x + 3 < m.d) o[x + 3] = v.w;
            }
        }
        if (lse) {
            const long long hw = (long long)m.H * m.W;
            lse[((long long)w.b * m.heads + head) * hw + pixel - w.b * hw] = sum[a] == 0.0f ? -INFINITY : fmaf(off[a], -kLn2, logf(sum[a]));
        }
    }
}

}  // namespace f32

// ---- bf16: tensor cores ---------------------------------------------------------------------------------------------------
// A warp has 16 or 32 queries (tiles of 16) as A operands in registers; the block's keys and values pass by in staged tiles of 128, copied ahead.
// s and p never leave the registers: the accumulators of q k^T, which start from the bias, are, rounded to bf16, the A operand of p v.
// p is rounded as an operand only: out is off by at most 2^-8 of sum p |v| more; the sum that divides it is of the fp32 values.
//
// Bound: the exponentials, 16 a clock and SM (measured; a row's other arithmetic runs beside them), then the issue slots.  640x360,
// windows of 32, 4 heads of 16 (0.93e9 pairs, 59 GFLOP, 118 MB): exponentials 204 us, products 103 at mma.sync's 955 multiply-adds
// a clock and SM, bytes 18; 400 us, 8 pairs a clock and SM, 9.7 instructions each and 0.65 of them issued per clock and scheduler.
// mma.sync and not tcgen05 because at 16 channels the products are not the limit: a kernel with s in tensor memory, a query per thread and
// p through shared memory, two groups of 128 queries per block, took 554 us here and 580 for 48 x 48 windows of 6 heads of 32 (449).
// Measured on the way, us: rescaling at every step 528; a base that moves seldom, places walked instead of divided 468; everything that a
// window decides once outside the loop and three blocks an SM with steps of 16 keys 400 (two blocks, 32 keys: 445).
namespace tc {
using bf16 = __nv_bfloat16;
constexpr int kKeys = 128, kMaxWarps = 8;          // keys of a staged tile
// Tiles of 16 queries of a warp: two halve the reads of keys and values per product.  One where that leaves SMs without work, or the registers
// no room for more than 64 channels' worth.
__host__ __device__ constexpr int most_tiles(int D) { return D <= 32 ? 2 : 1; }
__host__ __device__ constexpr int blocks_of(int D, int MT) { return D <= 16 ? (MT == 1 ? 4 : 3) : 2; }   // on an SM
__host__ __device__ constexpr int step_of(int D) { return D <= 16 ? 16 : 32; }      // keys of a step

// The table in shared memory backwards, so that neighbouring keys read upwards, with rows of 2 ww entries: entry (key j, query i) is at
// B(j) - A(i) + const, and in a window of even width the pair of keys that a lane holds starts at a place whose parity is
// the query's.  A second copy one entry further along makes the odd ones even: both read pairs.
struct Bias {
    int pitch, size;                               // entries of a row, of a copy
    __host__ __device__ Bias(int wh, int ww) : pitch(2 * ww), size((2 * wh - 1) * 2 * ww + 32) {}
};
__host__ __device__ constexpr int bias_gap() { return 16; }   // between the copies, so that their pairs lie in different banks

// Where the tokens of a staged tile are.  One warp walks them, kPer of a lane's own 32 apart, and leaves for each its distance in pixels
// from the window's first and 4 B, its distance in the table (tokens behind the last get the first one's, which is as even as theirs would be).
template <int ROWS> struct Walk {
    static constexpr int kPer = ROWS / 32;
    int y[kPer], x[kPer], step_y, step_x;
    __device__ __forceinline__ void start(const Window& w, int lane) {
        step_y = ROWS / w.w; step_x = ROWS - step_y * w.w;
#pragma unroll
        for (int i = 0; i < kPer; ++i) { const int r = lane + 32 * i; y[i] = r / w.w; x[i] = r - y[i] * w.w; }
    }
    __device__ __forceinline__ void next(const Window& w, int W, int pitch, int lane, long long* pixel, int* b) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const bool in = y[i] < w.h;
            pixel[lane + 32 * i] = in ? (long long)y[i] * W + x[i] : -1;
            b[lane + 32 * i] = in ? 4 * (y[i] * pitch + x[i]) : 0;
            y[i] += step_y; x[i] += step_x;
            if (x[i] >= w.w) { x[i] -= w.w; ++y[i]; }
        }
    }
};

// A 16-byte piece of a row into shared memory, zeros where there is none.
__device__ __forceinline__ void stage_piece(const bf16* p, uint32_t at, bool real, int left, bool wide) {
    if (wide) {
        wmma16::cp16(at, p, real);
    } else {
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t lo = real && 2 * i < left ? (uint32_t)__bfloat16_as_ushort(p[2 * i]) : 0u;
            const uint32_t hi = real && 2 * i + 1 < left ? (uint32_t)__bfloat16_as_ushort(p[2 * i + 1]) : 0u;
            v[i] = lo | hi << 16;
        }
        asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
    }
}
// ROWS rows of D channels of two tensors into a staged tile each, from the pixels (a negative one gives zeros) behind their first.
template <int D, int ROWS> struct Rows {
    using T = wmma16::Tile<D>;
    static __device__ __forceinline__ void stage(const bf16* __restrict__ one, long long stride1, bool wide1, uint32_t dst1, const bf16* __restrict__ two_, long long stride2,
                                                 bool wide2, uint32_t dst2, int d, const long long* pixel) {
        for (int e = threadIdx.x; e < ROWS * T::kPieces; e += blockDim.x) {
            const int r = e / T::kPieces, c = e % T::kPieces;
            long long px = pixel[r];
            const bool real = px >= 0 && c * 8 < d;
            px = real ? px : 0;
            const int ch = real ? c * 8 : 0;
            stage_piece(one + px * stride1 + ch, dst1 + T::at(r, c), real, d - ch, wide1);
            stage_piece(two_ + px * stride2 + ch, dst2 + T::at(r, c), real, d - ch, wide2);
        }
    }
};

// Whether rows of d channels can be read in pieces of 16 bytes.
__device__ __forceinline__ bool pieces(const void* p, long long stride, int d) {
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && stride % 8 == 0 && d % 8 == 0;
}

template <int D> struct Smem {
    static constexpr int kTile = kKeys * D * 2;
    static constexpr int kWalk = 3 * kKeys * (8 + 4);   // pixels and B of three tiles
    static __host__ __device__ size_t bytes(const Bias& b, bool twice) { return 4 * kTile + kWalk + (size_t)b.size * 4 * (twice ? 2 : 1) + (twice ? bias_gap() * 4 : 0); }
};

// The head's table for rows of queries (backwards: entry (dy, dx) at (wh - 1 - dy) pitch + ww - 1 - dx) or for rows of keys (as it is).
template <bool TWICE, bool BACKWARDS> __device__ __forceinline__ void stage_bias(const Maps<bf16>& m, int head, const Bias& bias, float* table) {
    const int cols = 2 * m.ww - 1, rows = 2 * m.wh - 1;
    int span = 1;                                                   // threads to a row of the table
    while (span < cols && span < 32) span *= 2;
    const int step = blockDim.x / span, c0 = threadIdx.x % span;
    for (int r = threadIdx.x / span; r < rows; r += step)
        for (int c = c0; c < cols; c += span) {
            const float v = bias_of(m, head, r * cols + c);
            const int at = BACKWARDS ? (rows - 1 - r) * bias.pitch + cols - 1 - c : r * bias.pitch + c;
            table[at] = v;
            if (TWICE) table[bias.size + bias_gap() + at + 1] = v;
        }
}
// Address in the staged table of the row (query or key) at (y, x), to which 4 (pitch y' + x') of the other one is added.
template <bool TWICE> __device__ __forceinline__ uint32_t bias_row(const Maps<bf16>& m, const Bias& bias, bool pairs, int y, int x, uint32_t table) {
    int at = (m.wh - 1 - y) * bias.pitch + m.ww - 1 - x;
    if (TWICE && pairs && (at & 1)) at += bias.size + bias_gap() + 1;
    return table + 4 * at;
}
// A row's channels as the A operand's registers of row g (half 0) or g + 8 (half 1).
template <int KC> __device__ __forceinline__ void load_operand(const bf16* __restrict__ p, int d, int t, int half, uint32_t (&q)[KC][4]) {
    const bool even = (reinterpret_cast<uintptr_t>(p) & 3) == 0;
#pragma unroll
    for (int k = 0; k < KC; ++k)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int c = 16 * k + 8 * h + 2 * t;
            uint32_t v = 0;
            if (even && c + 1 < d) v = *reinterpret_cast<const uint32_t*>(p + c);
            else {
                if (c < d) v = __bfloat16_as_ushort(p[c]);
                if (c + 1 < d) v |= (uint32_t)__bfloat16_as_ushort(p[c + 1]) << 16;
            }
            q[k][half + 2 * h] = v;
        }
}
// Where a lane reads 16 rows of a staged tile as B operands: for products along the channels (rows 8 (lane / 16) + lane % 8, piece lane / 8 % 2
// of 16 channels) and, transposed, for products along the rows (rows 8 (lane / 8 % 2) + lane % 8, piece lane / 16).  Rows in steps of 8
// are a constant further: they do not change how a row's pieces are exchanged.
template <int D> __device__ __forceinline__ void lane_offsets(int lane, uint32_t (&plain)[D / 16], uint32_t (&turned)[D / 16]) {
#pragma unroll
    for (int k = 0; k < D / 16; ++k) {
        plain[k] = wmma16::Tile<D>::at((lane >> 4) * 8 + (lane & 7), 2 * k + ((lane >> 3) & 1));
        turned[k] = wmma16::Tile<D>::at(((lane >> 3) & 1) * 8 + (lane & 7), 2 * k + (lane >> 4));
    }
}
// Two neighbouring channels of a result.
__device__ __forceinline__ void store_pair(bf16* to, int ch, int d, float u, float v) {
    if (ch + 1 < d && (reinterpret_cast<uintptr_t>(to) & 3) == 0) *reinterpret_cast<uint32_t*>(to + ch) = wmma16::pack(u, v);
    else {
        if (ch < d) to[ch] = __float2bfloat16_rn(u);
        if (ch + 1 < d) to[ch + 1] = __float2bfloat16_rn(v);
    }
}

template <int D, bool TWICE, int MT>
__global__ void __launch_bounds__(kMaxWarps * 32, blocks_of(D, MT))
forward(Maps<bf16> m, int tiles, bf16* __restrict__ out, float* __restrict__ lse) {
    using namespace wmma16;
    constexpr int KC = D / 16, kStep = step_of(D), NT = kStep / 8, ON = D / 8, R = 2 * MT;          // steps along the channels, tiles of 8 keys, of 8 channels of out
    constexpr int kTile = Smem<D>::kTile;
    extern __shared__ __align__(128) unsigned char raw[];
    long long* pixels = reinterpret_cast<long long*>(raw + 4 * kTile);
    int* bs = reinterpret_cast<int*>(pixels + 3 * kKeys);
    float* table = reinterpret_cast<float*>(bs + 3 * kKeys);
    const uint32_t tile0 = smem_addr(raw);
    int id = blockIdx.x;
    const int tile = id % tiles; id /= tiles;
    const int head = id % m.heads;
    const Window w = window_at(m, id / m.heads);
    const int n = w.tokens(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int block_first = tile * (blockDim.x >> 5) * (16 * MT), first = block_first + warp * (16 * MT);
    if (block_first >= n) return;
    const Bias bias(m.wh, m.ww);
    const int head_off = head * m.d;
    const bf16 *k0 = m.k + w.pixel * m.stride + head_off, *v0 = m.v + w.pixel * m.stride + head_off;
    const bool wide_k = pieces(m.k, m.stride, m.d), wide_v = pieces(m.v, m.stride, m.d);
    Walk<kKeys> walk;
    if (warp == 0) {
        walk.start(w, lane);
        walk.next(w, m.W, bias.pitch, lane, pixels, bs);
    }
    __syncthreads();
    auto stage = [&](int buf, int place) {
        Rows<D, kKeys>::stage(k0, m.stride, wide_k, tile0 + buf * 2 * kTile, v0, m.stride, wide_v, tile0 + (buf * 2 + 1) * kTile, m.d, pixels + place * kKeys);
        cp_commit();
    };
    stage(0, 0);
    stage_bias<TWICE, true>(m, head, bias, table);
    if (warp == 0 && kKeys < n) walk.next(w, m.W, bias.pitch, lane, pixels + kKeys, bs + kKeys);
    const bool pairs = TWICE && (w.w & 1) == 0;

    // queries: operands, and where their rows of the bias start
    uint32_t q[MT][KC][4], at[R];                                    // at + 4 B(j): where (i, j) is
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = min(first + 8 * r + g, n - 1);
        const int y = i / w.w, x = i - y * w.w;
        at[r] = bias_row<TWICE>(m, bias, pairs, y, x, smem_addr(table));
        load_operand<KC>(m.q + (w.pixel + (long long)y * m.W + x) * m.stride + head_off, m.d, t, r & 1, q[r >> 1]);
    }
    const float c = m.scale * kLog2e;
    const float slack = kSlack / c;
    float o[MT][ON][4], limit[R], off[R], sum[R];
#pragma unroll
    for (int r = 0; r < R; ++r) { limit[r] = -INFINITY; sum[r] = off[r] = 0.0f; }
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int x = 0; x < ON; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[a][x][e] = 0.0f;

    uint32_t plain[KC], turned[KC];
    lane_offsets<D>(lane, plain, turned);
    // Some keys of a staged tile; `paired`: two neighbours' bias is read at a time, `ends`: the window may end within them.
    auto keys_at = [&](int step, bool paired, bool ends, int buf, int place, int left) {
        const uint32_t ks = tile0 + buf * 2 * kTile + step * (kStep * D * 2), vs = ks + kTile;
        const int* b = bs + place * kKeys + step * kStep + 2 * t;
        float s[MT][NT][4];
#pragma unroll
        for (int x = 0; x < NT; ++x) {
            const int b0 = b[8 * x], b1 = paired ? 0 : b[8 * x + 1];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float2 v = paired ? lds2(at[r] + b0) : make_float2(lds1(at[r] + b0), lds1(at[r] + b1));
                s[r >> 1][x][2 * (r & 1)] = v.x; s[r >> 1][x][2 * (r & 1) + 1] = v.y;
            }
        }
#pragma unroll
        for (int x = 0; x < NT; x += 2)
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                uint32_t f[4];
                ldsm(f, ks + plain[k] + x * (8 * D * 2));
#pragma unroll
                for (int a = 0; a < MT; ++a) { mma(s[a][x], q[a][k], f[0], f[1]); mma(s[a][x + 1], q[a][k], f[2], f[3]); }
            }
        if (ends && left < (step + 1) * kStep) {
#pragma unroll
            for (int x = 0; x < NT; ++x)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    if (step * kStep + 8 * x + 2 * t + e >= left)
#pragma unroll
                        for (int a = 0; a < MT; ++a) s[a][x][e] = s[a][x][e + 2] = -INFINITY;
        }
        float high[R];
        bool over = false;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int a = r >> 1, e = 2 * (r & 1);
            high[r] = fmaxf(s[a][0][e], s[a][0][e + 1]);
#pragma unroll
            for (int y = 1; y < NT; ++y) high[r] = max3(high[r], s[a][y][e], s[a][y][e + 1]);
            over |= high[r] > limit[r];
        }
        if (__any_sync(0xffffffffu, over)) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float top = limit[r] - slack;                 // -inf the first time, and 2^-inf = 0
                float x = fmaxf(high[r], top);
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 1));
                x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, 2));
                limit[r] = x + slack;
                const float to = x == -INFINITY ? 0.0f : -x * c, old = top == -INFINITY ? 0.0f : ex2(to - off[r]);
                off[r] = to;
                sum[r] *= old;
#pragma unroll
                for (int y = 0; y < ON; ++y) { o[r >> 1][y][2 * (r & 1)] *= old; o[r >> 1][y][2 * (r & 1) + 1] *= old; }
            }
        }
#pragma unroll
        for (int y = 0; y < NT; ++y)
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int a = r >> 1, e = 2 * (r & 1);
                s[a][y][e] = ex2(fmaf(s[a][y][e], c, off[r]));
                s[a][y][e + 1] = ex2(fmaf(s[a][y][e + 1], c, off[r]));
                sum[r] += s[a][y][e] + s[a][y][e + 1];
            }
        // p v: 16 keys at a time, the values transposed on the way in
#pragma unroll
        for (int x = 0; x < NT; x += 2) {
            uint32_t p[MT][4];
#pragma unroll
            for (int a = 0; a < MT; ++a) {
                p[a][0] = pack(s[a][x][0], s[a][x][1]); p[a][1] = pack(s[a][x][2], s[a][x][3]);
                p[a][2] = pack(s[a][x + 1][0], s[a][x + 1][1]); p[a][3] = pack(s[a][x + 1][2], s[a][x + 1][3]);
            }
#pragma unroll
            for (int k = 0; k < KC; ++k) {
                uint32_t f[4];
                ldsm_t(f, vs + turned[k] + x * (8 * D * 2));
#pragma unroll
                for (int a = 0; a < MT; ++a) { mma(o[a][2 * k], p[a], f[0], f[1]); mma(o[a][2 * k + 1], p[a], f[2], f[3]); }
            }
        }
    };
    for (int tile_key = 0, buf = 0, place = 0; tile_key < n; tile_key += kKeys, buf ^= 1) {
        const int next = place == 2 ? 0 : place + 1, free = 3 - place - next;
        cp_wait<0>();
        __syncthreads();                                            // this tile and the next one's places are there; the other tile and the last one's places are free
        if (tile_key + kKeys < n) stage(buf ^ 1, next);
        if (warp == 0 && tile_key + 2 * kKeys < n) walk.next(w, m.W, bias.pitch, lane, pixels + free * kKeys, bs + free * kKeys);
        const int left = n - tile_key;
        if (TWICE && pairs) {
            if (left >= kKeys) {
#pragma unroll 2
                for (int step = 0; step < kKeys / kStep; ++step) keys_at(step, true, false, buf, place, left);
            } else {
#pragma unroll 1
                for (int step = 0; step * kStep < left; ++step) keys_at(step, true, true, buf, place, left);
            }
        } else {
#pragma unroll 1
            for (int step = 0; step < (min(kKeys, left) + kStep - 1) / kStep; ++step) keys_at(step, false, true, buf, place, left);
        }
        place = next;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float x = sum[r];
        x += __shfl_xor_sync(0xffffffffu, x, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        const int i = first + 8 * r + g, a = r >> 1, e = 2 * (r & 1);
        if (i >= n) continue;
        const long long pixel = pixel_of(m, w, i);
        const float inv = x == 0.0f ? 0.0f : 1.0f / x;
        bf16* to = out + (pixel * m.heads + head) * m.d;
#pragma unroll
        for (int y = 0; y < ON; ++y) store_pair(to, 8 * y + 2 * t, m.d, o[a][y][e] * inv, o[a][y][e + 1] * inv);
        if (lse && t == 0) {
            const long long hw = (long long)m.H * m.W;
            lse[((long long)w.b * m.heads + head) * hw + pixel - w.b * hw] = x == 0.0f ? -INFINITY : fmaf(off[r], -kLn2, logf(x));
        }
    }
}
}  // namespace tc
}}  // namespace esc::winatt
