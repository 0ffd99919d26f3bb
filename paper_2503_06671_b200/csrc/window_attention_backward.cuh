// Backward pass of the window self-attention (window_attention.cuh).  With go = dL/dout and p recomputed from lse:
//
//   D[i]     = go[i] . out[i]                      dp[i,j] = go[i] . v[j]
//   ds[i,j]  = p[i,j] (dp[i,j] - D[i])             (dL/ds; the bias enters s directly)
//   g_q[i]   = scale sum_j ds[i,j] k[j]            g_k[j]  = scale sum_i ds[i,j] q[i]
//   g_v[j]   = sum_i p[i,j] go[i]                  g_table[b,h] = sum of ds over all windows' pairs of bucket b
//
// Every sum has a fixed order.  A query without keys (lse = -inf) has p = 0 and so takes and gives nothing.  In a window of one pixel p is 1 whatever
// the score is: ds is zero, and is not left to the difference of dp and D, which are two roundings of one number.
#pragma once
#include "window_attention.cuh"

namespace esc { namespace winatt { namespace bwd {

// What the other kernels take of a row, in [B][heads][H][W] like lse: bases = -lse log2(e), so that p = 2^(c s' + base) (-inf where the row
// has no keys: p = 0), and dots = -D.  Bound: HBM, go and out are read once.
constexpr int kRowThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kRowThreads)
row_terms(const T* __restrict__ go, const T* __restrict__ out, const float* __restrict__ lse, long long pixels, long long hw, int heads, int d,
          float* __restrict__ bases, float* __restrict__ dots) {
    constexpr int V = Elem<T>::kVec;
    const bool wide = d % V == 0;
    for (long long e = (long long)blockIdx.x * kRowThreads + threadIdx.x; e < pixels * heads; e += (long long)gridDim.x * kRowThreads) {
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
        const long long image = pixel / hw, row = (image * heads + head) * hw + pixel - image * hw;
        dots[row] = -sum;
        bases[row] = lse[row] == -INFINITY ? -INFINITY : -lse[row] * kLog2e;
    }
}

// What the backward kernels need beyond Maps.
template <typename T> struct Grads {
    const T* go;                                   // dense
    const float* bases;
    float* dots;
    T *g_q, *g_k, *g_v;                            // pixels `stride` values apart
    float* part;                                   // [slices][heads][offsets] sums of ds, or null
    int windows, groups;
};
// The scale of g_q and g_k in a window of n pixels.
template <typename T> __device__ __forceinline__ float score_scale(const Maps<T>& m, int n) { return n > 1 ? m.scale : 0.0f; }
template <typename T> __device__ __forceinline__ long long row_of(const Maps<T>& m, const Window& w, int head, long long pixel) {
    const long long hw = (long long)m.H * m.W;
    return ((long long)w.b * m.heads + head) * hw + pixel - w.b * hw;
}

// ---- fp32: CUDA cores -----------------------------------------------------------------------------------------------------
// Two kernels, so that every gradient is a sum in one thread's registers: in the first a thread has a key (k, v and their gradients
// in registers) and the queries pass by, in the second it has a query.  A row of 64 channels is shared by two neighbouring lanes.
// Bound: the FP32 pipe, 7 D multiply-adds per pair.  4 x 64x64, windows of 24, 3 heads of 16: 153 and 187 us, one round of blocks whose threads
// walk 576 rows, four at a time (two blocks an SM instead of four for the second kernel: 234).
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
    // Pairs of channels, two multiply-adds at a time.
    static __device__ __forceinline__ void load(const float* __restrict__ src, int d, Two* f) {
#pragma unroll
        for (int c = 0; c < N; c += 2) f[c / 2] = two(first() + c < d ? src[first() + c] : 0.0f, first() + c + 1 < d ? src[first() + c + 1] : 0.0f);
    }
    static __device__ __forceinline__ void clear(Two* f) {
#pragma unroll
        for (int c = 0; c < N / 2; ++c) f[c] = two(0.0f, 0.0f);
    }
    static __device__ __forceinline__ void store(float* __restrict__ dst, int d, const Two* f, float by) {
#pragma unroll
        for (int c = 0; c < N; c += 2) {
            float x, y;
            apart(f[c / 2], x, y);
            if (first() + c < d) dst[first() + c] = x * by;
            if (first() + c + 1 < d) dst[first() + c + 1] = y * by;
        }
    }
    static __device__ __forceinline__ float dot(const Two* f, const float* row) {
        const ulonglong2* r = reinterpret_cast<const ulonglong2*>(row + first());
        Two s0 = two(0.0f, 0.0f), s1 = s0;
#pragma unroll
        for (int c = 0; c < N / 4; ++c) {
            const ulonglong2 v = r[c];
            s0 = fma2(f[2 * c], v.x, s0);
            s1 = fma2(f[2 * c + 1], v.y, s1);
        }
        float a, b, x, y;
        apart(s0, a, b);
        apart(s1, x, y);
        float sum = (a + b) + (x + y);
        if (S == 2) sum += __shfl_xor_sync(0xffffffffu, sum, 1);
        return sum;
    }
    static __device__ __forceinline__ void add(Two* f, const float* row, float by) {
        const ulonglong2* r = reinterpret_cast<const ulonglong2*>(row + first());
        const Two b = two(by, by);
#pragma unroll
        for (int c = 0; c < N / 4; ++c) {
            const ulonglong2 v = r[c];
            f[2 * c] = fma2(b, v.x, f[2 * c]);
            f[2 * c + 1] = fma2(b, v.y, f[2 * c + 1]);
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
    Two k[L::N / 2], v[L::N / 2], gk[L::N / 2], gv[L::N / 2];
    L::load(m.k + at, m.d, k);
    L::load(m.v + at, m.d, v);
    L::clear(gk);
    L::clear(gv);
    for (int row = 0; row < n; row += kRows) {
        __syncthreads();
        stage_rows<D>(m, m.q, m.stride, w, head, row, qs);
        stage_rows<D>(m, g.go, (long long)m.heads * m.d, w, head, row, gs);
        for (int r = threadIdx.x; r < kRows; r += blockDim.x) {
            const int i = row + r, y = i / w.w;
            const long long p = i < n ? row_of(m, w, head, pixel_of(m, w, i)) : 0;
            as[r] = i < n ? (y + m.wh - 1) * pitch + i - y * w.w + m.ww - 1 : (m.wh - 1) * pitch + m.ww - 1;
            base[r] = i < n ? g.bases[p] : -INFINITY;
            dots[r] = i < n ? g.dots[p] : 0.0f;
        }
        __syncthreads();
        // rows behind the last have p = 0; four at a time, so that their sums of products run side by side
#pragma unroll 1
        for (int r = 0; r < kRows; r += 4) {
            float p[4], ds[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                p[u] = ex2(fmaf(L::dot(k, qs + (r + u) * D) + table[as[r + u] - b], c, base[r + u]));
                ds[u] = p[u] * (L::dot(v, gs + (r + u) * D) + dots[r + u]);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                L::add(gv, gs + (r + u) * D, p[u]);
                L::add(gk, qs + (r + u) * D, ds[u]);
            }
        }
    }
    if (first + L::row() < n) {
        L::store(g.g_k + at, m.d, gk, score_scale(m, n));
        L::store(g.g_v + at, m.d, gv, 1.0f);
    }
}

// Also the sums for the table's gradient: a block keeps one copy of the head's offsets for each warp over all tiles of queries that
// it takes.  At one step the lanes of a warp have different queries and one key, so all their offsets differ.
template <int D>
__global__ void __launch_bounds__(kThreads, D <= 16 ? 4 : 2)
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
        const bool own = first + L::row() < n, adds = own && L::first() == 0 && n > 1;   // adds: to the table's sums
        const int i = min(first + L::row(), n - 1);
        const long long pixel = pixel_of(m, w, i), at = pixel * m.stride + (long long)head * m.d, row = row_of(m, w, head, pixel);
        const int a = (i / w.w + m.wh - 1) * pitch + i % w.w + m.ww - 1;
        const float base = own ? g.bases[row] : -INFINITY, dot = own ? g.dots[row] : 0.0f;
        Two q[L::N / 2], go[L::N / 2], gq[L::N / 2];
        L::load(m.q + at, m.d, q);
        L::load(g.go + (pixel * m.heads + head) * m.d, m.d, go);
        L::clear(gq);
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
#pragma unroll 1
            for (int r = 0; r < rows; r += 4) {
                float ds[4];
                int o[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    o[u] = a - bs[r + u];
                    const float p = r + u < rows ? ex2(fmaf(L::dot(q, ks + (r + u) * D) + table[o[u]], c, base)) : 0.0f;
                    ds[u] = p * (L::dot(go, vs + (r + u) * D) + dot);
                }
#pragma unroll
                for (int u = 0; u < 4; ++u) L::add(gq, ks + (r + u) * D, ds[u]);
                if (g.part) {
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        if (adds && r + u < rows) mine[o[u]] += ds[u];
                        __syncwarp();              // the next key's offsets are the neighbours'
                    }
                }
            }
        }
        if (own) L::store(g.g_q + at, m.d, gq, score_scale(m, n));
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

// ---- bf16: tensor cores ---------------------------------------------------------------------------------------------------
// Three kernels that each make p and dp anew from products of registers and staged tiles, so that every sum has one owner: the first
// with rows of queries (g_q), the second with rows of keys (g_k, g_v), the third with a tile of query-key pairs that all windows pass
// by (the table's gradient: the pairs' sums over the windows stay in registers, and go to their offsets once).  One pass would need g_q
// added up across the warps and 1e9 additions to a table whose neighbouring pairs share entries; p and ds as an operand are rounded
// to bf16 (2^-8 of each term), D is put right by the rows' own sums, the sums of ds for the table are of the fp32 values.
// Bound: the exponentials, three times 236 us for the pairs of 64 patches of 64x64 in windows of 32, 4 heads of 16 (1.07e9),
// and the issue slots.  There: 618 + 621 + 605 us (rows of queries, of keys, table) beside 476 of the forward pass.  Rows of queries took 515
// with D of the rounded out in g_q, without sum p k.
namespace tc {
using namespace winatt::tc;
constexpr int kCols = 128;                                          // staged columns: queries for rows of keys, keys for rows of queries
__host__ __device__ constexpr int grad_tiles(int D) { return D <= 32 ? 2 : 1; }    // tiles of 16 rows of a warp
__host__ __device__ constexpr int grad_blocks(int D) { return D <= 16 ? 2 : 1; }   // on an SM

template <int D> struct RowSmem {
    static constexpr int kTile = kCols * D * 2, kWalk = 3 * kCols * (8 + 4), kRows = 2 * kCols * 2 * 4;   // the columns' terms, two tiles
    static __host__ __device__ size_t bytes(const Bias& b, bool twice) { return 4 * kTile + kWalk + kRows + (size_t)b.size * 4 * (twice ? 2 : 1) + (twice ? bias_gap() * 4 : 0); }
};

// A row's terms into shared memory; a row that is none: p = 0.
__device__ __forceinline__ void stage_terms(const Grads<bf16>& gr, long long row0, long long px, bool in, float* base, int to_dot) {
    if (in) {
        wmma16::cp4(wmma16::smem_addr(base), gr.bases + row0 + px);
        wmma16::cp4(wmma16::smem_addr(base + to_dot), gr.dots + row0 + px);
    } else {
        base[0] = -INFINITY;
        base[to_dot] = 0.0f;
    }
}

// KEYS: rows are keys (operands k and v), columns queries (q and go): g_k += ds^T q, g_v += p^T go.
// Else: rows are queries (q and go), columns keys (k and v): g_q += ds k.  Here a row's ds add up to what D of the rounded out is off
// (sum_j p (dp - D) would be zero), so its dots are put right for the kernels that follow, and g_q by as much of sum_j p k: where few keys
// decide a row its ds are small beside D's error, which was up to 18 times what bf16 as such costs there.
template <int D, bool KEYS, bool TWICE>
__global__ void __launch_bounds__(kMaxWarps * 32, grad_blocks(D))
grad_rows(Maps<bf16> m, Grads<bf16> gr, int tiles) {
    using namespace wmma16;
    constexpr int KC = D / 16, ON = D / 8, MT = grad_tiles(D), R = 2 * MT;   // R: rows that a lane has a part of
    constexpr int kTile = RowSmem<D>::kTile;
    extern __shared__ __align__(128) unsigned char raw[];
    long long* pixels = reinterpret_cast<long long*>(raw + 4 * kTile);
    int* bs = reinterpret_cast<int*>(pixels + 3 * kCols);
    float* bases = reinterpret_cast<float*>(bs + 3 * kCols);        // [two tiles][bases, dots][kCols]
    float* table = bases + 4 * kCols;
    const uint32_t tile0 = smem_addr(raw);
    int id = blockIdx.x;
    const int tile = id % tiles; id /= tiles;
    const int head = id % m.heads;
    const Window w = window_at(m, id / m.heads);
    const int n = w.tokens(), warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int block_first = tile * (blockDim.x >> 5) * (16 * MT), first = block_first + warp * 16 * MT;
    if (block_first >= n) return;
    const Bias bias(m.wh, m.ww);
    const long long dense = (long long)m.heads * m.d, off = (long long)head * m.d, row0 = row_of(m, w, head, w.pixel);
    const bf16 *c1 = (KEYS ? m.q : m.k) + w.pixel * m.stride + off, *c2 = KEYS ? gr.go + w.pixel * dense + off : m.v + w.pixel * m.stride + off;
    const long long stride2 = KEYS ? dense : m.stride;
    const bool wide1 = pieces(KEYS ? m.q : m.k, m.stride, m.d), wide2 = pieces(KEYS ? gr.go : m.v, stride2, m.d);
    Walk<kCols> walk;
    if (warp == 0) {
        walk.start(w, lane);
        walk.next(w, m.W, bias.pitch, lane, pixels, bs);
    }
    __syncthreads();
    auto stage = [&](int buf, int place) {
        const long long* px = pixels + place * kCols;
        Rows<D, kCols>::stage(c1, m.stride, wide1, tile0 + buf * 2 * kTile, c2, stride2, wide2, tile0 + (buf * 2 + 1) * kTile, m.d, px);
        if (KEYS)
            for (int r = threadIdx.x; r < kCols; r += blockDim.x) stage_terms(gr, row0, px[r], px[r] >= 0, bases + 2 * buf * kCols + r, kCols);
        cp_commit();
    };
    stage(0, 0);
    stage_bias<TWICE, !KEYS>(m, head, bias, table);
    if (warp == 0 && kCols < n) walk.next(w, m.W, bias.pitch, lane, pixels + kCols, bs + kCols);
    const bool pairs = TWICE && (w.w & 1) == 0;

    uint32_t a1[MT][KC][4], a2[MT][KC][4], at[R];
    float dot[R], base[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool in = first + 8 * r + g < n;
        const int i = min(first + 8 * r + g, n - 1), y = i / w.w, x = i - y * w.w;
        const long long px = (long long)y * m.W + x;
        at[r] = bias_row<TWICE>(m, bias, pairs, y, x, smem_addr(table));
        load_operand<KC>((KEYS ? m.k : m.q) + (w.pixel + px) * m.stride + off, m.d, t, r & 1, a1[r >> 1]);
        load_operand<KC>(KEYS ? m.v + (w.pixel + px) * m.stride + off : gr.go + (w.pixel + px) * dense + off, m.d, t, r & 1, a2[r >> 1]);
        base[r] = KEYS || !in ? -INFINITY : gr.bases[row0 + px];
        dot[r] = KEYS ? 0.0f : gr.dots[row0 + px];
    }
    const float c = m.scale * kLog2e;
    float acc1[MT][ON][4], acc2[MT][ON][4], rest[R];               // acc2: g_v, or sum p k
#pragma unroll
    for (int r = 0; r < R; ++r) rest[r] = 0.0f;
#pragma unroll
    for (int x = 0; x < ON; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int a = 0; a < MT; ++a) acc1[a][x][e] = acc2[a][x][e] = 0.0f;

    uint32_t plain[KC], turned[KC];
    lane_offsets<D>(lane, plain, turned);
    // 16 staged columns; `paired`: two neighbours' bias is read at a time, `ends`: the window may end within them.
    auto cols_at = [&](int step, bool paired, bool ends, int buf, int place, int left) {
        const uint32_t s1 = tile0 + buf * 2 * kTile + step * (16 * D * 2), s2 = s1 + kTile;
        const int* b = bs + place * kCols + step * 16 + 2 * t;
        float s[MT][2][4], dp[MT][2][4];
        float2 col_base[2], col_dot[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int b0 = b[8 * x], b1 = paired ? 0 : b[8 * x + 1];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float2 v = paired ? lds2(at[r] + b0) : make_float2(lds1(at[r] + b0), lds1(at[r] + b1));
                s[r >> 1][x][2 * (r & 1)] = v.x; s[r >> 1][x][2 * (r & 1) + 1] = v.y;
            }
            if (KEYS) {
                const float* row = bases + 2 * buf * kCols + step * 16 + 8 * x + 2 * t;
                col_base[x] = *reinterpret_cast<const float2*>(row);
                col_dot[x] = *reinterpret_cast<const float2*>(row + kCols);
            }
        }
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            uint32_t f[4], h[4];
            ldsm(f, s1 + plain[k]);
            ldsm(h, s2 + plain[k]);
#pragma unroll
            for (int a = 0; a < MT; ++a) {
                mma(s[a][0], a1[a][k], f[0], f[1]); mma(s[a][1], a1[a][k], f[2], f[3]);
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    if (k > 0) mma(dp[a][x], a2[a][k], h[2 * x], h[2 * x + 1]);
                    else if (KEYS) mma(dp[a][x], a2[a][k], h[2 * x], h[2 * x + 1], col_dot[x].x, col_dot[x].y, col_dot[x].x, col_dot[x].y);
                    else mma(dp[a][x], a2[a][k], h[2 * x], h[2 * x + 1], dot[2 * a], dot[2 * a], dot[2 * a + 1], dot[2 * a + 1]);
                }
            }
        }
        uint32_t pp[MT][4], pd[MT][4];
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float u = ex2(fmaf(s[a][x][2 * e], c, KEYS ? col_base[x].x : base[2 * a + e])), v = ex2(fmaf(s[a][x][2 * e + 1], c, KEYS ? col_base[x].y : base[2 * a + e]));
                    if (!KEYS && ends) {
                        const int j = step * 16 + 8 * x + 2 * t;
                        if (j >= left) u = 0.0f;
                        if (j + 1 >= left) v = 0.0f;
                    }
                    pp[a][2 * x + e] = pack(u, v);
                    u *= dp[a][x][2 * e];
                    v *= dp[a][x][2 * e + 1];
                    if (!KEYS) rest[2 * a + e] += u + v;
                    pd[a][2 * x + e] = pack(u, v);
                }
#pragma unroll
        for (int k = 0; k < KC; ++k) {
            uint32_t f[4];
            ldsm_t(f, s1 + turned[k]);
#pragma unroll
            for (int a = 0; a < MT; ++a) { mma(acc1[a][2 * k], pd[a], f[0], f[1]); mma(acc1[a][2 * k + 1], pd[a], f[2], f[3]); }
            if (KEYS) ldsm_t(f, s2 + turned[k]);
#pragma unroll
            for (int a = 0; a < MT; ++a) { mma(acc2[a][2 * k], pp[a], f[0], f[1]); mma(acc2[a][2 * k + 1], pp[a], f[2], f[3]); }
        }
    };
    for (int tile_col = 0, buf = 0, place = 0; tile_col < n; tile_col += kCols, buf ^= 1) {
        const int next = place == 2 ? 0 : place + 1, free = 3 - place - next;
        cp_wait<0>();
        __syncthreads();
        if (tile_col + kCols < n) stage(buf ^ 1, next);
        if (warp == 0 && tile_col + 2 * kCols < n) walk.next(w, m.W, bias.pitch, lane, pixels + free * kCols, bs + free * kCols);
        const int left = n - tile_col;
        if (TWICE && pairs) {
            if (left >= kCols) {
#pragma unroll 2
                for (int step = 0; step < kCols / 16; ++step) cols_at(step, true, false, buf, place, left);
            } else {
#pragma unroll 1
                for (int step = 0; step * 16 < left; ++step) cols_at(step, true, true, buf, place, left);
            }
        } else {
#pragma unroll 1
            for (int step = 0; step < (min(kCols, left) + 15) / 16; ++step) cols_at(step, false, true, buf, place, left);
        }
        place = next;
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int i = first + 8 * r + g, a = r >> 1, e = 2 * (r & 1);
        float more = rest[r];
        more += __shfl_xor_sync(0xffffffffu, more, 1);
        more += __shfl_xor_sync(0xffffffffu, more, 2);
        if (i >= n) continue;
        const long long pixel = pixel_of(m, w, i), to = pixel * m.stride + off;
        if (!KEYS && t == 0) gr.dots[row_of(m, w, head, pixel)] = dot[r] - more;
#pragma unroll
        for (int x = 0; x < ON; ++x) {
            float u = acc1[a][x][e], v = acc1[a][x][e + 1];
            if (!KEYS) { u = fmaf(-more, acc2[a][x][e], u); v = fmaf(-more, acc2[a][x][e + 1], v); }
            store_pair((KEYS ? gr.g_k : gr.g_q) + to, 8 * x + 2 * t, m.d, u * score_scale(m, n), v * score_scale(m, n));
            if (KEYS) store_pair(gr.g_v + to, 8 * x + 2 * t, m.d, acc2[a][x][e], acc2[a][x][e + 1]);
        }
    }
}

// The table's gradient.  A block has one head, a tile of 64 keys, every `parts`-th tile of 128 queries and every `groups`-th window; for each
// tile of queries its windows pass by with the sums of ds of the 128 x 64 pairs in registers (a warp 32 x 32), their bias laid
// out as the products' C operands once.  Windows of one shape have the tokens at the same places; those that the border cuts come
// behind the whole ones.  Then every thread adds up the pairs of some offsets.
constexpr int kPairQ = 128, kPairK = 64, kList = 64;
template <int D> struct PairSmem {
    static constexpr int kQ = kPairQ * D * 2, kK = kPairK * D * 2, kBuf = 2 * kQ + 2 * kK;
    static constexpr int kSums = kPairQ * (kPairK + 1) * 4;         // the pairs' sums, over the staged tiles
    static constexpr int kData = 2 * kBuf > kSums ? 2 * kBuf : kSums;
    static constexpr int kBias = 256 * 8 * 16;                      // the pairs' bias, eight C operands a thread
    static __host__ __device__ size_t bytes(int offsets, bool staged) { return kData + kBias + 2 * kList * 16 + (4 * kPairQ + 2 * (kPairQ + kPairK) + (staged ? 2 : 1) * offsets) * 4; }
};
template <int D>
__global__ void __launch_bounds__(256, D <= 32 ? 2 : 1)
grad_table(Maps<bf16> m, Grads<bf16> gr, int key_tiles, int parts, bool staged) {   // staged: there is room for the head's table

    using namespace wmma16;
    constexpr int KC = D / 16, P = Tile<D>::kPieces, QN = kPairQ * P / 256, KN = kPairK * P > 256 ? kPairK * P / 256 : 1;   // pieces of q, of k that a thread stages
    using S = PairSmem<D>;
    extern __shared__ __align__(128) unsigned char raw[];
    float4* bias = reinterpret_cast<float4*>(raw + S::kData) + threadIdx.x;   // of this thread, 256 apart
    long long* list = reinterpret_cast<long long*>(raw + S::kData + S::kBias); // windows to come, two halves: first pixel, first row
    float* bases = reinterpret_cast<float*>(list + 2 * kList * 2);  // [two windows][bases, dots][kPairQ]
    int* px = reinterpret_cast<int*>(bases + 4 * kPairQ);           // places of the queries, of the keys; behind the window's first pixel
    int* lin = px + kPairQ + kPairK;                                // y pitch + x of them
    float* sums = reinterpret_cast<float*>(lin + kPairQ + kPairK);
    const uint32_t data = smem_addr(raw);
    const int head = blockIdx.x % m.heads, id = blockIdx.x / m.heads, key0 = id % key_tiles * kPairK, part = id / key_tiles % parts, group = id / key_tiles / parts;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3, wq = (warp >> 1) * 32, wk = (warp & 1) * 32;
    const int pitch = 2 * m.ww - 1, offsets = (2 * m.wh - 1) * pitch;
    const long long dense = (long long)m.heads * m.d, off = (long long)head * m.d, hw = (long long)m.H * m.W;
    const bool wide_q = pieces(m.q, m.stride, m.d), wide_k = pieces(m.k, m.stride, m.d), wide_v = pieces(m.v, m.stride, m.d), wide_g = pieces(gr.go, dense, m.d);
    const float c = m.scale * kLog2e;
    uint32_t plain[KC], turned[KC];
    lane_offsets<D>(lane, plain, turned);
    float* table = sums + offsets;
    for (int o = tid; o < offsets; o += 256) {
        if (staged) table[o] = bias_of(m, head, o);
        sums[o] = 0.0f;
    }
    const int full_x = m.W / m.ww, rest_x = m.W - full_x * m.ww, full_y = m.H / m.wh, rest_y = m.H - full_y * m.wh;   // whole windows, and what is left
    for (int kind = 0; kind < 4; ++kind) {
        const int per_row = kind & 1 ? (rest_x > 0) : full_x, width = kind & 1 ? rest_x : m.ww, per_col = kind & 2 ? (rest_y > 0) : full_y, height = kind & 2 ? rest_y : m.wh;
        const int count = m.B * per_col * per_row, tokens = height * width;
        const int mine = group < count ? (count - group + gr.groups - 1) / gr.groups : 0;
        if (mine == 0 || key0 >= tokens || tokens == 1) continue;
        auto look = [&](int i) {                                    // the group's windows i .. i + kList - 1 into the list
            if (tid < kList && i + tid < mine) {
                const int at = group + (i + tid) * gr.groups, line = at / per_row, b = line / per_col;
                const int wy = kind & 2 ? full_y : line - b * per_col, wx = kind & 1 ? full_x : at - line * per_row;
                const long long pixel = (long long)b * hw + (long long)wy * m.wh * m.W + wx * m.ww;
                long long* l = list + ((i / kList & 1) * kList + tid) * 2;
                l[0] = pixel;
                l[1] = ((long long)b * m.heads + head) * hw + pixel - b * hw;
            }
        };
        for (int q0 = part * kPairQ; q0 < tokens; q0 += parts * kPairQ) {
            __syncthreads();                                        // the last queries' sums and places are done with
            for (int r = tid; r < kPairQ + kPairK; r += 256) {
                const int i = r < kPairQ ? q0 + r : key0 + r - kPairQ, y = i / width, x = i - y * width;
                px[r] = i < tokens ? y * m.W + x : -1;
                lin[r] = y * pitch + x;
            }
            look(0);
            __syncthreads();
            float sum[2][4][4];
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    float v[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = wq + 16 * a + 8 * (e >> 1) + g, j = kPairQ + wk + 8 * x + 2 * t + (e & 1);
                        const int o = lin[i] - lin[j] + (m.wh - 1) * pitch + m.ww - 1;
                        v[e] = px[i] < 0 || px[j] < 0 ? -INFINITY : staged ? table[o] : bias_of(m, head, o);   // pairs that are none: p = 0
                        sum[a][x][e] = 0.0f;
                    }
                    bias[(4 * a + x) * 256] = make_float4(v[0], v[1], v[2], v[3]);
                }
            auto stage = [&](int i, int buf) {
                const long long* l = list + ((i / kList & 1) * kList + i % kList) * 2;
                const long long pixel = l[0], row0 = l[1];
                const uint32_t dst = data + buf * S::kBuf;
                const bf16 *q = m.q + pixel * m.stride + off, *go = gr.go + pixel * dense + off, *k = m.k + pixel * m.stride + off, *v = m.v + pixel * m.stride + off;
#pragma unroll
                for (int u = 0; u < QN; ++u) {
                    const int r = (tid + 256 * u) / P, c = (tid + 256 * u) % P * 8;
                    const bool real = px[r] >= 0 && c < m.d;
                    const long long at = real ? px[r] : 0;
                    stage_piece(q + at * m.stride + (real ? c : 0), dst + Tile<D>::at(r, c / 8), real, m.d - c, wide_q);
                    stage_piece(go + at * dense + (real ? c : 0), dst + S::kQ + Tile<D>::at(r, c / 8), real, m.d - c, wide_g);
                }
                if (kPairK * P >= 256 || tid < kPairK * P)
#pragma unroll
                    for (int u = 0; u < KN; ++u) {
                        const int r = (tid + 256 * u) / P, c = (tid + 256 * u) % P * 8, p = px[kPairQ + r];
                        const bool real = p >= 0 && c < m.d;
                        const long long at = real ? p * m.stride + c : 0;
                        stage_piece(k + at, dst + 2 * S::kQ + Tile<D>::at(r, c / 8), real, m.d - c, wide_k);
                        stage_piece(v + at, dst + 2 * S::kQ + S::kK + Tile<D>::at(r, c / 8), real, m.d - c, wide_v);
                    }
                if (tid < kPairQ) stage_terms(gr, row0, px[tid], px[tid] >= 0, bases + 2 * buf * kPairQ + tid, kPairQ);
                cp_commit();
            };
            stage(0, 0);
            for (int i = 0, buf = 0; i < mine; ++i, buf ^= 1) {
                cp_wait<0>();
                __syncthreads();
                if (i % kList == 0) look(i + kList);                // read from the next barrier on
                if (i + 1 < mine) stage(i + 1, buf ^ 1);
                const uint32_t dst = data + buf * S::kBuf;
                const uint32_t ks = dst + 2 * S::kQ + wk * (D * 2), vs = ks + S::kK;
#pragma unroll
                for (int a = 0; a < 2; ++a) {                       // 16 queries at a time
                    uint32_t q[KC][4], go[KC][4];
                    const uint32_t rows = dst + (wq + 16 * a) * (D * 2);
#pragma unroll
                    for (int k = 0; k < KC; ++k) { ldsm(q[k], rows + turned[k]); ldsm(go[k], rows + S::kQ + turned[k]); }   // as A operands: rows lane % 16, piece lane / 16
                    const float* terms = bases + 2 * buf * kPairQ + wq + 16 * a + g;
                    const float base[2] = {terms[0], terms[8]}, dot[2] = {terms[kPairQ], terms[kPairQ + 8]};
#pragma unroll
                    for (int x = 0; x < 4; x += 2) {
                        float s[2][4], dp[2][4];
#pragma unroll
                        for (int y = 0; y < 2; ++y) {
                            const float4 v = bias[(4 * a + x + y) * 256];
                            s[y][0] = v.x; s[y][1] = v.y; s[y][2] = v.z; s[y][3] = v.w;
                        }
#pragma unroll
                        for (int k = 0; k < KC; ++k) {
                            uint32_t f[4], h[4];
                            ldsm(f, ks + x * (8 * D * 2) + plain[k]);
                            ldsm(h, vs + x * (8 * D * 2) + plain[k]);
#pragma unroll
                            for (int y = 0; y < 2; ++y) {
                                mma(s[y], q[k], f[2 * y], f[2 * y + 1]);
                                if (k > 0) mma(dp[y], go[k], h[2 * y], h[2 * y + 1]);
                                else mma(dp[y], go[k], h[2 * y], h[2 * y + 1], dot[0], dot[0], dot[1], dot[1]);
                            }
                        }
#pragma unroll
                        for (int y = 0; y < 2; ++y)
#pragma unroll
                            for (int e = 0; e < 4; ++e) sum[a][x + y][e] = fmaf(ex2(fmaf(s[y][e], c, base[e >> 1])), dp[y][e], sum[a][x + y][e]);
                    }
                }
            }
            // the pairs' sums to their offsets: every thread takes some offsets and walks the keys
            __syncthreads();
            float* pair = reinterpret_cast<float*>(raw);
#pragma unroll
            for (int a = 0; a < 2; ++a)
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int e = 0; e < 4; ++e) pair[(wq + 16 * a + 8 * (e >> 1) + g) * (kPairK + 1) + wk + 8 * x + 2 * t + (e & 1)] = sum[a][x][e];
            __syncthreads();
            const int q_end = min(q0 + kPairQ, tokens), k_end = min(key0 + kPairK, tokens);
            const int dy_lo = q0 / width - (k_end - 1) / width, dy_hi = (q_end - 1) / width - key0 / width, cols = 2 * width - 1;
            for (int o = tid; o < (dy_hi - dy_lo + 1) * cols; o += 256) {
                const int dy = dy_lo + o / cols, dx = o % cols - (width - 1);
                float v = 0.0f;
                for (int yj = key0 / width, j0 = key0; j0 < k_end; ++yj, j0 = yj * width) {   // a row of keys; the queries next to it are a row too
                    const int shift = dy * width + dx;              // i - j
                    const int lo = max(max(j0, yj * width - dx), q0 - shift), hi = min(min(min(k_end, (yj + 1) * width), (yj + 1) * width - dx), q_end - shift);
                    const float* from = pair + (lo + shift - q0) * (kPairK + 1) + lo - key0;
                    for (int j = lo; j < hi; ++j, from += kPairK + 2) v += *from;
                }
                sums[(dy + m.wh - 1) * pitch + dx + m.ww - 1] += v;
            }
        }
    }
    __syncthreads();
    float* to = gr.part + ((size_t)id * m.heads + head) * offsets;
    for (int o = tid; o < offsets; o += 256) to[o] = sums[o];
}
}  // namespace tc
}}}  // namespace esc::winatt::bwd
