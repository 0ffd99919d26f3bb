// Learned relative position bias of a window of wh x ww pixels (ESC paper, Section 3.3: the block's window self-attention), and the
// gradient of its table:
//
//   bias[h, i, j]  = table[bucket[o(i, j)], h],     o(i, j) = (yi - yj + wh - 1) (2 ww - 1) + (xi - xj + ww - 1)
//   g_table[b, h]  = sum of g_bias[h, i, j] over all (i, j) with bucket[o(i, j)] = b
//
// Without buckets every offset o has a row of the table.  A bucket outside the table gives no bias and takes no gradient.
// o(i, j) = A(i) - B(j) with A(i) = o(i, 0), B(j) = yj (2 ww - 1) + xj: a row of the bias for one row yj of keys is a piece of
// the table read backwards.
#pragma once
#include "common.cuh"

namespace esc { namespace relpos {

constexpr int kMaxOffsets = 16384;       // (2 wh - 1) (2 ww - 1): one head's table in fp32 is at most 64 KB of shared memory

inline long long offsets_of(int wh, int ww) { return (2LL * wh - 1) * (2LL * ww - 1); }

// The bias of offset `o` for one head.
template <typename T>
__device__ __forceinline__ float table_at(const T* __restrict__ table, const int* __restrict__ bucket, int n_buckets, int heads, int head, int o) {
    if (!table) return 0.0f;
    const int b = bucket ? bucket[o] : o;
    return (unsigned)b < (unsigned)n_buckets ? Elem<T>::to_f32(table[(size_t)b * heads + head]) : 0.0f;
}

// ---- the bias as a matrix -------------------------------------------------------------------------------------------------
// A block takes kRows neighbouring queries of one row of the window: the wh (ww + kRows - 1) entries of the table that they
// read go to shared memory, then each warp writes rows of the matrix, 16 bytes a lane.  Eight neighbouring entries of the
// staged table are followed by a hole (`skew`): a warp's lanes read at a stride of 16 bytes' worth of values, which
// would fall into a few banks.  Bound: HBM, the matrix is written once.
constexpr int kRows = 16, kFillThreads = 256;
__host__ __device__ __forceinline__ int skew(int p) { return p + (p >> 3); }

template <typename T>
__global__ void __launch_bounds__(kFillThreads)
fill(const T* __restrict__ table, const int* __restrict__ bucket, int n_buckets, int heads, int wh, int ww, T* __restrict__ bias) {
    extern __shared__ float strip[];     // [wh][width]: dy from yi - (wh - 1) on, dx from x0 - (ww - 1) on
    const int groups = (ww + kRows - 1) / kRows;
    int id = blockIdx.x;
    const int group = id % groups; id /= groups;
    const int yi = id % wh, head = id / wh;
    const int x0 = group * kRows, rows = min(kRows, ww - x0), width = ww + rows - 1, pitch = 2 * ww - 1, tokens = wh * ww;
    for (int e = threadIdx.x; e < wh * width; e += kFillThreads) {
        const int r = e / width, c = e - r * width;
        strip[skew(e)] = table_at(table, bucket, n_buckets, heads, head, (yi + r) * pitch + x0 + c);
    }
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    constexpr int V = Elem<T>::kVec;
    const bool wide = tokens % V == 0;   // then every row starts on 16 bytes
    for (int r = warp; r < rows; r += kFillThreads / 32) {
        T* row = bias + ((size_t)head * tokens + (size_t)yi * ww + x0 + r) * tokens;
        // key (yj, xj): strip row wh - 1 - yj, column r + ww - 1 - xj
        if (wide) {
            for (int j = lane * V; j < tokens; j += 32 * V) {
                int yj = j / ww, xj = j - yj * ww;
                int at = (wh - 1 - yj) * width + r + ww - 1 - xj;
                __align__(16) T v[V];
#pragma unroll
                for (int e = 0; e < V; ++e) {
                    v[e] = Elem<T>::from_f32(strip[skew(at)]);
                    --at;
                    if (++xj == ww) { xj = 0; at += ww - width; }   // the row of keys below: one strip row up, back to its end
                }
                *reinterpret_cast<uint4*>(row + j) = *reinterpret_cast<const uint4*>(v);
            }
        } else {
            for (int j = lane; j < tokens; j += 32) {
                const int yj = j / ww, xj = j - yj * ww;
                row[j] = Elem<T>::from_f32(strip[skew((wh - 1 - yj) * width + r + ww - 1 - xj)]);
            }
        }
    }
}

// ---- the table's gradient -------------------------------------------------------------------------------------------------
// First the sums over the pairs of equal offset: a block takes one dy and 32 neighbouring dx, a lane each.  For a query a warp reads
// the 32 keys at those offsets, which are neighbours, and a lane adds its own: no two threads of the grid add to the same sum, and
// the order is fixed.  Offsets near zero have the most pairs, so the pairs of a block are cut into slices of kSlice, which `sum_slices` adds
// in order.  Bound: HBM, the matrix is read once (in pieces of 32 values, off the sectors' borders).
constexpr int kSumThreads = 256, kSlice = 512, kUnroll = 8;

// pairs of (query row, query column) that a block of dx from dx0 to dx0 + 31 walks
__host__ __device__ __forceinline__ int walk_columns(int ww, int dx0, int* first) {
    const int lo = dx0 > 0 ? dx0 : 0, hi = (dx0 + 31 < 0 ? dx0 + 31 : 0) + ww - 1;   // some lane's key column xi - dx lies in [0, ww)
    *first = lo;
    return hi - lo + 1;
}
__host__ __device__ __forceinline__ int slices_at(int wh, int ww, int dy, int dx0) {
    int first;
    const int n = (wh - (dy < 0 ? -dy : dy)) * walk_columns(ww, dx0, &first);
    return (n + kSlice - 1) / kSlice;
}
inline int most_slices(int wh, int ww) { return (int)(((long long)wh * ww + kSlice - 1) / kSlice); }

template <typename T>
__global__ void __launch_bounds__(kSumThreads)
sum_offsets(const T* __restrict__ g, int wh, int ww, float* __restrict__ part, int heads) {   // part [slices][heads][offsets]
    const int pitch = 2 * ww - 1, dys = 2 * wh - 1, groups = (pitch + 31) / 32, tokens = wh * ww;
    int id = blockIdx.x;
    const int group = id % groups; id /= groups;
    const int dy = id % dys - (wh - 1), head = id / dys, slice = blockIdx.y;
    const int dx0 = group * 32 - (ww - 1);
    int x_first;
    const int cols = walk_columns(ww, dx0, &x_first);
    const int n = (wh - abs(dy)) * cols, begin = slice * kSlice, end = min(n, begin + kSlice);
    if (begin >= n) return;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, y_first = max(dy, 0), dx = dx0 + lane;
    const T* gh = g + (size_t)head * tokens * tokens;
    float sum = 0.0f;
    for (int at = begin + warp; at < end; at += kUnroll * (kSumThreads / 32)) {
        float v[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int it = at + u * (kSumThreads / 32);
            const int row = it / cols, xi = x_first + it - row * cols, yi = y_first + row, xj = xi - dx;
            const bool ok = it < end && (unsigned)xj < (unsigned)ww;
            v[u] = ok ? Elem<T>::to_f32(gh[((size_t)yi * ww + xi) * tokens + (yi - dy) * ww + xj]) : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) sum += v[u];
    }
    __shared__ float warps[kSumThreads / 32][32];
    warps[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && group * 32 + lane < pitch) {
#pragma unroll
        for (int w = 1; w < kSumThreads / 32; ++w) sum += warps[w][lane];
        part[((size_t)slice * heads + head) * dys * pitch + (size_t)(dy + wh - 1) * pitch + group * 32 + lane] = sum;
    }
}

// Sum over the slices of an offset: a block takes 32 offsets, a lane each, and its warps every eighth slice.  per_offset: every offset has as many as
// slices_at says, else `slices` of them.  `dense` gets [heads][offsets] in fp32 for `sum_buckets`, else g_table gets [offsets][heads].
template <typename G>
__global__ void __launch_bounds__(256)
sum_slices(const float* __restrict__ part, int slices, bool per_offset, int heads, int wh, int ww, float* __restrict__ dense, G* __restrict__ g_table) {
    const int pitch = 2 * ww - 1, offsets = (2 * wh - 1) * pitch, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int o = blockIdx.x * 32 + lane, head = blockIdx.y;
    float sum = 0.0f;
    if (o < offsets) {
        if (per_offset) slices = slices_at(wh, ww, o / pitch - (wh - 1), (o % pitch) / 32 * 32 - (ww - 1));
        const float* p = part + (size_t)head * offsets + o;
        const size_t step = (size_t)heads * offsets;
#pragma unroll 4
        for (int s = warp; s < slices; s += 8) sum += p[s * step];
    }
    __shared__ float warps[8][32];
    warps[warp][lane] = sum;
    __syncthreads();
    if (warp != 0 || o >= offsets) return;
#pragma unroll
    for (int w = 1; w < 8; ++w) sum += warps[w][lane];
    if (dense) dense[(size_t)head * offsets + o] = sum;
    else g_table[(size_t)o * heads + head] = Elem<G>::from_f32(sum);
}

// Sums over the offsets of a bucket: a block takes 32 buckets of one head, a lane each; its warps walk the offsets, every value goes
// past all lanes, and the one whose bucket it is adds it.
template <typename G>
__global__ void __launch_bounds__(256)
sum_buckets(const float* __restrict__ dense, const int* __restrict__ bucket, int n_buckets, int heads, int offsets, G* __restrict__ g_table) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, head = blockIdx.y, mine = blockIdx.x * 32 + lane;
    float sum = 0.0f;
    for (int at = warp * 32; at < offsets; at += 256) {
        const bool ok = at + lane < offsets;
        const float v = ok ? dense[(size_t)head * offsets + at + lane] : 0.0f;
        const int b = ok ? bucket[at + lane] : -1;
        unsigned left = __ballot_sync(0xffffffffu, (unsigned)(b - (int)blockIdx.x * 32) < 32u);
        while (left) {                   // only the offsets of these buckets, in order
            const int src = __ffs(left) - 1;
            left &= left - 1;
            const float x = __shfl_sync(0xffffffffu, v, src);
            const int k = __shfl_sync(0xffffffffu, b, src);
            if (k == mine) sum += x;
        }
    }
    __shared__ float warps[8][32];
    warps[warp][lane] = sum;
    __syncthreads();
    if (warp == 0 && mine < n_buckets) {
#pragma unroll
        for (int w = 1; w < 8; ++w) sum += warps[w][lane];
        g_table[(size_t)mine * heads + head] = Elem<G>::from_f32(sum);
    }
}

}}  // namespace esc::relpos
