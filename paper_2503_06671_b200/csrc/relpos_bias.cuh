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
// read go to shared memory, then each warp writes rows of the matrix, 16 bytes a lane.  Bound: HBM, the matrix is written once.
// A lane's V values lie V places from the next lane's, which would be a few banks only.  Where ww is a multiple of V the entries
// are therefore staged in V planes, entry p in plane p % V: for one of its V values every lane of the warp reads the same plane, at
// neighbouring places, and the planes' order is the row's alone.  Elsewhere a lane's piece can run over the end of a row of keys: it is
// walked entry by entry, with a hole behind every eighth entry of the strip (`skew`) against the banks.
// 6 x 2304 x 2304 bf16 (64 MB): 24.6 us with the walk, 15.6 by planes (4.1 TB/s).
constexpr int kRows = 16, kFillThreads = 256;
__host__ __device__ __forceinline__ int skew(int p) { return p + (p >> 3); }
__host__ __device__ __forceinline__ int round_to(int v, int to) { return (v + to - 1) / to * to; }
// Floats of the strip.
__host__ __device__ __forceinline__ int strip_floats(int wh, int ww, int V) {
    const int rows = kRows < ww ? kRows : ww, width = ww + rows - 1;
    return ww % V == 0 ? V * (wh * (round_to(width, V) / V) + 1) : skew(wh * width) + 1;
}

template <typename T>
__global__ void __launch_bounds__(kFillThreads)
fill(const T* __restrict__ table, const int* __restrict__ bucket, int n_buckets, int heads, int wh, int ww, T* __restrict__ bias) {
    extern __shared__ float strip[];     // [wh][width]: dy from yi - (wh - 1) on, dx from x0 - (ww - 1) on
    constexpr int V = Elem<T>::kVec;
    const int groups = (ww + kRows - 1) / kRows;
    int id = blockIdx.x;
    const int group = id % groups; id /= groups;
    const int yi = id % wh, head = id / wh;
    const int x0 = group * kRows, rows = min(kRows, ww - x0), width = ww + rows - 1, pitch = 2 * ww - 1, tokens = wh * ww;
    const bool planes = ww % V == 0;
    const int per = round_to(width, V) / V, plane = wh * per + 1;   // one more, so that the planes start in different banks
    for (int r = threadIdx.x >> 5; r < wh; r += kFillThreads / 32)
        for (int c = threadIdx.x & 31; c < width; c += 32) {
            const float v = table_at(table, bucket, n_buckets, heads, head, (yi + r) * pitch + x0 + c);
            strip[planes ? (c % V) * plane + r * per + c / V : skew(r * width + c)] = v;
        }
    __syncthreads();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const bool wide = tokens % V == 0;   // then every row starts on 16 bytes
    for (int r = warp; r < rows; r += kFillThreads / 32) {
        T* row = bias + ((size_t)head * tokens + (size_t)yi * ww + x0 + r) * tokens;
        // key (yj, xj): strip row wh - 1 - yj, column r + ww - 1 - xj
        if (planes) {
            const int top = r + ww - 1;
            int from[V];                 // where value e of a piece at xj = 0 is, in a strip row that starts at 0
#pragma unroll
            for (int e = 0; e < V; ++e) from[e] = (top - e) % V * plane + (top - e) / V;
            for (int j = lane * V; j < tokens; j += 32 * V) {
                const int yj = j / ww, xj = j - yj * ww, at = (wh - 1 - yj) * per - xj / V;
                __align__(16) T v[V];
#pragma unroll
                for (int e = 0; e < V; ++e) v[e] = Elem<T>::from_f32(strip[from[e] + at]);
                *reinterpret_cast<uint4*>(row + j) = *reinterpret_cast<const uint4*>(v);
            }
        } else if (wide) {
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
// the order is fixed.  The warps take the queries' columns in turn, and a lane reads kUnroll queries ahead: one column's rows, which lie a
// constant apart, or (windows of few rows) columns.  Offsets near zero have the most pairs, so a block takes kRowSlice rows of queries, or
// kColSlice columns; `sum_slices` adds them in order.  Bound: HBM, the matrix is read once (in pieces of 32 values, off the sectors' borders).
constexpr int kSumThreads = 256, kSumWarps = kSumThreads / 32, kUnroll = 8, kRowSlice = 8, kColSlice = 256, kFewRows = 4;

// Columns of queries that a block of dx from dx0 to dx0 + 31 walks: those where some lane's key column xi - dx lies in [0, ww).
__host__ __device__ __forceinline__ int walk_columns(int ww, int dx0, int* first) {
    const int lo = dx0 > 0 ? dx0 : 0, hi = (dx0 + 31 < 0 ? dx0 + 31 : 0) + ww - 1;
    *first = lo;
    return hi - lo + 1;
}
__host__ __device__ __forceinline__ int slices_at(int wh, int ww, int dy, int dx0) {
    int first;
    return wh < kFewRows ? (walk_columns(ww, dx0, &first) + kColSlice - 1) / kColSlice : (wh - (dy < 0 ? -dy : dy) + kRowSlice - 1) / kRowSlice;
}
inline int most_slices(int wh, int ww) { return wh < kFewRows ? (ww + kColSlice - 1) / kColSlice : (wh + kRowSlice - 1) / kRowSlice; }

template <typename T>
__global__ void __launch_bounds__(kSumThreads)
sum_offsets(const T* __restrict__ g, int wh, int ww, float* __restrict__ part, int heads) {   // part [slices][heads][offsets]
    const int pitch = 2 * ww - 1, dys = 2 * wh - 1, groups = (pitch + 31) / 32, tokens = wh * ww;
    int id = blockIdx.x;
    const int group = id % groups; id /= groups;
    const int dy = id % dys - (wh - 1), head = id / dys, slice = blockIdx.y;
    const int dx0 = group * 32 - (ww - 1);
    if (slice >= slices_at(wh, ww, dy, dx0)) return;
    int x_first;
    const int cols = walk_columns(ww, dx0, &x_first);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, y_first = max(dy, 0), y_end = min(wh, wh + dy), dx = dx0 + lane;
    const T* gh = g + (size_t)head * tokens * tokens - (ptrdiff_t)dy * ww - dx;   // + i tokens + yi ww + xi: the pair of query i = (yi, xi)
    float sum[2] = {0.0f, 0.0f};
    if (wh < kFewRows) {
        const int end = x_first + min(cols, (slice + 1) * kColSlice);
        const size_t step = (size_t)kSumWarps * (tokens + 1);
        for (int yi = y_first; yi < y_end; ++yi) {
            int xi = x_first + slice * kColSlice + warp;
            const T* p = gh + ((size_t)yi * ww + xi) * tokens + yi * ww + xi;
            for (; xi < end; xi += kUnroll * kSumWarps, p += kUnroll * step) {
                float v[kUnroll];
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) {
                    const int x = xi + u * kSumWarps;
                    v[u] = x < end && (unsigned)(x - dx) < (unsigned)ww ? Elem<T>::to_f32(p[u * step]) : 0.0f;
                }
#pragma unroll
                for (int u = 0; u < kUnroll; ++u) sum[u & 1] += v[u];
            }
        }
    } else {
        const int from = y_first + slice * kRowSlice, rows = min(kRowSlice, y_end - from);
        const size_t step = (size_t)ww * tokens + ww;
        for (int xi = x_first + warp; xi < x_first + cols; xi += kSumWarps) {
            const bool in = (unsigned)(xi - dx) < (unsigned)ww;
            const T* p = gh + ((size_t)from * ww + xi) * tokens + from * ww + xi;
            float v[kRowSlice];
#pragma unroll
            for (int u = 0; u < kRowSlice; ++u) v[u] = in && u < rows ? Elem<T>::to_f32(p[u * step]) : 0.0f;
#pragma unroll
            for (int u = 0; u < kRowSlice; ++u) sum[u & 1] += v[u];
        }
    }
    __shared__ float warps[kSumWarps][32];
    float total = sum[0] + sum[1];
    warps[warp][lane] = total;
    __syncthreads();
    if (warp == 0 && group * 32 + lane < pitch) {
#pragma unroll
        for (int w = 1; w < kSumWarps; ++w) total += warps[w][lane];
        part[((size_t)slice * heads + head) * dys * pitch + (size_t)(dy + wh - 1) * pitch + group * 32 + lane] = total;
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
    __shared__ float2 past[8][32];
    float sum = 0.0f;
    for (int first = warp * 32; first < offsets; first += 4 * 256) {
        float v[4];
        int b[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int at = first + u * 256 + lane;
            v[u] = at < offsets ? dense[(size_t)head * offsets + at] : 0.0f;
            b[u] = at < offsets ? bucket[at] : -1;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            unsigned left = __ballot_sync(0xffffffffu, b[u] >= 0 && (unsigned)(b[u] - (int)blockIdx.x * 32) < 32u);
            if (left == 0) continue;     // none of the 32 offsets is of these buckets
            __syncwarp();
            past[warp][lane] = make_float2(v[u], __int_as_float(b[u]));
            __syncwarp();
            if (__popc(left) > 8) {
#pragma unroll
                for (int src = 0; src < 32; ++src) {
                    const float2 x = past[warp][src];
                    if (__float_as_int(x.y) == mine) sum += x.x;
                }
            } else {
                for (; left; left &= left - 1) {
                    const float2 x = past[warp][__ffs(left) - 1];
                    if (__float_as_int(x.y) == mine) sum += x.x;
                }
            }
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
