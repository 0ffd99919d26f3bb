// C ABI of the window self-attention and of its relative position bias: argument checks, kernel selection and launches.
#include "abi.h"

#include <algorithm>
#include <cmath>

#include "relpos_bias.cuh"
#include "window_attention.cuh"
#include "window_attention_backward.cuh"

namespace {

namespace abi = esc::abi;
namespace rp = esc::relpos;
namespace wa = esc::winatt;
using bf16 = __nv_bfloat16;

bool known(int dtype) { return dtype == ESC_F32 || dtype == ESC_BF16; }

constexpr size_t kMostSmem = 227 * 1024;           // of a block

// Shared memory beyond 48 KB, once more for every call: the attribute belongs to the kernel on the current device, and setting it
// again is cheaper than remembering which devices have it.  Always the same value: another thread may be between this and its launch.
template <typename K> int allow_smem(K kernel, size_t bytes) {
    if (bytes > 48 * 1024) ESC_ABI_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMostSmem));
    return ESC_OK;
}
#define ESC_TRY(call)                    \
    do {                                 \
        const int rc__ = (call);         \
        if (rc__ != ESC_OK) return rc__; \
    } while (0)

int launched() {
    ESC_ABI_CUDA(cudaGetLastError());
    abi::launched();
    return ESC_OK;
}

// ---- relative position bias ---------------------------------------------------------------------------------------------
int check_window(int heads, int win_h, int win_w) {
    if (heads <= 0 || win_h <= 0 || win_w <= 0) return ESC_ERR_SHAPE;
    if (heads > 65535 || win_h > rp::kMaxOffsets || win_w > rp::kMaxOffsets || rp::offsets_of(win_h, win_w) > rp::kMaxOffsets) return ESC_ERR_UNSUPPORTED;
    return ESC_OK;
}
int check_buckets(const int* bucket, int n_buckets, int win_h, int win_w) {
    if (n_buckets <= 0 || (!bucket && n_buckets != rp::offsets_of(win_h, win_w))) return ESC_ERR_SHAPE;
    if (n_buckets > 1 << 30) return ESC_ERR_UNSUPPORTED;   // sum_buckets numbers them in an int, 32 to a block
    if (!abi::aligned(bucket, 4)) return ESC_ERR_ALIGN;
    return ESC_OK;
}

// Behind the sums of `slices` partial sums per offset: into the table, through the offsets' buckets where there are any.
template <typename G>
int launch_table_sums(const float* part, float* dense, int slices, bool per_offset, int heads, int wh, int ww, const int* bucket, int n_buckets,
                      G* g_table, cudaStream_t st) {
    const int offsets = (int)rp::offsets_of(wh, ww);
    rp::sum_slices<G><<<dim3((offsets + 31) / 32, heads), 256, 0, st>>>(part, slices, per_offset, heads, wh, ww, bucket ? dense : nullptr, g_table);
    ESC_TRY(launched());
    if (!bucket) return ESC_OK;
    rp::sum_buckets<G><<<dim3((n_buckets + 31) / 32, heads), 256, 0, st>>>(dense, bucket, n_buckets, heads, offsets, g_table);
    return launched();
}

template <typename T>
int bias_forward_t(const void* table, const int* bucket, int n_buckets, int heads, int wh, int ww, void* bias, cudaStream_t st) {
    const int groups = (ww + rp::kRows - 1) / rp::kRows;
    const size_t smem = (size_t)rp::strip_floats(wh, ww, esc::Elem<T>::kVec) * sizeof(float);
    ESC_TRY(allow_smem(rp::fill<T>, smem));
    rp::fill<T><<<(unsigned)(heads * wh * groups), rp::kFillThreads, smem, st>>>(static_cast<const T*>(table), bucket, n_buckets, heads, wh, ww, static_cast<T*>(bias));
    return launched();
}

template <typename T>
int bias_backward_t(const void* grad_bias, const int* bucket, int n_buckets, int heads, int wh, int ww, float* g_table, float* ws, cudaStream_t st) {
    const int slices = rp::most_slices(wh, ww), groups = (2 * ww - 1 + 31) / 32;
    float* dense = ws + (size_t)slices * heads * rp::offsets_of(wh, ww);
    rp::sum_offsets<T><<<dim3((unsigned)(heads * (2 * wh - 1) * groups), slices), rp::kSumThreads, 0, st>>>(static_cast<const T*>(grad_bias), wh, ww, ws, heads);
    ESC_TRY(launched());
    return launch_table_sums<float>(ws, dense, slices, true, heads, wh, ww, bucket, n_buckets, g_table, st);
}

// ---- window attention ----------------------------------------------------------------------------------------------------
struct Call {
    const void *q, *k, *v;
    int B, heads, d, H, W;
    long long stride;
    int wh, ww;
    const void* table;
    const int* bucket;
    int n_buckets;
    float scale;
    int dtype;
    size_t es() const { return abi::elem_size(dtype); }
    long long pixels() const { return (long long)B * H * W; }
    size_t dense_bytes() const { return (size_t)pixels() * heads * d * es(); }
    size_t strided_bytes() const { return ((size_t)(pixels() - 1) * stride + (size_t)heads * d) * es(); }
    int ny() const { return (int)(((long long)H + wh - 1) / wh); }   // H + wh can be more than an int holds
    int nx() const { return (int)(((long long)W + ww - 1) / ww); }
    long long windows() const { return (long long)B * ny() * nx(); }
    int tokens() const { return std::min(wh, H) * std::min(ww, W); }   // of the largest window
};

int check_sizes(int B, int heads, int d, int H, int W, int wh, int ww) {
    if (B <= 0 || heads <= 0 || d <= 0 || H <= 0 || W <= 0) return ESC_ERR_SHAPE;
    if (d > wa::kMaxHeadDim) return ESC_ERR_UNSUPPORTED;
    ESC_TRY(check_window(heads, wh, ww));
    const long double n = (long double)B * heads * H * W;
    if (n * d > 1.0e15L) return ESC_ERR_SHAPE;
    if ((long double)std::min(wh, H) * W > 2.0e9L) return ESC_ERR_UNSUPPORTED;   // a pixel's distance from its window's first
    // one block per window, head and tile of queries (at least 32 of them)
    const long double blocks = (long double)B * (((long long)H + wh - 1) / wh) * (((long long)W + ww - 1) / ww) * heads * ((std::min(wh, H) * std::min(ww, W) + 31) / 32);
    return blocks > 1.0e9L ? ESC_ERR_UNSUPPORTED : ESC_OK;
}

int check_call(const Call& c) {
    ESC_TRY(check_sizes(c.B, c.heads, c.d, c.H, c.W, c.wh, c.ww));
    if (!known(c.dtype)) return ESC_ERR_UNSUPPORTED;
    if (!c.q || !c.k || !c.v) return ESC_ERR_NULL;
    if (c.stride < (long long)c.heads * c.d || (long double)c.pixels() * c.stride > 4.0e15L) return ESC_ERR_SHAPE;
    if (!(c.scale >= 1e-6f && c.scale <= 1e6f)) return ESC_ERR_UNSUPPORTED;
    for (const void* p : {c.q, c.k, c.v, c.table})
        if (!abi::aligned(p, c.es())) return ESC_ERR_ALIGN;
    return c.table ? check_buckets(c.bucket, c.n_buckets, c.wh, c.ww) : ESC_OK;
}

template <typename T> wa::Maps<T> maps_of(const Call& c) {
    wa::Maps<T> m;
    m.q = static_cast<const T*>(c.q); m.k = static_cast<const T*>(c.k); m.v = static_cast<const T*>(c.v);
    m.stride = c.stride;
    m.B = c.B; m.heads = c.heads; m.d = c.d; m.H = c.H; m.W = c.W; m.wh = c.wh; m.ww = c.ww; m.ny = c.ny(); m.nx = c.nx();
    m.table = static_cast<const T*>(c.table); m.bucket = c.bucket; m.n_buckets = c.n_buckets;
    m.scale = c.scale; m.inv_scale = 1.0f / c.scale;
    return m;
}

// Threads of a block whose threads take `per_thread` rows each, or `lanes` threads one: as few blocks per window as the most threads
// allow, and those evenly filled.
struct Tiling { int tiles, threads; };
Tiling tile_rows(int tokens, int most_threads, int per_thread, int lanes) {
    const int most = most_threads * per_thread / lanes, tiles = (tokens + most - 1) / most;
    const int rows = (tokens + tiles - 1) / tiles;
    const int threads = ((rows * lanes + per_thread - 1) / per_thread + 31) / 32 * 32;
    const int per_tile = threads * per_thread / lanes;
    return {(tokens + per_tile - 1) / per_tile, threads};
}

template <int D, int Q> int forward_f32_q(const Call& c, void* out, float* lse, cudaStream_t st) {
    using namespace wa::f32;
    const Tiling t = tile_rows(c.tokens(), kThreads, Q, 1);
    const size_t smem = (size_t)(2 * kKeys * D + kKeys + rp::offsets_of(c.wh, c.ww)) * sizeof(float);
    ESC_TRY(allow_smem(forward<D, Q>, smem));
    forward<D, Q><<<(unsigned)(c.windows() * c.heads * t.tiles), t.threads, smem, st>>>(maps_of<float>(c), t.tiles, static_cast<float*>(out), lse);
    return launched();
}
// Two queries a thread halve the reads of keys and values; not where that leaves the SMs fewer than 16 warps each, or a thread too many channels.
// 427x240, windows of 24, 4 heads of 16: 593 us with two, 637 with one; 4 x 64x64, 3 heads: 150 with two, 112 with one.
template <int D> int forward_f32(const Call& c, void* out, float* lse, cudaStream_t st) {
    const bool many = c.windows() * c.heads * c.tokens() >= 2LL * 16 * 32 * abi::sm_count();
    return D <= 16 && many ? forward_f32_q<D, D <= 16 ? 2 : 1>(c, out, lse, st) : forward_f32_q<D, 1>(c, out, lse, st);
}

template <int D, bool TWICE, int MT> int forward_bf16_t(const Call& c, void* out, float* lse, cudaStream_t st) {
    using namespace wa::tc;
    constexpr int rows = 16 * MT;
    const int most = (c.tokens() + rows - 1) / rows, tiles = (most + kMaxWarps - 1) / kMaxWarps, warps = (most + tiles - 1) / tiles;
    const size_t smem = Smem<D>::bytes(Bias(c.wh, c.ww), TWICE);
    ESC_TRY(allow_smem(forward<D, TWICE, MT>, smem));
    forward<D, TWICE, MT><<<(unsigned)(c.windows() * c.heads * tiles), warps * 32, smem, st>>>(maps_of<bf16>(c), tiles, static_cast<bf16*>(out), lse);
    return launched();
}
// The most queries a warp can have, unless that leaves fewer blocks than SMs: then a tile of queries a warp.  64x64, windows of 32, 4 heads of
// 16 (64 or 128 blocks): 30.6 us with two tiles, 22.5 with one; 640x360 (3,840 blocks): 400 with two, 515 with one.
template <int D, bool TWICE> int forward_bf16_b(const Call& c, void* out, float* lse, cudaStream_t st) {
    using namespace wa::tc;
    constexpr int MT = most_tiles(D);
    const long long blocks = c.windows() * c.heads * ((c.tokens() + 16 * MT * kMaxWarps - 1) / (16 * MT * kMaxWarps));
    if (blocks < abi::sm_count()) return forward_bf16_t<D, TWICE, 1>(c, out, lse, st);
    return forward_bf16_t<D, TWICE, MT>(c, out, lse, st);
}
// Two copies of the table where they leave room for two blocks on an SM.
template <int D> int forward_bf16(const Call& c, void* out, float* lse, cudaStream_t st) {
    return wa::tc::Smem<D>::bytes(wa::tc::Bias(c.wh, c.ww), true) <= 112 * 1024 ? forward_bf16_b<D, true>(c, out, lse, st) : forward_bf16_b<D, false>(c, out, lse, st);
}

// The fp32 kernel that adds up sums for the table's gradient: one copy of the offsets per warp beside the table and the staged rows of D
// channels.  Its groups: as many blocks as the SMs hold, at most four each.
struct SumsPlan { Tiling t; size_t smem; int groups; };
SumsPlan sums_plan(const Call& c, int D, bool sums) {
    using namespace wa::bwd::f32;
    const size_t offsets = (size_t)rp::offsets_of(c.wh, c.ww) * sizeof(float), rest = (2 * kRows * D + kRows) * sizeof(float);
    const int warps = sums ? (int)std::min<size_t>(kThreads / 32, (kMostSmem - rest) / offsets - 1) : kThreads / 32;
    SumsPlan p;
    p.t = tile_rows(c.tokens(), warps * 32, 1, lanes_of(D));
    p.smem = rest + offsets * (sums ? 1 + p.t.threads / 32 : 1);
    const long long units = c.windows() * p.t.tiles, per_sm = std::max<long long>(1, std::min<long long>(4, kMostSmem / (p.smem + 1024)));
    p.groups = (int)std::min<long long>(units, sums ? std::max(1LL, per_sm * abi::sm_count() / c.heads) : 0x7fffffff / c.heads);
    return p;
}
int padded(int d) { return d <= 16 ? 16 : d <= 32 ? 32 : 64; }
int table_groups(const Call& c) { return sums_plan(c, padded(c.d), true).groups; }

// And of the tensor-core kernel, whose blocks have a tile of keys each: the tiles of queries, then the windows are dealt to as many as fill
// two rounds of two blocks per SM.
int key_tiles(const Call& c) { return (c.tokens() + wa::bwd::tc::kPairK - 1) / wa::bwd::tc::kPairK; }
int pair_parts(const Call& c) {
    const long long want = std::max(1LL, 4LL * abi::sm_count() / ((long long)c.heads * key_tiles(c)));
    return (int)std::min<long long>(want, (c.tokens() + wa::bwd::tc::kPairQ - 1) / wa::bwd::tc::kPairQ);
}
int pair_groups(const Call& c) {
    const long long want = std::max(1LL, 4LL * abi::sm_count() / ((long long)c.heads * key_tiles(c) * pair_parts(c)));
    return (int)std::min(want, c.windows());
}
int pair_slices(const Call& c) { return pair_groups(c) * pair_parts(c) * key_tiles(c); }
int table_slices(const Call& c) { return c.dtype == ESC_BF16 ? pair_slices(c) : table_groups(c); }

struct BackwardWs { float *bases, *dots, *part, *dense; size_t bytes; };
BackwardWs carve(void* ws, const Call& c) {
    BackwardWs w;
    char* base = static_cast<char*>(ws);
    size_t off = 0;
    auto take = [&](size_t floats) { float* p = reinterpret_cast<float*>(base + off); off += abi::round_up(floats * sizeof(float), 256); return p; };
    const size_t offsets = (size_t)rp::offsets_of(c.wh, c.ww) * c.heads;
    w.bases = take((size_t)c.pixels() * c.heads);
    w.dots = take((size_t)c.pixels() * c.heads);
    w.part = take(offsets * std::max(table_groups(c), pair_slices(c)));
    w.dense = take(offsets);
    w.bytes = off;
    return w;
}

template <int D> int backward_f32(const Call& c, wa::bwd::Grads<float> g, cudaStream_t st) {
    using namespace wa::bwd::f32;
    const wa::Maps<float> m = maps_of<float>(c);
    const size_t offsets = (size_t)rp::offsets_of(c.wh, c.ww);
    const Tiling t = tile_rows(c.tokens(), kThreads, 1, lanes_of(D));
    const size_t smem = (2 * kRows * D + 3 * kRows + offsets) * sizeof(float);
    ESC_TRY(allow_smem(grad_kv<D>, smem));
    grad_kv<D><<<(unsigned)(c.windows() * c.heads * t.tiles), t.threads, smem, st>>>(m, g, t.tiles);
    ESC_TRY(launched());
    const SumsPlan p = sums_plan(c, D, g.part != nullptr);
    g.groups = p.groups;
    ESC_TRY(allow_smem(grad_q<D>, p.smem));
    grad_q<D><<<(unsigned)(g.groups * c.heads), p.t.threads, p.smem, st>>>(m, g, p.t.tiles);
    return launched();
}

template <int D, bool KEYS, bool TWICE> int grad_rows_bf16(const Call& c, const wa::bwd::Grads<bf16>& g, cudaStream_t st) {
    using namespace wa::bwd::tc;
    constexpr int rows = 16 * grad_tiles(D);
    const int most = (c.tokens() + rows - 1) / rows, tiles = (most + kMaxWarps - 1) / kMaxWarps, warps = (most + tiles - 1) / tiles;
    const size_t smem = RowSmem<D>::bytes(Bias(c.wh, c.ww), TWICE);
    ESC_TRY(allow_smem(grad_rows<D, KEYS, TWICE>, smem));
    grad_rows<D, KEYS, TWICE><<<(unsigned)(c.windows() * c.heads * tiles), warps * 32, smem, st>>>(maps_of<bf16>(c), g, tiles);
    return launched();
}
template <int D> int backward_bf16(const Call& c, wa::bwd::Grads<bf16> g, cudaStream_t st) {
    using namespace wa::bwd::tc;
    const bool twice = RowSmem<D>::bytes(Bias(c.wh, c.ww), true) <= (D <= 16 ? 112 : 224) * 1024;
    ESC_TRY(twice ? (grad_rows_bf16<D, false, true>(c, g, st)) : (grad_rows_bf16<D, false, false>(c, g, st)));   // first: it makes D exact
    ESC_TRY(twice ? (grad_rows_bf16<D, true, true>(c, g, st)) : (grad_rows_bf16<D, true, false>(c, g, st)));
    if (!g.part) return ESC_OK;
    g.groups = pair_groups(c);
    const int offsets = (int)rp::offsets_of(c.wh, c.ww);
    const bool staged = PairSmem<D>::bytes(offsets, true) <= kMostSmem;
    const size_t smem = PairSmem<D>::bytes(offsets, staged);
    ESC_TRY(allow_smem(grad_table<D>, smem));
    grad_table<D><<<(unsigned)(pair_slices(c) * c.heads), 256, smem, st>>>(maps_of<bf16>(c), g, key_tiles(c), pair_parts(c), staged);
    return launched();
}

template <typename T> int launch_row_terms(const Call& c, const void* go, const void* out, const float* lse, const BackwardWs& w, cudaStream_t st) {
    using namespace wa::bwd;
    const long long items = c.pixels() * c.heads;
    const unsigned blocks = (unsigned)std::min<long long>((items + kRowThreads - 1) / kRowThreads, 16LL * abi::sm_count());
    row_terms<T><<<blocks, kRowThreads, 0, st>>>(static_cast<const T*>(go), static_cast<const T*>(out), lse, c.pixels(), (long long)c.H * c.W, c.heads, c.d, w.bases, w.dots);
    return launched();
}

// Whether two runs of heads*d values every `stride` values share any: tensors of their own, or slices of one packed tensor.
bool interleave(const void* a, const void* b, const Call& c) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    const uintptr_t far = x > y ? x - y : y - x;
    const size_t run = (size_t)c.heads * c.d * c.es(), step = (size_t)c.stride * c.es();
    if (far >= c.strided_bytes()) return false;
    return far % step < run || step - far % step < run;
}

}  // namespace

extern "C" {

int esc_relpos_bias_forward(const void* table, const int* bucket, int n_buckets, int heads, int win_h, int win_w, void* bias, int dtype, void* stream) {
    abi::launches_reset();
    ESC_TRY(check_window(heads, win_h, win_w));
    ESC_TRY(check_buckets(bucket, n_buckets, win_h, win_w));
    if (!known(dtype)) return ESC_ERR_UNSUPPORTED;
    if (!table || !bias) return ESC_ERR_NULL;
    if (!abi::aligned(table, abi::elem_size(dtype)) || !abi::aligned(bias, 16)) return ESC_ERR_ALIGN;
    const size_t tokens = (size_t)win_h * win_w, es = abi::elem_size(dtype);
    if (abi::overlap(table, (size_t)n_buckets * heads * es, bias, tokens * tokens * heads * es)) return ESC_ERR_ALIAS;
    if ((long double)heads * win_h * ((win_w + rp::kRows - 1) / rp::kRows) > 2.0e9L) return ESC_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dtype == ESC_F32 ? bias_forward_t<float>(table, bucket, n_buckets, heads, win_h, win_w, bias, st)
                            : bias_forward_t<bf16>(table, bucket, n_buckets, heads, win_h, win_w, bias, st);
}

size_t esc_relpos_bias_workspace_bytes(int heads, int win_h, int win_w) {
    if (check_window(heads, win_h, win_w) != ESC_OK) return 0;
    return abi::round_up((size_t)(rp::most_slices(win_h, win_w) + 1) * heads * rp::offsets_of(win_h, win_w) * sizeof(float), 256);
}

int esc_relpos_bias_backward(const void* grad_bias, const int* bucket, int n_buckets, int heads, int win_h, int win_w, float* grad_table, int dtype,
                             void* workspace, size_t workspace_bytes, void* stream) {
    abi::launches_reset();
    ESC_TRY(check_window(heads, win_h, win_w));
    ESC_TRY(check_buckets(bucket, n_buckets, win_h, win_w));
    if (!known(dtype)) return ESC_ERR_UNSUPPORTED;
    if (!grad_bias || !grad_table) return ESC_ERR_NULL;
    if (!abi::aligned(grad_bias, abi::elem_size(dtype)) || !abi::aligned(grad_table, 4)) return ESC_ERR_ALIGN;
    const size_t tokens = (size_t)win_h * win_w;
    if (abi::overlap(grad_table, (size_t)n_buckets * heads * 4, grad_bias, tokens * tokens * heads * abi::elem_size(dtype))) return ESC_ERR_ALIAS;
    if (!workspace || !abi::aligned(workspace, 256) || workspace_bytes < esc_relpos_bias_workspace_bytes(heads, win_h, win_w)) return ESC_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    float* ws = static_cast<float*>(workspace);
    return dtype == ESC_F32 ? bias_backward_t<float>(grad_bias, bucket, n_buckets, heads, win_h, win_w, grad_table, ws, st)
                            : bias_backward_t<bf16>(grad_bias, bucket, n_buckets, heads, win_h, win_w, grad_table, ws, st);
}

int esc_window_attention_forward(const void* q, const void* k, const void* v, int B, int heads, int head_dim, int H, int W, long long pixel_stride,
                                 int win_h, int win_w, const void* table, const int* bucket, int n_buckets, float scale, void* out, float* lse,
                                 int dtype, void* stream) {
    abi::launches_reset();
    const Call c{q, k, v, B, heads, head_dim, H, W, pixel_stride, win_h, win_w, table, bucket, n_buckets, scale, dtype};
    ESC_TRY(check_call(c));
    if (!out) return ESC_ERR_NULL;
    if (!abi::aligned(out, 16) || !abi::aligned(lse, 4)) return ESC_ERR_ALIGN;
    for (const void* p : {q, k, v})
        if (abi::overlap(out, c.dense_bytes(), p, c.strided_bytes()) || (lse && abi::overlap(lse, (size_t)c.pixels() * heads * 4, p, c.strided_bytes()))) return ESC_ERR_ALIAS;
    if (lse && abi::overlap(lse, (size_t)c.pixels() * heads * 4, out, c.dense_bytes())) return ESC_ERR_ALIAS;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (dtype == ESC_BF16)
        return head_dim <= 16 ? forward_bf16<16>(c, out, lse, st) : head_dim <= 32 ? forward_bf16<32>(c, out, lse, st) : forward_bf16<64>(c, out, lse, st);
    return head_dim <= 16 ? forward_f32<16>(c, out, lse, st) : head_dim <= 32 ? forward_f32<32>(c, out, lse, st) : forward_f32<64>(c, out, lse, st);
}

size_t esc_window_attention_backward_workspace_bytes(int B, int heads, int head_dim, int H, int W, int win_h, int win_w) {
    if (check_sizes(B, heads, head_dim, H, W, win_h, win_w) != ESC_OK) return 0;
    const Call c{nullptr, nullptr, nullptr, B, heads, head_dim, H, W, 0, win_h, win_w, nullptr, nullptr, 0, 1.0f, ESC_F32};
    return carve(nullptr, c).bytes;
}

int esc_window_attention_backward(const void* q, const void* k, const void* v, int B, int heads, int head_dim, int H, int W, long long pixel_stride,
                                  int win_h, int win_w, const void* table, const int* bucket, int n_buckets, float scale, const void* out,
                                  const float* lse, const void* grad_out, void* grad_q, void* grad_k, void* grad_v, void* grad_table, int dtype,
                                  void* workspace, size_t workspace_bytes, void* stream) {
    abi::launches_reset();
    const Call c{q, k, v, B, heads, head_dim, H, W, pixel_stride, win_h, win_w, table, bucket, n_buckets, scale, dtype};
    ESC_TRY(check_call(c));
    if (!out || !lse || !grad_out || !grad_q || !grad_k || !grad_v) return ESC_ERR_NULL;
    if (grad_table && !table) return ESC_ERR_NULL;
    if (!abi::aligned(out, 16) || !abi::aligned(grad_out, 16) || !abi::aligned(lse, 4)) return ESC_ERR_ALIGN;
    for (const void* p : {static_cast<const void*>(grad_q), static_cast<const void*>(grad_k), static_cast<const void*>(grad_v), static_cast<const void*>(grad_table)})
        if (!abi::aligned(p, c.es())) return ESC_ERR_ALIGN;
    if (interleave(grad_q, grad_k, c) || interleave(grad_q, grad_v, c) || interleave(grad_k, grad_v, c)) return ESC_ERR_ALIAS;
    for (const void* g : {static_cast<const void*>(grad_q), static_cast<const void*>(grad_k), static_cast<const void*>(grad_v)}) {
        for (const void* p : {q, k, v})
            if (abi::overlap(g, c.strided_bytes(), p, c.strided_bytes())) return ESC_ERR_ALIAS;
        if (abi::overlap(g, c.strided_bytes(), out, c.dense_bytes()) || abi::overlap(g, c.strided_bytes(), grad_out, c.dense_bytes()) ||
            abi::overlap(g, c.strided_bytes(), lse, (size_t)c.pixels() * heads * 4)) return ESC_ERR_ALIAS;
    }
    const BackwardWs w = carve(workspace, c);
    if (!workspace || !abi::aligned(workspace, 256) || workspace_bytes < w.bytes) return ESC_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int slices = table_slices(c);
    float* part = grad_table ? w.part : nullptr;
    if (dtype == ESC_BF16) {
        ESC_TRY(launch_row_terms<bf16>(c, grad_out, out, lse, w, st));
        const wa::bwd::Grads<bf16> g{static_cast<const bf16*>(grad_out), w.bases, w.dots, static_cast<bf16*>(grad_q), static_cast<bf16*>(grad_k), static_cast<bf16*>(grad_v),
                                     part, (int)c.windows(), 0};
        ESC_TRY(head_dim <= 16 ? backward_bf16<16>(c, g, st) : head_dim <= 32 ? backward_bf16<32>(c, g, st) : backward_bf16<64>(c, g, st));
        if (!part) return ESC_OK;
        return launch_table_sums<bf16>(part, w.dense, slices, false, heads, win_h, win_w, bucket, n_buckets, static_cast<bf16*>(grad_table), st);
    }
    ESC_TRY(launch_row_terms<float>(c, grad_out, out, lse, w, st));
    const wa::bwd::Grads<float> g{static_cast<const float*>(grad_out), w.bases, w.dots, static_cast<float*>(grad_q), static_cast<float*>(grad_k), static_cast<float*>(grad_v),
                                  part, (int)c.windows(), table_groups(c)};
    ESC_TRY(head_dim <= 16 ? backward_f32<16>(c, g, st) : head_dim <= 32 ? backward_f32<32>(c, g, st) : backward_f32<64>(c, g, st));
    if (!part) return ESC_OK;
    return launch_table_sums<float>(part, w.dense, slices, false, heads, win_h, win_w, bucket, n_buckets, static_cast<float*>(grad_table), st);
}

}  // extern "C"
