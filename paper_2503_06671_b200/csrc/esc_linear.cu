// C ABI of the linear layers: argument checks, kernel selection and launches.
#include "rows.h"

#include <algorithm>
#include <type_traits>

#include "linear_backward_small.cuh"
#include "linear_few.cuh"

namespace {

namespace abi = esc::abi;
namespace lin = esc::linear;
namespace um = esc::linear::umma;
namespace sm = esc::linear::small;
namespace fw = esc::linear::few;
using namespace esc::rows;
using bf16 = __nv_bfloat16;

struct Call {
    const void* x;
    long long x_stride;
    const void* w;
    long long rows;
    int K, N, act, dtype;
    size_t es() const { return abi::elem_size(dtype); }
    Matrix mx() const { return Matrix{x, rows, x_stride, K, es()}; }
    Matrix mw() const { return flat(w, (long long)N * K, es()); }
    Matrix out(const void* p, long long width) const { return Matrix{p, rows, width, width, es()}; }
};

constexpr int kMaxWidth = 1 << 20;

int check_sizes(long long rows, int K, int N, int act, int dtype) {
    if (rows < 0 || K <= 0 || N <= 0) return ESC_ERR_SHAPE;
    if (!known(dtype) || act < ESC_ACT_NONE || act > ESC_ACT_GELU) return ESC_ERR_UNSUPPORTED;
    if (K > kMaxWidth || N > kMaxWidth || rows > 0x7fffffffLL - 4096) return ESC_ERR_UNSUPPORTED;
    return ESC_OK;
}
int check_call(const Call& c) {
    ESC_TRY(check_sizes(c.rows, c.K, c.N, c.act, c.dtype));
    ESC_TRY(check_rows(c.rows, c.K, c.x_stride));
    if (!c.w || (!c.x && c.rows > 0)) return ESC_ERR_NULL;
    for (const void* p : {c.x, c.w})
        if (!abi::aligned(p, c.es())) return ESC_ERR_ALIGN;
    return ESC_OK;
}

template <typename T> lin::Layer<T> layer_of(const Call& c) {
    lin::Layer<T> p{};
    p.x = static_cast<const T*>(c.x); p.w = static_cast<const T*>(c.w);
    p.x_stride = c.x_stride; p.rows = c.rows; p.K = c.K; p.N = c.N; p.act = c.act;
    return p;
}

// ---- tensor-core products ----------------------------------------------------------------------------------------------------

// What a product is cut into (`runs`: its sums end, after run_of blocks; otherwise its runs of rows have kLongRun blocks at most).  Times in cycles of an SM, from the rates below; the cheapest width of a tile and number of runs of rows.
struct Cut {
    int tiles_i, tiles_j, bn, splits, stages, grid;
    bool resident, single;
    size_t smem;
};
constexpr double kLoadRate = 35, kStoreRate = 20;   // bytes per cycle of one SM: from L2 into its ring, to memory
Cut cut(lin::Role role, long long I, int J, long long depth, size_t es, bool tma, bool runs) {
    const int sms = abi::sm_count(), step = role == lin::kForward ? 16 : 64, most = es == 4 ? um::most_columns<float> : um::most_columns<bf16>, most_run = es == 4 ? um::most_run_columns<float> : um::most_run_columns<bf16>;
    const int parts = es == 4 ? 3 : 1, products = es == 4 ? 6 : 1;
    const long long blocks = (depth + um::kBlockC - 1) / um::kBlockC, tiles_i = (I + um::kBlockI - 1) / um::kBlockI;
    const size_t out_es = role == lin::kGradW ? 4 : es, epi = tma ? um::epi_warps<true> : um::epi_warps<false>;
    const int unit = (int)(128 / out_es), run = um::run_of(role, es);   // unit: columns that leave together
    const long long least_splits = runs ? 1 : (blocks + um::kLongRun - 1) / um::kLongRun;
    Cut best{};
    double least = 1e300;
    for (int bn = std::min(most / step, (J + step - 1) / step) * step; bn >= step; bn -= step) {
        const long long tiles_j = ((long long)J + bn - 1) / bn;
        if (tiles_j > 1 && bn > unit && bn % unit != 0) continue;
        // w stays where it leaves room for a ring of rows and a block has several tiles
        const size_t b_bytes = (size_t)bn * 128 * parts, a_bytes = (size_t)um::kABytes * parts, fixed = epi * (um::kSlotBytes + 256) + 1024;   // with a strip of an epilogue warp, and the barriers
        const bool resident = role != lin::kGradW && blocks * b_bytes + fixed + 3 * a_bytes <= um::kMostSmem && tiles_j <= sms && tiles_i * tiles_j >= 2LL * sms;
        const size_t kept = resident ? blocks * b_bytes : 0, stage = a_bytes + (resident ? 0 : b_bytes);
        const int stages = (int)std::min<long long>(um::kMaxStages, ((long long)um::kMostSmem - (long long)(fixed + kept)) / (long long)stage);
        if (stages < 1 || (stages < 2 && bn > step)) continue;
        const double rows = (double)std::min<long long>(I, um::kBlockI), b_rows = resident ? 0 : bn;
        const double mma = 4.0 * products * std::max(40.0, bn / 2.0), load = (rows + b_rows) * um::kBlockC * es / kLoadRate, store = rows * bn * out_es / kStoreRate;
        // runs of rows: one, or as many as fill the SMs one to four times
        for (int fill = 0; fill <= (role == lin::kGradW ? 4 : 0); ++fill) {
            const long long splits = fill == 0 ? least_splits : std::min<long long>(blocks, (long long)fill * sms / (tiles_i * tiles_j));
            const long long units = tiles_i * tiles_j * splits, waves = (units + sms - 1) / sms;
            if (splits < least_splits || units > 0x7fffffffLL) continue;
            // runs of c: a narrow tile, or fp32 with one buffer for sums, which waits while they are added (about 1500 cycles)
            const long long each = (blocks + splits - 1) / splits;
            const bool single = runs && bn > most_run && each > run;
            if (single && es == 2) continue;
            const double body = (double)each * std::max(mma, load) + (single ? 1500.0 * (each / run) : 0.0);
            double cost = (double)waves * (std::max(body, store) + 200) + std::min(body, store) + 1500;
            if (role == lin::kGradW) cost += 2.0 * splits * I * J * 4 / (kStoreRate * sms);
            if (cost < least * 0.995) {
                least = cost;
                best = Cut{(int)tiles_i, (int)tiles_j, bn, (int)splits, stages, resident ? (int)(sms / tiles_j * tiles_j) : (int)std::min<long long>(units, sms), resident, single,
                           stages * stage + kept + fixed};
            }
        }
    }
    return best;
}

// Matrices [batch, rows, width] whose rows are `ld` values apart, in boxes of 128 bytes of `box_rows` rows.
template <typename T> bool map_of(CUtensorMap* m, const void* base, long long batch, long long rows, long long width, long long ld, int box_rows) {
    constexpr size_t es = sizeof(T);
    const bool flat = batch == 0;                                  // two dimensions
    const cuuint64_t dims[3] = {(cuuint64_t)width, (cuuint64_t)rows, (cuuint64_t)batch}, strides[2] = {(cuuint64_t)ld * es, (cuuint64_t)rows * ld * es};
    const cuuint32_t box[3] = {128 / es, (cuuint32_t)box_rows, 1}, ones[3] = {1, 1, 1};
    um::EncodeTiledFn fn = um::encode_fn();
    return fn && fn(m, es == 2 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, flat ? 2 : 3, const_cast<void*>(base), dims, strides, box, ones,
                    CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool whole_pieces(const void* p, long long ld, size_t es) { return abi::aligned(p, 16) && (size_t)ld * es % 16 == 0; }

// The result lies in memory as O [splits, I, J].  Returns the number of splits through `splits`.  `beside`: the kernel before it in the stream
// (the other product of the same g, or grad_out's column sums) need not have ended.
template <typename T, lin::Role ROLE> int launch_product(um::Args<T> p, long long depth, bool runs, cudaStream_t st, int* splits = nullptr, bool beside = false) {
    using O = typename um::Result<T, ROLE>::type;
    constexpr bool a_mn = ROLE == lin::kGradW, b_mn = ROLE != lin::kForward;
    constexpr int V = esc::Elem<T>::kVec;
    const bool a_pieces = whole_pieces(p.a.p, p.a.ld, sizeof(T)), b_pieces = whole_pieces(p.b.p, p.b.ld, sizeof(T));
    CUtensorMap ma{}, mb{}, mo{}, mr{}, mz{};
    p.a_rows = (int)std::min<long long>(um::kBlockI, (p.I + 7) / 8 * 8);
    p.a_tma = sizeof(T) == 2 && a_pieces && map_of<T>(&ma, p.a.p, 0, p.a.rows, p.a.width, p.a.ld, a_mn ? um::kBlockC : p.a_rows);
    const auto cut_for = [&] { return cut(ROLE, p.I, p.J, depth, sizeof(T), p.a_tma && p.b_tma, runs); };
    p.b_tma = sizeof(T) == 2 && b_pieces;
    Cut c = cut_for();
    if (p.b_tma && !map_of<T>(&mb, p.b.p, 0, p.b.rows, p.b.width, p.b.ld, b_mn ? um::kBlockC : c.bn)) {
        p.b_tma = false;
        c = cut_for();
    }
    const bool tma = p.a_tma && p.b_tma;
    if (c.bn == 0) return ESC_ERR_UNSUPPORTED;                     // more tiles than a launch can count
    p.tiles_i = c.tiles_i; p.tiles_j = c.tiles_j; p.bn = c.bn; p.splits = c.splits; p.stages = c.stages; p.resident = c.resident; p.single = c.single;
    p.blocks = (int)((depth + um::kBlockC - 1) / um::kBlockC);
    p.per_split = p.blocks / c.splits; p.longer = p.blocks % c.splits;
    p.units = (unsigned)((long long)c.tiles_i * c.tiles_j * c.splits);
    if (splits) *splits = c.splits;
    const void* out = p.out;
    if constexpr (ROLE == lin::kGradW) out = p.part;
    const bool out_tma = (c.tiles_j == 1 || c.bn % (int)(128 / sizeof(O)) == 0) && whole_pieces(out, p.J, sizeof(O)) && map_of<O>(&mo, out, c.splits, p.I, p.J, p.J, 32) &&
               (!p.residual || (whole_pieces(p.residual, p.J, sizeof(T)) && map_of<T>(&mr, p.residual, 1, p.I, p.J, p.J, 32))) &&
               (!p.z || (whole_pieces(p.z, p.J, sizeof(T)) && map_of<T>(&mz, p.z, 1, p.I, p.J, p.J, 32)));
    p.a.pieces = a_pieces && p.a.width % V == 0;
    p.b.pieces = b_pieces && p.b.width % V == 0;
    auto launch = [&](auto kernel, int warps) {
        ESC_ABI_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)um::kMostSmem));   // the same for every call
        if (beside) return launch_behind(kernel, (unsigned)c.grid, 32 * warps, st, c.smem, ma, mb, mo, mr, mz, p);
        kernel<<<(unsigned)c.grid, 32 * warps, c.smem, st>>>(ma, mb, mo, mr, mz, p);
        return launched();
    };
    auto pick = [&](auto in, auto out_by) {
        constexpr bool TMA = decltype(in)::value, OUT = decltype(out_by)::value;
        if (runs && (p.blocks + c.splits - 1) / c.splits > um::run_of(ROLE, sizeof(T))) return launch(um::product_umma<T, ROLE, TMA, true, OUT>, um::all_warps<TMA>);
        return launch(um::product_umma<T, ROLE, TMA, false, OUT>, um::all_warps<TMA>);
    };
    using yes = std::true_type;
    using no = std::false_type;
    if constexpr (sizeof(T) == 2)
        if (tma) return out_tma ? pick(yes{}, yes{}) : pick(yes{}, no{});
    return out_tma ? pick(no{}, yes{}) : pick(no{}, no{});
}

// grad_z_sums: pieces of a row to a block, and as many blocks as fill the SMs four times, which leave a partial sum each.
struct BiasCut { int blocks, across, parts; };
BiasCut bias_cut(const Call& c, int vec) {
    // 32 pieces at most, whole lines of 128 bytes where rows have them, and blocks alike (48 pieces: 24 and 24)
    const int all = c.N / vec, line = std::max(1, (int)(128 / (vec * c.es()))), blocks = (all + 31) / 32;
    const int across = blocks == 1 ? all : std::min(32, (int)abi::round_up((all + blocks - 1) / blocks, line));
    return {blocks, across, (int)std::max(1LL, std::min(((long long)lin::kSumBlocks * abi::sm_count() + blocks - 1) / blocks, (c.rows + 31) / 32))};
}
// A copy of ragged bf16 rows to rows of whole pieces costs two passes over them and a launch, and pays where a product reads them several times:
// 70640 x 906 to 441 backward 505 us, 654 without, 4000 x 777 to 1999 93 and 165.  Below a million values the launch costs more; x is read once for
// every 128 outputs (100000 x 61 to 64: 45 us with a copy of it, 39 without).
bool copied(long long rows, int K) { return rows * K >= 1 << 20; }
bool x_copied(const Call& c) { return copied(c.rows, c.K) && c.N > um::kBlockI; }
long long piece_stride(int K) { return (long long)abi::round_up(K, 8); }
// g lies in rows of whole 16-byte pieces, whatever N is.
long long g_stride(const Call& c) { return (long long)abi::round_up(c.N, 16 / c.es()); }
struct FewCut { int across, stretches; };
FewCut few_cut(const Call& c, int vec);
constexpr int kFewV = 4;
struct LinearWs { float *part, *bias; void* g; bf16 *x, *w; size_t bytes; };
LinearWs carve(void* ws, const Call& c) {
    LinearWs w;
    char* base = static_cast<char*>(ws);
    size_t off = 0;
    auto take = [&](size_t bytes) { char* p = base + off; off += abi::round_up(bytes, 256); return p; };
    const long long rows = std::max(c.rows, 1LL);
    const sm::Plan small = sm::plan(rows, c.K, c.N, c.act != ESC_ACT_NONE, false, abi::sm_count());   // its blocks, as many with fp32 gradients, leave a part each
    const int fused = c.dtype == ESC_BF16 && small.stages > 0 ? small.grid : 0;
    int splits = fused;
    for (int kind = 0; kind < 4; ++kind) splits = std::max(splits, cut(lin::kGradW, c.N, c.K, rows, c.es(), kind & 1, kind & 2).splits);   // whatever the call takes
    size_t part = (size_t)splits * c.N * c.K;
    if (rows <= fw::kMostRows) part = std::max(part, (size_t)(std::max(few_cut(c, 1).stretches, few_cut(c, kFewV).stretches) * rows * c.K));
    w.part = reinterpret_cast<float*>(take(part * sizeof(float)));
    int parts = fused;
    for (int vec = 16 / (int)c.es(); vec >= 1; vec /= 2)
        if (c.N % vec == 0) parts = std::max(parts, bias_cut(c, vec).parts);
    w.bias = reinterpret_cast<float*>(take((size_t)parts * c.N * sizeof(float)));
    w.g = take(c.act != ESC_ACT_NONE ? (size_t)c.rows * g_stride(c) * c.es() : 0);
    // bf16 with K that is no multiple of eight: x and the weights as rows of whole 16-byte pieces, where copying them pays
    const bool ragged = c.dtype == ESC_BF16 && c.K % 8 != 0;
    w.x = reinterpret_cast<bf16*>(take(ragged && x_copied(c) ? (size_t)c.rows * piece_stride(c.K) * 2 : 0));
    w.w = reinterpret_cast<bf16*>(take(ragged && copied(c.N, c.K) ? (size_t)c.N * piece_stride(c.K) * 2 : 0));
    w.bytes = off;
    return w;
}

template <typename T> um::Source<T> source(const void* p, long long rows, long long width, long long ld) {
    return um::Source<T>{static_cast<const T*>(p), rows, width, ld, false};
}

template <typename U> int launch_copy_of(const um::Source<bf16>& s, bf16* out, long long ld, cudaStream_t st) {
    constexpr int values = sizeof(U) / 2;
    const int width = (int)(s.width / values);
    const unsigned across = (unsigned)((width + 63) / 64);
    const long long want = (32LL * abi::sm_count() + across - 1) / across;
    lin::copy_rows<U><<<dim3(across, (unsigned)std::min({(s.rows + 63) / 64, want, 65535LL})), 256, 0, st>>>(reinterpret_cast<const U*>(s.p), s.ld / values, s.rows, width,
                                                                                                         reinterpret_cast<U*>(out), ld / values);
    return launched();
}
int launch_copy(const um::Source<bf16>& s, bf16* out, long long ld, cudaStream_t st) {
    return s.width % 2 == 0 && s.ld % 2 == 0 && abi::aligned(s.p, 4) ? launch_copy_of<unsigned>(s, out, ld, st) : launch_copy_of<unsigned short>(s, out, ld, st);
}

// The partial sums of the weights' and the bias' gradients, in one launch.
template <typename G> int launch_sums(const lin::Parts& w, const lin::Parts& b, void* gw, void* gb, cudaStream_t st) {
    return launch_behind(lin::sum_parts<G>, (unsigned)(lin::sum_blocks(w) + lin::sum_blocks(b)), esc::kSumThreads, st, 0, w, b, static_cast<G*>(gw), static_cast<G*>(gb));
}
int sum_to(const lin::Parts& w, const lin::Parts& b, void* gw, void* gb, int grad_dtype, cudaStream_t st) {
    if (w.count + b.count == 0) return ESC_OK;
    return grad_dtype == ESC_F32 ? launch_sums<float>(w, b, gw, gb, st) : launch_sums<bf16>(w, b, gw, gb, st);
}

// ---- a few rows --------------------------------------------------------------------------------------------------------------

// Whether rows of the tensors that a kernel reads in pieces of `vec` values are whole aligned ones.
bool even(const Call& c, int vec) {
    const size_t bytes = vec * c.es();
    return c.K % vec == 0 && c.x_stride % vec == 0 && abi::aligned(c.x, bytes) && abi::aligned(c.w, bytes);
}
template <int R> using rows_is = std::integral_constant<int, R>;
template <typename F> int for_rows(long long rows, F f) {
    return rows <= 1 ? f(rows_is<1>{}) : rows <= 2 ? f(rows_is<2>{}) : rows <= 4 ? f(rows_is<4>{}) : rows <= 8 ? f(rows_is<8>{}) : f(rows_is<16>{});
}

// Whether a call of that many rows is one for those kernels.  They take about 8 us (a backward pass 15) and 0.15 us for a million products,
// whichever way these lie; the tensor cores' 10 to 13 (21) and 3.5 for each thousand of inputs or, for fp32 and rows that are not whole pieces, 25.
// Forward: 16 x 8192 to 256 in bf16 11 us here, 29 there; 16 x 1024 to 4096 15 and 10; 8 x 4096 to 4096 in fp32 39 and 116; 4 and 16 x 4001 to
// 4001 in bf16 56 and 163, 111 there.  Backward: 4 x 1024 to 4096 in bf16 18 and 38, 16 x 1024 to 1024 25 and 23, 4 x 4001 to 4001 113 and 99, in
// fp32 125 and 232.
bool is_few(const Call& c, bool backward) {
    const bool wide = c.dtype == ESC_F32, pieces = even(c, 16 / (int)c.es());
    if (c.rows > (backward && !wide ? fw::kMostRows / 2 : fw::kMostRows)) return false;
    const double products = (double)c.rows * c.K * c.N;
    return (wide && pieces) || products <= (wide || (!backward && !pieces) ? 1 << 27 : 1 << 25);
}

template <typename T> int forward_few(const Call& c, const lin::Layer<T>& l, cudaStream_t st) {
    constexpr int V = esc::Elem<T>::kVec;
    const bool pieces = even(c, V);
    const int step = 32 * (pieces ? V : 1);
    // Four outputs to a warp, two where four would leave SMs short of warps (16 x 2050 to 64: 16.8 and 12.5 us; 8 x 4096 to 4096: 39 and 59).
    // Slices of the inputs: as many as have a step each, until every SM has eight warps (32 warps: 16 x 4096 to 4096 72 -> 84 us).
    const int columns = c.N < 4 * abi::sm_count() ? 2 : 4;
    int slices = 1;
    while (slices < fw::kWarps && slices * step < c.K && (long long)c.N * slices < 8LL * abi::sm_count() * columns) slices *= 2;
    const int per_block = fw::kWarps / slices * columns;
    const unsigned blocks = (unsigned)((c.N + per_block - 1) / per_block);
    return for_rows(c.rows, [&](auto r) {
        constexpr int R = decltype(r)::value;
        auto launch = [&](auto kernel) {
            kernel<<<blocks, 32 * fw::kWarps, 0, st>>>(l, slices);
            return launched();
        };
        if (columns == 2) return pieces ? launch(fw::forward<T, V, R, 2>) : launch(fw::forward<T, 1, R, 2>);
        return pieces ? launch(fw::forward<T, V, R, 4>) : launch(fw::forward<T, 1, R, 4>);
    });
}

// The backward pass: tiles of 32 V inputs, and stretches of outputs, so many that the SMs have 16 warps each, of 8 at least, and so long that
// the partial sums of gx are no more than half of w's values.
FewCut few_cut(const Call& c, int vec) {
    const int across = (c.K + 32 * vec - 1) / (32 * vec);
    return {across, (int)std::max(1LL, std::min(c.N / std::max(8LL, 2 * c.rows), (16LL * abi::sm_count() + across - 1) / across))};
}
template <typename T, typename G> int backward_few_to(const Call& c, const lin::Layer<T>& l, G* gw, G* gb, float* part, cudaStream_t st) {
    const int vec = even(c, kFewV) && abi::aligned(gw, kFewV * sizeof(G)) ? kFewV : 1;
    const FewCut d = few_cut(c, vec);
    const unsigned blocks = (unsigned)((d.across * (long long)d.stretches + 3) / 4);
    ESC_TRY(for_rows(c.rows, [&](auto r) {
        constexpr int R = decltype(r)::value;
        if (vec == kFewV) fw::backward<T, G, kFewV, R><<<blocks, 128, 0, st>>>(l, d.across, d.stretches, part, gw, gb);
        else fw::backward<T, G, 1, R><<<blocks, 128, 0, st>>>(l, d.across, d.stretches, part, gw, gb);
        return launched();
    }));
    if (!l.gx) return ESC_OK;
    const lin::Parts px{part, d.stretches, c.rows * c.K}, none{nullptr, 0, 0};
    return launch_sums<T>(px, none, l.gx, nullptr, st);
}
template <typename T> int backward_few(const Call& c, const lin::Layer<T>& l, void* gw, void* gb, int grad_dtype, float* part, cudaStream_t st) {
    return grad_dtype == ESC_F32 ? backward_few_to<T, float>(c, l, static_cast<float*>(gw), static_cast<float*>(gb), part, st)
                                 : backward_few_to<T, bf16>(c, l, static_cast<bf16*>(gw), static_cast<bf16*>(gb), part, st);
}

template <typename T> int linear_forward_t(const Call& c, const lin::Layer<T>& l, cudaStream_t st) {
    if (is_few(c, false)) return forward_few<T>(c, l, st);
    um::Args<T> p{};
    p.I = c.rows; p.J = c.N; p.act = c.act;
    p.a = source<T>(c.x, c.rows, c.K, c.x_stride); p.b = source<T>(c.w, c.N, c.K, c.K);
    p.bias = l.b; p.residual = l.residual; p.out = l.out; p.z = l.z;
    return launch_product<T, lin::kForward>(p, c.K, true, st);
}

// A small bf16 layer in one pass; kNotThis: it is not one, or its tensors are not rows of whole 16-byte pieces.
constexpr int kNotThis = -1;
int backward_small(const Call& c, const lin::Layer<bf16>& l, void* gw, void* gb, int grad_dtype, const LinearWs& w, cudaStream_t st) {
    const bool act = c.act != ESC_ACT_NONE;
    const sm::Plan d = sm::plan(c.rows, c.K, c.N, act, gw && grad_dtype == ESC_F32, abi::sm_count());
    if (d.stages == 0 || (!l.gx && !gw)) return kNotThis;
    if (!whole_pieces(l.go, c.N, 2) || !whole_pieces(c.x, c.x_stride, 2) || !whole_pieces(c.w, c.K, 2) || (act && !whole_pieces(l.kept, c.N, 2)) ||
        (l.gx && !whole_pieces(l.gx, c.K, 2))) return kNotThis;
    CUtensorMap go{}, z{}, x{}, wm{}, gx{}, part{};
    if (!map_of<bf16>(&go, l.go, 0, c.rows, c.N, c.N, sm::kRows) || !map_of<bf16>(&x, c.x, 0, c.rows, c.K, c.x_stride, sm::kRows) || !map_of<bf16>(&wm, c.w, 0, c.N, c.K, c.K, 64) ||
        (act && !map_of<bf16>(&z, l.kept, 0, c.rows, c.N, c.N, sm::kRows)) || (l.gx && !map_of<bf16>(&gx, l.gx, 1, c.rows, c.K, c.K, 32)) ||
        (gw && !map_of<float>(&part, w.part, d.grid, c.N, c.K, c.K, 32))) return kNotThis;
    const sm::Args p{(int)c.rows, c.N, c.K, d.tiles, c.act, d.stages, d.nb, d.kb, d.gx_buffers, l.gx != nullptr, gw != nullptr, gb != nullptr, w.bias};
    const auto kernel = d.runs ? sm::backward<true> : sm::backward<false>;
    ESC_ABI_CUDA(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)um::kMostSmem));   // the same for every call
    kernel<<<(unsigned)d.grid, sm::kThreads, d.smem, st>>>(go, z, x, wm, gx, part, p);
    ESC_TRY(launched());
    return sum_to({w.part, d.grid, gw ? (long long)c.N * c.K : 0}, {w.bias, d.grid, gb ? c.N : 0}, gw, gb, grad_dtype, st);
}

template <typename T> int linear_backward_t(const Call& c, const lin::Layer<T>& l, void* gw, void* gb, int grad_dtype, const LinearWs& w, cudaStream_t st) {
    constexpr int V = esc::Elem<T>::kVec;
    if (is_few(c, true)) return backward_few<T>(c, l, gw, gb, grad_dtype, w.part, st);
    if constexpr (sizeof(T) == 2) {
        const int rc = backward_small(c, l, gw, gb, grad_dtype, w, st);
        if (rc != kNotThis) return rc;
    }
    um::Source<T> g = source<T>(l.go, c.rows, c.N, c.N);
    lin::Parts pw{w.part, 0, 0}, pb{w.bias, 0, 0};
    const bool acts = c.act != ESC_ACT_NONE && (l.gx || gw);
    bool beside = gb && !acts;                                     // the next product needs nothing of the kernel before it
    if (acts || gb) {
        T* to = acts ? static_cast<T*>(w.g) : nullptr;
        const long long ld = g_stride(c);
        // the widest piece, of 16 bytes at most, that divides the rows and their alignment
        const auto fits = [&](int vec) {
            return c.N % vec == 0 && abi::aligned(l.go, vec * sizeof(T)) && (c.act == ESC_ACT_NONE || abi::aligned(l.kept, vec * sizeof(T)));
        };
        int vec = V;
        while (!fits(vec)) vec /= 2;
        const BiasCut b = bias_cut(c, vec);
        const dim3 grid(b.blocks, b.parts);
        float* sums = gb ? w.bias : nullptr;
        if (vec == 8) { if constexpr (V == 8) lin::grad_z_sums<T, 8><<<grid, 256, 0, st>>>(l, to, ld, sums, b.across); }
        else if (vec == 4) lin::grad_z_sums<T, 4><<<grid, 256, 0, st>>>(l, to, ld, sums, b.across);
        else if (vec == 2) lin::grad_z_sums<T, 2><<<grid, 256, 0, st>>>(l, to, ld, sums, b.across);
        else lin::grad_z_sums<T, 1><<<grid, 256, 0, st>>>(l, to, ld, sums, b.across);
        ESC_TRY(launched());
        if (gb) pb = lin::Parts{w.bias, b.parts, c.N};
        if (acts) g = source<T>(to, c.rows, c.N, ld);
    }
    um::Source<T> x = source<T>(c.x, c.rows, c.K, c.x_stride), weight = source<T>(c.w, c.N, c.K, c.K);
    if constexpr (sizeof(T) == 2) {
        if (c.K % 8 != 0) {
            const long long ld = piece_stride(c.K);
            if (gw && x_copied(c)) {
                ESC_TRY(launch_copy(x, w.x, ld, st));
                beside = false;
                x = source<T>(w.x, c.rows, c.K, ld);
            }
            if (l.gx && copied(c.N, c.K)) {
                ESC_TRY(launch_copy(weight, w.w, ld, st));
                beside = false;
                weight = source<T>(w.w, c.N, c.K, ld);
            }
        }
    }
    if (l.gx) {
        um::Args<T> p{};
        p.I = c.rows; p.J = c.K;
        p.a = g; p.b = weight; p.out = l.gx;
        ESC_TRY((launch_product<T, lin::kGradX>(p, c.N, true, st, nullptr, beside)));
        beside = true;
    }
    if (gw) {
        um::Args<T> p{};
        p.I = c.N; p.J = c.K;
        p.a = g; p.b = x; p.part = w.part;
        ESC_TRY((launch_product<T, lin::kGradW>(p, c.rows, sizeof(T) == 4 || grad_dtype == ESC_F32, st, &pw.parts, beside)));
        pw.count = (long long)c.N * c.K;
    }
    return sum_to(pw, pb, gw, gb, grad_dtype, st);
}

}  // namespace

extern "C" {

int esc_linear_device_status(void* stream) {
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
    ESC_ABI_CUDA(cudaStreamIsCapturing(st, &capturing));
    if (capturing != cudaStreamCaptureStatusNone) return ESC_ERR_UNSUPPORTED;
    unsigned status[2] = {0, 0};
    ESC_ABI_CUDA(cudaMemcpyFromSymbolAsync(status, um::wait_status, sizeof status, 0, cudaMemcpyDeviceToHost, st));
    ESC_ABI_CUDA(cudaStreamSynchronize(st));
    if (status[0] == 0) return ESC_OK;
    const unsigned clear[2] = {0, 0};
    ESC_ABI_CUDA(cudaMemcpyToSymbolAsync(um::wait_status, clear, sizeof clear, 0, cudaMemcpyHostToDevice, st));
    ESC_ABI_CUDA(cudaStreamSynchronize(st));
    return (int)status[0];
}

int esc_linear_selftest_bounded_wait(void* stream) {
    um::wait_in_vain<<<1, 32, 0, static_cast<cudaStream_t>(stream)>>>();
    ESC_ABI_CUDA(cudaGetLastError());
    return ESC_OK;
}

int esc_linear_forward(const void* x, long long x_stride, const void* weight, const void* bias, int activation, const void* residual, void* out, void* z,
                       long long rows, int K, int N, int dtype, void* stream) {
    abi::launches_reset();
    const Call c{x, x_stride, weight, rows, K, N, activation, dtype};
    ESC_TRY(check_call(c));
    if (!out && rows > 0) return ESC_ERR_NULL;
    for (const void* p : {bias, residual, static_cast<const void*>(out), static_cast<const void*>(z)})
        if (!abi::aligned(p, c.es())) return ESC_ERR_ALIGN;
    const Matrix read[] = {c.mx(), c.mw(), flat(bias, N, c.es()), c.out(residual, N)};
    for (const Matrix& i : read)
        if (touch(c.out(out, N), i) || touch(c.out(z, N), i)) return ESC_ERR_ALIAS;
    if (touch(c.out(out, N), c.out(z, N))) return ESC_ERR_ALIAS;
    if (rows == 0) return ESC_OK;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    auto go = [&](auto zero_value) {
        using T = decltype(zero_value);
        lin::Layer<T> p = layer_of<T>(c);
        p.b = static_cast<const T*>(bias); p.residual = static_cast<const T*>(residual);
        p.out = static_cast<T*>(out); p.z = static_cast<T*>(z);
        return linear_forward_t<T>(c, p, st);
    };
    return dtype == ESC_F32 ? go(float{}) : go(bf16{});
}

size_t esc_linear_backward_workspace_bytes(long long rows, int K, int N, int activation, int dtype) {
    if (check_sizes(rows, K, N, activation, dtype) != ESC_OK) return 0;
    return carve(nullptr, Call{nullptr, K, nullptr, rows, K, N, activation, dtype}).bytes;
}

int esc_linear_backward(const void* x, long long x_stride, const void* weight, const void* z, int activation, const void* grad_out, void* grad_x,
                        void* grad_weight, void* grad_bias, long long rows, int K, int N, int dtype, int grad_dtype, void* workspace,
                        size_t workspace_bytes, void* stream) {
    abi::launches_reset();
    const Call c{x, x_stride, weight, rows, K, N, activation, dtype};
    ESC_TRY(check_call(c));
    if (!known(grad_dtype)) return ESC_ERR_UNSUPPORTED;
    if (rows > 0 && (!grad_out || (activation != ESC_ACT_NONE && !z))) return ESC_ERR_NULL;
    const size_t gs = abi::elem_size(grad_dtype);
    for (const void* p : {z, grad_out, static_cast<const void*>(grad_x)})
        if (!abi::aligned(p, c.es())) return ESC_ERR_ALIGN;
    if (!abi::aligned(grad_weight, gs) || !abi::aligned(grad_bias, gs)) return ESC_ERR_ALIGN;
    const Matrix written[] = {c.out(grad_x, K), flat(grad_weight, (long long)N * K, gs), flat(grad_bias, N, gs)};
    const Matrix read[] = {c.mx(), c.mw(), c.out(activation != ESC_ACT_NONE ? z : nullptr, N), c.out(grad_out, N)};
    for (const Matrix& o : written)
        for (const Matrix& i : read)
            if (touch(o, i)) return ESC_ERR_ALIAS;
    if (touch(written[0], written[1]) || touch(written[0], written[2]) || touch(written[1], written[2])) return ESC_ERR_ALIAS;
    const LinearWs w = carve(workspace, c);
    if (!workspace || !abi::aligned(workspace, 256) || workspace_bytes < w.bytes) return ESC_ERR_WORKSPACE;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0) {
        ESC_TRY(zero(grad_weight, (size_t)N * K * gs, st));
        return zero(grad_bias, N * gs, st);
    }
    auto go = [&](auto zero_value) {
        using T = decltype(zero_value);
        lin::Layer<T> p = layer_of<T>(c);
        p.go = static_cast<const T*>(grad_out); p.kept = static_cast<const T*>(z); p.gx = static_cast<T*>(grad_x);
        return linear_backward_t<T>(c, p, grad_weight, grad_bias, grad_dtype, w, st);
    };
    return dtype == ESC_F32 ? go(float{}) : go(bf16{});
}

}  // extern "C"
