// The three products of a linear layer on the fifth-generation tensor cores (tcgen05.mma, sums in tensor memory):
//
//   D[i][j] = sum over c of A(i, c) B(j, c)
//     kForward  i a row, j an output, c an input:   A = x, B = w          both K-major (c runs along memory)
//     kGradX    i a row, j an input, c an output:   A = g, B = w          A K-major, B MN-major (j runs along memory)
//     kGradW    i an output, j an input, c a row:   A = g, B = x          both MN-major
//
// so nothing is transposed in memory: an operand is staged as lines of 64 values of a row, 128 bytes with the 128-byte swizzle, and the
// descriptor says which way the contraction runs.  A tile of D is 128 x bn (bn up to 256, a multiple of 16, or of 64 for MN-major B);
// c goes by blocks of 64.  Blocks are persistent, one per SM; two tiles' sums lie in tensor memory, so that one is written out while the
// next is summed.
//
// bf16 with rows of whole 16-byte pieces: TMA fills the ring.  Otherwise eight warps load values as they lie and store them swizzled:
// any stride and alignment, and fp32, where every value is split into three bf16 parts (24 bits: hi + mid + lo exactly) and six of
// the nine products are taken; what is left out is below 2^-26 of a product.  The largest of them has an accumulator of its own
// (the tensor cores add as fp32, and small terms would be rounded at the large sum's step).
//
// Epilogue: a warp reads 32 columns of 32 rows, turns them in 4 KB of shared memory so that lanes hold neighbouring columns, and there
// adds the bias, applies the activation, adds the residual and rounds once: all of its memory traffic is whole sectors.
//
// Small layers (K and N of a few hundred, many rows) are bound by memory: w then stays in shared memory for the whole life of a block
// (`resident`), and the ring holds rows alone.
#pragma once
#include <cuda.h>
#include "linear.cuh"

namespace esc { namespace linear { namespace umma {

constexpr int kBlockI = 128, kBlockC = 64;
constexpr int kABytes = kBlockI * kBlockC * 2;                     // of one part
constexpr int kEpiWarps = 8, kFillWarps = 8, kFirstEpi = 4, kFirstFill = kFirstEpi + kEpiWarps;
constexpr int kStageBytes = kEpiWarps * 32 * 32 * 4;               // staging of the epilogue
constexpr int kMaxStages = 8;
constexpr size_t kMostSmem = 227 * 1024;
constexpr int kTmemBuffer = 256;                                   // columns of one tile's sums
constexpr unsigned kPolls = 1u << 20, kHintNs = 1000;              // a wait gives up after about one second

__device__ unsigned wait_status[2];                                // ESC_DEV_TIMEOUT and where, if a wait ran out

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, unsigned count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void mbar_expect(uint32_t bar, unsigned bytes) { asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory"); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
// Bounded wait of a whole warp; all lanes get the same answer.
__device__ __forceinline__ bool wait_warp(uint32_t bar, unsigned parity, unsigned where) {
    for (unsigned n = 0; n < kPolls; ++n) {
        unsigned ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity), "r"(kHintNs) : "memory");
        if (__all_sync(0xffffffffu, ok)) return true;
    }
    if (threadIdx.x % 32 == 0) { atomicExch(&wait_status[0], kDevTimeout); atomicExch(&wait_status[1], where); }
    return false;
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1) : "memory");
}
// 128-byte swizzle.  K-major: rows of 128 bytes, eight rows 1024 bytes further on.  MN-major: atoms of 64 values x eight c (1024
// bytes); the next eight c 1024 bytes, the next 64 values kBlockC lines further on.
template <bool MN> __device__ __forceinline__ unsigned long long smem_desc(uint32_t addr) {
    constexpr unsigned long long lbo = MN ? (kBlockC * 128) >> 4 : 1, sbo = 1024 >> 4;
    return (unsigned long long)((addr >> 4) & 0x3FFFu) | (lbo << 16) | (sbo << 32) | (1ull << 46) | (2ull << 61);
}
template <bool MN> constexpr uint32_t step16 = MN ? 16 * 128 : 16 * 2;   // bytes to the next 16 of c
template <bool A_MN, bool B_MN> __device__ __forceinline__ uint32_t instr_desc(int n) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(kBlockI >> 4) << 24);
}
// By a whole warp with the same arguments in every lane; one elected lane issues.
__device__ __forceinline__ void mma(uint32_t d, unsigned long long a, unsigned long long b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\telect.sync _|q, 0xffffffff;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((unsigned)add) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t"
                 "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_ld32(uint32_t at, uint32_t (&r)[32]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

template <typename T> struct Args {
    long long I, depth;
    int J, tiles_i, tiles_j, bn, splits, stages;
    bool resident;                      // B stays in shared memory; a block keeps its tile of j
    long long units;
    const T *a, *b;                     // as they lie: rows of a_ld, b_ld values
    long long a_ld, b_ld;
    const T* kept;                      // with an activation: A = a act'(kept), laid out like a (plain loads only)
    int act;
    const T *bias, *residual;
    T *out, *z;
    float* part;                        // kGradW: [splits][I][J]
    bool pieces;                        // rows of the result, the bias and the residual are whole 16-byte pieces
};

template <typename T> constexpr int parts_of = sizeof(T) == 4 ? 3 : 1;
template <typename T> constexpr int most_columns = sizeof(T) == 4 ? 128 : 256;

struct Unit { int i, j, split; long long c0, c1; bool live; };
template <typename T> __device__ __forceinline__ Unit unit_of(const Args<T>& p, long long n) {
    Unit u{};
    const long long blocks = (p.depth + kBlockC - 1) / kBlockC;
    if (p.resident) {
        const long long i = blockIdx.x / p.tiles_j + n * (gridDim.x / p.tiles_j);
        u.live = i < p.tiles_i;
        u.i = (int)i; u.j = (int)(blockIdx.x % p.tiles_j); u.c0 = 0; u.c1 = blocks;
        return u;
    }
    const long long t = blockIdx.x + n * gridDim.x;
    u.live = t < p.units;
    u.j = (int)(t % p.tiles_j);
    u.i = (int)(t / p.tiles_j % p.tiles_i);
    u.split = (int)(t / p.tiles_j / p.tiles_i);
    u.c0 = blocks * u.split / p.splits; u.c1 = blocks * (u.split + 1) / p.splits;
    return u;
}

// ---- plain loads into swizzled lines ------------------------------------------------------------------------------------------

struct Pair { float lo, hi; };
__device__ __forceinline__ Pair load_pair(const float* p, int n, bool even) {
    Pair v{0.f, 0.f};
    if (n >= 2 && even) { const float2 f = *reinterpret_cast<const float2*>(p); v.lo = f.x; v.hi = f.y; return v; }
    if (n >= 1) v.lo = p[0];
    if (n >= 2) v.hi = p[1];
    return v;
}
__device__ __forceinline__ Pair load_pair(const __nv_bfloat16* p, int n, bool) {
    Pair v{0.f, 0.f};
    if (n >= 2 && (reinterpret_cast<uintptr_t>(p) & 3) == 0) {
        const uint32_t w = *reinterpret_cast<const uint32_t*>(p);
        v.lo = __uint_as_float(w << 16); v.hi = __uint_as_float(w & 0xffff0000u);
        return v;
    }
    if (n >= 1) v.lo = __bfloat162float(p[0]);
    if (n >= 2) v.hi = __bfloat162float(p[1]);
    return v;
}
__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void st_shared(uint32_t at, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }
__device__ __forceinline__ Pair less(Pair v, uint32_t part) { return Pair{v.lo - __uint_as_float(part << 16), v.hi - __uint_as_float(part & 0xffff0000u)}; }

// One operand's block: `lines` lines of 64 values, a warp a line, a lane two values of it.  Line L: K-major row mn0 + L, columns from c0;
// MN-major row c0 + L % 64, columns from mn0 + L / 64 * 64.  The parts of fp32 lie `part_bytes` apart.
template <typename T, bool MN> __device__ __forceinline__ void fill(uint32_t dst, int lines, uint32_t part_bytes, const T* src, long long ld, const T* kept, int act,
                                                                     long long mn0, long long mn_all, long long c0, long long c_all, int warp, int lane) {
    constexpr int kBatch = 8;
    const bool even = sizeof(T) == 4 && ld % 2 == 0 && (reinterpret_cast<uintptr_t>(src) & 7) == 0;
    const bool even_kept = even && (reinterpret_cast<uintptr_t>(kept) & 7) == 0;
    for (int first = warp; first < lines; first += kFillWarps * kBatch) {
        Pair v[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int L = first + u * kFillWarps;
            const long long row = MN ? c0 + L % kBlockC : mn0 + L, col = (MN ? mn0 + L / kBlockC * kBlockC : c0) + 2 * lane;
            const long long left = (MN ? mn_all : c_all) - col;
            const int n = L < lines && row < (MN ? c_all : mn_all) ? (left >= 2 ? 2 : left == 1 ? 1 : 0) : 0;
            v[u] = load_pair(src + row * ld + col, n, even);
            if (kept) {
                const Pair z = load_pair(kept + row * ld + col, n, even_kept);
                v[u].lo *= act_slope(act, z.lo);
                v[u].hi *= act_slope(act, z.hi);
            }
        }
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const int L = first + u * kFillWarps;
            if (L >= lines) break;
            const uint32_t at = dst + L * 128 + (((lane >> 2) ^ (L & 7)) << 4) + (lane & 3) * 4;
            const uint32_t hi = pack(v[u].lo, v[u].hi);
            st_shared(at, hi);
            if (sizeof(T) == 4) {
                const Pair r = less(v[u], hi);
                const uint32_t mid = pack(r.lo, r.hi);
                st_shared(at + part_bytes, mid);
                const Pair q = less(r, mid);
                st_shared(at + 2 * part_bytes, pack(q.lo, q.hi));
            }
        }
    }
}

// ---- epilogue ---------------------------------------------------------------------------------------------------------------

// Eight (bf16) or four (fp32) neighbouring columns of one row, which is a 16-byte piece of it.
template <typename T> __device__ __forceinline__ void store16(T* p, const float* f);
template <> __device__ __forceinline__ void store16<float>(float* p, const float* f) { *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]); }
template <> __device__ __forceinline__ void store16<__nv_bfloat16>(__nv_bfloat16* p, const float* f) {
    *reinterpret_cast<uint4*>(p) = make_uint4(pack(f[0], f[1]), pack(f[2], f[3]), pack(f[4], f[5]), pack(f[6], f[7]));
}

// 32 rows x 32 columns that this warp has staged, from row i0 and column j0 on; rows below `rows`, columns below `cols` of them are real.
// O: type of the result; the epilogue of kForward adds bias, activation and residual.
template <typename T, typename O, Role ROLE> __device__ __forceinline__ void write_chunk(const float* st, const Args<T>& p, O* out, long long i0, int rows, int j0, int cols, int lane) {
    constexpr int V = Elem<O>::kVec, per_row = 32 / V, at_once = 32 / per_row, turns = 32 / at_once;
    const float4* st4 = reinterpret_cast<const float4*>(st);
    if (p.pieces) {
        const int c = lane % per_row * V;
        if (c >= cols) return;
        float bias[V];
        if (ROLE == kForward && p.bias) unpack16<T>(*reinterpret_cast<const uint4*>(p.bias + j0 + c), bias);
        uint4 res[turns];
        if (ROLE == kForward && p.residual)
#pragma unroll
            for (int t = 0; t < turns; ++t) {
                const int r = t * at_once + lane / per_row;
                if (r < rows) res[t] = *reinterpret_cast<const uint4*>(p.residual + (i0 + r) * p.J + j0 + c);
            }
#pragma unroll
        for (int t = 0; t < turns; ++t) {
            const int r = t * at_once + lane / per_row;
            if (r >= rows) break;
            float f[V];
#pragma unroll
            for (int q = 0; q < V / 4; ++q) {
                const float4 v = st4[r * 8 + ((c / 4 + q) ^ (r & 7))];
                f[4 * q] = v.x; f[4 * q + 1] = v.y; f[4 * q + 2] = v.z; f[4 * q + 3] = v.w;
            }
            const long long at = (i0 + r) * p.J + j0 + c;
            if (ROLE == kForward) {
                if (p.bias)
#pragma unroll
                    for (int e = 0; e < V; ++e) f[e] += bias[e];
                if (p.z) store16<T>(p.z + at, f);
                if (p.act != kActNone)
#pragma unroll
                    for (int e = 0; e < V; ++e) f[e] = act_of(p.act, f[e]);
                if (p.residual) {
                    float rf[V];
                    unpack16<T>(res[t], rf);
#pragma unroll
                    for (int e = 0; e < V; ++e) f[e] += rf[e];
                }
            }
            store16<O>(out + at, f);
        }
        return;
    }
    if (lane >= cols) return;
    const float bias = ROLE == kForward && p.bias ? Elem<T>::to_f32(p.bias[j0 + lane]) : 0.f;
#pragma unroll 4
    for (int r = 0; r < rows; ++r) {
        float f = st[r * 32 + (((lane >> 2) ^ (r & 7)) << 2) + (lane & 3)];
        const long long at = (i0 + r) * p.J + j0 + lane;
        if (ROLE == kForward) {
            f += bias;
            if (p.z) p.z[at] = Elem<T>::from_f32(f);
            f = act_of(p.act, f);
            if (p.residual) f += Elem<T>::to_f32(p.residual[at]);
        }
        out[at] = Elem<O>::from_f32(f);
    }
}

// ---- the kernel ---------------------------------------------------------------------------------------------------------------

template <typename T, Role ROLE, bool TMA>
__global__ void __launch_bounds__(32 * (TMA ? kFirstFill : kFirstFill + kFillWarps), 1)
product_umma(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ Args<T> p)
{
    constexpr bool A_MN = ROLE == kGradW, B_MN = ROLE != kForward;
    constexpr int PARTS = parts_of<T>;
    static_assert(!TMA || PARTS == 1, "TMA brings bf16 as it is");
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t base = smem_u32(smem);
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const long long blocks = (p.depth + kBlockC - 1) / kBlockC;
    const uint32_t b_part = (uint32_t)p.bn * 128, b_bytes = b_part * PARTS, stage_bytes = kABytes * PARTS + (p.resident ? 0 : b_bytes);
    const uint32_t resident = base + p.stages * stage_bytes;
    const uint32_t staging = resident + (p.resident ? (uint32_t)blocks * b_bytes : 0), bars = staging + kStageBytes;
    const uint32_t full = bars, empty = full + 8 * kMaxStages, acc_full = empty + 8 * kMaxStages, acc_empty = acc_full + 16, b_full = acc_empty + 16, slot = b_full + 8;
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) { mbar_init(full + 8 * s, TMA ? 1 : kFillWarps); mbar_init(empty + 8 * s, 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(acc_full + 8 * s, 1); mbar_init(acc_empty + 8 * s, kEpiWarps); }
        mbar_init(b_full, TMA ? 1 : kFillWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    uint32_t tmem;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(slot));

    bool alive = true;
    if (TMA ? warp == 0 : warp >= kFirstFill) {
        // ---- fill the ring --------------------------------------------------------------------------------------------------
        unsigned k = 0;                                            // blocks so far
        for (long long n = 0; alive; ++n) {
            const Unit u = unit_of(p, n);
            if (!u.live) break;
            const long long i0 = (long long)u.i * kBlockI;
            const int j0 = u.j * p.bn;
            if (TMA) {
                if (p.resident && n == 0 && lane == 0) {
                    mbar_expect(b_full, (unsigned)(blocks * b_bytes));
                    for (int c = 0; c < blocks; ++c) {
                        if (B_MN) for (int m = 0; m < p.bn; m += 64) tma_load_2d(resident + c * b_bytes + m * 128, &map_b, b_full, j0 + m, c * kBlockC);
                        else tma_load_2d(resident + c * b_bytes, &map_b, b_full, c * kBlockC, j0);
                    }
                }
                __syncwarp();
                for (long long c = u.c0; c < u.c1; ++c, ++k) {
                    const int s = (int)(k % p.stages);
                    if (k >= (unsigned)p.stages) alive = wait_warp(empty + 8 * s, (k / p.stages - 1) & 1, 0x10000000u | k);
                    if (!alive) break;
                    if (lane == 0) {
                        const uint32_t at = base + s * stage_bytes, bar = full + 8 * s;
                        const int c0 = (int)(c * kBlockC);
                        mbar_expect(bar, stage_bytes);
                        if (A_MN) for (int m = 0; m < kBlockI; m += 64) tma_load_2d(at + m * 128, &map_a, bar, (int)i0 + m, c0);
                        else tma_load_2d(at, &map_a, bar, c0, (int)i0);
                        if (!p.resident) {
                            if (B_MN) for (int m = 0; m < p.bn; m += 64) tma_load_2d(at + kABytes + m * 128, &map_b, bar, j0 + m, c0);
                            else tma_load_2d(at + kABytes, &map_b, bar, c0, j0);
                        }
                    }
                    __syncwarp();
                }
                if (!alive)                                        // what is still on its way here lands before the block goes
                    for (unsigned q = k > (unsigned)p.stages ? k - p.stages : 0; q < k; ++q) wait_warp(full + 8 * (q % p.stages), (q / p.stages) & 1, 0x70000000u | q);
            } else {
                const int w = warp - kFirstFill;
                if (p.resident && n == 0) {
                    for (int c = 0; c < blocks; ++c)
                        fill<T, B_MN>(resident + c * b_bytes, p.bn, b_part, p.b, p.b_ld, nullptr, 0, j0, p.J, (long long)c * kBlockC, p.depth, w, lane);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(b_full);
                }
                for (long long c = u.c0; c < u.c1; ++c, ++k) {
                    const int s = (int)(k % p.stages);
                    if (k >= (unsigned)p.stages) alive = wait_warp(empty + 8 * s, (k / p.stages - 1) & 1, 0x20000000u | k);
                    if (!alive) break;
                    const uint32_t at = base + s * stage_bytes;
                    fill<T, A_MN>(at, kBlockI, kABytes, p.a, p.a_ld, p.kept, p.act, i0, p.I, c * kBlockC, p.depth, w, lane);
                    if (!p.resident) fill<T, B_MN>(at + PARTS * kABytes, p.bn, b_part, p.b, p.b_ld, nullptr, 0, j0, p.J, c * kBlockC, p.depth, w, lane);
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(full + 8 * s);
                }
            }
        }
    } else if (warp == 1) {
        // ---- issue ------------------------------------------------------------------------------------------------------------
        const uint32_t idesc = instr_desc<A_MN, B_MN>(p.bn);
        unsigned k = 0;
        for (long long n = 0; alive; ++n) {
            const Unit u = unit_of(p, n);
            if (!u.live) break;
            const int buf = (int)(n & 1);
            if (n >= 2) alive = wait_warp(acc_empty + 8 * buf, (unsigned)((n >> 1) - 1) & 1, 0x30000000u | (unsigned)n);
            if (alive && p.resident && n == 0) alive = wait_warp(b_full, 0, 0x40000000u);
            if (!alive) break;
            fence_after();
            const uint32_t d = tmem + buf * kTmemBuffer;
            for (long long c = u.c0; c < u.c1; ++c, ++k) {
                const int s = (int)(k % p.stages);
                alive = wait_warp(full + 8 * s, (k / p.stages) & 1, 0x50000000u | k);
                if (!alive) break;
                fence_after();
                const uint32_t a_at = base + s * stage_bytes, b_at = p.resident ? resident + (uint32_t)c * b_bytes : a_at + PARTS * kABytes;
                const unsigned long long da = smem_desc<A_MN>(a_at), db = smem_desc<B_MN>(b_at);
#pragma unroll
                for (int t = 0; t < kBlockC / 16; ++t) {
                    const unsigned long long at = da + t * (step16<A_MN> >> 4), bt = db + t * (step16<B_MN> >> 4);
                    const bool add = c > u.c0 || t > 0;
                    mma(d, at, bt, idesc, add);
                    if (PARTS == 3) {
                        const unsigned long long pa = kABytes >> 4, pb = b_part >> 4;
                        const uint32_t d2 = d + kTmemBuffer / 2;
                        mma(d2, at + 2 * pa, bt, idesc, add);
                        mma(d2, at + pa, bt + pb, idesc, true);
                        mma(d2, at, bt + 2 * pb, idesc, true);
                        mma(d2, at + pa, bt, idesc, true);
                        mma(d2, at, bt + pb, idesc, true);
                    }
                }
                commit(empty + 8 * s);
            }
            commit(acc_full + 8 * buf);
        }
    } else if (warp >= kFirstEpi && warp < kFirstFill) {
        // ---- write out ------------------------------------------------------------------------------------------------------
        const int e = warp - kFirstEpi, quarter = warp & 3;
        const uint32_t mine = staging + e * 4096;
        const float* st = reinterpret_cast<const float*>(smem + (mine - base));
        for (long long n = 0; alive; ++n) {
            const Unit u = unit_of(p, n);
            if (!u.live) break;
            const int buf = (int)(n & 1);
            alive = wait_warp(acc_full + 8 * buf, (unsigned)(n >> 1) & 1, 0x60000000u | (unsigned)n);
            if (!alive) break;
            fence_after();
            const long long i0 = (long long)u.i * kBlockI + quarter * 32;
            const int rows = (int)(p.I - i0 < 32 ? p.I - i0 : 32);
            const int j0 = u.j * p.bn, wide = p.J - j0 < p.bn ? p.J - j0 : p.bn;
            const uint32_t d = tmem + buf * kTmemBuffer + ((uint32_t)(quarter * 32) << 16);
            for (int c = e / 4 * 32; c < wide; c += 64) {
                uint32_t acc[32];
                tmem_ld32(d + c, acc);
                tmem_wait_ld();
                if (PARTS == 3) {
                    uint32_t small[32];
                    tmem_ld32(d + kTmemBuffer / 2 + c, small);
                    tmem_wait_ld();
#pragma unroll
                    for (int q = 0; q < 32; ++q) acc[q] = __float_as_uint(__uint_as_float(acc[q]) + __uint_as_float(small[q]));
                }
#pragma unroll
                for (int q = 0; q < 8; ++q)
                    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(mine + lane * 128 + ((q ^ (lane & 7)) << 4)),
                                 "r"(acc[4 * q]), "r"(acc[4 * q + 1]), "r"(acc[4 * q + 2]), "r"(acc[4 * q + 3]) : "memory");
                __syncwarp();
                const int cols = wide - c < 32 ? wide - c : 32;
                if (rows > 0) {
                    if (ROLE == kGradW) {
                        write_chunk<T, float, ROLE>(st, p, p.part + u.split * p.I * p.J, i0, rows, j0 + c, cols, lane);
                    } else {
                        write_chunk<T, T, ROLE>(st, p, p.out, i0, rows, j0 + c, cols, lane);
                    }
                }
                __syncwarp();
            }
            fence_before();
            if (lane == 0) mbar_arrive(acc_empty + 8 * buf);
        }
    }
    fence_before();
    __syncthreads();
    if (warp == 2) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// ---- host side ------------------------------------------------------------------------------------------------------------------
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*, const cuuint32_t*, const cuuint32_t*,
                                  CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
inline EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = []() -> EncodeTiledFn {
        void* sym = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &sym, cudaEnableDefault, &found) != cudaSuccess || found != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            return nullptr;
        }
        return reinterpret_cast<EncodeTiledFn>(sym);
    }();
    return fn;
}

}}}  // namespace esc::linear::umma
