// The backward pass of a small linear layer (bf16; K and N of a few hundred at most) in one pass over its rows:
//
//   g = go act'(z)     gx = g w     gw = sum over rows of g^T x     gb = sum over rows of g
//
// Such layers are bound by memory: go, z and x are read once, gx is written once, and g never leaves shared memory.  A block takes tiles of
// 128 rows, one after another.  TMA brings go, z and x as boxes of 128 rows x 64 columns (128 bytes a row, 128-byte swizzle); eight warps
// turn go into g in place and add up its columns; then the same boxes of g are the operand of both products: with 128 rows and the columns
// as contraction (K-major) for gx, with the columns as rows of the result and 128 rows as contraction (MN-major) for gw.  w stays in shared
// memory and the sums of gw in tensor memory for the life of the block (N / 128 x K columns beside one or two tiles of gx); each block leaves
// one partial sum of gw and gb.  64 x 64x64 rows, 64 to 128 channels, GELU: 52 us (3.9 TB/s), with gradients of the weights in bf16 or fp32, where
// three kernels that wrote and read g took 96 and 87.  What bounds it: the act' of 33 million values on eight warps of an SM, and latency.
#pragma once
#include "linear_umma.cuh"

namespace esc { namespace linear { namespace small {

using namespace esc::linear::umma;
using bf16 = __nv_bfloat16;

constexpr int kRows = 128, kBox = kRows * 128, kActWarps = 8, kOutWarps = 4, kFirstAct = 4, kFirstOut = kFirstAct + kActWarps, kThreads = 32 * (kFirstOut + kOutWarps);
constexpr int kMostBoxes = 4;                                      // of go: N up to 256
constexpr int kMostStages = 4;
constexpr int kRunTiles = kRun * kBlockC / kRows, kLongTiles = kLongRun * kBlockC / kRows;   // tiles after which a sum of gw has to end, where gw is fp32, and bf16

struct Args {
    int rows, N, K, tiles, act, stages;
    int nb, kb;                                                    // boxes of 64 columns of go and of x
    int gx_buffers;
    bool gx, gw, gb;
    float* part_b;                                                 // [gridDim.x][N]
};

__device__ __forceinline__ unsigned long long desc(uint32_t addr, uint32_t lbo) {
    return (unsigned long long)((addr >> 4) & 0x3FFFu) | ((unsigned long long)(lbo >> 4) << 16) | ((unsigned long long)(1024 >> 4) << 32) | (1ull << 46) | (2ull << 61);
}

// RUNS: a block has more tiles than a sum of gw may: that of kRunTiles is added to a running one beside it in tensor memory (see kRun).
template <bool RUNS> __global__ void __launch_bounds__(kThreads, 1)
backward(const __grid_constant__ CUtensorMap map_go, const __grid_constant__ CUtensorMap map_z, const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_w,
         const __grid_constant__ CUtensorMap map_gx, const __grid_constant__ CUtensorMap map_part, const __grid_constant__ Args p)
{
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t base = smem_u32(smem);
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const bool has_act = p.act != kActNone;
    // a tile: go, x, z in this order (the last rows of gw's products may come from the box behind go's, and go nowhere)
    const uint32_t x_at = p.nb * kBox, z_at = x_at + p.kb * kBox, stage_bytes = z_at + (has_act ? p.nb * kBox : 0);
    const uint32_t w_at = base + p.stages * stage_bytes, w_block = p.kb * 64 * 128, staging = w_at + p.nb * w_block;
    const uint32_t full = staging + kOutWarps * kSlotBytes, ready = full + 8 * kMostStages, empty = ready + 8 * kMostStages, gx_full = empty + 8 * kMostStages,
                   gx_empty = gx_full + 16, w_full = gx_empty + 16, gw_done = w_full + 8, gb_done = gw_done + 8, gw_taken = gb_done + 8, finished = gw_taken + 8, slot = finished + 8,
                   strip = slot + 16;                              // [kActWarps][256] floats: columns of g
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) { mbar_init(full + 8 * s, 1); mbar_init(ready + 8 * s, kActWarps); mbar_init(empty + 8 * s, 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(gx_full + 8 * s, 1); mbar_init(gx_empty + 8 * s, kOutWarps); }
        mbar_init(w_full, 1);
        mbar_init(gw_done, 1);
        mbar_init(gb_done, kActWarps);
        mbar_init(gw_taken, kOutWarps);
        mbar_init(finished, 1);
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
    tmem = __shfl_sync(0xffffffffu, tmem, 0);
    const uint32_t columns = p.kb * 64, gw_at = tmem + p.gx_buffers * columns;   // sums: gx of one or two tiles, then gw by 128 outputs

    bool alive = true;
    int n = 0;                                                     // tiles so far
    Ring r{};
    if (warp == 0) {
        if (lane == 0) {
            mbar_expect(w_full, p.nb * w_block);
            for (int c = 0; c < p.nb; ++c)
                for (int m = 0; m < p.kb; ++m) tma_load_2d(w_at + c * w_block + m * 64 * 128, &map_w, w_full, m * 64, c * 64);
            for (int t = blockIdx.x; t < p.tiles && alive; t += gridDim.x, r.next(p.stages)) {
                if (r.round > 0) alive = wait_lane(empty + 8 * r.s, (r.round - 1) & 1, 0x11000000u | r.round);
                if (!alive) break;
                const uint32_t at = base + r.s * stage_bytes, bar = full + 8 * r.s;
                mbar_expect(bar, stage_bytes);
                for (int c = 0; c < p.nb; ++c) {
                    tma_load_2d(at + c * kBox, &map_go, bar, c * 64, t * kRows);
                    if (has_act) tma_load_2d(at + z_at + c * kBox, &map_z, bar, c * 64, t * kRows);
                }
                for (int c = 0; c < p.kb; ++c) tma_load_2d(at + x_at + c * kBox, &map_x, bar, c * 64, t * kRows);
            }
            wait_lane(w_full, 0, 0x7B000000u);
            landed(full, p.stages, r);
        }
        __syncwarp();
    } else if (warp == 1) {
        const uint32_t idesc_x = instr_desc<false, true>(columns), idesc_w = instr_desc<true, true>(columns);
        alive = wait_warp(w_full, 0, 0x41000000u);
        for (int t = blockIdx.x; t < p.tiles && alive; t += gridDim.x, r.next(p.stages), ++n) {
            const int buf = p.gx_buffers == 2 ? n & 1 : 0, use = p.gx_buffers == 2 ? n >> 1 : n;
            alive = wait_warp(ready + 8 * r.s, r.round & 1, 0x51000000u | r.round);
            if (alive && p.gx && use > 0) alive = wait_warp(gx_empty + 8 * buf, (use - 1) & 1, 0x31000000u | (unsigned)n);
            if (!alive) break;
            fence_after();
            const uint32_t at = base + r.s * stage_bytes;
            if (p.gx) {
#pragma unroll 1
                for (int c = 0; c < p.nb; ++c) {
                    const unsigned long long a = desc(at + c * kBox, 16), b = desc(w_at + c * w_block, 64 * 128);
#pragma unroll
                    for (int k = 0; k < 4; ++k) mma(tmem + buf * columns, a + k * 2, b + k * 128, idesc_x, c > 0 || k > 0);
                }
                commit(gx_full + 8 * buf);
            }
            const int in_run = RUNS ? n % kRunTiles : n;
            if (p.gw) {
                if (RUNS && n > 0 && in_run == 0) {                // the sum of the run before has been read
                    alive = wait_warp(gw_taken, (unsigned)(n / kRunTiles - 1) & 1, 0xB1000000u | (unsigned)n);
                    if (!alive) break;
                    fence_after();
                }
#pragma unroll 1
                for (int m = 0; m < p.nb; m += 2) {
                    const unsigned long long a = desc(at + m * kBox, kBox), b = desc(at + x_at, kBox);
#pragma unroll
                    for (int k = 0; k < 8; ++k) mma(gw_at + m / 2 * columns, a + k * 128, b + k * 128, idesc_w, in_run > 0 || k > 0);
                }
            }
            commit(empty + 8 * r.s);
            if (RUNS && in_run == kRunTiles - 1 && t + gridDim.x < p.tiles) commit(gw_done);
        }
        commit(gw_done);
        finish(finished);
    } else if (warp >= kFirstAct && warp < kFirstOut) {
        // ---- g in place, and its columns' sums ------------------------------------------------------------------------------
        // A lane has the eight columns of one piece in every box, a warp four rows at a time.
        const int w = warp - kFirstAct, row = w * 4 + lane / 8, q = lane % 8;
        float sum[kMostBoxes][8] = {};
        const GaussConst k;
        for (int t = blockIdx.x; t < p.tiles && alive; t += gridDim.x, r.next(p.stages)) {
            alive = wait_warp(full + 8 * r.s, r.round & 1, 0x21000000u | r.round);
            if (!alive) break;
            const uint32_t at = base + r.s * stage_bytes + staged(row, q * 16);   // rows 4 kActWarps apart are exchanged alike
            if (has_act || p.gb) {
#pragma unroll
                for (int c = 0; c < kMostBoxes; ++c) {
                    if (c >= p.nb) break;
#pragma unroll 1
                    for (int i = 0; i < kRows; i += 4 * kActWarps) {
                        const uint32_t piece = at + c * kBox + i * 128;
                        float f[8];
                        unpack16<bf16>(ld_shared(piece), f);
                        if (has_act) {
                            float z[8];
                            unpack16<bf16>(ld_shared(piece + z_at), z);
                            times_slope<8>(p.act, k, f, z);
                            st_shared(piece, pack16<bf16>(f));
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e) sum[c][e] += f[e];
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(ready + 8 * r.s);
        }
        if (p.gb && alive) {
            // the rows of a warp, then the warps in order
#pragma unroll
            for (int c = 0; c < kMostBoxes; ++c) {
                if (c >= p.nb) break;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    sum[c][e] += __shfl_xor_sync(0xffffffffu, sum[c][e], 8);
                    sum[c][e] += __shfl_xor_sync(0xffffffffu, sum[c][e], 16);
                    if (lane < 8) st_value(strip + (w * 256 + c * 64 + lane * 8 + e) * 4, sum[c][e]);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(gb_done);
            alive = wait_warp(gb_done, 0, 0x91000000u);
            const int col = w * 32 + lane;
            if (alive && col < p.N) {
                float s = 0.f;
#pragma unroll
                for (int v = 0; v < kActWarps; ++v) s += get_value(strip + (v * 256 + col) * 4, 0.f);
                p.part_b[(size_t)blockIdx.x * p.N + col] = s;
            }
        }
    } else if (warp >= kFirstOut) {
        // ---- gx of each tile, gw at the end: 128 bytes of 32 rows at a time ---------------------------------------------------
        static_assert(kOutWarps == 4, "a warp to each quarter of the lanes");
        const int quarter = warp & 3;
        const uint32_t mine = staging + (warp - kFirstOut) * kSlotBytes, lane_at = lane * 128 + ((lane & 7) << 4), lanes = (uint32_t)(quarter * 32) << 16;
        const int across = (int)(columns / 32), units = (p.nb + 1) / 2 * across;
        const uint32_t run_at = gw_at + (p.nb + 1) / 2 * columns;  // the running sum
        int runs = 0;
        for (int t = blockIdx.x; t < p.tiles && alive; t += gridDim.x, ++n) {
            if (p.gx) {
                const int buf = p.gx_buffers == 2 ? n & 1 : 0, use = p.gx_buffers == 2 ? n >> 1 : n;
                alive = wait_warp(gx_full + 8 * buf, use & 1, 0x61000000u | (unsigned)n);
                if (!alive) break;
                fence_after();
                const int i0 = t * kRows + quarter * 32;
                for (int c = 0; c < p.kb; ++c) {
                    if (i0 >= p.rows) break;
                    if (lane == 0) bulk_wait_read<0>();
                    __syncwarp();
#pragma unroll 1
                    for (int q = 0; q < 8; q += 2) {
                        float f[16];
                        tmem_ld(tmem + lanes + buf * columns + c * 64 + q * 8, f);
                        tmem_wait_ld();
                        st_shared(mine + (lane_at ^ (uint32_t)(q << 4)), pack16<bf16>(f));
                        st_shared(mine + (lane_at ^ (uint32_t)((q + 1) << 4)), pack16<bf16>(f + 8));
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) { tma_store_3d(&map_gx, mine, c * 64, i0, 0); bulk_commit(); }
                    __syncwarp();
                }
                fence_before();
                if (lane == 0) mbar_arrive(gx_empty + 8 * buf);
            }
            if (RUNS && p.gw && n % kRunTiles == kRunTiles - 1 && t + gridDim.x < p.tiles) {
                alive = wait_warp(gw_done, (unsigned)runs & 1, 0x82000000u | (unsigned)runs);
                if (!alive) break;
                fence_after();
                for (int v = 0; v < units; ++v) add_run<1, 16, 32>(gw_at + lanes + v * 32, run_at + lanes + v * 32, runs > 0);
                ++runs;
                fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(gw_taken);
            }
        }
        if (p.gw && alive) alive = wait_warp(gw_done, (unsigned)runs & 1, 0x81000000u);
        if (p.gw && alive) {
            fence_after();
            for (int v = 0; v < units; ++v) {
                const int m = v / across, c = v - m * across, n0 = m * 128 + quarter * 32;
                if (n0 >= p.N || c * 32 >= p.K) continue;
                if (lane == 0) bulk_wait_read<0>();
                __syncwarp();
#pragma unroll 1
                for (int q = 0; q < 8; q += 2) {
                    float f[8];
                    sums<1>(f, gw_at + lanes + v * 32 + q * 4, run_at + lanes + v * 32 + q * 4, RUNS && runs > 0);
                    st_shared(mine + (lane_at ^ (uint32_t)(q << 4)), pack16<float>(f));
                    st_shared(mine + (lane_at ^ (uint32_t)((q + 1) << 4)), pack16<float>(f + 4));
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) { tma_store_3d(&map_part, mine, c * 32, n0, (int)blockIdx.x); bulk_commit(); }
                __syncwarp();
            }
        }
        if (lane == 0) bulk_wait_read<0>();                        // shared memory outlives what is read from it
    }
    pdl_launch_dependents();
    fence_before();
    __syncthreads();
    if (warp == 2) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// Sizes: whether a layer is one of these, and how its block is laid out (stages 0: it is not).  wide: gw is fp32.
struct Plan { int stages, gx_buffers, nb, kb, tiles, grid; bool runs; size_t smem; };
inline Plan plan(long long rows, int K, int N, bool act, bool wide, int sms) {
    Plan d{};
    if (N > 64 * kMostBoxes || K > 256 || rows < 1 || rows > 0x7fffffffLL - kRows) return d;
    d.nb = (N + 63) / 64; d.kb = (K + 63) / 64;
    d.tiles = (int)((rows + kRows - 1) / kRows);
    d.grid = d.tiles < sms ? d.tiles : sms;
    d.runs = (d.tiles + d.grid - 1) / d.grid > (wide ? kRunTiles : kLongTiles);
    const int gw_columns = (d.nb + 1) / 2 * d.kb * 64 * (d.runs ? 2 : 1);
    d.gx_buffers = gw_columns + 2 * d.kb * 64 <= 512 ? 2 : 1;
    if (gw_columns + d.kb * 64 > 512) return d;
    const size_t stage = (size_t)(d.nb * (act ? 2 : 1) + d.kb) * kBox, fixed = (size_t)d.nb * d.kb * 64 * 128 + kOutWarps * kSlotBytes + 1024 + kActWarps * 1024;
    if (fixed + stage > kMostSmem) return d;
    size_t stages = (kMostSmem - fixed) / stage;
    if (stages > kMostStages) stages = kMostStages;
    if (stages < 2 && d.tiles > sms) return d;                     // without a second tile on its way the three kernels are faster
    d.stages = (int)stages;
    d.smem = stages * stage + fixed;
    return d;
}

}}}  // namespace esc::linear::small
