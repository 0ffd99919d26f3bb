// The window self-attention's forward pass for bf16 (window_attention.cuh has the formulas) on the fifth-generation tensor cores, for
// windows of many pixels.  A block has 256 queries of one window and head: two groups of four warps, a query per thread, so that a row's
// maximum, sum and base belong to one thread.  Per tile of 64 keys and group
//
//   S [128 x 64] = q k^T                  tcgen05.mma into tensor memory, operands in shared memory
//   p = 2^(c S + bias - base)             a thread reads its row, adds its bias (two at a time from the staged table), writes p as bf16
//   out [128 x d] += p v                  tcgen05.mma, out stays in tensor memory
//
// Warp 9 stages keys and values (three tiles), warp 8 issues: the next tile's S as soon as a group has read the last one, so that the
// products run while powers are taken.  Rows of a tile are 32 bytes for 16 channels (one plane of the tile for each 16), their two
// halves exchanged where bit 7 of the address is set (the 32-byte swizzle): k and q are read along the channels, v along its rows.
// Every wait is bounded; where one runs out the block's rows are left as NaN.
#pragma once
#include "window_attention.cuh"

namespace esc { namespace winatt { namespace umma {

using bf16 = __nv_bfloat16;
using winatt::tc::Bias; using winatt::tc::bias_gap; using winatt::tc::bias_row; using winatt::tc::Walk; using winatt::tc::pieces; using winatt::tc::stage_piece;
using wmma16::smem_addr;
constexpr int kGroups = 2, kRows = 128, kKeys = 64, kStages = 3;
constexpr int kIssuer = kGroups * 4, kLoader = kIssuer + 1, kThreads = (kLoader + 1) * 32;
constexpr unsigned kSpinLimit = 1u << 20;          // polls of a wait, each suspended for up to kPollNs by the hardware
constexpr unsigned kPollNs = 1000;

// ---- barriers and tensor memory --------------------------------------------------------------------------------------------
__device__ __forceinline__ void bar_init(uint32_t bar, unsigned count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void bar_arrive(uint32_t bar) { asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory"); }
__device__ __forceinline__ bool bar_try(uint32_t bar, unsigned parity) {
    unsigned ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity), "r"(kPollNs) : "memory");
    return ok != 0;
}
// By all lanes of a warp.  False, in all of them, where the phase does not come or another warp has given up.
__device__ __forceinline__ bool bar_wait(uint32_t bar, unsigned parity, volatile int* gave_up) {
    for (unsigned n = 0; n < kSpinLimit; ++n) {
        if (__all_sync(0xffffffffu, bar_try(bar, parity))) return true;
        if (__any_sync(0xffffffffu, *gave_up)) return false;
    }
    *gave_up = 1;
    return false;
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
template <int COLS> __device__ __forceinline__ void tmem_alloc(uint32_t slot) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
template <int COLS> __device__ __forceinline__ void tmem_free(uint32_t tmem) { asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(COLS) : "memory"); }
// 16 or 32 columns of a warp's 32 lanes.
__device__ __forceinline__ void tmem_ld(uint32_t a, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]) : "r"(a) : "memory");
}
__device__ __forceinline__ void tmem_st(uint32_t a, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(a), "r"(r[0]), "r"(r[1]),
                 "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]),
                 "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Operands in shared memory with the 32-byte swizzle: rows of 16 channels, eight of them 256 bytes.  Along the channels (K-major); or along
// the rows (MN-major): the next 16 channels lie `plane` bytes further on.
__device__ __forceinline__ unsigned long long desc_k(uint32_t addr) {
    return (unsigned long long)((addr >> 4) & 0x3FFFu) | (1ull << 16) | ((unsigned long long)(256u >> 4) << 32) | (1ull << 46) | (6ull << 61);
}
__device__ __forceinline__ unsigned long long desc_mn(uint32_t addr, uint32_t plane) {
    return (unsigned long long)((addr >> 4) & 0x3FFFu) | ((unsigned long long)((plane >> 4) & 0x3FFFu) << 16) | ((unsigned long long)(256u >> 4) << 32) |
           (1ull << 46) | (6ull << 61);
}
// D fp32, A and B bf16, M = 128, N = n; B along its rows or not.
__device__ __forceinline__ constexpr uint32_t instr(int n, bool b_mn) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | (8u << 24);
}
// By a whole warp with the same arguments; one elected lane issues.
__device__ __forceinline__ void mma(uint32_t d, unsigned long long a, unsigned long long b, uint32_t idesc, bool add) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %4, 0;\n\telect.sync _|q, 0xffffffff;\n\t@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(add ? 1u : 0u) : "memory");
}
__device__ __forceinline__ void commit(uint32_t bar) {
    asm volatile("{\n\t.reg .pred q;\n\telect.sync _|q, 0xffffffff;\n\t@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(bar) : "memory");
}
// Piece (16 bytes) `c` of row `r` in planes of `rows` rows.
__device__ __forceinline__ uint32_t place(int r, int c, int rows) { return (uint32_t)((c >> 1) * rows * 32 + r * 32 + (((c & 1) ^ ((r >> 2) & 1)) << 4)); }

template <int D> struct Smem {
    static constexpr int kQ = kRows * D * 2, kTile = kKeys * D * 2, kP = kRows * kKeys * 2;
    static constexpr int kOffTiles = kGroups * kQ, kOffP = kOffTiles + kStages * 2 * kTile, kOffPlaces = kOffP + kGroups * kP, kOffBars = kOffPlaces + kStages * kKeys * 4,
                         kOffTable = kOffBars + 256;
    static constexpr int kCols = 256;              // of tensor memory: per group 64 of S and D of out
    static __host__ __device__ size_t bytes(const Bias& b, bool twice) { return 1024 + kOffTable + (size_t)b.size * 4 * (twice ? 2 : 1) + (twice ? bias_gap() * 4 : 0); }
};

template <int D, bool TWICE>
__global__ void __launch_bounds__(kThreads, 2)
forward(Maps<bf16> m, int tiles, bf16* __restrict__ out, float* __restrict__ lse) {
    using S = Smem<D>;
    constexpr int kSteps = D / 16, kGroupCols = kKeys + D;
    static_assert(kGroups * kGroupCols <= S::kCols, "tensor memory");
    extern __shared__ unsigned char raw_[];
    unsigned char* raw = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw_) + 1023) & ~(uintptr_t)1023);
    const uint32_t base_smem = smem_addr(raw);
    int* places = reinterpret_cast<int*>(raw + S::kOffPlaces);      // 4 B of the staged keys
    float* table = reinterpret_cast<float*>(raw + S::kOffTable);
    const uint32_t bars = base_smem + S::kOffBars;
    const uint32_t tile_full = bars, tile_free = bars + 8 * kStages, s_full = tile_free + 8 * kStages, s_free = s_full + 8 * kGroups, p_full = s_free + 8 * kGroups,
                   p_free = p_full + 8 * kGroups;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(raw + S::kOffBars + 192);
    volatile int* gave_up = reinterpret_cast<volatile int*>(tmem_slot + 1);
    static_assert(16 * kStages + 32 * kGroups <= 192, "barriers");

    const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
    int id = blockIdx.x;
    const int tile = id % tiles; id /= tiles;
    const int head = id % m.heads;
    const Window w = window_at(m, id / m.heads);
    const int n = w.tokens(), block_first = tile * kGroups * kRows;
    if (block_first >= n) return;
    const int count = (n + kKeys - 1) / kKeys, groups = n - block_first > kRows ? 2 : 1;   // tiles of keys; groups that have queries
    const Bias bias(m.wh, m.ww);
    const int head_off = head * m.d;
    if (tid == 0) {
        for (int s = 0; s < kStages; ++s) { bar_init(tile_full + 8 * s, 1); bar_init(tile_free + 8 * s, 1); }
        for (int g = 0; g < kGroups; ++g) { bar_init(s_full + 8 * g, 1); bar_init(s_free + 8 * g, 4); bar_init(p_full + 8 * g, 4); bar_init(p_free + 8 * g, 1); }
        *gave_up = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kIssuer) tmem_alloc<S::kCols>(smem_addr(tmem_slot));
    // the table, in units of 2^x, backwards as for every kernel with rows of queries
    {
        const int cols = 2 * m.ww - 1, rows = 2 * m.wh - 1;
        int span = 1;
        while (span < cols && span < 32) span *= 2;
        const int step = kThreads / span, c0 = tid % span;
        for (int r = tid / span; r < rows; r += step)
            for (int c = c0; c < cols; c += span) {
                const float x = relpos::table_at(m.table, m.bucket, m.n_buckets, m.heads, head, r * cols + c);
                const float v = x <= kMasked ? -INFINITY : x * kLog2e;
                const int at = (rows - 1 - r) * bias.pitch + cols - 1 - c;
                table[at] = v;
                if (TWICE) table[bias.size + bias_gap() + at + 1] = v;
            }
    }
    const int group = warp >> 2, row = (warp & 3) * 32 + lane, i = block_first + group * kRows + row;   // of the first eight warps
    if (warp < kIssuer) {                                           // a thread stages its own query
        const bf16* src = m.q + (i < n ? pixel_of(m, w, i) * m.stride + head_off : 0);
        const bool wide = pieces(m.q, m.stride, m.d);
#pragma unroll
        for (int c = 0; c < D / 8; ++c) {
            const bool real = i < n && c * 8 < m.d;
            const uint32_t to = base_smem + group * S::kQ + place(row, c, kRows);
            if (wide) {
                const uint4 v = real ? *reinterpret_cast<const uint4*>(src + c * 8) : make_uint4(0u, 0u, 0u, 0u);
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
            } else {
                stage_piece(src + (real ? c * 8 : 0), to, real, m.d - c * 8, false);
            }
        }
        fence_async();
    }
    fence_before();
    __syncthreads();
    fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_slot, 0);
    bool alive = true;

    if (warp == kLoader) {
        const bf16 *k0 = m.k + w.pixel * m.stride + head_off, *v0 = m.v + w.pixel * m.stride + head_off;
        const bool wide_k = pieces(m.k, m.stride, m.d), wide_v = pieces(m.v, m.stride, m.d);
        Walk<kKeys> walk;
        walk.start(w, lane);
        for (int t = 0; t <= count && alive; ++t) {
            if (t < count) {
                const int s = t % kStages;
                if (t >= kStages) alive = bar_wait(tile_free + 8 * s, (t / kStages - 1) & 1, gave_up);
                if (!alive) break;
                const uint32_t ks = base_smem + S::kOffTiles + s * 2 * S::kTile, vs = ks + S::kTile;
#pragma unroll
                for (int u = 0; u < kKeys / 32; ++u) {
                    const bool in = walk.y[u] < w.h;
                    const long long px = in ? ((long long)walk.y[u] * m.W + walk.x[u]) * m.stride : 0;
                    places[s * kKeys + lane + 32 * u] = in ? 4 * (walk.y[u] * bias.pitch + walk.x[u]) : 0;
#pragma unroll
                    for (int c = 0; c < D / 8; ++c) {
                        const bool real = in && c * 8 < m.d;
                        const long long from = real ? px + c * 8 : 0;
                        stage_piece(k0 + from, ks + place(lane + 32 * u, c, kKeys), real, m.d - c * 8, wide_k);
                        stage_piece(v0 + from, vs + place(lane + 32 * u, c, kKeys), real, m.d - c * 8, wide_v);
                    }
                }
                walk.step(w);
                wmma16::cp_commit();
            }
            if (t > 0) {                                            // the tile before is there
                if (t < count) wmma16::cp_wait<1>(); else wmma16::cp_wait<0>();
                fence_async();
                __syncwarp();
                if (lane == 0) bar_arrive(tile_full + 8 * ((t - 1) % kStages));
            }
        }
        wmma16::cp_wait<0>();
    } else if (warp == kIssuer) {
        auto product = [&](int g, int t) {                          // S of tile t
            const uint32_t a = base_smem + g * S::kQ, b = base_smem + S::kOffTiles + (t % kStages) * 2 * S::kTile;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) mma(tmem + g * kGroupCols, desc_k(a + k * kRows * 32), desc_k(b + k * kKeys * 32), instr(kKeys, false), k > 0);
            commit(s_full + 8 * g);
        };
        alive = bar_wait(tile_full, 0, gave_up);
        fence_after();
        for (int g = 0; g < groups && alive; ++g) product(g, 0);
        for (int t = 0; t < count && alive; ++t) {
            for (int g = 0; g < groups && alive; ++g) {
                if (t + 1 < count) {
                    if (g == 0) alive = bar_wait(tile_full + 8 * ((t + 1) % kStages), ((t + 1) / kStages) & 1, gave_up);
                    if (alive) alive = bar_wait(s_free + 8 * g, t & 1, gave_up);
                    if (!alive) break;
                    fence_after();
                    product(g, t + 1);
                }
                alive = bar_wait(p_full + 8 * g, t & 1, gave_up);
                if (!alive) break;
                fence_after();
                const uint32_t a = base_smem + S::kOffP + g * S::kP, b = base_smem + S::kOffTiles + (t % kStages) * 2 * S::kTile + S::kTile;
#pragma unroll
                for (int k = 0; k < kKeys / 16; ++k)
                    mma(tmem + g * kGroupCols + kKeys, desc_k(a + k * kRows * 32), desc_mn(b + k * 512, kKeys * 32), instr(D, true), t > 0 || k > 0);
                commit(p_free + 8 * g);
            }
            if (alive) commit(tile_free + 8 * (t % kStages));
        }
    } else if (group < groups) {
        const int q = min(i, n - 1), y = q / w.w, x = q - y * w.w;
        const bool pairs = TWICE && (w.w & 1) == 0, eights = TWICE && (w.w & 7) == 0;
        const uint32_t at = bias_row<TWICE>(m, bias, pairs, y, x, smem_addr(table));
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16) + group * kGroupCols, acc = lanes + kKeys;
        const uint32_t p_row = base_smem + S::kOffP + group * S::kP + row * 32, swap = (uint32_t)((row >> 2) & 1) << 4;
        const float c = m.scale * kLog2e;
        const Two by = two(c, c);
        float top = -INFINITY, limit = -INFINITY;
        Two off = two(0.0f, 0.0f), sum0 = off, sum1 = off;
        for (int t = 0; t < count && alive; ++t) {
            const int s = t % kStages, left = n - t * kKeys;
            alive = bar_wait(tile_full + 8 * s, (t / kStages) & 1, gave_up) && bar_wait(s_full + 8 * group, t & 1, gave_up);
            if (!alive) break;
            fence_after();
            uint32_t r[4][16];
#pragma unroll
            for (int u = 0; u < 4; ++u) tmem_ld(lanes + 16 * u, r[u]);
            tmem_wait_ld();
            fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(s_free + 8 * group);
            const int* b = places + s * kKeys;
            if (eights) {
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    const uint32_t from = at + b[8 * u];
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        uint32_t* to = &r[u >> 1][(u & 1) * 8 + 2 * e];
                        const float2 v = lds2(from + 8 * e);
                        float f, g;
                        apart(fma2(two(__uint_as_float(to[0]), __uint_as_float(to[1])), by, two(v.x, v.y)), f, g);
                        to[0] = __float_as_uint(f); to[1] = __float_as_uint(g);
                    }
                }
            } else {
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    uint32_t* to = &r[e >> 3][2 * (e & 7)];
                    const float2 v = pairs ? lds2(at + b[2 * e]) : make_float2(lds1(at + b[2 * e]), lds1(at + b[2 * e + 1]));
                    float f, g;
                    apart(fma2(two(__uint_as_float(to[0]), __uint_as_float(to[1])), by, two(v.x, v.y)), f, g);
                    to[0] = __float_as_uint(f); to[1] = __float_as_uint(g);
                }
            }
            if (left < kKeys) {
#pragma unroll
                for (int e = 0; e < kKeys; ++e)
                    if (e >= left) r[e >> 4][e & 15] = __float_as_uint(-INFINITY);
            }
            float high = fmaxf(__uint_as_float(r[0][0]), __uint_as_float(r[0][1])), high1 = fmaxf(__uint_as_float(r[2][0]), __uint_as_float(r[2][1]));
#pragma unroll
            for (int e = 2; e < 32; e += 2) {
                high = max3(high, __uint_as_float(r[e >> 4][e & 15]), __uint_as_float(r[e >> 4][(e & 15) + 1]));
                high1 = max3(high1, __uint_as_float(r[2 + (e >> 4)][e & 15]), __uint_as_float(r[2 + (e >> 4)][(e & 15) + 1]));
            }
            high = fmaxf(high, high1);
            if (t > 0) {                                            // the last p has been read, and out is complete up to here
                alive = bar_wait(p_free + 8 * group, (t - 1) & 1, gave_up);
                if (!alive) break;
            }
            if (__any_sync(0xffffffffu, high > limit)) {            // rows whose base moves: what they have so far is scaled
                fence_after();
                const float to = fmaxf(high, top), base = to == -INFINITY ? 0.0f : to, old = ex2(top - base);
                top = to;
                limit = to + tc::kSlack;
                off = two(-base, -base);
                sum0 = mul2(sum0, two(old, old)); sum1 = mul2(sum1, two(old, old));
                if (t > 0) {
#pragma unroll 1
                    for (int k = 0; k < kSteps; ++k) {
                        uint32_t o[16];
                        tmem_ld(acc + 16 * k, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * old);
                        tmem_st(acc + 16 * k, o);
                    }
                    tmem_wait_st();
                }
                fence_before();
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                uint32_t p[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    float f, g;
                    apart(add2(two(__uint_as_float(r[u][2 * e]), __uint_as_float(r[u][2 * e + 1])), off), f, g);
                    f = ex2(f); g = ex2(g);
                    if (e & 1) sum1 = add2(sum1, two(f, g)); else sum0 = add2(sum0, two(f, g));
                    p[e] = wmma16::pack(f, g);
                }
                const uint32_t to = p_row + u * kRows * 32;
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to + swap), "r"(p[0]), "r"(p[1]), "r"(p[2]), "r"(p[3]) : "memory");
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(to + (swap ^ 16u)), "r"(p[4]), "r"(p[5]), "r"(p[6]), "r"(p[7]) : "memory");
            }
            fence_async();
            __syncwarp();
            if (lane == 0) bar_arrive(p_full + 8 * group);
        }
        if (alive) alive = bar_wait(p_free + 8 * group, (count - 1) & 1, gave_up);
        fence_after();
        float f0, g0, f1, g1;
        apart(sum0, f0, g0); apart(sum1, f1, g1);
        const float total = (f0 + g0) + (f1 + g1), inv = !alive ? __int_as_float(0x7fffffff) : total == 0.0f ? 0.0f : 1.0f / total;
        const long long pixel = pixel_of(m, w, q);
        bf16* to = out + (pixel * m.heads + head) * m.d;
        const bool wide = m.d % 8 == 0;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            uint32_t o[16];
            __syncwarp();
            tmem_ld(acc + 16 * k, o);
            tmem_wait_ld();
            if (i >= n) continue;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int ch = 16 * k + 8 * h;
                float f[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = __uint_as_float(o[8 * h + e]) * inv;
                if (wide) {
                    if (ch < m.d) *reinterpret_cast<uint4*>(to + ch) = make_uint4(wmma16::pack(f[0], f[1]), wmma16::pack(f[2], f[3]), wmma16::pack(f[4], f[5]), wmma16::pack(f[6], f[7]));
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (ch + e < m.d) to[ch + e] = __float2bfloat16_rn(f[e]);
                }
            }
        }
        if (lse && i < n) {
            const long long hw = (long long)m.H * m.W;
            lse[((long long)w.b * m.heads + head) * hw + pixel - w.b * hw] = !alive ? inv : total == 0.0f ? -INFINITY : fmaf(top, kLn2, logf(total));
        }
        fence_before();
    }
    __syncthreads();
    if (warp == kIssuer) {
        fence_after();
        tmem_free<S::kCols>(tmem);
    }
}

}}}  // namespace esc::winatt::umma
