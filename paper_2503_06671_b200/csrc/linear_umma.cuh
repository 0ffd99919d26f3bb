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
// bf16 with rows of whole 16-byte pieces: TMA fills the ring.  Otherwise two groups of eight warps load values as they lie and store them
// swizzled, a group every other block: any stride and alignment, and fp32, where every value is split into three bf16 parts (24 bits: hi + mid
// + lo exactly, down to 2^-110; smaller values lose what lies below bf16's last bit, 2^-133) and six of the nine products are taken; the parts are 2^-8
// of one another at most, so what is left out is two products of 2^-25 (rms of all: 2^-27).  The largest of them has an accumulator
// of its own (the tensor cores add as fp32, and small terms would be rounded at the large sum's step).  An infinity has no such parts: a row
// or column with one comes out as NaN.
//
// Epilogue: a lane of a warp reads a row's 128 bytes of results from tensor memory, 32 bytes at a time, adds the bias, applies the activation,
// adds the residual, rounds once and puts them, exchanged as the 128-byte swizzle has it, into the warp's 4 KB of shared memory; TMA brings the
// residual there and takes the results from there.  Rows that TMA cannot take leave through the same 4 KB by plain stores of whole warps.
//
// Large products run at the tensor cores' rate under the power limit: 16384 x 4096 x 4096 in bf16 410 us, 1.33 PFLOP/s.  fp32 is bound by the warps
// that split: 57600 x 192 to 384 78 us, 8192 x 512 to 512 44 us, with the tensor cores busy a quarter to a third of the time.
// Small layers (K and N of a few hundred, many rows) are bound by memory: w then stays in shared memory for the whole life of a block
// (`resident`), and the ring holds rows alone.
#pragma once
#include <cuda.h>
#include "linear.cuh"

namespace esc { namespace linear { namespace umma {

constexpr int kBlockI = 128, kBlockC = 64;
constexpr int kABytes = kBlockI * kBlockC * 2;                     // of one part
// Warps: one that asks for TMA loads, one that issues (two idle), those that write out, those that fill (a group fills every other block).
constexpr int kFillWarps = 16, kGroupWarps = 8, kFirstEpi = 4;
template <bool TMA> constexpr int epi_warps = TMA ? 12 : 8;
template <bool TMA> constexpr int all_warps = kFirstEpi + epi_warps<TMA> + (TMA ? 0 : kFillWarps);
constexpr int kMostEpi = 12;
constexpr int kSlotBytes = 32 * 128;                               // staging of an epilogue warp: 128 bytes of 32 rows
constexpr int kMaxStages = 8;
constexpr size_t kMostSmem = 227 * 1024;
constexpr int kTmemBuffer = 256;                                   // columns of one tile's sums
constexpr unsigned kPolls = 1u << 20, kHintNs = 1000;              // a wait gives up after about one second

__device__ unsigned wait_status[2];                                // ESC_DEV_TIMEOUT and where, if a wait ran out

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, unsigned count) { asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory"); }
__device__ __forceinline__ void mbar_expect(uint32_t bar, unsigned bytes) { asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory"); }
// Bytes alone: who asks for them arrives later.
__device__ __forceinline__ void mbar_bytes(uint32_t bar, unsigned bytes) { asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(bytes) : "memory"); }
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
// The same of one lane.
__device__ __forceinline__ bool wait_lane(uint32_t bar, unsigned parity, unsigned where) {
    for (unsigned n = 0; n < kPolls; ++n) {
        unsigned ok;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(ok) : "r"(bar), "r"(parity), "r"(kHintNs) : "memory");
        if (ok) return true;
    }
    atomicExch(&wait_status[0], kDevTimeout);
    atomicExch(&wait_status[1], where);
    return false;
}
// A place in the ring, and how often it came round.
struct Ring {
    unsigned s, round;
    __device__ __forceinline__ void next(int stages) { if (++s == (unsigned)stages) { s = 0; ++round; } }
};
// Loads into the ring up to place r have landed, by the lane that asked for them: also where the block gave up, shared memory outlives what is written to it.
__device__ __forceinline__ void landed(uint32_t full, int stages, Ring r) {
#pragma unroll 1
    for (unsigned s = 0; s < (unsigned)stages; ++s)
        if (r.round > 0 || s < r.s) wait_lane(full + 8 * s, (s < r.s ? r.round : r.round - 1) & 1, 0x70000000u | s);
}
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
                 ::"r"(dst), "l"(map), "r"(bar), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void tma_store_3d(const CUtensorMap* map, uint32_t src, int c0, int c1, int c2) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];" ::"l"(map), "r"(src), "r"(c0), "r"(c1), "r"(c2) : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(N) : "memory"); }
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
// All products issued so far have been done, likewise.
__device__ __forceinline__ void finish(uint32_t bar) {
    commit(bar);
    wait_warp(bar, 0, 0xC0000000u);
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_ld(uint32_t at, float (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]), "=f"(r[10]), "=f"(r[11]),
                   "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_ld(uint32_t at, float (&r)[8]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]) : "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_st(uint32_t at, const float (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(at), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]), "f"(r[8]), "f"(r[9]), "f"(r[10]), "f"(r[11]),
                   "f"(r[12]), "f"(r[13]), "f"(r[14]), "f"(r[15]) : "memory");
}
__device__ __forceinline__ void tmem_st(uint32_t at, const float (&r)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(at), "f"(r[0]), "f"(r[1]), "f"(r[2]), "f"(r[3]), "f"(r[4]), "f"(r[5]), "f"(r[6]), "f"(r[7]) : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Loads that stay where they are written: a batch of them is under way before the first value is used.
__device__ __forceinline__ uint4 ld_piece(const void* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ float ld_value(const float* p) {
    float v;
    asm volatile("ld.global.nc.b32 %0, [%1];" : "=f"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ uint32_t ld_bits(const float* p) { return __float_as_uint(ld_value(p)); }
__device__ __forceinline__ uint32_t ld_bits(const __nv_bfloat16* p) {
    unsigned short v;
    asm volatile("ld.global.nc.b16 %0, [%1];" : "=h"(v) : "l"(p));
    return v;
}
__device__ __forceinline__ __nv_bfloat16 ld_value(const __nv_bfloat16* p) {
    unsigned short v;
    asm volatile("ld.global.nc.b16 %0, [%1];" : "=h"(v) : "l"(p));
    return __ushort_as_bfloat16(v);
}

// 16 aligned bytes, or zeros and no access.
__device__ __forceinline__ uint4 ld_piece_if(bool in, unsigned long long at) {
    uint4 v;
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b32 %0, 0;\n\tmov.b32 %1, 0;\n\tmov.b32 %2, 0;\n\tmov.b32 %3, 0;\n\t"
                 "@p ld.global.nc.v4.b32 {%0, %1, %2, %3}, [%4];\n\t}" : "=&r"(v.x), "=&r"(v.y), "=&r"(v.z), "=&r"(v.w) : "l"(at), "r"((unsigned)in));
    return v;
}
// 16 aligned bytes of which those outside [begin, end) are not read: the first and the last of a matrix.
__device__ __noinline__ uint4 ld_edge(unsigned long long at, unsigned long long begin, unsigned long long end) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        w[i] = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const unsigned long long a = at + 4 * i + 2 * h;
            if (a >= begin && a < end) w[i] |= ld_bits(reinterpret_cast<const __nv_bfloat16*>(a)) << (16 * h);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// What a warp group loads of one operand: rows of `width` values, `ld` apart; `pieces`: rows are whole aligned 16-byte pieces.
template <typename T> struct Source {
    const T* p;
    long long rows, width, ld;
    bool pieces;
};

template <typename T> struct Args {
    long long I;
    int J, tiles_i, tiles_j, bn, blocks, stages;           // blocks: of c
    int splits, per_split, longer;      // a split has per_split blocks, the first `longer` of them one more
    bool single;                        // RUNS of fp32: a run's sums have one buffer
    bool resident;                      // B stays in shared memory; a block keeps its tile of j
    unsigned units;
    Source<T> a, b;
    int a_rows;                         // lines of A that TMA brings (K-major; the others' sums go nowhere)
    bool a_tma, b_tma;                  // beside plain loads: this operand comes by TMA
    int act;
    const T *bias, *residual;
    T *out, *z;
    float* part;                        // kGradW: [splits][I][J]
};

template <typename T> constexpr int parts_of = sizeof(T) == 4 ? 3 : 1;
// The tensor cores add to a sum by truncation, always towards zero, of the sum and of the products: where all have one sign 512 values lose 2.4e-7 of
// their sum, and from some 16384 on, when the sum has left the products' low bits behind, every 16 values lose 1e-7 (65536 values 3.7e-4, 2^20
// 6.6e-3).  A sum therefore ends after a number of blocks of c and is added, rounded to nearest, to a running sum beside it in tensor memory:
// after kRun where the result is fp32 (4096 values: 4.4e-6 -> below 1e-6 of the result's norm; 16 x 8000: 9.1e-6 -> 3e-7), after kLongRun where it
// is bf16, when 2^-12 are lost at most (65536: 3.7e-4 -> 1.7e-4, 2^20: 6.6e-3 -> 1.9e-4).  That takes columns: tiles are narrower or, in fp32,
// which waits for its operands and not for the tensor cores, have one buffer for a run's sums instead of two (`single`).  Gradients of weights
// in bf16 are cut into runs of rows, which are added in fp32 anyway, of kLongRun blocks at most.
constexpr int kRun = 8, kLongRun = 512;
__host__ __device__ constexpr int run_of(Role role, size_t es) { return role == kGradW || es == 4 ? kRun : kLongRun; }
template <typename T> constexpr int most_columns = sizeof(T) == 4 ? 128 : 256;
template <typename T> constexpr int most_run_columns = sizeof(T) == 4 ? 96 : 128;

// A block's tiles, in the order of its loops.  32-bit arithmetic: a warp that does little else spends a tile's time on divisions.
struct Walk {
    unsigned t, step;                   // resident: tiles of i; else units
    int i, j, split, c0, c1;
    bool live;
};
template <typename T> __device__ __forceinline__ void place(Walk& w, const Args<T>& p) {
    w.live = w.t < (p.resident ? (unsigned)p.tiles_i : p.units);
    if (p.resident) { w.i = (int)w.t; return; }
    const unsigned r = p.tiles_j == 1 ? w.t : w.t / (unsigned)p.tiles_j;
    w.j = (int)(w.t - r * (unsigned)p.tiles_j);
    w.split = p.splits == 1 ? 0 : (int)(r / (unsigned)p.tiles_i);
    w.i = (int)(r - (unsigned)w.split * (unsigned)p.tiles_i);
    w.c0 = w.split * p.per_split + min(w.split, p.longer);
    w.c1 = w.c0 + p.per_split + (w.split < p.longer);
}
template <typename T> __device__ __forceinline__ Walk walk(const Args<T>& p) {
    Walk w{blockIdx.x, gridDim.x, 0, 0, 0, 0, p.blocks, false};
    if (p.resident) { w.step /= (unsigned)p.tiles_j; w.t /= (unsigned)p.tiles_j; w.j = (int)(blockIdx.x % (unsigned)p.tiles_j); }
    place(w, p);
    return w;
}
template <typename T> __device__ __forceinline__ void next(Walk& w, const Args<T>& p) { w.t += w.step; place(w, p); }

// ---- plain loads into swizzled lines ------------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t pack(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void st_shared(uint32_t at, uint32_t v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "r"(v) : "memory"); }
__device__ __forceinline__ void st_shared(uint32_t at, uint32_t v, uint32_t w) { asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(at), "r"(v), "r"(w) : "memory"); }
__device__ __forceinline__ void st_shared(uint32_t at, uint4 v) { asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory"); }
// The three bf16 parts of two values; the differences are exact, and lo is too where the value is not below 2^-110.
__device__ __forceinline__ void split(float a, float b, uint32_t& hi, uint32_t& mid, uint32_t& lo) {
    hi = pack(a, b);
    const F2 minus = f2(-1.f, -1.f);
    un2(fma2(f2(__uint_as_float(hi << 16), __uint_as_float(hi & 0xffff0000u)), minus, f2(a, b)), a, b);
    mid = pack(a, b);
    un2(fma2(f2(__uint_as_float(mid << 16), __uint_as_float(mid & 0xffff0000u)), minus, f2(a, b)), a, b);
    lo = pack(a, b);
}

// Staged rows of 128 bytes: the 16-byte pieces of row r are exchanged by r % 8, so that eight rows' pieces of a column lie in different
// banks.  Byte b of row r:
__device__ __forceinline__ uint32_t staged(int r, uint32_t b) { return r * 128 + (b ^ ((uint32_t)(r & 7) << 4)); }

// 64 lines of 64 values of an operand: line l is row r0 + l from column c0 on.  What lies outside the matrix is zero, lines from `lines` on
// are left out.  The warps of a group take every kGroupWarps-th line, a lane two values of it, or 16 bytes where rows allow that.  Loads are
// issued by `get` and used by `put`, another chunk's in between.
template <typename T> struct Chunk;

// bf16: 16 bytes of a line to a lane, out of the two aligned pieces in which they lie, whatever the rows' alignment.  (Two loads of one value
// each for two values: 38391 x 96 to 1580 backward 218 us, 194 so; 17467 x 605 to 3664 468 and 395.)
template <> struct Chunk<__nv_bfloat16> {
    static constexpr int kStep = kGroupWarps * 4, kTurns = kBlockC / kStep;
    static_assert(kGroupWarps == 8, "the pieces of a lane's lines are exchanged alike");
    uint4 a[kTurns], b[kTurns];
    uint32_t to, shifts;                // shifts: where the 16 bytes begin in a, a byte for each turn
    int rows, lines, count;             // below a lane's first line; values inside the matrix

    __device__ __forceinline__ void get(const Source<__nv_bfloat16>& s, uint32_t dst, int left_lines, long long r0, long long c0, int warp, int lane) {
        const int line = warp * 4 + lane / 8, col = lane % 8 * 8;
        count = (int)max(0LL, min(8LL, s.width - c0 - col));
        lines = left_lines - line;
        rows = count > 0 ? (int)min(s.rows - r0 - line, (long long)lines) : 0;
        to = dst + staged(line, col * 2);
        shifts = 0;
        const unsigned long long begin = reinterpret_cast<unsigned long long>(s.p), end = begin + 2 * ((s.rows - 1) * s.ld + s.width);
        unsigned long long p = begin + 2 * ((r0 + line) * s.ld + c0 + col);
#pragma unroll
        for (int u = 0; u < kTurns; ++u, p += 2 * kStep * s.ld) {
            const uint32_t shift = (uint32_t)p & 15;
            const unsigned long long q = p - shift;
            const bool one = u * kStep < rows, two = one && shift + 2 * count > 16, one_in = q >= begin && q + 16 <= end, two_in = q + 32 <= end;
            a[u] = ld_piece_if(one && one_in, q);
            b[u] = ld_piece_if(two && two_in, q + 16);
            if (one && !one_in) a[u] = ld_edge(q, begin, end);
            if (two && !two_in) b[u] = ld_edge(q + 16, begin, end);
            shifts |= shift << (8 * u);
        }
    }
    __device__ __forceinline__ void put(uint32_t) {
#pragma unroll
        for (int u = 0; u < kTurns; ++u) {
            if (u * kStep >= lines) break;
            const uint32_t shift = shifts >> (8 * u);
            uint32_t w[8] = {a[u].x, a[u].y, a[u].z, a[u].w, b[u].x, b[u].y, b[u].z, b[u].w};
#pragma unroll
            for (int i = 0; i < 6; ++i) w[i] = shift & 8 ? w[i + 2] : w[i];
#pragma unroll
            for (int i = 0; i < 5; ++i) w[i] = shift & 4 ? w[i + 1] : w[i];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                w[i] = __funnelshift_r(w[i], w[i + 1], (shift & 2) * 8);
                w[i] &= count >= 2 * i + 2 ? 0xffffffffu : count == 2 * i + 1 ? 0xffffu : 0u;
            }
            st_shared(to + u * kStep * 128, make_uint4(w[0], w[1], w[2], w[3]));
        }
    }
};

// fp32: a lane has two values of every eighth line, or 16 bytes where rows are whole aligned pieces, and splits them.
template <> struct Chunk<float> {
    static constexpr int V = 4, kLanes = 64 / V, kStep = kGroupWarps * (32 / kLanes), kTurns = kBlockC / kStep;   // of pieces
    static_assert(kGroupWarps == 8, "the pieces of a lane's lines are exchanged alike");
    uint32_t v[16];
    uint32_t to;
    int rows, lines;                    // below a lane's first line
    bool pieces, one, two;              // values: which of a lane's two lie inside

    // No load is conditional: one that has nothing to read reads the matrix' first value.
    __device__ __forceinline__ void get(const Source<float>& s, uint32_t dst, int left_lines, long long r0, long long c0, int warp, int lane) {
        pieces = s.pieces;
        const int line = pieces ? warp * (32 / kLanes) + lane / kLanes : warp, col = pieces ? lane % kLanes * V : 2 * lane;
        one = c0 + col < s.width;
        two = c0 + col + 1 < s.width;
        lines = left_lines - line;
        rows = (int)min(s.rows - r0 - line, (long long)lines);
        if (pieces && !one) rows = 0;
        to = dst + staged(line, col * 2);
        const float* p = s.p + (r0 + line) * s.ld + c0 + col;
        if (pieces) {
            const long long step = s.ld * kStep;
#pragma unroll
            for (int u = 0; u < kTurns; ++u, p += step) {
                const uint4 w = ld_piece(u * kStep < rows ? p : s.p);
                v[4 * u] = w.x; v[4 * u + 1] = w.y; v[4 * u + 2] = w.z; v[4 * u + 3] = w.w;
            }
        } else {
            const long long step = s.ld * kGroupWarps;
#pragma unroll
            for (int u = 0; u < 8; ++u, p += step) {
                const bool in = u * kGroupWarps < rows;
                v[2 * u] = ld_bits(in && one ? p : s.p);
                v[2 * u + 1] = ld_bits(in && two ? p + 1 : s.p);
            }
        }
    }
    __device__ __forceinline__ void put(uint32_t part_bytes) {
        if (pieces) {
#pragma unroll
            for (int u = 0; u < kTurns; ++u) {
                if (u * kStep >= lines) break;
                const uint4 w = u * kStep < rows ? make_uint4(v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]) : make_uint4(0, 0, 0, 0);
                const uint32_t at = to + u * kStep * 128;
                uint32_t h[2], m[2], l[2];
                split(__uint_as_float(w.x), __uint_as_float(w.y), h[0], m[0], l[0]);
                split(__uint_as_float(w.z), __uint_as_float(w.w), h[1], m[1], l[1]);
                st_shared(at, h[0], h[1]);
                st_shared(at + part_bytes, m[0], m[1]);
                st_shared(at + 2 * part_bytes, l[0], l[1]);
            }
        } else {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (u * kGroupWarps >= lines) break;
                const bool in = u * kGroupWarps < rows;
                const uint32_t a = in && one ? v[2 * u] : 0u, b = in && two ? v[2 * u + 1] : 0u, at = to + u * kGroupWarps * 128;
                uint32_t h, m, l;
                split(__uint_as_float(a), __uint_as_float(b), h, m, l);
                st_shared(at, h);
                st_shared(at + part_bytes, m);
                st_shared(at + 2 * part_bytes, l);
            }
        }
    }
};

// ---- epilogue ---------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ uint4 ld_shared(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
template <typename O> __device__ __forceinline__ uint4 pack16(const float* f);
template <> __device__ __forceinline__ uint4 pack16<float>(const float* f) { return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3])); }
template <> __device__ __forceinline__ uint4 pack16<__nv_bfloat16>(const float* f) { return make_uint4(pack(f[0], f[1]), pack(f[2], f[3]), pack(f[4], f[5]), pack(f[6], f[7])); }
template <typename T, Role ROLE> struct Result { using type = T; };
template <typename T> struct Result<T, kGradW> { using type = float; };

template <typename T> __device__ __forceinline__ void add_piece(float* f, uint4 v) {
    float g[Elem<T>::kVec];
    unpack16<T>(v, g);
#pragma unroll
    for (int e = 0; e < Elem<T>::kVec; ++e) f[e] += g[e];
}

__device__ __forceinline__ void st_value(uint32_t at, float v) { asm volatile("st.shared.b32 [%0], %1;" ::"r"(at), "f"(v) : "memory"); }
__device__ __forceinline__ void st_value(uint32_t at, __nv_bfloat16 v) { asm volatile("st.shared.b16 [%0], %1;" ::"r"(at), "h"(__bfloat16_as_ushort(v)) : "memory"); }
__device__ __forceinline__ float get_value(uint32_t at, float) {
    float v;
    asm volatile("ld.shared.b32 %0, [%1];" : "=f"(v) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ __nv_bfloat16 get_value(uint32_t at, __nv_bfloat16) {
    unsigned short v;
    asm volatile("ld.shared.b16 %0, [%1];" : "=h"(v) : "r"(at) : "memory");
    return __ushort_as_bfloat16(v);
}
// Where rows are not whole aligned 16-byte pieces: 32 staged rows, the first `rows` of them and `cols` values of each, from or to a matrix.
template <typename T> __device__ __forceinline__ void rows_in(uint32_t slot, const T* src, long long ld, int rows, int cols, int lane) {
    constexpr int per_lane = 128 / sizeof(T) / 32, kBatch = 16;
#pragma unroll 1
    for (int r = 0; r < rows; r += kBatch) {
        T v[kBatch][per_lane];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
#pragma unroll
            for (int q = 0; q < per_lane; ++q) v[u][q] = ld_value(src + (r + u < rows && lane + 32 * q < cols ? (r + u) * ld + lane + 32 * q : 0));
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
#pragma unroll
            for (int q = 0; q < per_lane; ++q) st_value(slot + staged(r + u, (lane + 32 * q) * sizeof(T)), v[u][q]);
    }
}
template <typename T> __device__ __forceinline__ void rows_out(uint32_t slot, T* dst, long long ld, int rows, int cols, int lane) {
    constexpr int per_lane = 128 / sizeof(T) / 32, kBatch = 8;
    dst += lane;
#pragma unroll 1
    for (int r = 0; r < rows; r += kBatch) {
        T v[kBatch][per_lane];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
#pragma unroll
            for (int q = 0; q < per_lane; ++q) v[u][q] = get_value(slot + staged(r + u, (lane + 32 * q) * sizeof(T)), T{});
#pragma unroll
        for (int u = 0; u < kBatch; ++u, dst += ld)
#pragma unroll
            for (int q = 0; q < per_lane; ++q)
                if (r + u < rows && lane + 32 * q < cols) dst[32 * q] = v[u][q];
    }
}

// Columns of this run, of its small parts, and of the runs before.
template <int PARTS, int N> __device__ __forceinline__ void sums(float (&f)[N], uint32_t d, uint32_t sum_at, bool begun) {
    float more[N];
    tmem_ld(d, f);
    tmem_wait_ld();
    if (PARTS == 3) {
        tmem_ld(d + kTmemBuffer / 2, more);
        tmem_wait_ld();
#pragma unroll
        for (int v = 0; v < N; ++v) f[v] += more[v];
    }
    if (begun) {
        tmem_ld(sum_at, more);
        tmem_wait_ld();
#pragma unroll
        for (int v = 0; v < N; ++v) f[v] += more[v];
    }
}
// A unit's columns of a run that is not its tile's last, onto the running sum.  Out of the way of the code that every tile runs.
template <int PARTS, int N, int COLUMNS> __device__ __noinline__ void add_run(uint32_t d, uint32_t sum_at, bool begun) {
#pragma unroll 1
    for (int c = 0; c < COLUMNS; c += N) {
        float f[N];
        sums<PARTS>(f, d + c, sum_at + c, begun);
        tmem_st(sum_at + c, f);
    }
    tmem_wait_st();
}

// ---- the kernel ---------------------------------------------------------------------------------------------------------------

// RUNS: the contraction is longer than a run (run_of).  Of its own: the code of the running sum, though it did not run,
// cost 427x240, 64 to 64 channels in fp32 six of 33 us.
// OUT: results leave and residuals come by TMA: rows of whole aligned 16-byte pieces.
template <typename T, Role ROLE, bool TMA, bool RUNS, bool OUT>
__global__ void __launch_bounds__(32 * all_warps<TMA>, 1)
product_umma(const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b, const __grid_constant__ CUtensorMap map_out,
             const __grid_constant__ CUtensorMap map_res, const __grid_constant__ CUtensorMap map_z, const __grid_constant__ Args<T> p)
{
    constexpr bool A_MN = ROLE == kGradW, B_MN = ROLE != kForward;
    constexpr int PARTS = parts_of<T>, EPI = epi_warps<TMA>, kIssue = 1, kFirstFill = kFirstEpi + EPI, run = run_of(ROLE, sizeof(T));
    static_assert(!TMA || PARTS == 1, "TMA brings bf16 as it is");
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t base = smem_u32(smem);
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const uint32_t b_part = (uint32_t)p.bn * 128, b_bytes = b_part * PARTS, stage_bytes = kABytes * PARTS + (p.resident ? 0 : b_bytes);
    const uint32_t resident = base + p.stages * stage_bytes;
    const uint32_t staging = resident + (p.resident ? (uint32_t)p.blocks * b_bytes : 0);
    const uint32_t strips = staging + EPI * kSlotBytes;    // of an epilogue warp: the bias of its columns
    const uint32_t full = strips + EPI * 256, empty = full + 8 * kMaxStages, acc_full = empty + 8 * kMaxStages, acc_empty = acc_full + 16,
                   b_full = acc_empty + 16, res_full = b_full + 8, finished = res_full + 8 * kMostEpi, slot = finished + 8;
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) { mbar_init(full + 8 * s, TMA ? 1 : kGroupWarps); mbar_init(empty + 8 * s, 1); }
        for (int s = 0; s < 2; ++s) { mbar_init(acc_full + 8 * s, 1); mbar_init(acc_empty + 8 * s, EPI); }
        mbar_init(b_full, TMA ? 1 : kFillWarps);
        mbar_init(finished, 1);
        for (int s = 0; s < EPI; ++s) mbar_init(res_full + 8 * s, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == kIssue) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    fence_before();
    __syncthreads();
    fence_after();
    // The product of the weights' gradient may start on SMs that this one leaves.  Not before this block has its tensor memory: the other
    // kernel keeps its own until this one has ended.
    if (ROLE == kGradX) pdl_launch_dependents();
    uint32_t tmem;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(tmem) : "r"(slot));
    tmem = __shfl_sync(0xffffffffu, tmem, 0);                      // known to be uniform, as an instruction's operands have to be

    const bool single = RUNS && PARTS == 3 && p.single;
    bool alive = true;
    int n = 0;                                                     // tiles so far
    if (TMA && warp == 0) {
        const uint32_t a_expect = stage_bytes - (A_MN ? 0 : (kBlockI - p.a_rows) * 128);
        // ---- the ring, by TMA -------------------------------------------------------------------------------------------------
        // by one lane: a block of c takes little more than its loads' issue
        if (lane == 0) {
            Ring r{};
            for (Walk u = walk(p); u.live && alive; next(u, p), ++n) {
                const int i0 = u.i * kBlockI, j0 = u.j * p.bn;
                if (p.resident && n == 0) {
                    mbar_expect(b_full, (unsigned)p.blocks * b_bytes);
                    for (int c = 0; c < p.blocks; ++c) {
                        if (B_MN) for (int m = 0; m < p.bn; m += 64) tma_load_2d(resident + c * b_bytes + m * 128, &map_b, b_full, j0 + m, c * kBlockC);
                        else tma_load_2d(resident + c * b_bytes, &map_b, b_full, c * kBlockC, j0);
                    }
                }
                for (int c = u.c0; c < u.c1; ++c, r.next(p.stages)) {
                    if (r.round > 0) alive = wait_lane(empty + 8 * r.s, (r.round - 1) & 1, 0x10000000u | r.round);
                    if (!alive) break;
                    const uint32_t at = base + r.s * stage_bytes, bar = full + 8 * r.s;
                    const int c0 = c * kBlockC;
                    mbar_expect(bar, a_expect);
                    if (A_MN) for (int m = 0; m < kBlockI; m += 64) tma_load_2d(at + m * 128, &map_a, bar, i0 + m, c0);
                    else tma_load_2d(at, &map_a, bar, c0, i0);
                    if (!p.resident) {
                        if (B_MN) for (int m = 0; m < p.bn; m += 64) tma_load_2d(at + kABytes + m * 128, &map_b, bar, j0 + m, c0);
                        else tma_load_2d(at + kABytes, &map_b, bar, c0, j0);
                    }
                }
            }
            if (p.resident) wait_lane(b_full, 0, 0x7B000000u);
            landed(full, p.stages, r);
        }
        __syncwarp();
    } else if (!TMA && warp >= kFirstFill) {
        // ---- the ring, by plain loads -------------------------------------------------------------------------------------------
        // A group walks its blocks' operands in chunks; a chunk's loads are under way while the one before is stored.
        const int group = (warp - kFirstFill) / kGroupWarps, w = (warp - kFirstFill) % kGroupWarps;
        static_assert(kFillWarps == 2 * kGroupWarps, "groups take turns");
        const bool ta = PARTS == 1 && p.a_tma, tb = PARTS == 1 && p.b_tma;
        const int a_chunks = ta ? 0 : kBlockI / kBlockC, b_chunks = tb ? 0 : (p.bn + kBlockC - 1) / kBlockC;
        // chunk q of the block c of tile u (of B alone: q from a_chunks on), to `at`
        auto get = [&](Chunk<T>& x, int q, const Walk& u, int c, uint32_t a_at, uint32_t b_at) {
            const bool of_b = q >= a_chunks, mn = of_b ? B_MN : A_MN;
            const int L = (of_b ? q - a_chunks : q) * kBlockC;
            const long long m0 = of_b ? (long long)u.j * p.bn : (long long)u.i * kBlockI, c0 = (long long)c * kBlockC;
            x.get(of_b ? p.b : p.a, (of_b ? b_at : a_at) + L * 128, of_b ? p.bn - L : kBlockI - L, mn ? c0 : m0 + L, mn ? m0 + L : c0, w, lane);
        };
        auto put = [&](Chunk<T>& x, int q) { x.put(q >= a_chunks ? b_part : (uint32_t)kABytes); };
        struct Place { Walk u; int c; Ring r; };                   // a block, and its place in the ring
        auto forth = [&](Place& k) {
            if (++k.c >= k.u.c1) { next(k.u, p); k.c = k.u.c0; }
            k.r.next(p.stages);
        };
        Place here{walk(p), 0, Ring{}};
        here.c = here.u.c0;
        if (p.resident) {
            if (tb && group == 1 && w == 0 && lane == 0) {
                mbar_bytes(b_full, (unsigned)p.blocks * b_bytes);
                for (int c = 0; c < p.blocks; ++c) {
                    if (B_MN) for (int m = 0; m < p.bn; m += 64) tma_load_2d(resident + c * b_bytes + m * 128, &map_b, b_full, here.u.j * p.bn + m, c * kBlockC);
                    else tma_load_2d(resident + c * b_bytes, &map_b, b_full, c * kBlockC, here.u.j * p.bn);
                }
            }
            for (int c = 1 - group; c < p.blocks; c += kFillWarps / kGroupWarps)   // of one block group 0 has none: it has the first tile
                for (int q = a_chunks; q < a_chunks + b_chunks; ++q) {
                    Chunk<T> x;
                    get(x, q, here.u, c, 0, resident + c * b_bytes);
                    put(x, q);
                }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(b_full);
        }
        const int chunks = a_chunks + (p.resident ? 0 : b_chunks);
        if (group == 1) forth(here);
        auto at_of = [&](const Place& k) { return base + k.r.s * stage_bytes; };
        Chunk<T> x;
        if (chunks > 0 && here.u.live) get(x, 0, here.u, here.c, at_of(here), at_of(here) + PARTS * kABytes);
        while (here.u.live) {
            Place after = here;
            forth(after);
            if (after.u.live) forth(after);
            if (here.r.round > 0) alive = wait_warp(empty + 8 * here.r.s, (here.r.round - 1) & 1, 0x20000000u | here.r.round);
            if (!alive) break;
            const uint32_t at = at_of(here), bar = full + 8 * here.r.s;
            if ((ta || (tb && !p.resident)) && w == 0 && lane == 0) {
                const int i0 = here.u.i * kBlockI, j0 = here.u.j * p.bn, c0 = here.c * kBlockC;
                mbar_bytes(bar, (ta ? (A_MN ? kABytes : p.a_rows * 128) : 0) + (tb && !p.resident ? b_bytes : 0));
                if (ta) {
                    if (A_MN) for (int m = 0; m < kBlockI; m += 64) tma_load_2d(at + m * 128, &map_a, bar, i0 + m, c0);
                    else tma_load_2d(at, &map_a, bar, c0, i0);
                }
                if (tb && !p.resident) {
                    if (B_MN) for (int m = 0; m < p.bn; m += 64) tma_load_2d(at + kABytes + m * 128, &map_b, bar, j0 + m, c0);
                    else tma_load_2d(at + kABytes, &map_b, bar, c0, j0);
                }
            }
#pragma unroll 1
            for (int q = 0; q < chunks; ++q) {                     // the next chunk, or the next block's first, is loaded meanwhile
                const bool more = q + 1 < chunks;
                const Place& k = more ? here : after;
                if constexpr (PARTS == 3) {
                    Chunk<T> y;
                    if (k.u.live) get(y, more ? q + 1 : 0, k.u, k.c, at_of(k), at_of(k) + PARTS * kABytes);
                    put(x, q);
                    x = y;
                } else {                                           // bf16 has no registers for two
                    put(x, q);
                    if (k.u.live) get(x, more ? q + 1 : 0, k.u, k.c, at_of(k), at_of(k) + PARTS * kABytes);
                }
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(bar);
            here = after;
        }
        if ((ta || tb) && w == 0 && lane == 0) {
            if (tb && p.resident) wait_lane(b_full, 0, 0x7B000000u);
            landed(full, p.stages, here.r);
        }
        __syncwarp();
    } else if (warp == kIssue) {
        // ---- issue --------------------------------------------------------------------------------------------------------------
        const uint32_t idesc = instr_desc<A_MN, B_MN>(p.bn);
        Ring r{};
        if (p.resident) alive = wait_warp(b_full, 0, 0x40000000u);
        for (Walk u = walk(p); u.live && alive; next(u, p))
            for (int c = u.c0; c < u.c1 && alive; ++n) {           // n: runs so far
                const int first = c, end = RUNS ? min(c + run, u.c1) : u.c1, buf = single ? 0 : n & 1, use = single ? n : n >> 1;
                if (use > 0) alive = wait_warp(acc_empty + 8 * buf, (unsigned)(use - 1) & 1, 0x30000000u | (unsigned)n);
                if (!alive) break;
                fence_after();
                const uint32_t d = tmem + buf * kTmemBuffer;
                for (; c < end; ++c, r.next(p.stages)) {
                    alive = wait_warp(full + 8 * r.s, r.round & 1, 0x50000000u | r.round);
                    if (!alive) break;
                    fence_after();
                    const uint32_t a_at = base + r.s * stage_bytes, b_at = p.resident ? resident + (uint32_t)c * b_bytes : a_at + PARTS * kABytes;
                    const unsigned long long da = smem_desc<A_MN>(a_at), db = smem_desc<B_MN>(b_at);
#pragma unroll
                    for (int t = 0; t < kBlockC / 16; ++t) {
                        const unsigned long long at = da + t * (step16<A_MN> >> 4), bt = db + t * (step16<B_MN> >> 4);
                        const bool add = c > first || t > 0;
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
                    commit(empty + 8 * r.s);
                }
                commit(acc_full + 8 * buf);
            }
        finish(finished);
    } else if (warp >= kFirstEpi && warp < kFirstFill) {
        // ---- write out ------------------------------------------------------------------------------------------------------
        // A unit: 128 bytes of 32 rows.  The warps of a quarter of the lanes take units in turn, over the tiles.
        using O = typename Result<T, ROLE>::type;
        constexpr int UC = 128 / sizeof(O), V = Elem<O>::kVec, TEAM = EPI / 4;
        const int e = warp - kFirstEpi, quarter = warp & 3, member = e / 4, per_tile = (p.bn + UC - 1) / UC;
        const uint32_t mine = staging + e * kSlotBytes, res_bar = res_full + e * 8;
        const uint32_t lane_at = lane * 128 + ((lane & 7) << 4), strip = strips + e * 256;   // a piece q of this lane's row: xor q << 4
        const bool has_z = ROLE == kForward && p.z, has_res = ROLE == kForward && p.residual, has_bias = ROLE == kForward && p.bias;
        unsigned units = 0;                                        // of this warp so far
        // the residual of this warp's next unit, from unit c of tile u on, into its slot; `turn` is whose c is
        auto fetch = [&](Walk u, int c, int turn) {
            for (; u.live; next(u, p), c = 0, turn = RUNS ? 0 : turn) {
                const int i0 = u.i * kBlockI + quarter * 32, j0 = u.j * p.bn, wide = min(p.J - j0, p.bn);
                for (; c < per_tile; ++c) {
                    const bool ours = turn == member && c * UC < wide && i0 < p.I;
                    turn = turn + 1 == TEAM ? 0 : turn + 1;
                    if (!ours) continue;
                    mbar_expect(res_bar, kSlotBytes);
                    tma_load_3d(mine, &map_res, res_bar, j0 + c * UC, i0, 0);
                    return;
                }
            }
        };
        Walk u = walk(p);
        if (OUT && has_res && !has_z && lane == 0) fetch(u, 0, 0);
        __syncwarp();
        int turn = 0;                                              // which member of the team has the next unit
        int done = 0;                                              // blocks of c of this tile that are summed; n: runs so far
        for (; u.live && alive; ++n) {
            const int buf = single ? 0 : n & 1;
            alive = wait_warp(acc_full + 8 * buf, (unsigned)(single ? n : n >> 1) & 1, 0x60000000u | (unsigned)n);
            if (!alive) break;
            fence_after();
            const bool begun = RUNS && done > 0, last = !RUNS || done + run >= u.c1 - u.c0;
            done = last ? 0 : done + run;
            const int i0 = u.i * kBlockI + quarter * 32, j0 = u.j * p.bn, wide = min(p.J - j0, p.bn), rows = (int)min(p.I - i0, 32LL);
            const uint32_t d = tmem + buf * kTmemBuffer + ((uint32_t)(quarter * 32) << 16);
            for (int c = 0; c < per_tile; ++c) {
                const bool ours = turn == member && c * UC < wide && rows > 0;
                turn = turn + 1 == TEAM ? 0 : turn + 1;
                if (!ours) continue;
                const uint32_t sum_at = tmem + ((uint32_t)(quarter * 32) << 16) + (single ? kTmemBuffer + c * UC : most_run_columns<T> + c * (PARTS == 3 ? kTmemBuffer / 2 : UC));
                if (RUNS && !last) {                              // the same warp has this unit in every run
                    add_run<PARTS, 2 * V, UC>(d + c * UC, sum_at, begun);
                    continue;
                }
                const int col = j0 + c * UC, cols = min(wide - c * UC, UC);
                if (has_bias)
#pragma unroll
                    for (int v = lane; v < UC; v += 32) st_value(strip + v * 4, v < cols ? Elem<T>::to_f32(ld_value(p.bias + col + v)) : 0.f);
                if (OUT && lane == 0) bulk_wait_read<0>();    // the slot has been read
                __syncwarp();
                // Loops that stay loops: a role's code has to stay in the instruction cache beside the others' (unrolled, waiting for
                // instructions was most of this kernel's time).  z leaves first, through the same slot.
#pragma unroll 1
                for (int pass = has_z ? 0 : 1; pass < 2; ++pass) {
                    if (pass == 1 && has_res) {
                        if constexpr (!OUT) {
                            if constexpr (ROLE == kForward) rows_in<T>(mine, p.residual + (long long)i0 * p.J + col, p.J, rows, cols, lane);
                            __syncwarp();
                        } else {
                            if (has_z && lane == 0) fetch(u, c, member);
                            alive = wait_warp(res_bar, units & 1, 0x80000000u | (unsigned)n);
                            if (!alive) break;
                        }
                    }
#pragma unroll 1
                    for (int q = 0; q * V < cols; q += 2) {
                        float f[2 * V];
                        sums<PARTS>(f, d + c * UC + q * V, sum_at + q * V, begun);
                        const uint32_t left = lane_at ^ (uint32_t)(q << 4), right = lane_at ^ (uint32_t)((q + 1) << 4);
                        if (has_bias)
#pragma unroll
                            for (int v = 0; v < 2 * V; v += 4) add_piece<float>(f + v, ld_shared(strip + (q * V + v) * 4));
                        if (ROLE == kForward && pass == 1) {
                            if (p.act == kActGelu)
#pragma unroll
                                for (int v = 0; v < 2 * V; ++v) f[v] = gelu<O>(f[v]);
                            else if (p.act == kActRelu)
#pragma unroll
                                for (int v = 0; v < 2 * V; ++v) f[v] = max_nan(f[v], 0.f);
                            if (has_res) {
                                add_piece<O>(f, ld_shared(mine + left));
                                add_piece<O>(f + V, ld_shared(mine + right));
                            }
                        }
                        st_shared(mine + left, pack16<O>(f));
                        st_shared(mine + right, pack16<O>(f + V));
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (pass == 0) {
                        if constexpr (OUT) {
                            if (lane == 0) { tma_store_3d(&map_z, mine, col, i0, 0); bulk_commit(); bulk_wait_read<0>(); }
                        } else {
                            if constexpr (ROLE == kForward) rows_out<T>(mine, p.z + (long long)i0 * p.J + col, p.J, rows, cols, lane);
                        }
                        __syncwarp();
                    }
                }
                if (!alive) break;
                ++units;
                if constexpr (OUT) {
                    if (lane == 0) {
                        tma_store_3d(&map_out, mine, col, i0, u.split); bulk_commit();
                        if (has_res && !has_z) {
                            bulk_wait_read<0>();
                            fetch(u, c + 1, turn);
                        }
                    }
                } else {
                    O* out;
                    if constexpr (ROLE == kGradW) out = p.part + u.split * p.I * p.J; else out = p.out;
                    rows_out<O>(mine, out + (long long)i0 * p.J + col, p.J, rows, cols, lane);
                }
                __syncwarp();
            }
            if (!alive) break;
            fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(acc_empty + 8 * buf);
            if (last) next(u, p);
            if (RUNS) turn = 0;                                    // a unit's running sum belongs to one warp, in every tile
        }
        if (OUT && has_res && !alive && lane == 0) wait_lane(res_bar, units & 1, 0x7E000000u);   // a residual on its way, as in `landed`
        if (lane == 0) bulk_wait_read<0>();                        // shared memory outlives what is read from it
        __syncwarp();
    }
    pdl_launch_dependents();
    if (ROLE != kForward) pdl_wait_primary();                      // it may have started beside the kernel before it: what comes next waits for both
    fence_before();
    __syncthreads();
    if (warp == kIssue) {
        fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    }
}

// One warp's wait for a barrier that nothing signals: gives up after its poll limit and records that.
__global__ void __launch_bounds__(32) wait_in_vain()
{
    __shared__ __align__(8) unsigned long long bar;
    if (threadIdx.x == 0) mbar_init(smem_u32(&bar), 1);
    __syncwarp();
    wait_warp(smem_u32(&bar), 0, 0xA0000000u);
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
