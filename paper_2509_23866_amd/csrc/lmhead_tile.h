// libdart internal: the bf16 MFMA tile that the LM-head kernels share, and what their
// epilogues have in common.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>
#include <utility>

#include "internal.h"
#include "dart.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));

// Waits until at most N loads of this wave are outstanding (vmcnt), leaving
// the LDS and export counters alone.
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
    static_assert(N >= 0 && N < 64, "vmcnt");
    __builtin_amdgcn_s_waitcnt((N & 0xF) | ((N >> 4) << 14) | (0x7 << 4) | (0xF << 8));
}

// A buffer resource over [base, base + bytes) (bytes capped at 2^32 - 1): raw
// loads past its end return zero. Dword 3 selects 32-bit data, untyped.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_rsrc(const void* base, int64_t bytes) {
    const uint32_t n = bytes > 0xFFFFFFFFll ? 0xFFFFFFFFu : (uint32_t)bytes;
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, (int)n, 0x00020000);
}

// Bytes from a matrix's row to the end of the last of `rows` rows of K bf16: the
// padding after that one need not belong to the caller's allocation (the last
// columns of a wider matrix), so a K slice that runs past K must not read it.
__host__ __device__ constexpr int64_t rows_bytes(int64_t rows, int64_t ld, int64_t K) {
    return ((rows - 1) * ld + K) * 2;
}
static_assert(rows_bytes(1, 80, 72) == 72 * 2 && rows_bytes(3, 80, 72) == (2 * 80 + 72) * 2,
              "the last row's padding is left out");

__device__ __forceinline__ __attribute__((address_space(3))) void* lds_ptr(void* p) {
    return (__attribute__((address_space(3))) void*)p;
}

// Workgroup barrier of the LDS ring: the caller has waited for its own loads
// into LDS (vmcnt); lgkmcnt(0) retires its LDS reads; the empty asm
// statements keep the compiler from moving memory accesses across it. Unlike
// __syncthreads it carries no fence, which would wait for every load in flight.
[[maybe_unused]] __device__ __forceinline__ void lds_ring_barrier() {
    __builtin_amdgcn_s_waitcnt(0xF | (0x3 << 14) | (0x7 << 4));  // lgkmcnt(0)
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Orders a wave's LDS accesses before it against those after it, across its lanes
// (which the convergent barrier brings together): the hardware runs them in the
// program's order, so nothing is waited for.
[[maybe_unused]] __device__ __forceinline__ void lds_wave_order() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_wave_barrier();
    asm volatile("" ::: "memory");
}

// Tile configuration: BM tokens x BN vocabulary entries per workgroup, K in
// slices of 64 through an NS-buffer LDS ring filled by direct global->LDS
// loads (no staging registers), WM x WN waves each owning a (BM/WM) x (BN/WN)
// block of 32 x 32 MFMA tiles.
// A K slice of BK bf16 per tile row is BK/8 chunks of 16 B. Chunk c of row r
// sits in LDS slot c ^ swz(r). gfx950's LDS serves 16-byte-per-lane reads 16
// lanes at a time across 64 four-byte banks (16 bank quads); a row of CH
// chunks covers CH quads, so 16 / CH consecutive rows tile the banks once and
// the swizzle shifts each such run of rows: the 16 rows that one read cycle
// takes (same chunk c) land in 16 distinct quads. With the plain c ^ (r % 8)
// of a 32-bank LDS, the bank-conflict counter showed half of all LDS cycles
// in two-way conflicts.
template <int CH>
__device__ __forceinline__ int swz(int r) { return (r / (16 / CH)) % CH; }

// Columns of a row that the statistics reduce together, in every configuration.
constexpr int kStatsUnit = 64;

template <int BM_, int BN_, int WM_, int WN_, int NS_, int BK_ = 64>
struct Cfg {
    static constexpr int BM = BM_, BN = BN_, BK = BK_, WM = WM_, WN = WN_, NS = NS_;
    static_assert(NS == 2 || NS == 3, "buffers of the K loop");
    static constexpr int CH = BK / 8;          // 16-byte chunks per row and slice
    static constexpr int LROWS = 64 / CH;      // rows one load instruction fills
    static constexpr int KSTEPS = BK / 16;     // MFMA k-steps per slice
    static constexpr int THREADS = 64 * WM * WN, WAVES = WM * WN;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;  // MFMA tiles per wave
    // a wave's TM row blocks of 32 sit RS = WM * 32 rows apart, so that each
    // epilogue pass over EPI = RS rows takes one block from every wave
    static constexpr int RS = BM / TM;
    static constexpr int IA = BM / LROWS / WAVES, IB = BN / LROWS / WAVES;  // loads per slice
    // LDS rows of a result tile: 16 bytes beyond BN elements, so that
    // consecutive rows start one bank quad apart and the rows that the lanes of
    // one write cycle hold fall in distinct banks. A bf16 tile goes through LDS
    // whole, an fp32 one EPI rows at a time: one 32-row block of every wave
    static constexpr int CROW = BN + 4, CROW16 = BN + 8;
    static constexpr int EPI = RS;
    static_assert(BK == 32 || BK == 64, "slice depth");
    static_assert(BM % (32 * WM) == 0 && BN % (32 * WN) == 0, "tile shape");
    static_assert(IA * LROWS * WAVES == BM && IB * LROWS * WAVES == BN, "rows per wave");
    static_assert(THREADS % EPI == 0 || EPI % THREADS == 0, "epilogue rows");
    struct alignas(16) Smem {
        union {
            struct {
                // slice buffers: BK bf16 per row, chunk c of row r in slot c ^ swz(r)
                uint16_t a[NS][BM][BK];
                uint16_t b[NS][BN][BK];
            } in;
            float c[EPI][CROW];
            uint16_t c16[BM][CROW16];
            float4 red[BN / kStatsUnit][BM];  // per-row partial triples of the statistics
        };
    };
};
// Measured on MI355X at T = 4096, d = 3584, V = 152064 among 128/256-square
// tiles, 4 or 8 waves, 2-4 buffers, 32- or 64-wide slices and register-staged
// loads: 256 x 256 with 8 waves as 4 x 2 (64 x 128 per wave) and two 64-wide
// buffers is the fastest.
using LmCfg = Cfg<256, 256, 4, 2, 2>;
// Tiles of fewer rows, for few rows in all: a third buffer fits the LDS, so that
// two slices are in flight where W comes from HBM and little is multiplied per
// byte of it. Measured (d = 3584, V = 152064; statistics and dlogits, us): 64
// rows 213 and 204 with the 64-row tile (243 and 241 with two buffers), 279 and
// 270 with the 256-row one; 128 rows 231 and 220 with the 128-row tile (274 and
// 267 with two buffers), 285 and 281.
using LmCfg128 = Cfg<128, 256, 2, 4, 3>;
using LmCfg64 = Cfg<64, 256, 2, 4, 3>;
static_assert(sizeof(LmCfg::Smem) <= 160 * 1024 && sizeof(LmCfg128::Smem) <= 160 * 1024 &&
                  sizeof(LmCfg64::Smem) <= 160 * 1024,
              "LDS per workgroup");
constexpr int kMergeWaves = 4;
constexpr int kMergeBatch = 5;

struct Triple {
    float m, s, w;  // reference, sum of e^{z-m}, sum of e^{z-m} (z-m), natural units
};

// float -> bf16 bits, round to nearest even, a NaN kept quiet with its
// payload: the __bf16 conversion, which is gfx950's v_cvt_pk_bf16_f32 (two
// values per instruction; the same bits as the integer rounding
// u + 0x7FFF + ((u >> 16) & 1) for every one of the 2^32 fp32 inputs, checked
// on the GPU)
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint16_t bf16_bits(float f) {
    return __builtin_bit_cast(uint16_t, (__bf16)f);
}

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    const bf16x2_t v = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, v);
}

// Exact merge of two partial triples; an empty triple has s == 0. Contracted by
// hand alone, so that every kernel it is inlined into rounds the same.
__device__ __forceinline__ Triple merge(const Triple& a, const Triple& b) {
#pragma clang fp contract(off)
    if (b.s == 0.f) return a;
    if (a.s == 0.f) return b;
    const float m = fmaxf(a.m, b.m);
    const float ca = expf(a.m - m), cb = expf(b.m - m);
    Triple r;
    r.m = m;
    r.s = fmaf(ca, a.s, cb * b.s);
    r.w = fmaf(ca, fmaf(a.m - m, a.s, a.w), cb * fmaf(b.m - m, b.s, b.w));
    return r;
}

// acc = this wave's part of the tile A[m0:m0+BM, :] B[n0:n0+BN, :]^T (A [M, K]
// and B [N, K] row-major bf16, rows 16-byte aligned, K % 8 == 0). Rows past M
// or N read as zero (their results are not used); K past the end is zeroed in
// LDS. Layout of acc[i][j]: value v of lane l is
// tile row (wave / WN) * 32 + i * RS + l%32, column
// (wave % WN) * BN/WN + j*32 + (v/4)*8 + (l/32)*4 + v%4: the MFMA takes B's rows
// as its first operand, so that a lane holds 16 TN columns of one row, four
// adjacent ones in consecutive registers. (With A's rows first a lane holds
// one column of 16 rows, and every epilogue had to turn the fp32 tile round in
// LDS, one value at a time. Measured at d = 3584, V = 152064, the same card:
// statistics 3450 -> 3378 us at T = 4096 and 950 -> 925 at 1000, the backward
// with bf16 gradients 10702 -> 10565 and 2953 -> 2856, dlogits 928 -> 917 at
// 1000, the fp32 gradients within 0.3%.) Ends on a barrier with no loads in
// flight, so the caller may reuse the LDS.
template <class C>
__device__ __forceinline__ void gemm_tile(const uint16_t* __restrict__ A, int64_t M, int64_t lda,
                                          const uint16_t* __restrict__ B, int64_t N, int64_t ldb,
                                          int64_t K, int64_t m0, int64_t n0,
                                          typename C::Smem& sm,
                                          f32x16 (&acc)[C::TM][C::TN]) {
#if defined(__HIP_DEVICE_COMPILE__)  // the gfx950 builtins below have no host form
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);  // uniform: addresses in SGPRs
    const int wr = (wave / C::WN) * 32, wc = (wave % C::WN) * (C::BN / C::WN);
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int j = 0; j < C::TN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

    // One load instruction fills LROWS rows x CH slots (1 KB): lane l writes
    // slot l % CH of row r0 + l / CH, i.e. chunk (l % CH) ^ swz(row) of that
    // row. The loads are buffer loads into LDS: each operand's tile rows are a
    // buffer resource whose range ends at the matrix's last element, so rows
    // past M or N read as zero (their results are not used). A lane's byte
    // offset within its instruction's rows is the same for every instruction
    // and slice (the swizzle repeats every 16 rows, and the rows of one
    // instruction of every wave together are a multiple of that), so one VGPR
    // serves all of an operand's loads; the instruction's rows and the slice
    // enter as a scalar offset.
    constexpr int CH = C::CH, BK = C::BK;
    const int lrow = lane / CH, lslot = lane % CH;
    static_assert((C::WAVES * C::LROWS) % (16 / CH * CH) == 0, "swizzle period");
    const int r_lane = wave * C::LROWS + lrow;  // row of the lane in instruction 0
    const uint32_t voff_a = (uint32_t)((r_lane * lda + (lslot ^ swz<CH>(r_lane)) * 8) * 2);
    const uint32_t voff_b = (uint32_t)((r_lane * ldb + (lslot ^ swz<CH>(r_lane)) * 8) * 2);
    const uint32_t qstride_a = (uint32_t)(C::WAVES * C::LROWS * lda * 2);
    const uint32_t qstride_b = (uint32_t)(C::WAVES * C::LROWS * ldb * 2);
    const __amdgpu_buffer_rsrc_t rsrc_a = tile_rsrc(A + m0 * lda, rows_bytes(M - m0, lda, K));
    const __amdgpu_buffer_rsrc_t rsrc_b = tile_rsrc(B + n0 * ldb, rows_bytes(N - n0, ldb, K));
    // rows of instruction q of wave `wave + hh * HW`
    auto lds_a = [&](int buf, int q, int hh) {
        return &sm.in.a[buf][(q * C::WAVES + wave + hh * (C::WAVES / 2)) * C::LROWS][0];
    };
    auto lds_b = [&](int buf, int q, int hh) {
        return &sm.in.b[buf][(q * C::WAVES + wave + hh * (C::WAVES / 2)) * C::LROWS][0];
    };
    const int64_t nk = (K + BK - 1) / BK;
    // slice kt into buffer buf; a slice that ends past K reads chunks past K
    // (in the row padding, the next row or, at the end, as zero) that are
    // zeroed after landing
    // The first half of the waves (one per SIMD) issue every load of a
    // slice: their own rows and those of the wave HW above, with the same lane
    // offsets (the rows between them are a whole number of swizzle periods).
    // Issuing a slice's 64 loads holds each issuing wave for ~700 cycles; the
    // other wave of its SIMD multiplies meanwhile.
    constexpr int HW = C::WAVES / 2;
    static_assert((HW * C::LROWS) % 16 == 0, "swizzle period");
    const uint32_t hstride_a = (uint32_t)(HW * C::LROWS * lda * 2);
    const uint32_t hstride_b = (uint32_t)(HW * C::LROWS * ldb * 2);
    auto issue = [&](int64_t kt, int buf) {
        if (wave >= HW) return;
        const uint32_t kb = (uint32_t)(kt * BK * 2);
#pragma unroll
        for (int q = 0; q < C::IA; ++q)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_a, lds_ptr(lds_a(buf, q, hh)), 16,
                                                        voff_a, kb + q * qstride_a + hh * hstride_a,
                                                        0, 0);
#pragma unroll
        for (int q = 0; q < C::IB; ++q)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_b, lds_ptr(lds_b(buf, q, hh)), 16,
                                                        voff_b, kb + q * qstride_b + hh * hstride_b,
                                                        0, 0);
    };
    // a partial last slice: zero the chunks past K
    auto zero_tail = [&](int64_t kt, int buf) {
        const u32x4 z = {0u, 0u, 0u, 0u};
        for (int e = tid; e < (C::BM + C::BN) * CH; e += C::THREADS) {
            const int r = e / CH, c = e % CH;
            if (kt * BK + c * 8 < K) continue;
            if (r < C::BM)
                *reinterpret_cast<u32x4*>(&sm.in.a[buf][r][(c ^ swz<CH>(r)) * 8]) = z;
            else
                *reinterpret_cast<u32x4*>(
                    &sm.in.b[buf][r - C::BM][(c ^ swz<CH>(r - C::BM)) * 8]) = z;
        }
    };

    // MFMA operands: lane l reads row (l % 32) of each 32-row block, chunk
    // 2 ks + l / 32. The rows' swizzle depends only on l % 32 (blocks start at
    // multiples of 32), so one byte offset per k-step serves every block, the
    // block and the buffer entering as immediate offsets.
    // The B offsets include the B buffers' start (64 KB into the LDS) and are
    // kept opaque to the compiler, so that the buffer and the 32-column block
    // enter as the read's 16-bit immediate (below 64 KB); folded into the
    // immediate, they did not fit, and every B read cost an address add.
    uint32_t rda[C::KSTEPS], rdb[C::KSTEPS];
    const char* const lds0 = reinterpret_cast<const char*>(&sm);
    const uint32_t b_at = (uint32_t)(reinterpret_cast<const char*>(&sm.in.b[0][0][0]) - lds0);
#pragma unroll
    for (int ks = 0; ks < C::KSTEPS; ++ks) {
        const int c = ks * 2 + (lane >> 5), ra = wr + (lane & 31), rb = wc + (lane & 31);
        rda[ks] = (uint32_t)(ra * BK + (c ^ swz<CH>(ra)) * 8) * 2;
        rdb[ks] = b_at + (uint32_t)(rb * BK + (c ^ swz<CH>(rb)) * 8) * 2;
        asm volatile("" : "+v"(rdb[ks]));
    }
    bf16x8 af[2][C::TM], bfr[2][C::TN];
    auto read_step = [&](auto bufc, int ks, int set) {
        constexpr int buf = decltype(bufc)::value;
        const char* ba = reinterpret_cast<const char*>(&sm.in.a[buf][0][0]);
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
            af[set][i] = __builtin_bit_cast(
                bf16x8, *reinterpret_cast<const u32x4*>(ba + rda[ks] + i * C::RS * BK * 2));
#pragma unroll
        for (int j = 0; j < C::TN; ++j)
            bfr[set][j] = __builtin_bit_cast(
                bf16x8, *reinterpret_cast<const u32x4*>(lds0 + rdb[ks] + buf * C::BN * BK * 2 +
                                                        j * 32 * BK * 2));
    };
    // the MFMAs of row blocks [i0, i1) of k-step ks
    auto mfmas = [&](int ks, int i0 = 0, int i1 = C::TM) {
        const int set = ks & 1;
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j)
                if (i >= i0 && i < i1)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bfr[set][j], af[set][i],
                                                                        acc[i][j], 0, 0, 0);
    };
    // Every wave holds back the last k-step's MFMAs of its last row block
    // and issues them after the next slice's barrier (and its loads), while
    // the first operand reads of that slice are in flight.
    constexpr int LAST = C::KSTEPS - 1;

    // NS LDS buffers: slices kt+1 .. kt+NS-1 load while slice kt is multiplied
    constexpr int LOADS = 2 * (C::IA + C::IB);  // of an issuing wave and slice
    auto slice = [&](auto bufc, int64_t kt) {
        constexpr int buf = decltype(bufc)::value;
        // slice kt has landed for this wave; the barrier makes it so for all,
        // and every wave has finished reading the buffer of slice kt-1
        if (C::NS == 2 || kt + C::NS - 2 >= nk)
            wait_vmcnt<0>();
        else
            wait_vmcnt<(C::NS - 2) * LOADS>();
        lds_ring_barrier();
        if ((K % BK) && kt == nk - 1) {
            zero_tail(kt, buf);
            lds_ring_barrier();
        }
        if (kt + C::NS - 1 < nk) issue(kt + C::NS - 1, (buf + C::NS - 1) % C::NS);
        // the operands of k-step ks+1 are read while the MFMAs of k-step ks issue
        read_step(bufc, 0, 0);
        __builtin_amdgcn_s_setprio(1);
        if (kt > 0) mfmas(LAST, C::TM - 1, C::TM);
#pragma unroll
        for (int ks = 0; ks < C::KSTEPS; ++ks) {
            const int cs = ks & 1;
            if (ks < C::KSTEPS - 1) read_step(bufc, ks + 1, cs ^ 1);
            mfmas(ks, 0, ks == C::KSTEPS - 1 ? C::TM - 1 : C::TM);
            if (ks < C::KSTEPS - 1) {
                // interleave: one LDS read, then a share of the MFMAs
#pragma unroll
                for (int g = 0; g < C::TM + C::TN; ++g) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x008, (C::TM * C::TN) / (C::TM + C::TN), 0);
                }
            }
        }
        __builtin_amdgcn_s_setprio(0);
    };
    // the loop body has no condition on the accumulators: the last slices that
    // do not fill a round of the buffers run after it (a conditional second
    // slice in the body made the compiler copy every accumulator at the join)
#pragma unroll
    for (int b = 0; b < C::NS - 1; ++b)
        if (b == 0 || b < nk) issue(b, b);
    int64_t kt = 0;
    for (; kt + C::NS - 1 < nk; kt += C::NS) {
        slice(std::integral_constant<int, 0>{}, kt);
        slice(std::integral_constant<int, 1>{}, kt + 1);
        if constexpr (C::NS > 2) slice(std::integral_constant<int, 2 % C::NS>{}, kt + 2);
    }
    if (kt < nk) slice(std::integral_constant<int, 0>{}, kt);
    if (C::NS > 2 && kt + 1 < nk) slice(std::integral_constant<int, 1>{}, kt + 1);
    mfmas(LAST, C::TM - 1, C::TM);
    __syncthreads();
#else
    (void)A, (void)M, (void)lda, (void)B, (void)N, (void)ldb, (void)K, (void)m0, (void)n0;
    (void)sm, (void)acc;
#endif
}

// NJ 32-column blocks (acc[0] is block j0) of the wave's row block i in the
// workgroup's result tile in LDS, rounded to bf16: four adjacent columns of a row
// leave a lane as one 8-byte write.
template <class C, int NJ>
__device__ __forceinline__ void blocks_to_lds_bf16(const f32x16* acc, int i, int j0,
                                                   typename C::Smem& sm) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wr = (wave / C::WN) * 32 + (lane & 31), wc = (wave % C::WN) * (C::BN / C::WN);
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int v = 0; v < 16; v += 4) {
            u32x2 pk;
            pk.x = pack_bf16x2(acc[j][v], acc[j][v + 1]);
            pk.y = pack_bf16x2(acc[j][v + 2], acc[j][v + 3]);
            *reinterpret_cast<u32x2*>(
                &sm.c16[wr + i * C::RS][wc + (j0 + j) * 32 + (v >> 2) * 8 + (lane >> 5) * 4]) = pk;
        }
}

// Logical tile of workgroup b: the hardware places workgroup b on XCD b % 8,
// so each XCD gets a contiguous run of logical tiles. Logical tiles come in
// groups of G token tiles x every vocabulary tile, token tile fastest within
// a group, so the ~32 tiles an XCD runs at once share G tiles of h and a few
// slices of W in its L2. (Token tile fastest over all of them made each XCD
// read a different h tile per workgroup: at T = 152569 that re-read the 1.09
// GB of h from HBM once per vocabulary slice, 15% slower than groups of 4.)
constexpr int64_t kTileGroup = 4;  // token tiles per group
__device__ __forceinline__ void tile_of_block(int64_t nmt, int64_t nvt, int64_t& mt, int64_t& vt) {
    const int64_t nb = nmt * nvt, q = nb / 8, rr = nb % 8;
    const int64_t b = blockIdx.x, x = b % 8, sl = b / 8;
    const int64_t lg = x * q + min(x, rr) + sl;
    constexpr int64_t G = kTileGroup;
    const int64_t g = lg / (G * nvt), first = g * G;
    const int64_t gm = nmt - first < G ? nmt - first : G;
    const int64_t in = lg - first * nvt;
    mt = first + in % gm;
    vt = in / gm;
}

// The configuration of a last row tile of at most 128 rows where the others have
// 256: the 128-row one, in the place the order gives it, among the tiles that read
// the same slice of W. Only with 3 or 4 row tiles, one group of the order: with 2
// it saves nothing, beyond 4 the last group's tiles are one XCD's, and the gain
// is lost waiting for the others. Measured at d = 3584, V = 152064 (statistics,
// us): 800 rows 945 -> 832, 600 rows 639 -> 616; put after all others, where they
// read W from HBM once more, 600 rows 655.
__host__ __device__ constexpr bool has_rest(int64_t nmt) { return nmt == 3 || nmt == 4; }
template <class C>
struct Rest {
    using type = typename std::conditional<C::BM == LmCfg::BM, LmCfg128, C>::type;
};
// f(configuration, LDS, first row, vocabulary tile) for this workgroup's tile of M
// rows x nvt vocabulary tiles, if it has one.
template <class C, class F>
__device__ __forceinline__ void with_row_tile(int64_t M, int64_t nvt, F&& f) {
    using R = typename Rest<C>::type;
    __shared__ union {
        typename C::Smem full;
        typename R::Smem rest;
    } sm;
    const int64_t nmt = (M + C::BM - 1) / C::BM;
    if ((int64_t)blockIdx.x >= nmt * nvt) return;
    int64_t mt, vt;
    tile_of_block(nmt, nvt, mt, vt);
    const int64_t m0 = mt * C::BM;
    if constexpr (R::BM < C::BM) {
        if (has_rest(nmt) && M - m0 <= R::BM) {
            f(R{}, sm.rest, m0, vt);
            return;
        }
    }
    f(C{}, sm.full, m0, vt);
}

// The statistics of tile (m0, vt) of logits whose values (not scaled) tile(n0, acc)
// leaves in acc: part[t * nvt + vt] receives the triple of row t over the tile's columns
// other than target[t]; the workgroup holding target[t] writes z_y[t].
template <class C, class F>
__device__ __forceinline__ void stats_of_tile(F&& tile, int64_t T, int64_t V,
                                              const int32_t* __restrict__ target, float scale,
                                              int64_t nvt, float4* __restrict__ part,
                                              float* __restrict__ z_y, typename C::Smem& sm,
                                              int64_t m0, int64_t vt) {
#pragma clang fp contract(off)  // the same roundings in every configuration
    const int64_t n0 = vt * C::BN;
    f32x16 acc[C::TM][C::TN];
    tile(n0, acc);

    // The row's 256 columns are reduced in units of 64, in whatever configuration:
    // a lane's 32 columns of a unit (two 32-column blocks of its half-wave): their
    // maximum, then the sums in base-2 units against it, one partial sum per
    // block; merged with the lane that holds the unit's other columns; the four
    // units merged in column order through LDS. So a row's triple does not depend
    // on the tile height its call takes, or on the tile the row falls in: equal
    // rows have equal statistics, and a step recomputed in another batch the same.
    // (Reducing all of a wave's columns of a row at once, 64 or 128 by the
    // configuration, is 0.3 to 0.7% faster: 3373 against 3384 us at T = 4096, 913
    // against 922 at 1000, d = 3584, V = 152064.) The whole epilogue stays in
    // registers until the last merge.
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const int wr = (wave / C::WN) * 32 + (lane & 31), wc = (wave % C::WN) * (C::BN / C::WN);
    // the inverse temperature enters the base-2 exponent's factor (1 at scale
    // 1: the same bits)
    const float c2 = scale * 1.4426950408889634f;
    static_assert(C::TN % 2 == 0, "units of two 32-column blocks");
#pragma unroll
    for (int i = 0; i < C::TM; ++i) {
        const int64_t t = m0 + wr + i * C::RS;
        const int64_t y = t < T ? (int64_t)target[t] : -1;
#pragma unroll
        for (int u = 0; u < C::TN / 2; ++u) {
            const int64_t u0 = n0 + wc + u * kStatsUnit;
            // columns below vlim (counted from the unit's first) exist
            const int vlim = (int)max(min(V - u0, (int64_t)kStatsUnit), (int64_t)0);
            // the target's column within the unit's (-1: not here)
            const int64_t yrel = y - u0;
            const int y64 = yrel >= 0 && yrel < vlim ? (int)yrel : -1;
            // only the tile's last columns past V and a row's target column drop
            // out: the selects run only in lanes that hold such a column
            const bool masked = vlim < kStatsUnit || (y64 >= 0 && ((y64 >> 2) & 1) == half);
            if (masked) {
                float zy = 0.f;
                // opaque, so that the compiler does not take the comparisons of
                // every row block's columns together, and spill their masks
                int vl = vlim - half * 4, yl = y64 - half * 4;
                asm volatile("" : "+v"(vl), "+v"(yl));
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int col = j * 32 + (v >> 2) * 8 + (v & 3);
                        const float x = acc[i][2 * u + j][v];
                        const bool at_y = col == yl;
                        zy = at_y ? x : zy;
                        acc[i][2 * u + j][v] = col >= vl || at_y ? -INFINITY : x;
                    }
                if (y64 >= 0 && ((y64 >> 2) & 1) == half) z_y[t] = zy * scale;
            }
            float mx = -INFINITY;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) mx = fmaxf(mx, acc[i][2 * u + j][v]);
            // scale > 0: the maximum of the scaled row is the scaled maximum
            Triple mine = {mx * scale, 0.f, 0.f};
            // e = 2^xl with xl = (x - mx) scale log2(e); where a column was
            // dropped (-inf) xl is floored at -200, where 2^xl is already 0 in
            // fp32, so that it adds 0. A maximum of -inf says that every column
            // was dropped or is a NaN (which a maximum passes over): the sums run
            // all the same, from 0, and a NaN shows in them
            const float ml = mx == -INFINITY ? 0.f : mx * c2;
            float s2[2], w2[2];
            auto sums = [&](auto floored) {
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    s2[j] = w2[j] = 0.f;
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        float xl = fmaf(acc[i][2 * u + j][v], c2, -ml);
                        if constexpr (decltype(floored)::value) xl = xl < -200.f ? -200.f : xl;
                        const float e = __builtin_amdgcn_exp2f(xl);
                        s2[j] += e;
                        w2[j] = fmaf(e, xl, w2[j]);
                    }
                }
            };
            if (masked)
                sums(std::true_type{});
            else
                sums(std::false_type{});
            mine.s = s2[0] + s2[1];
            mine.w = (w2[0] + w2[1]) * 0.6931471805599453f;
            Triple o;
            o.m = __shfl_xor(mine.m, 32);
            o.s = __shfl_xor(mine.s, 32);
            o.w = __shfl_xor(mine.w, 32);
            mine = half ? merge(o, mine) : merge(mine, o);
            if (half == 0)
                sm.red[wc / kStatsUnit + u][wr + i * C::RS] =
                    make_float4(mine.m, mine.s, mine.w, 0.f);
        }
    }
    lds_ring_barrier();
    for (int r = tid; r < C::BM && m0 + r < T; r += C::THREADS) {
        Triple x = {-INFINITY, 0.f, 0.f};
#pragma unroll
        for (int k = 0; k < C::BN / kStatsUnit; ++k) {
            const float4 q = sm.red[k][r];
            x = merge(x, Triple{q.x, q.y, q.z});
        }
        part[(m0 + r) * nvt + vt] = make_float4(x.m, x.s, x.w, 0.f);
    }
}

// One wave per row: the row's nvt triples merged lane-strided in index order,
// then across lanes by a butterfly; the target logit is added last, as in
// tok_stats_kernel: lse = M + log S, H = log S - W / S, and logp from
// -log1p(s_rest / e_y) when the target dominates.
[[maybe_unused]] __global__ void __launch_bounds__(kMergeWaves * 64)
lmhead_merge_kernel(const float4* __restrict__ part, const float* __restrict__ z_y, int64_t T,
                    int64_t nvt, int64_t V, const int32_t* __restrict__ target,
                    float* __restrict__ logp, float* __restrict__ entropy,
                    float* __restrict__ lse) {
    const int lane = threadIdx.x & 63;
    const int64_t t = (int64_t)blockIdx.x * kMergeWaves + (threadIdx.x >> 6);
    if (t >= T) return;
    Triple acc = {-INFINITY, 0.f, 0.f};
    // a lane's next kMergeBatch triples are loaded together (an empty triple
    // past the last): one after the other, their latency was the kernel's time
    for (int64_t j0 = lane; j0 < nvt; j0 += 64 * kMergeBatch) {
        float4 p[kMergeBatch];
#pragma unroll
        for (int k = 0; k < kMergeBatch; ++k) {
            const int64_t j = j0 + 64 * k;
            p[k] = j < nvt ? part[t * nvt + j] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int k = 0; k < kMergeBatch; ++k) acc = merge(acc, Triple{p[k].x, p[k].y, p[k].z});
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        Triple o;
        o.m = __shfl_xor(acc.m, off);
        o.s = __shfl_xor(acc.s, off);
        o.w = __shfl_xor(acc.w, off);
        acc = merge(acc, o);
    }
    if (lane != 0) return;
    const int64_t y = target[t];
    const float zy = (y >= 0 && y < V) ? z_y[t] : __builtin_nanf("");
    const bool others = acc.s != 0.f;  // also where it is a NaN
    const float M = others ? fmaxf(acc.m, zy) : zy;
    float sx = 0.f, wx = 0.f;
    if (others) {
        const float dx = acc.m - M;
        const float cx = expf(dx);
        sx = cx * acc.s;
        wx = cx * fmaf(dx, acc.s, acc.w);
    }
    const float xy = zy - M;
    const float ey = expf(xy);
    const float S = sx + ey;
    const float W = fmaf(ey, xy, wx);
    const float ln_s = logf(S);
    const float h = ln_s - W / S;
    lse[t] = M + ln_s;
    entropy[t] = h < 0.f ? 0.f : h;
    logp[t] = sx < ey ? -log1pf(sx / ey) : xy - ln_s;
}

inline int64_t vocab_tiles(int64_t V) { return (V + LmCfg::BN - 1) / LmCfg::BN; }

// The MFMA tile addresses its rows by 32-bit byte offsets from the tile's first
// row: (BM - 1) rows of ld elements must stay below 2^31 bytes.
constexpr int64_t kMaxLd = int64_t(1) << 22;

// Rows of the tile that forms rows x V logits fastest: 64, 128 or 256. One
// workgroup runs per compute unit, so a launch takes its tiles in rounds of
// kUnits, and a round of 256-, 128- or 64-row tiles takes 92, 54 or 45 us at
// d = 3584 (T = 1000, 1000 and 256): the tile with the least rounds x time. So
// 64 rows go as one 64-row tile, up to 128 and 129 - 256 as 128-row tiles at
// V = 152064, more as 256-row ones (the last one of up to 128 rows as in Rest),
// unless those would leave units idle (1000 rows of V = 8000).
// The times' ratios at d = 3584 serve every depth: of 99 sizes (d = 512, 1024 and 2048;
// V = 8000, 32000 and 152064; T from 16 to 2100) the choice is within 5% of the fastest
// of the three but for 600 rows of V = 32000 (58.1 against 54.4 us at d = 1024, 96.6
// against 88.3 at 2048, by the last tile's rule), and none takes longer than with
// 256-row tiles alone (statistics).
// A round of 128-row tiles of dlogits is worth 57 us up to d = 1024, where the two
// heights come within 5% of each other (129 to 256 rows of V = 152064): the taller tile
// reads W once and has fewer first slices to wait for. 130 rows 50.0 us in 128-row
// tiles and 45.8 in 256-row ones at d = 512, 87.0 and 83.0 at 1024; 170 and 181 at 2048.
constexpr int64_t kUnits = 256;
inline int tile_rows(int64_t rows, int64_t V, double t128 = 54) {
    const double nvt = (double)((V + LmCfg::BN - 1) / LmCfg::BN), t256 = 92, t64 = 45;
    auto rounds = [](double tiles) { return ceil(tiles / kUnits); };
    const int64_t nmt = (rows + 255) / 256, r = rows % 256;
    double least = rounds((double)nmt * nvt) * t256;
    // short tiles among the long ones take 71 us, and half a tile's wait at the end
    if (has_rest(nmt) && r > 0 && r <= 128)
        least = fmin(least, fmax(((double)(nmt - 1) * t256 + 71) * nvt / kUnits + 27, t256));
    int best = 256;
    const double c128 = rounds((double)((rows + 127) / 128) * nvt) * t128;
    const double c64 = rounds((double)((rows + 63) / 64) * nvt) * t64;
    if (c128 < least) best = 128, least = c128;
    if (c64 < least) best = 64;
    return best;
}

// f(configuration of bm-row tiles) for rows x V logits. The launch's limits are checked
// with 256-row tiles, as ever; smaller ones are taken where they fit too.
template <class F>
void with_tile(int bm, int64_t rows, int64_t V, F&& f) {
    if (!grid_fits((rows + bm - 1) / bm * vocab_tiles(V), LmCfg::THREADS)) bm = 256;
    if (bm == 64)
        f(LmCfg64{});
    else if (bm == 128)
        f(LmCfg128{});
    else
        f(LmCfg{});
}

// The part of a tile of configuration C that is left where its wave's first row blocks have all
// of the matrix's rows: one row block a wave, the first C::RS rows.
template <class C>
struct FirstRows : C {
    static constexpr int BM = C::RS, TM = 1;
};

// f(C, or FirstRows<C> where that has the last of the M rows) for a tile whose first row is m0.
template <class C, class F>
__device__ __forceinline__ void with_rows_of(int64_t M, int64_t m0, F&& f) {
    if constexpr (C::TM > 1)
        if (M - m0 <= C::RS) return f(FirstRows<C>{});
    f(C{});
}

// Tiles of 64, 128 or 256 rows x 128 columns, of which two run on a compute unit: the height
// that forms rows x (128 column_tiles) fastest. A tile alone on its unit takes `alone`, with a
// second one there `second` times that; where many wait, a unit finishes one every `each` (any
// unit of time, and the same ratios at every depth measured).
[[maybe_unused]] inline int fastest_height(int64_t rows, int64_t column_tiles,
                                           const double (&alone)[3], const double (&each)[3],
                                           double second) {
    int best = 0;
    double least = 0;
    for (int k = 0; k < 3; ++k) {
        const int bm = 64 << k;
        // the last height of 256 is shorter work where it has 128 rows at most (FirstRows)
        const int64_t tail = rows % bm;
        const double last = tail == 0 ? 0 : k == 2 && tail <= 128 ? 0.75 : 1;
        const double per_unit = ((double)(rows / bm) + last) * (double)column_tiles / kUnits;
        const double cost = fmax(per_unit > 1 ? second * alone[k] : alone[k],
                                 each[k] * (per_unit + 0.4));
        if (best == 0 || cost < least) best = bm, least = cost;
    }
    return best;
}

}  // namespace
