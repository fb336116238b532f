// libdart, four-bit part: matrices in MXFP4 (blocks of 32 values along a row, each value
// in E2M1, the block's scale a power of two in E8M0), their product on the matrix cores,
// and the token statistics of the LM head kept so.
//
// Paper: DART, arXiv 2509.23866. Its truncated importance weight (Sec. 4.4) corrects for
// a rollout policy that differs from the trainer's by quantisation; this part makes that
// policy's head (quantise), its logits (product) and its log-probs (statistics).
//
//   mxfp4_quantize_kernel    one workgroup per panel: four lanes a block, their largest
//                            size by two exchanges, E2M1 by the hardware's conversion.
//                            Bound by memory.
//   mxfp4_dequantize_kernel  a panel back.
//   mxfp4_few_kernel         the product of up to 32 rows: a workgroup per 32 rows of B, its
//                            four waves on different panels of them, joined in LDS.
//                            Bound by B's bytes.
//   mxfp4_matmul_kernel      the product of more rows: mxfp4_tile, the fp32 tile written
//                            in bf16 or fp32.
//   mxfp4_stats_kernel       mxfp4_tile and the epilogue of lmhead_stats_kernel: the
//                            logits are not written.
//
// Layout of a quantised R x K matrix: panels of 32 rows x 256 columns, padded with zeros at
// the matrix's edges, [ceil(R / 32)][ceil(K / 256)], each the operands of four
// v_mfma_scale_f32_32x32x64_f8f6f4 as a wave holds them:
//   bytes ks * 1024 + l * 16 ..  (ks < 4, l < 64): lane l's operand of product ks, the block
//                               (l / 32) * 4 + ks of row l % 32, value j in the low (j even)
//                               or high half of byte j / 2;
//   bytes 4096 + l * 4 + ks     its scale.
// So a lane's four operands have their scales in one dword, a wave reads an operand as 1 KB
// in a row, from memory or from LDS, without a bank conflict, and no edge needs a check.
#include "lmhead_tile.h"

namespace {

constexpr int64_t kSlice = 256;  // columns of a panel
constexpr int64_t kRun = 32;     // rows of a panel
constexpr uint32_t kPanel = 4352, kScalesAt = 4096;  // bytes
constexpr int kQuantThreads = 256;

int64_t slices_of(int64_t K) { return (K + kSlice - 1) / kSlice; }
int64_t runs_of(int64_t R) { return (R + kRun - 1) / kRun; }

// Where values [8 c8, 8 c8 + 8) of row r of a panel are (four bytes), and their block's scale.
__device__ __forceinline__ uint32_t value_at(int r, int c8) {
    const int b = c8 >> 2;
    return (uint32_t)((b & 3) * 1024 + ((b >> 2) * 32 + r) * 16 + (c8 & 3) * 4);
}
__device__ __forceinline__ uint32_t scale_at(int r, int b) {
    return kScalesAt + (uint32_t)(((b >> 2) * 32 + r) * 4 + (b & 3));
}

// x of the lane that differs in bit 0 (B = 1) or 1 (B = 2) of its number.
template <int B>
__device__ __forceinline__ uint32_t quad_xor(uint32_t x) {
#if defined(__HIP_DEVICE_COMPILE__)
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, B == 1 ? 0xB1 : 0x4E, 0xF, 0xF, true);
#else
    return x;
#endif
}

// Four-bit codes of eight values already divided by their scale: E2M1, nearest, ties to
// even, saturating at 6 (the hardware's conversion at scale 1), value 0 lowest.
__device__ __forceinline__ uint32_t e2m1x8(const float (&v)[8]) {
#if defined(__HIP_DEVICE_COMPILE__)
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], 1.f, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], 1.f, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], 1.f, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], 1.f, 3);
    return w;
#else
    return (uint32_t)v[0];
#endif
}

// The hardware takes 16-byte vectors at any multiple of an element's size.
typedef u32x4 __attribute__((aligned(2))) u32x4_at2;
typedef u32x4 __attribute__((aligned(4))) u32x4_at4;
typedef u32x2 __attribute__((aligned(2))) u32x2_at2;

// Eight values of a row, the first `left` of them, then zeros.
__device__ __forceinline__ void load8(const float* p, int64_t left, float (&v)[8]) {
    if (left >= 8) {
        const u32x4 a = reinterpret_cast<const u32x4_at4*>(p)[0];
        const u32x4 b = reinterpret_cast<const u32x4_at4*>(p)[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(a[i]), v[4 + i] = __uint_as_float(b[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? p[i] : 0.f;
    }
}
__device__ __forceinline__ void load8(const uint16_t* p, int64_t left, float (&v)[8]) {
    if (left >= 8) {
        const u32x4 a = *reinterpret_cast<const u32x4_at2*>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(a[i] << 16);
            v[2 * i + 1] = __uint_as_float(a[i] & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < left ? __uint_as_float((uint32_t)p[i] << 16) : 0.f;
    }
}

// The scale of a block whose largest size has the bits top: 2^(floor(log2) - 2) not below
// 2^-127 as its E8M0 byte, 255 (a NaN) for a block with an infinity or a NaN. The fp32
// exponent field is floor(log2) + 127, and 0 (below 2^-126) ends at byte 0 all the same.
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    const uint32_t field = top >> 23;
    return field == 255u ? 255u : field > 2u ? field - 2u : 0u;
}

template <class X>
__global__ void __launch_bounds__(kQuantThreads)
mxfp4_quantize_kernel(const X* __restrict__ x, int64_t R, int64_t K, int64_t ld, int64_t slices,
                      uint8_t* __restrict__ out) {
    __shared__ alignas(16) uint8_t panel[kPanel];
    const int64_t run = blockIdx.x / slices, slice = blockIdx.x % slices;
    const int tid = threadIdx.x, c8 = tid & 31;
    const int64_t k = slice * kSlice + c8 * 8;
    float v[4][8];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int64_t r = run * kRun + p * 8 + (tid >> 5);
        load8(x + min(r, R - 1) * ld + min(k, K - 1), r < R ? K - k : 0, v[p]);
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int row = p * 8 + (tid >> 5);
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(v[p][i]) & 0x7FFFFFFFu);
        top = max(top, quad_xor<1>(top));
        top = max(top, quad_xor<2>(top));
        const uint32_t byte = scale_byte(top);
        // values / 2^(byte - 127), exact: the factor's exponent field is 2 at least
        const float inv = __uint_as_float((254u - min(byte, 252u)) << 23);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[p][i] *= inv;
        *reinterpret_cast<uint32_t*>(panel + value_at(row, c8)) = byte == 255u ? 0u : e2m1x8(v[p]);
        if ((c8 & 3) == 0) panel[scale_at(row, c8 >> 2)] = (uint8_t)byte;
    }
    __syncthreads();
    u32x4* dst = reinterpret_cast<u32x4*>(out + (int64_t)blockIdx.x * kPanel);
    const u32x4* src = reinterpret_cast<const u32x4*>(panel);
    dst[tid] = src[tid];
    static_assert(kPanel / 16 - kQuantThreads == 16, "the scales: sixteen more vectors");
    if (tid < 16) dst[kQuantThreads + tid] = src[kQuantThreads + tid];
}

// Up to eight results at p, the first `left` of them.
__device__ __forceinline__ void store8(float* p, int64_t left, const float (&v)[8]) {
    if (left >= 8) {
        u32x4 a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = __float_as_uint(v[i]), b[i] = __float_as_uint(v[4 + i]);
        reinterpret_cast<u32x4_at4*>(p)[0] = a;
        reinterpret_cast<u32x4_at4*>(p)[1] = b;
    } else {
        for (int i = 0; i < 8 && i < left; ++i) p[i] = v[i];
    }
}
__device__ __forceinline__ void store8(uint16_t* p, int64_t left, const float (&v)[8]) {
    if (left >= 8) {
        *reinterpret_cast<u32x4_at2*>(p) = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                                 pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    } else {
        for (int i = 0; i < 8 && i < left; ++i) p[i] = bf16_bits(v[i]);
    }
}

template <class X>
__global__ void __launch_bounds__(kQuantThreads)
mxfp4_dequantize_kernel(const uint8_t* __restrict__ q, int64_t R, int64_t K, int64_t slices,
                        X* __restrict__ out, int64_t ld) {
    __shared__ alignas(16) uint8_t panel[kPanel];
    const int64_t run = blockIdx.x / slices, slice = blockIdx.x % slices;
    const int tid = threadIdx.x, c8 = tid & 31;
    const u32x4* src = reinterpret_cast<const u32x4*>(q + (int64_t)blockIdx.x * kPanel);
    u32x4* dst = reinterpret_cast<u32x4*>(panel);
    dst[tid] = src[tid];
    if (tid < 16) dst[kQuantThreads + tid] = src[kQuantThreads + tid];
    __syncthreads();
    const int64_t k = slice * kSlice + c8 * 8;
    if (k >= K) return;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int row = p * 8 + (tid >> 5);
        const int64_t r = run * kRun + row;
        if (r >= R) return;
        const uint32_t w = *reinterpret_cast<const uint32_t*>(panel + value_at(row, c8));
        const uint32_t byte = panel[scale_at(row, c8 >> 2)];
        // the scale as fp32 (2^-127 is a denormal, byte 255 a NaN); a code's three bits
        // below the sign as the low exponent and high mantissa bits of an fp32, times
        // 2^126, are its size (0.5 from the denormal 2^-127)
        const float scale = byte == 255u ? __builtin_nanf("")
                            : byte == 0u ? __uint_as_float(0x00400000u)
                                         : __uint_as_float(byte << 23);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t code = w >> (4 * i);
            const float size = __uint_as_float((code & 7u) << 22) * 0x1p126f;
            v[i] = __uint_as_float(__float_as_uint(size) | (code & 8u) << 28) * scale;
        }
        store8(out + r * ld + k, K - k, v);
    }
}

// One 32 x 32 x 64 product of MXFP4 operands: byte ks of the scale dwords.
__device__ __forceinline__ f32x16 mfma_mxfp4(int ks, u32x4 b, u32x4 a, f32x16 c, uint32_t sb,
                                             uint32_t sa) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef int i32x8 __attribute__((ext_vector_type(8)));
    const i32x8 x = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    const i32x8 y = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
    switch (ks) {  // the byte is part of the instruction; 4: both operands in E2M1
        case 0: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, 0, sb, 0, sa);
        case 1: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, 1, sb, 1, sa);
        case 2: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, 2, sb, 2, sa);
        default: return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 4, 3, sb, 3, sa);
    }
#else
    (void)ks, (void)b, (void)a, (void)sb, (void)sa;
    return c;
#endif
}

// A lane's vector (or dword) at a byte offset of a run of panels, the slice's part of the
// offset in a scalar.
__device__ __forceinline__ u32x4 load_operand(__amdgpu_buffer_rsrc_t r, uint32_t lane_at,
                                              uint32_t wave_at) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane_at, wave_at, 0));
#else
    (void)r, (void)lane_at, (void)wave_at;
    return u32x4{0u, 0u, 0u, 0u};
#endif
}
__device__ __forceinline__ uint32_t load_scales(__amdgpu_buffer_rsrc_t r, uint32_t lane_at,
                                                uint32_t wave_at) {
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_raw_buffer_load_b32(r, lane_at, wave_at, 0);
#else
    (void)r, (void)lane_at, (void)wave_at;
    return 0u;
#endif
}

// Tile configuration: BM rows of A x 128 of B per workgroup of four waves, WM x WN, each
// owning (BM / WM) x (128 / WN) as 32 x 32 MFMA tiles; K in slices of 256, one panel of every
// 32 rows. A wave's panels of A go from memory (L2) to registers, those of B to an LDS ring of
// NS slices, from which the waves share them: an operand byte read from LDS serves one
// product, and with both operands there (the bf16 tile's way) the LDS was the limit. Two
// workgroups run per compute unit, so that one multiplies while the other is in its epilogue.
// T = 4096, V = 152064, d = 3584: the statistics 1.02 ms and the product, which stores 1.25 GB,
// 1.11 (4.4 and 4.0 PFLOP/s), where both operands through LDS in one workgroup a unit took 1.29 and
// 1.32. The matrix cores are busy 65% of the cycles at 1.5 to 1.6 GHz, which power has already lowered
// (the same instruction on registers alone is 94% busy at 1.65 GHz, 6.3 to 6.6 PFLOP/s): so what bounds
// the tile is taken to be power, as rings of other depths, more waves or stores that pass the caches
// move it by less than 2%.
template <int BM_, int WM_, int WN_, int NS_>
struct Cfg4 {
    static constexpr int BM = BM_, BN = 128, WM = WM_, WN = WN_, NS = NS_;
    static constexpr int WAVES = 4, THREADS = 256;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;  // MFMA tiles per wave
    static constexpr int SETS = NS % 2 == 0 ? 2 : 1;  // of registers for A's panels
    static constexpr int RS = WM * 32;  // rows between a wave's row blocks
    static constexpr int RUNS = BN / 32;  // panels of B a slice: one for each wave to bring
    static constexpr int CROW = BN + 4, CROW16 = BN + 8;  // as in Cfg
    static_assert(WM * WN == WAVES && RUNS == WAVES && TM * WM * 32 == BM && TN * WN * 32 == BN,
                  "four waves");
    struct alignas(16) Smem {
        union {
            uint8_t b[NS][RUNS][kPanel];
            float c[RS][CROW];
            uint16_t c16[BM][CROW16];
            float4 red[BN / kStatsUnit][BM];
        };
    };
    static_assert(sizeof(Smem) <= 80 * 1024, "two workgroups per compute unit");
};
// 256 rows; fewer for few rows, where B comes from HBM and little is multiplied per byte of it. 128
// rows with a slice more in flight (and its set of registers): 128 rows of V = 152064, d = 3584
// 61 us to 70. 64 rows with three workgroups a unit in its place: 64 rows of V = 152064, d = 1024 22.4
// us to 24.7, 48 x 32003 of K = 2056 13.6 to 14.1, d = 3584 66.8 to 66.2.
using Mx256 = Cfg4<256, 4, 1, 3>;
using Mx128 = Cfg4<128, 4, 1, 4>;
using Mx64 = Cfg4<64, 2, 2, 3>;

// The operands of a product: panels, and panels per row of panels.
struct Mxfp4Pair {
    const uint8_t *a, *b;
    int64_t runs_a, runs_b, slices;
};

// acc = this wave's part of the tile of A's rows [m0, m0 + BM) x B's rows [n0, n0 + 128) of
// A B^T; rows past the matrices' last panels read as zero. Layout of acc as gemm_tile's. Ends on
// a barrier with no loads in flight, so the caller may reuse the LDS.
template <class C>
__device__ __forceinline__ void mxfp4_tile(const Mxfp4Pair& x, int64_t m0, int64_t n0,
                                           typename C::Smem& sm, f32x16 (&acc)[C::TM][C::TN]) {
#if defined(__HIP_DEVICE_COMPILE__)
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int j = 0; j < C::TN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

    // a run of panels is a resource of its own, so that loads past its last slice read as zero
    // without going to memory: the loop below needs no condition on them
    const int64_t nk = x.slices, run_bytes = nk * kPanel;
    auto run_rsrc = [&](const uint8_t* p, int64_t run, int64_t runs) {
        return tile_rsrc(p + (run < runs ? run : 0) * run_bytes, run < runs ? run_bytes : 0);
    };
    __amdgpu_buffer_rsrc_t ra[C::TM];
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
        ra[i] = run_rsrc(x.a, m0 / kRun + wave / C::WN + i * C::WM, x.runs_a);
    const __amdgpu_buffer_rsrc_t rb = run_rsrc(x.b, n0 / kRun + wave, x.runs_b);
    const uint32_t l16 = (uint32_t)lane * 16, l4 = (uint32_t)lane * 4, s4 = kScalesAt + l4;

    // slice kt's panels of B into buffer buf: every wave one run, four operands and the scales
    auto issue = [&](int64_t kt, int buf) {
        const uint32_t at = (uint32_t)kt * kPanel;
        uint8_t* dst = &sm.b[buf][wave][0];
#pragma unroll
        for (uint32_t ks = 0; ks < 4; ++ks)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, lds_ptr(dst + ks * 1024), 16, l16,
                                                    at + ks * 1024, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, lds_ptr(dst + kScalesAt), 4, l4, at + kScalesAt,
                                                0, 0);
    };
    u32x4 af[C::SETS][4][C::TM];
    uint32_t sa[C::TM], sa_next[C::TM], sb[C::TN];
    auto load_a = [&](int64_t kt, int ks, int a_set) {
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
            af[a_set][ks][i] = load_operand(ra[i], l16, (uint32_t)kt * kPanel + (uint32_t)ks * 1024);
    };
    auto load_sa = [&](int64_t kt) {
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
            sa_next[i] = load_scales(ra[i], s4, (uint32_t)kt * kPanel);
    };
    // the wave's first column block; opaque, so that buffer, block and product are the
    // reads' immediates
    uint32_t rd = (uint32_t)((wave % C::WN) * C::TN) * kPanel + l16;
    uint32_t rs = (uint32_t)((wave % C::WN) * C::TN) * kPanel + s4;
    asm volatile("" : "+v"(rd), "+v"(rs));
    const char* const lds0 = reinterpret_cast<const char*>(&sm);
    u32x4 bf[2][C::TN];
    auto read_b = [&](auto bufc, int ks, int set) {
        constexpr uint32_t buf = decltype(bufc)::value;
#pragma unroll
        for (uint32_t j = 0; j < C::TN; ++j)
            bf[set][j] = *reinterpret_cast<const u32x4*>(lds0 + rd + (buf * C::RUNS + j) * kPanel +
                                                         ks * 1024);
    };
    // When slice kt begins, the loads of B's slices kt + 1 .. kt + NS - 2, five each, were issued
    // after those of kt; waiting until no more than so many loads are left has slice kt landed,
    // wherever the compiler put A's.
    constexpr int AHEAD = 5 * (C::NS - 2);
    auto slice = [&](auto bufc, int64_t kt) {
        constexpr int buf = decltype(bufc)::value;
        wait_vmcnt<AHEAD>();
        lds_ring_barrier();
        // A's next slice: with two sets of registers now, before the loads of B, which may then
        // stay in flight when it is waited for; with one as the products let go of it
        constexpr int set_a = C::SETS == 2 ? buf & 1 : 0;
        if constexpr (C::SETS == 2) {
#pragma unroll
            for (int i = 0; i < C::TM; ++i) sa[i] = sa_next[i];
            load_sa(kt + 1);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) load_a(kt + 1, ks, set_a ^ 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        issue(kt + C::NS - 1, (buf + C::NS - 1) % C::NS);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t j = 0; j < C::TN; ++j)
            sb[j] = *reinterpret_cast<const uint32_t*>(lds0 + rs + (buf * C::RUNS + j) * kPanel);
        read_b(bufc, 0, 0);
        if constexpr (C::SETS == 1) {
#pragma unroll
            for (int i = 0; i < C::TM; ++i) sa[i] = sa_next[i];
            load_sa(kt + 1);
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int ks = 0; ks < 4; ++ks) {
            const int set = ks & 1;
            if (ks < 3) read_b(bufc, ks + 1, set ^ 1);
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
#pragma unroll
                for (int j = 0; j < C::TN; ++j)
                    acc[i][j] = mfma_mxfp4(ks, bf[set][j], af[set_a][ks][i], acc[i][j], sb[j], sa[i]);
            if constexpr (C::SETS == 1) load_a(kt + 1, ks, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        // the products stay in their slice (the compiler moved them to the next branch, with
        // every operand on the way in registers)
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j) asm volatile("" : "+v"(acc[i][j]));
    };
    load_sa(0);
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) load_a(0, ks, 0);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int b = 0; b < C::NS - 1; ++b) issue(b, b);
    int64_t kt = 0;
    for (; kt + C::NS - 1 < nk; kt += C::NS) {
        slice(std::integral_constant<int, 0>{}, kt);
        slice(std::integral_constant<int, 1>{}, kt + 1);
        slice(std::integral_constant<int, 2>{}, kt + 2);
        if constexpr (C::NS > 3) slice(std::integral_constant<int, 3 % C::NS>{}, kt + 3);
    }
    if (kt < nk) slice(std::integral_constant<int, 0>{}, kt);
    if (kt + 1 < nk) slice(std::integral_constant<int, 1>{}, kt + 1);
    if (C::NS > 3 && kt + 2 < nk) slice(std::integral_constant<int, 2>{}, kt + 2);
    static_assert(C::NS == 3 || C::NS == 4, "buffers of the K loop");
    wait_vmcnt<0>();  // the zeros of slices past the last are in LDS
    __syncthreads();
#else
    (void)x, (void)m0, (void)n0, (void)sm, (void)acc;
#endif
}

// This wave's part of a result tile to out [M, ld] through the wave's own part of the
// LDS (its accesses run in order: no barrier), 32 rows at a time, as in
// lmhead_dlogits_tile: bf16 rows of the wave's columns, fp32 ones 64 columns at a time.
template <class C, class O>
__device__ __forceinline__ void store_tile(f32x16 (&acc)[C::TM][C::TN], int64_t M, int64_t N,
                                           O* __restrict__ out, int64_t ld, typename C::Smem& sm,
                                           int64_t m0, int64_t n0) {
    constexpr bool BF16 = sizeof(O) == 2;
    constexpr int NJ = BF16 ? C::TN : 2;  // 32-column blocks a piece
    constexpr int EPC = 16 / sizeof(O), CPR = NJ * 32 / EPC, RPI = 64 / CPR;
    using vec_t = typename std::conditional<BF16, u32x4_at2, u32x4_at4>::type;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int wr = (wave / C::WN) * 32, wc = (wave % C::WN) * (C::BN / C::WN);
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int u = 0; u < C::TN / NJ; ++u) {
            lds_wave_order();  // fp32 pieces share their rows of the LDS
            if constexpr (BF16) {
                blocks_to_lds_bf16<C, NJ>(&acc[i][NJ * u], i, NJ * u, sm);
            } else {
#pragma unroll
                for (int j = 0; j < NJ; ++j)
#pragma unroll
                    for (int v = 0; v < 16; v += 4) {
                        const f32x16& t = acc[i][NJ * u + j];
                        *reinterpret_cast<f32x4*>(
                            &sm.c[wr + (lane & 31)][wc + (NJ * u + j) * 32 + (v >> 2) * 8 +
                                                    (lane >> 5) * 4]) =
                            f32x4{t[v], t[v + 1], t[v + 2], t[v + 3]};
                    }
            }
            lds_wave_order();
#pragma unroll
            for (int q = 0; q < 32 / RPI; ++q) {
                const int rr = wr + q * RPI + lane / CPR, c = wc + u * NJ * 32 + lane % CPR * EPC;
                const int64_t m = m0 + rr + i * C::RS, n = n0 + c;
                if (m >= M || n >= N) continue;
                const O* src;
                if constexpr (BF16)
                    src = &sm.c16[rr + i * C::RS][c];
                else
                    src = &sm.c[rr][c];
                O* dst = out + m * ld + n;
                if (n + EPC <= N)
                    *reinterpret_cast<vec_t*>(dst) = *reinterpret_cast<const u32x4*>(src);
                else
                    for (int e = 0; e < EPC && n + e < N; ++e) dst[e] = src[e];
            }
        }
}

// f(configuration, LDS, first row, column tile) for this workgroup's tile of M rows x nnt column
// tiles.
template <class C, class F>
__device__ __forceinline__ void with_mxfp4_tile(int64_t M, int64_t nnt, F&& f) {
    __shared__ typename C::Smem sm;
    int64_t mt, nt;
    tile_of_block((M + C::BM - 1) / C::BM, nnt, mt, nt);
    with_rows_of<C>(M, mt * C::BM, [&](auto c) { f(c, sm, mt * C::BM, nt); });
}

template <class C, class O>
__global__ void __launch_bounds__(C::THREADS, 2)
mxfp4_matmul_kernel(Mxfp4Pair x, int64_t M, int64_t N, int64_t nnt, O* __restrict__ out,
                    int64_t ld) {
    with_mxfp4_tile<C>(M, nnt, [&](auto c, auto& sm, int64_t m0, int64_t nt) {
        using P = decltype(c);
        f32x16 acc[P::TM][P::TN];
        mxfp4_tile<P>(x, m0, nt * P::BN, sm, acc);
        store_tile<P, O>(acc, M, N, out, ld, sm, m0, nt * P::BN);
    });
}

template <class C>
__global__ void __launch_bounds__(C::THREADS, 2)
mxfp4_stats_kernel(Mxfp4Pair x, int64_t T, int64_t V, const int32_t* __restrict__ target,
                   float scale, int64_t nvt, float4* __restrict__ part, float* __restrict__ z_y) {
    with_mxfp4_tile<C>(T, nvt, [&](auto c, auto& sm, int64_t m0, int64_t vt) {
        using P = decltype(c);
        stats_of_tile<P>(
            [&](int64_t n0, f32x16(&acc)[P::TM][P::TN]) { mxfp4_tile<P>(x, m0, n0, sm, acc); }, T, V,
            target, scale, nvt, part, z_y, sm, m0, vt);
    });
}

// One workgroup per row: the row's nvt triples merged in index order by thread, lane and wave, and
// the target logit last, as lmhead_merge_kernel does, whose single wave a row took 9 us for 64
// rows of V = 152064 (1188 triples each), where this takes 6 (17 and 19 for 4096). A NaN among
// the logits shows in the row's results.
constexpr int kMergeThreads = 256;
__global__ void __launch_bounds__(kMergeThreads)
mxfp4_merge_kernel(const float4* __restrict__ part, const float* __restrict__ z_y, int64_t nvt,
                   int64_t V, const int32_t* __restrict__ target, float* __restrict__ logp,
                   float* __restrict__ entropy, float* __restrict__ lse) {
    __shared__ Triple waves[kMergeThreads / 64];
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63;
    const int32_t y = target[t];
    const float zy = y >= 0 && y < V ? z_y[t] : __builtin_nanf("");
    Triple acc = {-INFINITY, 0.f, 0.f};
    for (int64_t j0 = tid; j0 < nvt; j0 += kMergeThreads * kMergeBatch) {
        float4 p[kMergeBatch];
#pragma unroll
        for (int k = 0; k < kMergeBatch; ++k) {
            const int64_t j = j0 + kMergeThreads * k;
            p[k] = j < nvt ? part[t * nvt + j] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int k = 0; k < kMergeBatch; ++k) acc = merge(acc, Triple{p[k].x, p[k].y, p[k].z});
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1)
        acc = merge(acc, Triple{__shfl_xor(acc.m, off), __shfl_xor(acc.s, off),
                                __shfl_xor(acc.w, off)});
    if (lane == 0) waves[tid >> 6] = acc;
    __syncthreads();
    if (tid) return;
#pragma unroll
    for (int k = 1; k < kMergeThreads / 64; ++k) acc = merge(acc, waves[k]);
    const bool others = acc.s != 0.f;  // also where it is a NaN
    const float M = others ? fmaxf(acc.m, zy) : zy, dx = acc.m - M;
    const float cx = others ? expf(dx) : 0.f;
    const float sx = others ? cx * acc.s : 0.f, wx = others ? cx * fmaf(dx, acc.s, acc.w) : 0.f;
    const float xy = zy - M, ey = expf(xy), S = sx + ey, ln_s = logf(S);
    const float h = ln_s - fmaf(ey, xy, wx) / S;
    lse[t] = M + ln_s;
    entropy[t] = h < 0.f ? 0.f : h;
    logp[t] = sx < ey ? -log1pf(sx / ey) : xy - ln_s;
}

// out = A B^T for up to 32 rows of A (one row of panels): the workgroup takes 32 rows of B, its
// waves panels w, w + 4, ... of both, kInFlight at a time all loaded before the first is
// multiplied; the waves' sums are added in order through LDS. No LDS on the way in: a panel of
// B is used once, and memory bounds it. One row by V = 152064, d = 3584: 50 us, 290 MB at 5.8 TB/s,
// where the tile of 64 rows takes 57.
constexpr int kFewRows = 32, kFewWaves = 4, kInFlight = 4;
template <class O>
__global__ void __launch_bounds__(kFewWaves * 64)
mxfp4_few_kernel(Mxfp4Pair x, int64_t M, int64_t N, O* __restrict__ out, int64_t ld) {
    __shared__ f32x4 sums[kFewWaves][4][64];
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int64_t n0 = (int64_t)blockIdx.x * kRun;
    const u32x4* a = reinterpret_cast<const u32x4*>(x.a);
    const u32x4* b = reinterpret_cast<const u32x4*>(x.b + (int64_t)blockIdx.x * x.slices * kPanel);
    f32x16 acc = {};
    for (int64_t s0 = wave; s0 < x.slices; s0 += kFewWaves * kInFlight) {
        u32x4 bv[kInFlight][4], av[kInFlight][4];
        uint32_t sb[kInFlight], sa[kInFlight];
#pragma unroll
        for (int p = 0; p < kInFlight; ++p) {
            const int64_t s = s0 + p * kFewWaves;
            if (s >= x.slices) break;
            const u32x4* pb = b + s * (kPanel / 16);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) bv[p][ks] = __builtin_nontemporal_load(pb + ks * 64 + lane);
            sb[p] = reinterpret_cast<const uint32_t*>(pb + kScalesAt / 16)[lane];
        }
#pragma unroll
        for (int p = 0; p < kInFlight; ++p) {
            const int64_t s = s0 + p * kFewWaves;
            if (s >= x.slices) break;
            const u32x4* pa = a + s * (kPanel / 16);
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) av[p][ks] = pa[ks * 64 + lane];
            sa[p] = reinterpret_cast<const uint32_t*>(pa + kScalesAt / 16)[lane];
        }
#pragma unroll
        for (int p = 0; p < kInFlight; ++p) {
            if (s0 + p * kFewWaves >= x.slices) break;
#pragma unroll
            for (int ks = 0; ks < 4; ++ks)
                acc = mfma_mxfp4(ks, bv[p][ks], av[p][ks], acc, sb[p], sa[p]);
        }
    }
#pragma unroll
    for (int v = 0; v < 4; ++v)
        sums[wave][v][lane] = f32x4{acc[4 * v], acc[4 * v + 1], acc[4 * v + 2], acc[4 * v + 3]};
    __syncthreads();
    // the wave's quarter of the columns: four adjacent ones of a row a lane
    f32x4 t = sums[0][wave][lane];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) t += sums[w][wave][lane];
    const int64_t m = lane & 31, n = n0 + wave * 8 + (lane >> 5) * 4;
    if (m >= M || n >= N) return;
    O* dst = out + m * ld + n;
    if constexpr (sizeof(O) == 2) {
        const u32x2 pk = {pack_bf16x2(t[0], t[1]), pack_bf16x2(t[2], t[3])};
        if (n + 4 <= N)
            *reinterpret_cast<u32x2_at2*>(dst) = pk;
        else
            for (int e = 0; n + e < N; ++e) dst[e] = bf16_bits(t[e]);
    } else {
        if (n + 4 <= N)
            *reinterpret_cast<u32x4_at4*>(dst) = __builtin_bit_cast(u32x4, t);
        else
            for (int e = 0; n + e < N; ++e) dst[e] = t[e];
    }
}

bool bad_size(int64_t n) { return n < 1 || n > 0x7FFFFFFFll; }
bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
bool bad_quantized(const void* q, int64_t R, int64_t K) {
    return !q || bad_size(R) || bad_size(K) || misaligned(q, 16);
}
size_t size_of(dart_dtype_t t) { return t == DART_BF16 ? 2 : 4; }
bool bad_dtype(dart_dtype_t t) { return t != DART_BF16 && t != DART_F32; }
// a run of panels is addressed by 32-bit byte offsets
constexpr int64_t kMaxK = int64_t(1) << 24;
static_assert((kMaxK / kSlice + 4) * kPanel < int64_t(1) << 31, "offsets of a run");

Mxfp4Pair pair_of(const void* a, int64_t M, const void* b, int64_t N, int64_t K) {
    return {static_cast<const uint8_t*>(a), static_cast<const uint8_t*>(b), runs_of(M), runs_of(N),
            slices_of(K)};
}

int64_t column_tiles(int64_t N) { return (N + Mx256::BN - 1) / Mx256::BN; }

// f(configuration that forms M x N results fastest); times in us at K = 3584 (fastest_height).
// Of 270 calls measured (M from 40 to 4000, N from 1088 to 152064, K = 256, 1024 and 3584,
// products and statistics) the choice is within 18% of the fastest of the three, 1.1% on average.
template <class F>
void with_mxfp4_cfg(int64_t M, int64_t N, F&& f) {
    const int bm = fastest_height(M, column_tiles(N), {6.4, 8.6, 12.6}, {6.2, 8.7, 15}, 1.3);
    if (bm == 64)
        f(Mx64{});
    else if (bm == 128)
        f(Mx128{});
    else
        f(Mx256{});
}

}  // namespace

extern "C" {

size_t dart_mxfp4_bytes(int64_t R, int64_t K) {
    if (bad_size(R) || bad_size(K)) return 0;
    return (size_t)runs_of(R) * (size_t)slices_of(K) * kPanel;
}

dart_status_t dart_mxfp4_quantize(const void* x, dart_dtype_t dtype, int64_t R, int64_t K,
                                  int64_t ld, void* q, hipStream_t stream) {
    if (bad_dtype(dtype) || !x || ld < K || bad_quantized(q, R, K) || misaligned(x, size_of(dtype)))
        return DART_ERR_INVALID_ARG;
    const int64_t blocks = runs_of(R) * slices_of(K);
    if (!grid_fits(blocks, kQuantThreads)) return DART_ERR_UNSUPPORTED;
    auto launch = [&](auto kernel, auto* p) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kQuantThreads), 0, stream, p, R, K,
                           ld, slices_of(K), static_cast<uint8_t*>(q));
    };
    if (dtype == DART_BF16)
        launch(mxfp4_quantize_kernel<uint16_t>, static_cast<const uint16_t*>(x));
    else
        launch(mxfp4_quantize_kernel<float>, static_cast<const float*>(x));
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

dart_status_t dart_mxfp4_dequantize(const void* q, int64_t R, int64_t K, dart_dtype_t dtype,
                                    void* out, int64_t ld_out, hipStream_t stream) {
    if (bad_dtype(dtype) || !out || ld_out < K || bad_quantized(q, R, K) ||
        misaligned(out, size_of(dtype)))
        return DART_ERR_INVALID_ARG;
    const int64_t blocks = runs_of(R) * slices_of(K);
    if (!grid_fits(blocks, kQuantThreads)) return DART_ERR_UNSUPPORTED;
    auto launch = [&](auto kernel, auto* p) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kQuantThreads), 0, stream,
                           static_cast<const uint8_t*>(q), R, K, slices_of(K), p, ld_out);
    };
    if (dtype == DART_BF16)
        launch(mxfp4_dequantize_kernel<uint16_t>, static_cast<uint16_t*>(out));
    else
        launch(mxfp4_dequantize_kernel<float>, static_cast<float*>(out));
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

dart_status_t dart_mxfp4_matmul(const void* a, int64_t M, const void* b, int64_t N, int64_t K,
                                dart_dtype_t dtype, void* out, int64_t ld_out, hipStream_t stream) {
    if (bad_dtype(dtype) || !out || ld_out < N || bad_quantized(a, M, K) ||
        bad_quantized(b, N, K) || misaligned(out, size_of(dtype)))
        return DART_ERR_INVALID_ARG;
    const int64_t nnt = column_tiles(N);
    if (!grid_fits((M + Mx64::BM - 1) / Mx64::BM * nnt, Mx64::THREADS) ||
        !grid_fits(runs_of(N), kFewWaves * 64) || K > kMaxK)
        return DART_ERR_UNSUPPORTED;
    const Mxfp4Pair x = pair_of(a, M, b, N, K);
    auto launch = [&](auto* p) {
        using O = typename std::remove_pointer<decltype(p)>::type;
        if (M <= kFewRows)
            hipLaunchKernelGGL(mxfp4_few_kernel<O>, dim3((unsigned)runs_of(N)), dim3(kFewWaves * 64),
                               0, stream, x, M, N, p, ld_out);
        else
            with_mxfp4_cfg(M, N, [&](auto cfg) {
                using C = decltype(cfg);
                hipLaunchKernelGGL((mxfp4_matmul_kernel<C, O>),
                                   dim3((unsigned)((M + C::BM - 1) / C::BM * nnt)),
                                   dim3(C::THREADS), 0, stream, x, M, N, nnt, p, ld_out);
            });
    };
    if (dtype == DART_BF16)
        launch(static_cast<uint16_t*>(out));
    else
        launch(static_cast<float*>(out));
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

size_t dart_lmhead_mxfp4_stats_workspace_bytes(int64_t T, int64_t V) {
    if (bad_size(T) || bad_size(V)) return 0;
    return (size_t)T * (size_t)column_tiles(V) * sizeof(float4) + (size_t)T * sizeof(float);
}

dart_status_t dart_lmhead_mxfp4_tok_stats(const void* hidden, int64_t T, const void* weight,
                                          int64_t V, int64_t d, const int32_t* target,
                                          float inv_temp, float* logp, float* entropy, float* lse,
                                          void* workspace, size_t workspace_bytes,
                                          hipStream_t stream) {
    if (bad_quantized(hidden, T, d) || bad_quantized(weight, V, d)) return DART_ERR_INVALID_ARG;
    if (!(inv_temp > 0.f) || isinf(inv_temp)) return DART_ERR_INVALID_ARG;
    if (!target || !logp || !entropy || !lse || !workspace || misaligned(workspace, 16) ||
        workspace_bytes < dart_lmhead_mxfp4_stats_workspace_bytes(T, V))
        return DART_ERR_INVALID_ARG;
    const int64_t nvt = column_tiles(V);
    if (!grid_fits((T + Mx64::BM - 1) / Mx64::BM * nvt, Mx64::THREADS) ||
        !grid_fits(T, kMergeThreads) || d > kMaxK)
        return DART_ERR_UNSUPPORTED;
    if (const dart_status_t ck = dart_check::run(
            stream, {{dart_check::Item::Ids, target, T, V}}); ck != DART_OK)
        return ck;
    const Mxfp4Pair x = pair_of(hidden, T, weight, V, d);
    float4* part = static_cast<float4*>(workspace);
    float* z_y = reinterpret_cast<float*>(part + T * nvt);
    with_mxfp4_cfg(T, V, [&](auto cfg) {
        using C = decltype(cfg);
        hipLaunchKernelGGL(mxfp4_stats_kernel<C>, dim3((unsigned)((T + C::BM - 1) / C::BM * nvt)),
                           dim3(C::THREADS), 0, stream, x, T, V, target, inv_temp, nvt, part, z_y);
    });
    hipLaunchKernelGGL(mxfp4_merge_kernel, dim3((unsigned)T), dim3(kMergeThreads), 0, stream, part,
                       z_y, nvt, V, target, logp, entropy, lse);
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

}  // extern "C"
