// libdart, supervised part: the cross entropy of the LM head and its gradient, straight
// from the hidden states and the head's weight.
//
// For the rows t whose target y_t lies in [0, V), with z = h W^T and lse_t = log sum_v e^z_tv:
//   l_t   = (1 - eps) (lse_t - z_ty) + eps (lse_t - mean_v z_tv) + lambda lse_t^2
//   dl/dz = (1 + 2 lambda lse_t) p_tv - (1 - eps) [v = y_t] - eps / V
// and 0 for the others. Forward alone: z is formed tile by tile, each row's columns of a tile
// reduced to (largest, normaliser, sum), and these merged per row. With the gradient, rows are
// taken a block at a time, and the product z is formed once:
//   xent_tile_kernel  forms z tile by tile on the matrix cores, reduces each row's 64-column
//                     units to (m = the largest, the normaliser) and the sum of z, and keeps
//                     e = 2^15 e^(z - m) in fp16;
//   xent_rows_kernel  merges a row's triples to lse, and turns its e in place into the
//                     bf16 dz / (1 - eps), from which no logit is needed;
//   the GEMMs of the LM head's backward (dh = dz W, dW = dz^T h), times (1 - eps) / N.
// The rows with a label are gathered first, so that the others cost no product, and
// whatever their hidden states hold (NaNs in the padding of a batch) reaches no result.
// So three products of T V d instead of the four of a loss whose coefficients only a
// second pass knows (dart_lmhead_backward): at T = 4096, V = 152064, d = 3584 the kept
// exponentials cost a read and a write of 1.25 GB, the fourth product took 3.4 ms.
// What is rounded: e to fp16, by 2^-11 of its value at most (half a step of 11 bits) down to 2^-29
// of its 64 columns' largest, below that by 2^-40 of that: an eighth of the bf16 rounding that follows,
// where 32 bits would be twice the bytes to write and read. dz to bf16, by 2^-8 at most, for the matrix
// cores, as in dart_lmhead_dlogits: the other operand is bf16, and two bf16 of dz would double two of the
// three products. Gradients are off from 64 bits by 1.8e-3 to 2.0e-3 of their size in the cases
// measured; a bf16 result's own rounding is 1.7e-3 of it. dz is kept divided by 1 - eps and not yet by N,
// so that the target's element of an unsure row, the largest of all, is next to -1 and
// loses nothing by its rounding.
#include "lmhead_tile.h"

namespace {

using lmhead::Grad;

constexpr float kLog2e = 1.4426950408889634f;
// exponentials are kept times 2^kShift: fp16 holds up to 65504 and 2^-14 at full width
constexpr int kShift = 15;

__device__ __forceinline__ bool has_label(int32_t y, int64_t V) { return y >= 0 && y < V; }

// Four adjacent columns as fp16.
__device__ __forceinline__ u32x2 pack_half4(float a, float b, float c, float d) {
    typedef _Float16 h4 __attribute__((ext_vector_type(4)));
    const h4 v = {(_Float16)a, (_Float16)b, (_Float16)c, (_Float16)d};
    return __builtin_bit_cast(u32x2, v);
}

// Tile configuration: BM rows x 128 vocabulary entries per workgroup of four waves, WM x WN, each
// owning (BM / WM) x (128 / WN) as 32 x 32 MFMA tiles; K in slices of 64. The hidden rows, which
// the call gathers anyway, lie in panels of 32 rows x 64 columns in the order in which a wave's
// MFMAs take them (below) and go from memory (L2) to registers; W's rows go through an LDS ring of NS
// slices, from which the waves share them. With both operands in the LDS, as in gemm_tile, the
// LDS is the limit; and two such workgroups fit a compute unit, so that one multiplies while the
// other is in its epilogue. T = 4096, V = 152064, d = 3584: 3.40 ms with the exponentials kept and
// 3.30 without (1.35 PFLOP/s; a library product of the size reaches 1.47 and stores its logits), where
// gemm_tile with the same epilogues took 3.50 and 3.44; 12 rows of V = 4864, d = 2328: 19 us to 28.
constexpr int kTileN = 128, kSliceK = 64;
constexpr uint32_t kPanel = 4096;  // bytes
template <int BM_, int WM_, int WN_, int NS_>
struct XCfg {
    static constexpr int BM = BM_, BN = kTileN, WM = WM_, WN = WN_, NS = NS_;
    static constexpr int WAVES = 4, THREADS = 256;
    static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;  // MFMA tiles per wave
    static constexpr int SETS = TM == 1 ? 2 : 1;  // of registers for the hidden rows' panels
    static constexpr int RS = WM * 32;            // rows between a wave's row blocks
    static constexpr int CROW16 = BN + 8;         // as in Cfg
    static_assert(WM * WN == WAVES && TM * WM * 32 == BM && TN * WN * 32 == BN && TN % 2 == 0,
                  "four waves, units of two column blocks");
    static_assert(SETS == 1 || NS % 2 == 0, "a slice's set goes by its buffer");
    static_assert(NS == 3 || NS == 4, "buffers of the K loop");
    struct alignas(16) Smem {
        union {
            // chunk c (16 bytes) of row r in slot c ^ swz(r), as in gemm_tile
            uint16_t b[NS][BN][kSliceK];
            uint16_t c16[BM][CROW16];
        };
        // a row's maxima, normalisers and sums of the tile's units of 64 columns
        float units[3][BN / kStatsUnit][BM];
    };
    static_assert(sizeof(Smem) <= 80 * 1024, "two workgroups per compute unit");
};
using X256 = XCfg<256, 4, 1, 3>;
using X128 = XCfg<128, 4, 1, 4>;
using X64 = XCfg<64, 2, 2, 4>;

// Where the 16 bytes of columns [8 c, 8 c + 8) of row r of a block's rows are: the panel of its
// run of 32 rows and slice, in it product c % 8 / 2, lane (c % 2) * 32 + r % 32.
__host__ __device__ constexpr int64_t panel_at(int64_t r, int64_t c, int64_t slices) {
    return (r / 32 * slices + c / 8) * kPanel + c % 8 / 2 * 1024 + (c % 2 * 32 + r % 32) * 16;
}
int64_t slices_of(int64_t d) { return (d + kSliceK - 1) / kSliceK; }
int64_t column_tiles(int64_t V) { return (V + kTileN - 1) / kTileN; }

// acc = this wave's part of h's rows [m0, m0 + BM) (panels of `runs` runs) times W's rows
// [n0, n0 + 128) of N (row-major, d columns). K past d: zeros in h's panels, and read as zero of
// W. Layout of acc as gemm_tile's. Ends on a barrier with no loads in flight.
template <class C>
__device__ __forceinline__ void xent_product(const uint8_t* __restrict__ h, int64_t runs,
                                             const uint16_t* __restrict__ w, int64_t N, int64_t ldw,
                                             int64_t d, int64_t m0, int64_t n0,
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

    // every run of panels a resource of its own: loads past its last slice read as zero without
    // going to memory (a raw load's whole offset is checked, its scalar part too)
    const int64_t nk = (d + kSliceK - 1) / kSliceK, run_bytes = nk * kPanel;
    __amdgpu_buffer_rsrc_t ra[C::TM];
#pragma unroll
    for (int i = 0; i < C::TM; ++i) {
        const int64_t run = m0 / 32 + wave / C::WN + i * C::WM;
        ra[i] = tile_rsrc(h + (run < runs ? run : 0) * run_bytes, run < runs ? run_bytes : 0);
    }
    const __amdgpu_buffer_rsrc_t rb = tile_rsrc(w + n0 * ldw, rows_bytes(N - n0 < C::BN ? N - n0 : C::BN, ldw, d));
    const uint32_t l16 = (uint32_t)lane * 16;
    // one load of W fills 8 rows x 8 chunks; load q of a wave rows (q * 4 + wave) * 8 .. + 7
    const int r_lane = wave * 8 + (lane >> 3), c_lane = (lane & 7) ^ swz<8>(r_lane);
    const uint32_t vb = (uint32_t)((r_lane * ldw + c_lane * 8) * 2);
    const uint32_t qstride = (uint32_t)(32 * ldw * 2);
    // the last slice's chunks past d, and slices past the last, are out of the resource's range (of
    // less than 2^31 bytes, as the scalar offsets are)
    constexpr uint32_t kNowhere = 0x80000000u;
    const uint32_t vb_last = (nk - 1) * kSliceK + c_lane * 8 < d ? vb : kNowhere;
    auto issue = [&](int64_t kt, int buf) {
        const uint32_t v = kt < nk - 1 ? vb : kt == nk - 1 ? vb_last : kNowhere;
        const uint32_t k = kt < nk ? (uint32_t)kt * (kSliceK * 2) : 0u;
#pragma unroll
        for (uint32_t q = 0; q < 4; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rb, lds_ptr(&sm.b[buf][(q * 4 + wave) * 8][0]), 16, v,
                kt < nk ? k + q * qstride : 0u, 0, 0);
    };
    bf16x8 af[C::SETS][4][C::TM];
    auto load_a = [&](int64_t kt, int ks, int a_set) {
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
            af[a_set][ks][i] = __builtin_bit_cast(
                bf16x8, __builtin_amdgcn_raw_buffer_load_b128(
                            ra[i], l16, (uint32_t)kt * kPanel + (uint32_t)ks * 1024, 0));
    };
    const int wc = (wave % C::WN) * (C::BN / C::WN);
    uint32_t rd[4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) {
        const int c = ks * 2 + (lane >> 5), r = wc + (lane & 31);
        rd[ks] = (uint32_t)(r * kSliceK + (c ^ swz<8>(r)) * 8) * 2;
        asm volatile("" : "+v"(rd[ks]));  // opaque: buffer and block are the reads' immediates
    }
    const char* const lds0 = reinterpret_cast<const char*>(&sm);
    bf16x8 bf[2][C::TN];
    auto read_b = [&](auto bufc, int ks, int set) {
        constexpr int buf = decltype(bufc)::value;
#pragma unroll
        for (int j = 0; j < C::TN; ++j)
            bf[set][j] = __builtin_bit_cast(
                bf16x8, *reinterpret_cast<const u32x4*>(
                            lds0 + rd[ks] + (buf * C::BN + j * 32) * kSliceK * 2));
    };
    // When slice kt begins, the loads of W's slices kt + 1 .. kt + NS - 2, four each, were issued
    // after those of kt; waiting until no more than so many are left has slice kt landed,
    // wherever the compiler put the others.
    constexpr int AHEAD = 4 * (C::NS - 2);
    auto slice = [&](auto bufc, int64_t kt) {
        constexpr int buf = decltype(bufc)::value;
        wait_vmcnt<AHEAD>();
        lds_ring_barrier();
        // h's next slice: with two sets of registers now, before the loads of W, which may then
        // stay in flight when it is waited for; with one as the products let go of it
        constexpr int set_a = C::SETS == 2 ? buf & 1 : 0;
        if constexpr (C::SETS == 2) {
#pragma unroll
            for (int ks = 0; ks < 4; ++ks) load_a(kt + 1, ks, set_a ^ 1);
            __builtin_amdgcn_sched_barrier(0);
        }
        issue(kt + C::NS - 1, (buf + C::NS - 1) % C::NS);
        __builtin_amdgcn_sched_barrier(0);
        read_b(bufc, 0, 0);
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
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf[set][j], af[set_a][ks][i],
                                                                        acc[i][j], 0, 0, 0);
            if constexpr (C::SETS == 1) load_a(kt + 1, ks, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        // the products stay in their slice
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j) asm volatile("" : "+v"(acc[i][j]));
    };
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
    wait_vmcnt<0>();  // the zeros of slices past the last are in LDS
    __syncthreads();
#else
    (void)h, (void)runs, (void)w, (void)N, (void)ldw, (void)d, (void)m0, (void)n0, (void)sm, (void)acc;
#endif
}

// Tile (m0, vt) of the logits of h's first M rows: part[t * nvt + vt] = (m, s, m', s'), the
// maximum and the sum of 2^15 e^(z - m) of row t over each of the tile's two units of 64 columns, the
// target's column left out; with sums z_sum[t * nvt + vt], the sum of z over the tile, that
// column included; the workgroup holding target[t] writes z_y[t]. With KEEP e [M, ld_e] receives
// 2^15 e^(z - m) in fp16 (0 in the target's column). Each unit has a maximum of its own so that a
// wave needs no other for its exponentials: with one for 256 columns, and a barrier
// before it, the tile took 4% longer. Sums run in the same order whatever the tile's height, so
// that equal rows have equal results.
template <class C, bool KEEP>
__device__ __forceinline__ void xent_tile(const uint8_t* __restrict__ h, int64_t M,
                                          const uint16_t* __restrict__ w, int64_t V, int64_t ldw,
                                          int64_t d, const int32_t* __restrict__ target, bool sums,
                                          int64_t nvt, float4* __restrict__ part,
                                          float* __restrict__ z_sum, float* __restrict__ z_y,
                                          uint16_t* __restrict__ e, int64_t ld_e,
                                          typename C::Smem& sm, int64_t m0, int64_t vt) {
#pragma clang fp contract(off)  // the same roundings in every configuration
    const int64_t n0 = vt * C::BN;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const int wr = (wave / C::WN) * 32 + (lane & 31), wc = (wave % C::WN) * (C::BN / C::WN);
    // the targets before the K loop, which their latency hides behind
    int32_t ys[C::TM];
#pragma unroll
    for (int i = 0; i < C::TM; ++i) {
        const int64_t t = m0 + wr + i * C::RS;
        ys[i] = t < M ? target[t] : -1;
    }
    f32x16 acc[C::TM][C::TN];
    xent_product<C>(h, (M + 31) / 32, w, V, ldw, d, m0, n0, sm, acc);

    constexpr int CPR = C::TN * 4, RPI = 64 / CPR;  // 16-byte chunks a row, rows a store
#pragma unroll
    for (int i = 0; i < C::TM; ++i) {
        const int row = wr + i * C::RS;
#pragma unroll
        for (int u = 0; u < C::TN / 2; ++u) {
            const int64_t u0 = n0 + wc + u * kStatsUnit;
            // the columns and the target within the unit, as in stats_of_tile
            const int vlim = (int)max(min(V - u0, (int64_t)kStatsUnit), (int64_t)0);
            const int64_t yrel = (int64_t)ys[i] - u0;
            const int y64 = yrel >= 0 && yrel < vlim ? (int)yrel : -1;
            float zs = 0.f;
            const bool masked = vlim < kStatsUnit || (y64 >= 0 && ((y64 >> 2) & 1) == half);
            if (masked) {
                float zy = 0.f;
                int vl = vlim - half * 4, yl = y64 - half * 4;
                asm volatile("" : "+v"(vl), "+v"(yl));  // as in stats_of_tile
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v) {
                        const int col = j * 32 + (v >> 2) * 8 + (v & 3);
                        const float x = acc[i][2 * u + j][v];
                        const bool at_y = col == yl;
                        zy = at_y ? x : zy;
                        zs += col >= vl ? 0.f : x;
                        acc[i][2 * u + j][v] = col >= vl || at_y ? -INFINITY : x;
                    }
                if (y64 >= 0 && ((y64 >> 2) & 1) == half) z_y[m0 + row] = zy;
            } else if (sums) {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int v = 0; v < 16; ++v) zs += acc[i][2 * u + j][v];
            }
            float m = -INFINITY;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) m = fmaxf(m, acc[i][2 * u + j][v]);
            m = fmaxf(m, __shfl_xor(m, 32));
            // nothing but the target: every exponential is 0
            const float ml = (m == -INFINITY ? 0.f : m * kLog2e) - (float)kShift;
            float s2[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                s2[j] = 0.f;
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const float x =
                        __builtin_amdgcn_exp2f(fmaf(acc[i][2 * u + j][v], kLog2e, -ml));
                    acc[i][2 * u + j][v] = x;
                    s2[j] += x;
                }
            }
            float s = s2[0] + s2[1];
            s += __shfl_xor(s, 32);
            if (sums) zs += __shfl_xor(zs, 32);
            if (half == 0) {
                const int unit = wc / kStatsUnit + u;
                sm.units[0][unit][row] = m;
                sm.units[1][unit][row] = s;
                sm.units[2][unit][row] = zs;
            }
        }
        if constexpr (KEEP) {
            // through the wave's own part of the LDS, as in lmhead_dlogits_tile
#pragma unroll
            for (int j = 0; j < C::TN; ++j)
#pragma unroll
                for (int v = 0; v < 16; v += 4) {
                    const f32x16& a = acc[i][j];
                    *reinterpret_cast<u32x2*>(&sm.c16[row][wc + j * 32 + (v >> 2) * 8 + half * 4]) =
                        pack_half4(a[v], a[v + 1], a[v + 2], a[v + 3]);
                }
            lds_wave_order();
#pragma unroll
            for (int q = 0; q < 32 / RPI; ++q) {
                const int r = (wave / C::WN) * 32 + i * C::RS + q * RPI + lane / CPR;
                const int c = wc + lane % CPR * 8;
                const int64_t t = m0 + r, col = n0 + c;
                if (t >= M || col >= V) continue;
                // rows are padded to whole vectors
                const u32x4 pk = *reinterpret_cast<const u32x4*>(&sm.c16[r][c]);
                __builtin_nontemporal_store(pk, reinterpret_cast<u32x4*>(e + t * ld_e + col));
            }
        }
    }
    lds_ring_barrier();
    for (int r = tid; r < C::BM && m0 + r < M; r += C::THREADS) {
        const int64_t at = (m0 + r) * nvt + vt;
        part[at] = make_float4(sm.units[0][0][r], sm.units[1][0][r], sm.units[0][1][r],
                               sm.units[1][1][r]);
        if (sums) z_sum[at] = sm.units[2][0][r] + sm.units[2][1][r];
    }
}

// The block's rows are its first *n_rows - base: the tiles are laid over theirs, so that they
// spread over every XCD, and the workgroups past them have nothing to do.
template <class C, bool KEEP>
__global__ void __launch_bounds__(C::THREADS, 2)
xent_tile_kernel(const uint8_t* __restrict__ h, int64_t M, const uint16_t* __restrict__ w, int64_t V,
                 int64_t ldw, int64_t d, const int32_t* __restrict__ target, int sums, int64_t nvt,
                 float4* __restrict__ part, float* __restrict__ z_sum, float* __restrict__ z_y,
                 uint16_t* __restrict__ e, int64_t ld_e, const int32_t* __restrict__ n_rows,
                 int64_t base) {
    __shared__ typename C::Smem sm;
    const int64_t live = (int64_t)*n_rows - base;
    M = live < M ? (live > 0 ? live : 0) : M;
    const int64_t nmt = (M + C::BM - 1) / C::BM;
    if ((int64_t)blockIdx.x >= nmt * nvt) return;
    int64_t mt, vt;
    tile_of_block(nmt, nvt, mt, vt);
    with_rows_of<C>(M, mt * C::BM, [&](auto c) {
        xent_tile<decltype(c), KEEP>(h, M, w, V, ldw, d, target, sums != 0, nvt, part, z_sum, z_y, e,
                                     ld_e, sm, mt * C::BM, vt);
    });
}

// The objective's constants.
struct XentTerms {
    float eps, lambda;
};

// A row's maximum, normaliser and sum.
struct RowSums {
    float m, s;
    double z;
};
__device__ __forceinline__ RowSums joined(const RowSums& a, const RowSums& b) {
    RowSums r = {fmaxf(a.m, b.m), 0.f, a.z + b.z};
    // an empty part's s is 0, and its maximum may be that of both
    r.s = (a.s == 0.f ? 0.f : a.s * expf(a.m - r.m)) + (b.s == 0.f ? 0.f : b.s * expf(b.m - r.m));
    return r;
}

// One workgroup of THREADS per row r of the block (of its first *n_rows - base): merges the
// row's triples (lane-strided in index order, then a butterfly, then the waves in order),
// adds the target logit last as lmhead_merge_kernel does, and writes the row's loss to
// tok_loss[map[r]]. With KEEP the row of e becomes dz / (1 - eps) in bf16, in place; where there
// are few rows by segs workgroups, which all merge the row and then take a segment of it each.
template <int THREADS, bool KEEP>
__global__ void __launch_bounds__(THREADS)
xent_rows_kernel(const float4* __restrict__ part, const float* __restrict__ z_sum,
                 const float* __restrict__ z_y, int64_t nvt, int64_t V,
                 const int32_t* __restrict__ target, const int32_t* __restrict__ map,
                 XentTerms terms, uint16_t* __restrict__ e, int64_t ld_e,
                 float* __restrict__ tok_loss, const int32_t* __restrict__ n_rows, int64_t base,
                 int64_t segs) {
    constexpr int WAVES = THREADS / 64;
    __shared__ RowSums waves[WAVES];
    const int tid = threadIdx.x, lane = tid & 63;
    const int64_t r = blockIdx.x / segs, seg = blockIdx.x % segs;
    // (the row's own values all at once: they exist also past the labelled rows)
    const int32_t y = target[r], row_to = map[r];
    const float zy = z_y[r];
    if (r >= (int64_t)*n_rows - base) return;
    const int64_t chunks = (V + 7) / 8;
    [[maybe_unused]] u32x4* row = KEEP ? reinterpret_cast<u32x4*>(e + r * ld_e) : nullptr;
    RowSums x = {-INFINITY, 0.f, 0.0};
    for (int64_t j = tid; j < nvt; j += THREADS) {
        const float4 p = part[r * nvt + j];
        const double z = terms.eps > 0.f ? (double)z_sum[r * nvt + j] : 0.0;
        x = joined(x, joined(RowSums{p.x, p.y, z}, RowSums{p.z, p.w, 0.0}));
    }
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) {
        const RowSums o = {__shfl_xor(x.m, off), __shfl_xor(x.s, off), __shfl_xor(x.z, off)};
        // the lower lane's first, so that both lanes round the same
        x = lane & off ? joined(o, x) : joined(x, o);
    }
    if constexpr (WAVES > 1) {
        if (lane == 0) waves[tid >> 6] = x;
        __syncthreads();
        x = waves[0];
        for (int k = 1; k < WAVES; ++k) x = joined(x, waves[k]);
    }
    // the target last: lse = M + log S, logp from -log1p(s_rest / e_y) when it dominates
    // (x.s is 0 where there is no other column, a NaN where a logit is none)
    x.s *= 0x1p-15f;
    const float M = x.s != 0.f ? fmaxf(x.m, zy) : zy;
    const float sx = x.s != 0.f ? x.s * expf(x.m - M) : 0.f, ey = expf(zy - M);
    const float ln_s = logf(sx + ey), lse = M + ln_s;
    const float logp = sx < ey ? -log1pf(sx / ey) : (zy - M) - ln_s;
    if (tid == 0 && seg == 0) {
        const double l = (double)lse;
        double loss = -(double)logp * (1.0 - (double)terms.eps) + (double)terms.lambda * l * l;
        if (terms.eps > 0.f) loss += (double)terms.eps * (l - x.z / (double)V);
        tok_loss[row_to] = (float)loss;
    }
    if constexpr (KEEP) {
        const float keep = 1.f / (1.f - terms.eps), g = 1.f + 2.f * terms.lambda * lse;
        const float flat = terms.eps / (float)V * keep, a = g * keep * 0x1p-15f;
        // (p g - (1 - eps) - eps / V) / (1 - eps), p - 1 = expm1(log p)
        const float dy =
            (expm1f(logp) + terms.eps + 2.f * terms.lambda * lse * expf(logp)) * keep - flat;
        typedef _Float16 h8 __attribute__((ext_vector_type(8)));
        const float* units = reinterpret_cast<const float*>(part + r * nvt);  // (m, s) of each
        const int64_t each = (chunks + segs - 1) / segs, end = min(chunks, (seg + 1) * each);
        for (int64_t c = seg * each + tid; c < end; c += THREADS) {
            const h8 q = __builtin_bit_cast(h8, row[c]);
            // the maximum of the chunk's unit
            const float m = units[c / (kStatsUnit / 8) * 2];
            const float f = m == -INFINITY ? 0.f : a * expf(m - lse);
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = fmaf((float)q[k], f, -flat);
            if (c == y >> 3)
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = k == (y & 7) ? dy : v[k];
            row[c] = u32x4{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                           pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
        }
    }
}

// The labels' count and the gradients' factor, written by one work-item: (1 - eps) / n, or
// 1 - eps for a sum; 0 without labels.
struct LabelOut {
    int32_t *count, *n_valid;
    float* scale;
    float eps;
    int mean;
};
__device__ __forceinline__ void put_labels(const LabelOut& o, int64_t n) {
    o.count[0] = (int32_t)n;
    o.n_valid[0] = (int32_t)n;
    const double f = 1.0 - (double)o.eps;
    o.scale[0] = n == 0 ? 0.f : (float)(o.mean ? f / (double)n : f);
}

// Where the labelled rows go: their hidden rows in panels, block by block of R rows, and (unless
// null) row-major, and their targets.
struct Placed {
    uint8_t* panels;
    uint16_t* rows;
    int32_t* target;
    int64_t R;
};

// Row t with a label: its hidden row and target to row `at` of the labelled ones. Without: its
// row of dh (unless null) and its loss set to 0. By a workgroup of THREADS.
template <int THREADS>
__device__ __forceinline__ void place_row(int64_t t, int64_t at, const uint16_t* __restrict__ h,
                                          int64_t ld_h, int64_t d, int32_t y, const Placed& to) {
    const u32x4* src = reinterpret_cast<const u32x4*>(h + t * ld_h);
    u32x4* dst = to.rows ? reinterpret_cast<u32x4*>(to.rows + at * d) : nullptr;
    const int64_t slices = (d + kSliceK - 1) / kSliceK, block = at / to.R, r = at - block * to.R;
    uint8_t* panels = to.panels + block * ((to.R + 31) / 32) * slices * kPanel;
    for (int64_t c = threadIdx.x; c < slices * 8; c += THREADS) {
        const u32x4 v = c < d / 8 ? src[c] : u32x4{0u, 0u, 0u, 0u};
        *reinterpret_cast<u32x4*>(panels + panel_at(r, c, slices)) = v;
        if (dst && c < d / 8) dst[c] = v;
    }
    if (threadIdx.x == 0) to.target[at] = y;
}
template <int THREADS>
__device__ __forceinline__ void clear_row(int64_t t, int64_t d, float* __restrict__ tok_loss,
                                          uint16_t* __restrict__ dh, int64_t ld_dh) {
    if (dh)
        for (int64_t c = threadIdx.x; c < d; c += THREADS) dh[t * ld_dh + c] = 0;
    if (threadIdx.x == 0) tok_loss[t] = 0.f;
}

// One workgroup per row t: finds the row's place among the labelled ones by counting the labels
// before it, and places or clears it; the first workgroup counts them all. For few rows
// (kFewRows), as its counting grows with T^2 and a launch less counts in short calls. Half the
// rows labelled, us by it and by the two kernels below (which are a launch more, about 5 us where
// the launches bound the call):
//   T          48          1000         4096          8192          16384          32768
//   d = 512    3.4  5.3    4.2  5.8     8.8  9.6      13.9  16.0    27.7   26.5    72.0   49.0
//   d = 3584   3.7  6.6    7.8  9.9     19.0 23.9     35.2  41.8    120    142     198    200
// They cross between 12288 (20.4 and 22.2 at d = 512) and 32768 rows; kFewRows is well below it, at
// sizes where the call takes milliseconds and either is within 7 us of the other.
constexpr int kPrepareThreads = 256;
constexpr int64_t kFewRows = 4096;
__global__ void __launch_bounds__(kPrepareThreads)
xent_prepare_kernel(const int32_t* __restrict__ target, int64_t T, int64_t V,
                    const uint16_t* __restrict__ h, int64_t ld_h, int64_t d,
                    int32_t* __restrict__ map, Placed to, float* __restrict__ tok_loss,
                    uint16_t* __restrict__ dh, int64_t ld_dh, LabelOut out) {
    __shared__ int waves[kPrepareThreads / 64];
    const int64_t t = blockIdx.x;
    const int tid = threadIdx.x;
    const int32_t y = target[t];
    const bool labelled = has_label(y, V);
    if (!labelled) clear_row<kPrepareThreads>(t, d, tok_loss, dh, ld_dh);
    if (!labelled && t > 0) return;
    // the first row's workgroup, which has none before it, counts all
    const int64_t end = t > 0 ? t : T;
    int n = 0;
#pragma unroll 4
    for (int64_t i = tid; i < end; i += kPrepareThreads) n += has_label(target[i], V);
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) n += __shfl_xor(n, off);
    if ((tid & 63) == 0) waves[tid >> 6] = n;
    __syncthreads();
    n = 0;
    for (int k = 0; k < kPrepareThreads / 64; ++k) n += waves[k];
    if (t == 0) {
        if (tid == 0) put_labels(out, n);
        if (!labelled) return;
        n = 0;
    }
    if (tid == 0) map[n] = (int32_t)t;
    place_row<kPrepareThreads>(t, n, h, ld_h, d, y, to);
}

// One workgroup: the rows with a label in increasing order in map, and their number.
constexpr int kLabelThreads = 1024;
__global__ void __launch_bounds__(kLabelThreads)
xent_labels_kernel(const int32_t* __restrict__ target, int64_t T, int64_t V,
                   int32_t* __restrict__ map, LabelOut out) {
    __shared__ int wave_n[2][kLabelThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int64_t base = 0;
    for (int64_t t0 = 0, k = 0; t0 < T; t0 += kLabelThreads, ++k) {
        const int64_t t = t0 + tid;
        const bool keep = t < T && has_label(target[t], V);
        const uint64_t ballot = __ballot(keep);
        const int before = __popcll(ballot & ((uint64_t(1) << lane) - 1));
        if (lane == 0) wave_n[k & 1][wave] = __popcll(ballot);
        __syncthreads();  // the other half is free: its readers are past the last barrier
        int off = 0, total = 0;
        for (int w = 0; w < kLabelThreads / 64; ++w) {
            off += w < wave ? wave_n[k & 1][w] : 0;
            total += wave_n[k & 1][w];
        }
        if (keep) map[base + off + before] = (int32_t)t;
        base += total;
    }
    if (tid == 0) put_labels(out, base);
}

// Row i < count: row map[i] placed; and row i cleared where it has no label. One workgroup per
// row, grid-stride.
__global__ void __launch_bounds__(128)
xent_gather_kernel(const int32_t* __restrict__ map, const int32_t* __restrict__ count, int64_t T,
                   int64_t V, const uint16_t* __restrict__ h, int64_t ld_h, int64_t d,
                   const int32_t* __restrict__ target, Placed to, float* __restrict__ tok_loss,
                   uint16_t* __restrict__ dh, int64_t ld_dh) {
    const int64_t n = count[0];
    for (int64_t i = blockIdx.x; i < T; i += gridDim.x) {
        if (!has_label(target[i], V)) clear_row<128>(i, d, tok_loss, dh, ld_dh);
        if (i < n) place_row<128>(map[i], i, h, ld_h, d, target[map[i]], to);
    }
}

// The last launch. Workgroup 0 (where loss is not null): the loss, summed in fp64 in a fixed
// order. The others (where parts is not null): the ksplit parts of the block's rows of dh
// ([rows, d] fp32 each, stride elements apart) added up in part order, rounded to bf16 and put
// where they belong (row map[r]), rows below *n_rows - base; four columns a work-item at a time,
// grid-stride.
constexpr int kFinishThreads = 512;
struct DhParts {
    const float* parts;
    int64_t ksplit, stride, rows, d;
    const int32_t* map;
    uint16_t* dh;
    int64_t ld_dh, base;
};
__global__ void __launch_bounds__(kFinishThreads)
xent_finish_kernel(const float* __restrict__ tok_loss, int64_t T, int mean,
                   const int32_t* __restrict__ n_rows, float* __restrict__ loss, DhParts p) {
    const int tid = threadIdx.x;
    const int64_t n = *n_rows;
    if (blockIdx.x > 0 || !loss) {
        const int64_t live = n - p.base, rows = live < p.rows ? live : p.rows;
        const int64_t first = blockIdx.x - (loss ? 1 : 0), wgs = gridDim.x - (loss ? 1 : 0);
        for (int64_t i = first * kFinishThreads + tid; i * 4 < rows * p.d; i += wgs * kFinishThreads) {
            const f32x4* q = reinterpret_cast<const f32x4*>(p.parts) + i;  // d % 8 == 0
            f32x4 x = q[0];
#pragma unroll 8
            for (int64_t k = 1; k < p.ksplit; ++k) x += q[k * (p.stride / 4)];
            const int64_t r = i * 4 / p.d;
            uint16_t* o = p.dh + p.map[r] * p.ld_dh + (i * 4 - r * p.d);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = bf16_bits(x[e]);
        }
        return;
    }
    __shared__ double waves[kFinishThreads / 64];
    double x = 0.0;
    for (int64_t t = tid; t < T; t += kFinishThreads) x += (double)tok_loss[t];
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) x += __shfl_xor(x, off);
    if ((tid & 63) == 0) waves[tid >> 6] = x;
    __syncthreads();
    if (tid) return;
    for (int k = 1; k < kFinishThreads / 64; ++k) x += waves[k];
    loss[0] = (float)(mean && n > 0 ? x / (double)n : x);
}

__device__ __forceinline__ void scale_by(float& x, float f) { x *= f; }
__device__ __forceinline__ void scale_by(uint16_t& x, float f) {
    x = bf16_bits(__uint_as_float((uint32_t)x << 16) * f);
}

// x *= *factor, rows of it by a workgroup, grid-stride; 16 bytes a lane with VEC.
constexpr int kScaleThreads = 256;
template <class X, bool VEC>
__global__ void __launch_bounds__(kScaleThreads)
grad_scale_kernel(X* __restrict__ x, int64_t rows, int64_t cols, int64_t ld,
                  const float* __restrict__ factor) {
    const float f = *factor;
    if (f == 1.f) return;
    constexpr int N = VEC ? 16 / sizeof(X) : 1;
    typedef X Some __attribute__((ext_vector_type(N)));
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = (int64_t)threadIdx.x * N; c < cols; c += kScaleThreads * N) {
            Some* p = reinterpret_cast<Some*>(x + r * ld + c);
            Some v = *p;
#pragma unroll
            for (int k = 0; k < N; ++k) {
                X one = v[k];
                scale_by(one, f);
                v[k] = one;
            }
            *p = v;
        }
}

constexpr int64_t kRowBlocksMost = 65536;
int64_t ceil8(int64_t x) { return (x + 7) / 8 * 8; }

// Parts of a block's dh sum over the vocabulary, as in the LM head's backward: dh's few tiles have
// long sums, and the launch waits for them while they fill only some of the units. At most as
// many as give every unit a part (of small tiles two); none shorter than four slices of 64; and, as a slice takes
// kSliceUs where few tiles run, and a part is written and read once more (rows * d * 8 bytes at 4
// TB/s) and waited for (kPartUs), the n that makes slices * kSliceUs / n + n * part least. (48
// rows of V = 4000, d = 512: the products 66 us in one part, 15 in 7, 12 in 15.)
constexpr double kSliceUs = 0.75, kPartUs = 0.1;
int64_t dh_parts(int64_t rows, int64_t d, int64_t V, bool small) {
    const int64_t side = small ? 128 : 256, room = small ? 2 * kUnits : kUnits;
    const int64_t tiles = ((rows + side - 1) / side) * ((d + side - 1) / side);
    const int64_t by_units = room / tiles, by_k = V / (LmCfg::BK * 4);
    const double slices = (double)V / LmCfg::BK;
    const double part_us = (double)rows * (double)d * 8 / 4e6 + kPartUs;
    const int64_t best = (int64_t)sqrt(slices * kSliceUs / part_us);
    const int64_t n = by_units < by_k ? by_units : by_k;
    return n < best ? (n > 1 ? n : 1) : (best > 1 ? best : 1);
}

// Whether a block's two products take the small tiles: three of them share a unit, so that their
// beginnings and stores, most of a dW tile where it has few slices (rows), are hidden; they fill
// the units where the large ones are few, and half as many columns are empty where d is
// short of a large one. The large ones load half as much for each product and win elsewhere. Of
// 110 calls measured (T from 16 to 4096, V from 1000 to 152064, d from 64 to 3584; whole calls) the
// rule takes the small ones in 75: 74 of them are faster, by 10% on average and 23% at most (2007 rows of
// V = 2864, d = 152: 73 -> 56 us; 48 of V = 4000, d = 512: 33.4 -> 29.7), one slower (49 of V =
// 113040, d = 1024: 182 -> 190). 4096 rows of V = 152064, d = 3584 would go from 11.2 to 16.8 ms.
bool small_tiles(int64_t rows, int64_t d, int64_t V) {
    const double large = ceil((double)V / 256) * ceil((double)d / 256);  // dW's
    return d <= 128 || large <= 52 || (rows <= 320 && large <= 2000);
}

// Where a call's parts sit in the workspace (byte offsets, each 256-byte aligned).
struct XentPlan {
    int64_t rows;   // a block's
    bool acc_w;     // dW summed over blocks in fp32
    int64_t ksplit; // parts of dh's sum over the vocabulary
    bool small;     // tiles of the two products
    size_t e, part, z_sum, z_y, count, scale, map, target_c, h_c, panels, accw, parts, total;
};

// total = 0 when the sizes do not fit the address arithmetic. rows: a block's (grad), or
// T (forward alone).
XentPlan plan_xent(int64_t T, int64_t d, int64_t V, int64_t rows, bool grad, bool want_w) {
    XentPlan P = {};
    P.rows = rows < T ? rows : T;
    P.acc_w = grad && want_w && P.rows < T;
    P.small = grad && small_tiles(P.rows, d, V);
    P.ksplit = grad ? dh_parts(P.rows, d, V, P.small) : 1;
    const double big = double(int64_t(1) << 60), nvt = (double)column_tiles(V);
    if ((double)P.rows * (double)ceil8(V) * 2 > big || (double)V * (double)d * 4 > big ||
        (double)T * ((double)d + 64) * 128 > big || (double)P.rows * nvt * 16 > big)
        return P;
    size_t end = 0;
    auto take = [&](size_t bytes) {
        const size_t at = (end + 255) / 256 * 256;
        end = at + bytes;
        return at;
    };
    P.count = take(4);
    P.scale = take(4);
    P.part = take((size_t)P.rows * (size_t)column_tiles(V) * sizeof(float4));
    P.z_sum = take((size_t)P.rows * (size_t)column_tiles(V) * sizeof(float));
    P.z_y = take((size_t)P.rows * 4);
    P.map = take((size_t)T * 4);
    P.target_c = take((size_t)T * 4);
    if (grad) P.h_c = take((size_t)T * (size_t)d * 2);
    const int64_t blocks = (T + P.rows - 1) / P.rows, runs = (P.rows + 31) / 32;
    P.panels = take((size_t)blocks * (size_t)runs * (size_t)slices_of(d) * kPanel);
    if (grad) P.e = take((size_t)P.rows * (size_t)ceil8(V) * 2);
    if (P.acc_w) P.accw = take((size_t)V * (size_t)d * 4);
    if (P.ksplit > 1) P.parts = take((size_t)P.ksplit * (size_t)P.rows * (size_t)d * 4);
    P.total = end;
    return P;
}

bool bad_terms(const dart_xent_config_t* c) {
    return !c || !(c->label_smoothing >= 0.f) || !(c->label_smoothing < 1.f) ||
           !(c->z_loss >= 0.f) || isinf(c->z_loss) ||
           (c->reduction != DART_XENT_MEAN && c->reduction != DART_XENT_SUM);
}

bool bad_inputs(const void* hidden, int64_t T, int64_t d, int64_t ld_h, const void* weight,
                int64_t V, int64_t ld_w, const int32_t* target) {
    if (!hidden || !weight || !target) return true;
    if (T < 1 || V < 1 || d < 8 || T > 0x7FFFFFFFll || V > 0x7FFFFFFFll || d > 0x7FFFFFFFll)
        return true;
    if (d % 8 || ld_h < d || ld_w < d || ld_h % 8 || ld_w % 8) return true;
    return reinterpret_cast<uintptr_t>(hidden) % 16 || reinterpret_cast<uintptr_t>(weight) % 16;
}

// f(configuration that forms rows x V logits fastest); times in us at d = 3584 (fastest_height).
// Of 135 calls measured (T from 40 to 4000, V from 1088 to 152064, d = 256, 1024 and 3584) the
// choice is within 11% of the fastest of the three, 0.4% on average.
template <class F>
void with_xent_cfg(int64_t rows, int64_t V, F&& f) {
    const int bm = fastest_height(rows, column_tiles(V), {33, 40, 52}, {22, 29, 48}, 1.5);
    if (bm == 64)
        f(X64{});
    else if (bm == 128)
        f(X128{});
    else
        f(X256{});
}

// f(threads of a row's workgroup): about 16 vectors of eight columns each, which take turns with
// the row's other latencies. 1220 rows of V = 1088: 16 us with 512, 7.6 with 64.
template <class F>
void with_row_threads(int64_t V, F&& f) {
    if (V <= 2048)
        f(std::integral_constant<int, 64>{});
    else if (V <= 8192)
        f(std::integral_constant<int, 128>{});
    else if (V <= 32768)
        f(std::integral_constant<int, 256>{});
    else
        f(std::integral_constant<int, 512>{});
}

// Workgroups that share a row of e: as many as there is room for beside the other rows, each with
// two rounds of its threads at least. 36 rows of V = 62036: 15 us by one each, 12 by 7.
int64_t row_segments(int64_t rows, int64_t V, int threads) {
    const int64_t room = 1024 / rows, most = (V + 7) / 8 / (2 * threads);
    const int64_t n = room < most ? room : most;
    return n > 1 ? n : 1;
}

// The whole call; without grads the loss alone.
struct XentGrads {
    void* dh;
    int64_t ld_dh;
    void* dw;
    int64_t ld_dw;
};
dart_status_t run_xent(const uint16_t* h, int64_t T, int64_t d, int64_t ld_h, const uint16_t* w,
                       int64_t V, int64_t ld_w, const int32_t* target,
                       const dart_xent_config_t& config, float* loss, float* tok_loss,
                       int32_t* n_valid, const XentGrads* grads, const XentPlan& P, char* ws,
                       hipStream_t stream) {
    const int64_t nvt = column_tiles(V);
    const int mean = config.reduction == DART_XENT_MEAN;
    const XentTerms terms = {config.label_smoothing, config.z_loss};
    int32_t* count = reinterpret_cast<int32_t*>(ws + P.count);
    float* scale = reinterpret_cast<float*>(ws + P.scale);
    float4* part = reinterpret_cast<float4*>(ws + P.part);
    float* z_sum = reinterpret_cast<float*>(ws + P.z_sum);
    float* z_y = reinterpret_cast<float*>(ws + P.z_y);
    const int sums = config.label_smoothing > 0.f;
    int32_t* map = reinterpret_cast<int32_t*>(ws + P.map);
    // row-major for dW's product alone
    uint16_t* h_c = grads ? reinterpret_cast<uint16_t*>(ws + P.h_c) : nullptr;
    const uint8_t* panels = reinterpret_cast<uint8_t*>(ws + P.panels);
    int32_t* target_c = reinterpret_cast<int32_t*>(ws + P.target_c);
    const LabelOut out = {count, n_valid, scale, config.label_smoothing, mean};
    uint16_t* dh_rows = grads ? static_cast<uint16_t*>(grads->dh) : nullptr;
    const int64_t ld_dh = grads ? grads->ld_dh : 0;
    const Placed to = {reinterpret_cast<uint8_t*>(ws + P.panels), h_c, target_c, P.rows};
    if (T <= kFewRows) {
        hipLaunchKernelGGL(xent_prepare_kernel, dim3((unsigned)T), dim3(kPrepareThreads), 0, stream,
                           target, T, V, h, ld_h, d, map, to, tok_loss, dh_rows, ld_dh, out);
    } else {
        hipLaunchKernelGGL(xent_labels_kernel, dim3(1), dim3(kLabelThreads), 0, stream, target, T, V,
                           map, out);
        hipLaunchKernelGGL(xent_gather_kernel,
                           dim3((unsigned)(T < kRowBlocksMost ? T : kRowBlocksMost)), dim3(128), 0,
                           stream, map, count, T, V, h, ld_h, d, target, to, tok_loss, dh_rows, ld_dh);
    }
    uint16_t* e = grads ? reinterpret_cast<uint16_t*>(ws + P.e) : nullptr;
    const int64_t ld_e = ceil8(V);
    float* parts = P.ksplit > 1 ? reinterpret_cast<float*>(ws + P.parts) : nullptr;
    const Grad dh{grads ? grads->dh : nullptr, grads ? grads->ld_dh : 0, true};
    const Grad dw{grads ? grads->dw : nullptr, grads ? grads->ld_dw : 0, true};
    const Grad sum_w = P.acc_w ? Grad{ws + P.accw, d, false} : dw;
    auto launch_finish = [&](int64_t blocks, float* to, const DhParts& to_add) {
        hipLaunchKernelGGL(xent_finish_kernel, dim3((unsigned)(blocks + (to ? 1 : 0))),
                           dim3(kFinishThreads), 0, stream, tok_loss, T, mean, count, to, to_add);
    };
    for (int64_t r0 = 0; r0 < T; r0 += P.rows) {
        const int64_t rows = T - r0 < P.rows ? T - r0 : P.rows;
        const uint16_t* hr = grads ? h_c + r0 * d : nullptr;
        const uint8_t* hp = panels + r0 / P.rows * ((P.rows + 31) / 32) * slices_of(d) * kPanel;
        with_xent_cfg(rows, V, [&](auto cfg) {
            using C = decltype(cfg);
            const dim3 grid((unsigned)((rows + C::BM - 1) / C::BM * nvt));
            auto launch = [&](auto kernel) {
                hipLaunchKernelGGL(kernel, grid, dim3(C::THREADS), 0, stream, hp, rows, w, V, ld_w, d,
                                   target_c + r0, sums, nvt, part, z_sum, z_y, e, ld_e, count, r0);
            };
            grads ? launch(xent_tile_kernel<C, true>) : launch(xent_tile_kernel<C, false>);
        });
        if (!grads) {
            hipLaunchKernelGGL((xent_rows_kernel<64, false>), dim3((unsigned)rows), dim3(64), 0,
                               stream, part, z_sum, z_y, nvt, V, target_c + r0, map + r0, terms, e, ld_e,
                               tok_loss, count, r0, int64_t(1));
            continue;
        }
        with_row_threads(V, [&](auto threads) {
            constexpr int N = decltype(threads)::value;
            const int64_t segs = row_segments(rows, V, N);
            hipLaunchKernelGGL((xent_rows_kernel<N, true>), dim3((unsigned)(rows * segs)), dim3(N), 0,
                               stream,
                               part, z_sum, z_y, nvt, V, target_c + r0, map + r0, terms, e, ld_e, tok_loss,
                               count, r0, segs);
        });
        const dart_status_t st = lmhead::launch_bwd_gemms(
            e, ld_e, rows, V, w, ld_w, hr, d, d, parts && dh.p ? Grad{parts, d, false} : dh, false,
            parts ? P.ksplit : 1, P.rows * d, sum_w, P.acc_w && r0 > 0, stream, parts ? nullptr : map + r0,
            count, r0, scale, P.small);
        if (st != DART_OK) return st;
        const DhParts to_add = {parts, P.ksplit, P.rows * d, rows, d, map + r0, dh_rows, ld_dh, r0};
        const bool last = r0 + rows == T;
        const int64_t blocks = (rows * d / 4 + kFinishThreads - 1) / kFinishThreads;
        if (parts && dh.p)
            launch_finish(blocks < kRowBlocksMost ? blocks : kRowBlocksMost, last ? loss : nullptr,
                          to_add);
        else if (last)
            launch_finish(0, loss, to_add);
    }
    if (P.acc_w) lmhead::launch_to_bf16(reinterpret_cast<float*>(ws + P.accw), V, d, dw, stream);
    if (!grads) launch_finish(0, loss, DhParts{});
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

// Launch limits: the tiles (the least of them, 64 rows), one workgroup of 512 per row of a block,
// and the tiles' 32-bit offsets.
bool too_large(int64_t rows, int64_t V, int64_t ld_h, int64_t ld_w) {
    return !grid_fits((rows + X64::BM - 1) / X64::BM * column_tiles(V), X64::THREADS) ||
           !grid_fits(rows, 512) || ld_h > kMaxLd || ld_w > kMaxLd;
}
// the tile's rows of W and, slices past its last included, a run of panels (d <= kMaxLd)
static_assert(rows_bytes(kTileN, kMaxLd, kMaxLd) < int64_t(1) << 31 &&
                  (kMaxLd / kSliceK + 4) * kPanel < int64_t(1) << 31,
              "32-bit offsets");

}  // namespace

extern "C" {

size_t dart_lmhead_xent_fwd_workspace_bytes(int64_t T, int64_t d, int64_t V) {
    if (T < 1 || d < 1 || V < 1 || T > 0x7FFFFFFFll || d > 0x7FFFFFFFll || V > 0x7FFFFFFFll) return 0;
    return plan_xent(T, d, V, T, false, false).total;
}

size_t dart_lmhead_xent_workspace_bytes(int64_t T, int64_t d, int64_t V, int64_t chunk_rows) {
    if (T < 1 || d < 1 || V < 1 || chunk_rows < 1 || T > 0x7FFFFFFFll || d > 0x7FFFFFFFll ||
        V > 0x7FFFFFFFll)
        return 0;
    return plan_xent(T, d, V, chunk_rows, true, true).total;
}

dart_status_t dart_lmhead_xent_fwd(const void* hidden, int64_t T, int64_t d, int64_t ld_h,
                                   const void* weight, int64_t V, int64_t ld_w,
                                   const int32_t* target, const dart_xent_config_t* config,
                                   float* loss, float* tok_loss, int32_t* n_valid, void* workspace,
                                   size_t workspace_bytes, hipStream_t stream) {
    if (bad_inputs(hidden, T, d, ld_h, weight, V, ld_w, target) || bad_terms(config) || !loss ||
        !tok_loss || !n_valid || !workspace || reinterpret_cast<uintptr_t>(workspace) % 16)
        return DART_ERR_INVALID_ARG;
    if (too_large(T, V, ld_h, ld_w)) return DART_ERR_UNSUPPORTED;
    const XentPlan P = plan_xent(T, d, V, T, false, false);
    if (P.total == 0) return DART_ERR_UNSUPPORTED;
    if (workspace_bytes < P.total) return DART_ERR_INVALID_ARG;
    if (const dart_status_t ck = dart_check::run(
            stream, {{dart_check::Item::Labels, target, T, V}}); ck != DART_OK)
        return ck;
    return run_xent(static_cast<const uint16_t*>(hidden), T, d, ld_h,
                    static_cast<const uint16_t*>(weight), V, ld_w, target, *config, loss, tok_loss,
                    n_valid, nullptr, P, static_cast<char*>(workspace), stream);
}

dart_status_t dart_lmhead_xent_fwd_bwd(const void* hidden, int64_t T, int64_t d, int64_t ld_h,
                                       const void* weight, int64_t V, int64_t ld_w,
                                       const int32_t* target, const dart_xent_config_t* config,
                                       float* loss, float* tok_loss, int32_t* n_valid,
                                       void* dhidden, int64_t ld_dh, void* dweight, int64_t ld_dw,
                                       int64_t chunk_rows, void* workspace, size_t workspace_bytes,
                                       hipStream_t stream) {
    if (bad_inputs(hidden, T, d, ld_h, weight, V, ld_w, target) || bad_terms(config) || !loss ||
        !tok_loss || !n_valid || !workspace || reinterpret_cast<uintptr_t>(workspace) % 16)
        return DART_ERR_INVALID_ARG;
    if ((!dhidden && !dweight) || (dhidden && ld_dh < d) || (dweight && ld_dw < d) ||
        chunk_rows < 1 || reinterpret_cast<uintptr_t>(dhidden) % 2 ||
        reinterpret_cast<uintptr_t>(dweight) % 2)
        return DART_ERR_INVALID_ARG;
    const int64_t rows = chunk_rows < T ? chunk_rows : T;
    if (too_large(rows, V, ld_h, ld_w) || ceil8(V) > kMaxLd || (dhidden && ld_dh > kMaxLd) ||
        (dweight && ld_dw > kMaxLd))
        return DART_ERR_UNSUPPORTED;
    const XentPlan P = plan_xent(T, d, V, rows, true, dweight != nullptr);
    if (P.total == 0) return DART_ERR_UNSUPPORTED;
    if (workspace_bytes < P.total) return DART_ERR_INVALID_ARG;
    if (const dart_status_t ck = dart_check::run(
            stream, {{dart_check::Item::Labels, target, T, V}}); ck != DART_OK)
        return ck;
    const XentGrads grads = {dhidden, dhidden ? ld_dh : 0, dweight, dweight ? ld_dw : 0};
    return run_xent(static_cast<const uint16_t*>(hidden), T, d, ld_h,
                    static_cast<const uint16_t*>(weight), V, ld_w, target, *config, loss, tok_loss,
                    n_valid, &grads, P, static_cast<char*>(workspace), stream);
}

dart_status_t dart_grad_scale(void* x, dart_dtype_t dtype, int64_t rows, int64_t cols, int64_t ld,
                              const float* factor, hipStream_t stream) {
    const size_t size = dtype == DART_BF16 ? 2 : 4;
    if ((dtype != DART_BF16 && dtype != DART_F32) || !x || !factor || rows < 1 || cols < 1 ||
        rows > 0x7FFFFFFFll || cols > 0x7FFFFFFFll || ld < cols ||
        reinterpret_cast<uintptr_t>(x) % size || reinterpret_cast<uintptr_t>(factor) % 4)
        return DART_ERR_INVALID_ARG;
    const bool vec = reinterpret_cast<uintptr_t>(x) % 16 == 0 && ld * (int64_t)size % 16 == 0 &&
                     cols * (int64_t)size % 16 == 0;
    const dim3 grid((unsigned)(rows < kRowBlocksMost ? rows : kRowBlocksMost)), block(kScaleThreads);
    auto launch = [&](auto kernel, auto* p) {
        hipLaunchKernelGGL(kernel, grid, block, 0, stream, p, rows, cols, ld, factor);
    };
    if (dtype == DART_BF16)
        vec ? launch(grad_scale_kernel<uint16_t, true>, static_cast<uint16_t*>(x))
            : launch(grad_scale_kernel<uint16_t, false>, static_cast<uint16_t*>(x));
    else
        vec ? launch(grad_scale_kernel<float, true>, static_cast<float*>(x))
            : launch(grad_scale_kernel<float, false>, static_cast<float*>(x));
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

}  // extern "C"
