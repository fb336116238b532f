// libdart, LM-head part: the token statistics and the gradient of the
// policy-update hot path computed straight from the LM head's inputs, so that
// the [T, V] logits are never written to memory.
//
// Paper: DART, arXiv 2509.23866. The statistics are those of Sec. 4.3 (token
// entropy, the target's log-prob of Eq. 1) for logits z = h W^T, where h [T, d]
// are the final hidden states of the T action tokens and W [V, d] the LM-head
// weight of the policy (the 7B VLM of Sec. 5.1); the gradient is the chain
// rule of Eq. 2's loss through them. Both kernels apply an inverse sampling
// temperature s (1 in the paper, App. A.4) in their epilogues: the fp32 tile
// stays unscaled, and s enters the factor of the base-2 exponent (s log2 e)
// and the row maximum (s > 0), so that s = 1 changes no bit.
//
//   lmhead_stats_kernel   one 256 x 256 tile of z per workgroup (64 or 128 rows
//                         where T is small) on MFMA
//                         (v_mfma_f32_32x32x16_bf16, fp32 accumulation), K = d
//                         in slices of 64 loaded straight into two LDS buffers;
//                         the tile is reduced in the epilogue to one (max,
//                         normaliser, entropy) triple per row over its 256
//                         columns (the target column kept apart), written to a
//                         workspace.
//   lmhead_merge_kernel   one wave per row: merges the row's V / 256 triples in
//                         a fixed order, adds the target logit, writes logp, H
//                         and lse exactly as tok_stats_kernel defines them.
//   lmhead_dlogits_kernel the same tile, its epilogue writing
//                         dz = g (onehot - softmax) in bf16.
// The backward forms dz block by block (rows x vocabulary entries, the blocked
// entry point optionally over the rows with a non-zero coefficient only) and
// adds dh = dz W and dW = dz^T h per block in one launch of
// lmhead_bwd_gemms_kernel (the same MFMA tile, its operands stored with K as
// their row index read through LDS transpose loads).
#include "lmhead_tile.h"

namespace {

template <class C>
__global__ void __launch_bounds__(C::THREADS)
lmhead_stats_kernel(const uint16_t* __restrict__ h, int64_t T, int64_t ldh,
                    const uint16_t* __restrict__ w, int64_t V, int64_t ldw, int64_t d,
                    const int32_t* __restrict__ target, float scale, int64_t nvt,
                    float4* __restrict__ part, float* __restrict__ z_y) {
    with_row_tile<C>(T, nvt, [&](auto cfg, auto& sm, int64_t m0, int64_t vt) {
        using R = decltype(cfg);
        stats_of_tile<R>(
            [&](int64_t n0, f32x16(&acc)[R::TM][R::TN]) {
                gemm_tile<R>(h, T, ldh, w, V, ldw, d, m0, n0, sm, acc);
            },
            T, V, target, scale, nvt, part, z_y, sm, m0, vt);
    });
}

// dlogits = s g_t (onehot(y_t) - exp(s z - lse_t)) (s = scale, the inverse
// temperature; lse_t that of s z) for rows [0, M) of the block
// (h and out already offset to the block's first row) and the V vocabulary
// entries vbase .. vbase + V - 1 (w already offset to entry vbase), written in
// bf16 (nearest even) to out [M, ld_out]: the gradient pass of the logits
// path with the logits formed on the fly. The target element is
// s g_t * -expm1(logp_t), accurate when p_y -> 1.
template <class C>
__device__ __forceinline__ void lmhead_dlogits_tile(
    const uint16_t* __restrict__ h, int64_t M, int64_t ldh, const uint16_t* __restrict__ w,
    int64_t V, int64_t ldw, int64_t d, const int32_t* __restrict__ target,
    const float* __restrict__ lse, const float* __restrict__ logp, const float* __restrict__ coef,
    float scale, uint16_t* __restrict__ out, int64_t ld_out, int64_t vbase, typename C::Smem& sm,
    int64_t m0, int64_t vt) {
    const int64_t n0 = vt * C::BN;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
    const int wr = (wave / C::WN) * 32 + (lane & 31), wc = (wave % C::WN) * (C::BN / C::WN);
    f32x16 acc[C::TM][C::TN];
    gemm_tile<C>(h, M, ldh, w, V, ldw, d, m0, n0, sm, acc);

    // the inverse temperature enters the base-2 exponent's factor (1 at scale
    // 1: the same bits)
    const float c2 = scale * 1.4426950408889634f;
    // the constants of all of the lane's rows ahead of the first store, which a later
    // load would wait for
    float gs[C::TM], lses[C::TM];
    int32_t ys[C::TM];
#pragma unroll
    for (int i = 0; i < C::TM; ++i) {
        const int64_t t = min(m0 + wr + i * C::RS, M - 1);  // rows past M are not stored
        gs[i] = coef[t], lses[i] = lse[t], ys[i] = target[t];
    }
    // Row blocks of 32 rows x the wave's columns: turned into bf16 in registers, then
    // through the wave's own part of the LDS (its accesses run in order: no barrier), so
    // that a row's 256 bytes leave together while the next block is formed. With the
    // whole tile formed, a barrier, and then every store, the stores came in one burst
    // behind the exponentials, which a short K loop does not hide: at d = 512 1000 rows
    // of V = 32000 took 42.2 us, now 39.9, 4096 of 8000 43.9 and 42.7, at d = 3584 4096
    // of 152064 3439 and 3394. (128 bytes at a time are 1 to 3% better where they are
    // whole lines, but rows of 60328 elements took 343 us in place of 300.)
    constexpr int CPR = C::TN * 4, RPI = 64 / CPR;  // 16-byte chunks a row, rows a store
#pragma unroll
    for (int i = 0; i < C::TM; ++i) {
        // -g, -lse log2(e), the target's gradient g (-expm1(logp)) (accurate when
        // p_y -> 1), the target's column; g carries the inverse temperature (the
        // chain rule through scale z)
        const float g = gs[i] * scale;
        const float neg_g = -g, neg_lse = -lses[i] * 1.4426950408889634f;
        const int64_t yrel = (int64_t)ys[i] - vbase - n0 - wc;
        const int y32 = yrel >= 0 && yrel < C::BN / C::WN ? (int)yrel : -1;
#pragma unroll
        for (int j = 0; j < C::TN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v)
                acc[i][j][v] = neg_g * __builtin_amdgcn_exp2f(fmaf(acc[i][j][v], c2, neg_lse));
        if (y32 >= 0 && ((y32 >> 2) & 1) == half) {
            const float dy = g * -expm1f(logp[min(m0 + wr + i * C::RS, M - 1)]);
#pragma unroll
            for (int j = 0; j < C::TN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) {
                    const int col = j * 32 + (v >> 2) * 8 + (v & 3);
                    acc[i][j][v] = col == y32 - half * 4 ? dy : acc[i][j][v];
                }
        }
        blocks_to_lds_bf16<C, C::TN>(acc[i], i, 0, sm);
        lds_wave_order();
#pragma unroll
        for (int q = 0; q < 32 / RPI; ++q) {
            const int r = (wave / C::WN) * 32 + i * C::RS + q * RPI + lane / CPR;
            const int c = wc + lane % CPR * 8;
            const int64_t t = m0 + r, col = n0 + c;
            if (t >= M || col >= V) continue;
            const u32x4 pk = *reinterpret_cast<const u32x4*>(&sm.c16[r][c]);
            uint16_t* dst = out + t * ld_out + col;
            if (col + 8 <= V)
                __builtin_nontemporal_store(pk, reinterpret_cast<u32x4*>(dst));
            else
                for (int k = 0; k < 8 && col + k < V; ++k) dst[k] = sm.c16[r][c + k];
        }
    }
}

// With dyn_rows, the block holds only rows below *dyn_rows - dyn_base (the grid
// covers the most it can hold): the tiles are laid over the live rows' tiles,
// so that they spread over every XCD, and the workgroups past them (the last
// ones dispatched) have nothing to do.
template <class C>
__global__ void __launch_bounds__(C::THREADS)
lmhead_dlogits_kernel(const uint16_t* __restrict__ h, int64_t M, int64_t ldh,
                      const uint16_t* __restrict__ w, int64_t V, int64_t ldw, int64_t d,
                      const int32_t* __restrict__ target, const float* __restrict__ lse,
                      const float* __restrict__ logp, const float* __restrict__ coef,
                      float scale, uint16_t* __restrict__ out, int64_t ld_out, int64_t vbase,
                      int64_t nvt, const int32_t* __restrict__ dyn_rows, int64_t dyn_base) {
    if (dyn_rows) {
        const int64_t live = (int64_t)*dyn_rows - dyn_base;
        M = live < M ? (live > 0 ? live : 0) : M;
    }
    with_row_tile<C>(M, nvt, [&](auto cfg, auto& sm, int64_t m0, int64_t vt) {
        lmhead_dlogits_tile<decltype(cfg)>(h, M, ldh, w, V, ldw, d, target, lse, logp, coef, scale,
                                           out, ld_out, vbase, sm, m0, vt);
    });
}

// ---------------------------------------------------------------------------
// Backward GEMMs on the matrix cores: C[M, N] (+)= A B with B stored [K][N]
// (N contiguous), for dh = dz W (A = the dz block read along its rows, K
// contiguous; B = the block's rows of W) and dW = dz^T h (A = the dz block
// read down its columns, M contiguous; B = the block's rows of h). The tile,
// waves, K slices and LDS ring are those of the forward tile; what differs is
// how an operand stored with K as its row index reaches the MFMA.
//
// Such an operand's slice sits in LDS as BK rows of 256 elements (its k rows
// as they are stored), chunk c (8 elements, 16 bytes) of row k in slot
// c ^ (4 (k mod 4)). The MFMA wants, in lane l, 8 consecutive k of one column;
// ds_read_b64_tr_b16 transposes 4 x 16 blocks within each 16 lanes: lane l
// receives element l % 4 of the 8 bytes that lane 16 (l / 16) + 4 j + (l % 16) / 4
// loaded, for j = 0..3 (whatever addresses the lanes gave). So lane L of a
// group points at row k0 + L / 4, columns 4 (L % 4) .. + 3 of its group's 16
// columns, and receives column L at rows k0 .. k0 + 3; two such reads give the
// 8 k of one MFMA operand. In one read, the 32 lanes of a half-wave take 4
// rows x 32 columns; the swizzle puts the 4 rows' chunks in 16 distinct bank
// quads (gfx950: 64 banks of 4 bytes), so the reads do not conflict.
// ---------------------------------------------------------------------------

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4_ptr;

// Elements of one transposed operand row in LDS (the tile width).
constexpr int kTw = 256;
static_assert(LmCfg::BM == kTw && LmCfg::BN == kTw, "transposed rows are one tile wide");

// Slot of chunk c of row k of a transposed operand tile.
__device__ __forceinline__ int tr_slot(int c, int k) { return c ^ (4 * (k & 3)); }

// acc = this wave's part of C[m0:m0+BM, n0:n0+BN] = A B over k in [kbeg, K), kbeg
// a multiple of BK.
// A_KMAJ: A(m, k) = A[m lda + k], else A(m, k) = A[k lda + m]. B(k, n) =
// B[k ldb + n]. Rows and columns past M, N read zero or whatever lies there
// in the matrices (their results are not stored); k past K is zero in LDS
// (also inside a chunk that straddles K), so the stored row padding up to a
// multiple of 8 may hold anything. lda >= ceil8(K) (A_KMAJ) or ceil8(M),
// ldb >= ceil8(N); rows 16-byte aligned. Layout of acc as in gemm_tile. Ends
// on a barrier with no loads in flight.
template <class C, bool A_KMAJ>
__device__ __forceinline__ void gemm_tile_bwd(const uint16_t* __restrict__ A, int64_t lda,
                                              const uint16_t* __restrict__ B, int64_t ldb,
                                              int64_t M, int64_t N, int64_t kbeg, int64_t K,
                                              int64_t m0, int64_t n0, typename C::Smem& sm,
                                              f32x16 (&acc)[C::TM][C::TN]) {
#if defined(__HIP_DEVICE_COMPILE__)
    static_assert(C::BK == 64 && C::BM == kTw && C::BN == kTw, "backward tile");
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = (wave / C::WN) * 32, wc = (wave % C::WN) * (C::BN / C::WN);
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int j = 0; j < C::TN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;

    constexpr int CH = C::CH, BK = C::BK;
    // transposed operands: one load instruction fills 2 rows of 32 chunks
    constexpr int TQ = BK / 2 / C::WAVES;  // load instructions per wave and slice
    static_assert(TQ * 2 * C::WAVES == BK, "transposed rows per wave");
    const int trow = lane >> 5, tslot = lane & 31;
    const int64_t nk = (K + BK - 1) / BK;

    // Buffer loads into LDS, as in gemm_tile: one per-lane offset VGPR per
    // operand, the instruction's rows and the slice as scalar offsets (or,
    // for a transposed operand, the slice in the resource base). A transposed
    // operand's resource ends at the last element of row K - 1 that exists
    // (columns < ceil8(len)), so k rows past K read as zero; chunks past len
    // within a row read the row padding or the next row (their results are
    // not stored).
    const int lrow = lane / CH, lslot = lane % CH;
    static_assert((C::WAVES * C::LROWS) % (16 / CH * CH) == 0, "swizzle period");
    static_assert(C::WAVES % 2 == 0, "transposed swizzle period");
    const int tr_k = wave * 2 + trow;  // transposed row of the lane in instruction 0
    const int tr_c = 8 * tr_slot(tslot, tr_k);
    uint32_t voff_a, qstride_a;
    if constexpr (A_KMAJ) {
        const int r_lane = wave * C::LROWS + lrow;
        voff_a = (uint32_t)((r_lane * lda + (lslot ^ swz<CH>(r_lane)) * 8) * 2);
        qstride_a = (uint32_t)(C::WAVES * C::LROWS * lda * 2);
    } else {
        voff_a = (uint32_t)((tr_k * lda + tr_c) * 2);
        qstride_a = (uint32_t)(C::WAVES * 2 * lda * 2);
    }
    const uint32_t voff_b = (uint32_t)((tr_k * ldb + tr_c) * 2);
    const uint32_t qstride_b = (uint32_t)(C::WAVES * 2 * ldb * 2);
    const __amdgpu_buffer_rsrc_t rsrc_ak = tile_rsrc(A + m0 * lda, (M - m0) * lda * 2);
    // resource of a transposed operand's slice kt: rows kt*BK .. K-1 from column t0
    auto tr_rsrc = [&](const uint16_t* X, int64_t ld, int64_t t0, int64_t len, int64_t kt) {
        const int64_t first = kt * BK * ld + t0;
        const int64_t end = (K - 1) * ld + (len + 7) / 8 * 8;
        return tile_rsrc(X + first, (end - first) * 2);
    };

    // instruction q of wave `wave + hh * HW`
    constexpr int HW = C::WAVES / 2;
    auto lds_a = [&](int buf, int q, int hh) {
        constexpr int per = A_KMAJ ? C::LROWS * BK : 2 * kTw;  // elements per instruction
        return &sm.in.a[buf][0][0] + (q * C::WAVES + wave + hh * HW) * per;
    };
    auto lds_b = [&](int buf, int q, int hh) {
        return &sm.in.b[buf][0][0] + (q * C::WAVES + wave + hh * HW) * 2 * kTw;
    };

    // As in gemm_tile, the first half of the waves issue every load, their
    // own rows and those of the wave HW above (HW * LROWS K-major rows or
    // 2 HW transposed rows further: whole swizzle periods, so the same lane
    // offsets)
    static_assert((HW * C::LROWS) % 16 == 0 && (2 * HW) % 4 == 0, "swizzle periods");
    const uint32_t hstride_ak = (uint32_t)(HW * C::LROWS * lda * 2);
    const uint32_t hstride_at = (uint32_t)(2 * HW * lda * 2);
    const uint32_t hstride_b = (uint32_t)(2 * HW * ldb * 2);
    auto issue = [&](int64_t kt, int buf) {
        if (wave >= HW) return;
        if constexpr (A_KMAJ) {
            const uint32_t kb = (uint32_t)(kt * BK * 2);
#pragma unroll
            for (int q = 0; q < C::IA; ++q)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(
                        rsrc_ak, lds_ptr(lds_a(buf, q, hh)), 16, voff_a,
                        kb + q * qstride_a + hh * hstride_ak, 0, 0);
        } else {
            const __amdgpu_buffer_rsrc_t ra = tr_rsrc(A, lda, m0, M, kt);
#pragma unroll
            for (int q = 0; q < TQ; ++q)
#pragma unroll
                for (int hh = 0; hh < 2; ++hh)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, lds_ptr(lds_a(buf, q, hh)), 16,
                                                            voff_a, q * qstride_a + hh * hstride_at,
                                                            0, 0);
        }
        const __amdgpu_buffer_rsrc_t rb = tr_rsrc(B, ldb, n0, N, kt);
#pragma unroll
        for (int q = 0; q < TQ; ++q)
#pragma unroll
            for (int hh = 0; hh < 2; ++hh)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rb, lds_ptr(lds_b(buf, q, hh)), 16, voff_b,
                                                        q * qstride_b + hh * hstride_b, 0, 0);
    };
    // the partial last slice of a K-major A: k >= K set to 0, also inside the
    // chunk that straddles K (transposed operands read zero rows there)
    auto zero_tail = [&](int64_t kt, int buf) {
        const int kv = (int)(K - kt * BK);  // valid k in this slice, 1 .. BK-1
        uint16_t* a = &sm.in.a[buf][0][0];
        for (int e = tid; e < BK * kTw; e += C::THREADS) {
            // [BM][BK] rows with swizzled chunks: element e is row e / BK,
            // slot (e % BK) / 8, holding chunk slot ^ swz(row)
            const int r = e / BK, sl = (e % BK) / 8;
            const int kk = ((sl ^ swz<CH>(r)) * 8) + (e % 8);
            if (kk >= kv) a[e] = 0;
        }
    };

    // MFMA operand offsets. A (K-major): as gemm_tile. Transposed: lane l
    // points at row ks*16 + 8 (l / 32) + 4 h + (l / 4) % 4 and columns
    // mb + 16 ((l / 16) % 2) + 4 (l % 4) of its 32-column block mb (a multiple
    // of 32, so the chunk is (mb / 8) | ((l / 16) % 2) * 2 | (l % 4) / 2).
    const int kq = (lane >> 2) & 3;
    const int tr_lane_row = 8 * (lane >> 5) + kq;
    const int tr_delta = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    auto tr_off = [&](int mb) -> uint32_t {
        const int slot = ((mb / 8) ^ (4 * kq)) | tr_delta;
        return (uint32_t)(tr_lane_row * kTw * 2 + slot * 16 + 8 * (lane & 1));
    };
    uint32_t rda[A_KMAJ ? C::KSTEPS : C::TM], rdb[C::TN];
    if constexpr (A_KMAJ) {
#pragma unroll
        for (int ks = 0; ks < C::KSTEPS; ++ks) {
            const int c = ks * 2 + (lane >> 5), ra = wr + (lane & 31);
            rda[ks] = (uint32_t)(ra * BK + (c ^ swz<CH>(ra)) * 8) * 2;
        }
    } else {
#pragma unroll
        for (int i = 0; i < C::TM; ++i) rda[i] = tr_off(wr + i * C::RS);
    }
    // B's offsets carry its buffers' start (64 KB into the LDS), opaque to the
    // compiler, so that the buffer, the k-step and the half enter as the
    // read's 16-bit immediate (as in gemm_tile)
    const char* const lds0 = reinterpret_cast<const char*>(&sm);
    const uint32_t b_at = (uint32_t)(reinterpret_cast<const char*>(&sm.in.b[0][0][0]) - lds0);
#pragma unroll
    for (int j = 0; j < C::TN; ++j) {
        rdb[j] = b_at + tr_off(wc + j * 32);
        asm volatile("" : "+v"(rdb[j]));
    }
    static_assert(C::NS == 2, "two buffers");
    static_assert((C::NS - 1) * C::BN * BK * 2 + (C::KSTEPS - 1) * 16 * kTw * 2 + 4 * kTw * 2 <
                      65536,
                  "B read immediates");

    auto tr_pair = [&](const char* base, uint32_t off, int ks) -> bf16x8 {
        const int k0 = ks * 16 * kTw * 2;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4_ptr)(base + off + k0));
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (lds_s16x4_ptr)(base + off + k0 + 4 * kTw * 2));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        return __builtin_bit_cast(bf16x8, v);
    };
    bf16x8 af[2][C::TM], bfr[2][C::TN];
    auto read_step = [&](auto bufc, int ks, int set) {
        constexpr int buf = decltype(bufc)::value;
        const char* ba = reinterpret_cast<const char*>(&sm.in.a[buf][0][0]);
        const char* bb = lds0 + buf * C::BN * BK * 2;
#pragma unroll
        for (int i = 0; i < C::TM; ++i) {
            if constexpr (A_KMAJ)
                af[set][i] = __builtin_bit_cast(
                    bf16x8, *reinterpret_cast<const u32x4*>(ba + rda[ks] + i * C::RS * BK * 2));
            else
                af[set][i] = tr_pair(ba, rda[i], ks);
        }
#pragma unroll
        for (int j = 0; j < C::TN; ++j) bfr[set][j] = tr_pair(bb, rdb[j], ks);
    };
    auto mfmas = [&](int set) {
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j)
                acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bfr[set][j], af[set][i],
                                                                    acc[i][j], 0, 0, 0);
    };
    auto slice = [&](auto bufc, int64_t kt) {
        constexpr int buf = decltype(bufc)::value;
        wait_vmcnt<0>();
        lds_ring_barrier();
        if (A_KMAJ && (K % BK) && kt == nk - 1) {
            zero_tail(kt, buf);
            lds_ring_barrier();
        }
        if (kt + 1 < nk) issue(kt + 1, buf ^ 1);
        read_step(bufc, 0, 0);
        __builtin_amdgcn_s_setprio(1);
        constexpr int NREAD = (A_KMAJ ? C::TM : 2 * C::TM) + 2 * C::TN;
#pragma unroll
        for (int ks = 0; ks < C::KSTEPS; ++ks) {
            const int cs = ks & 1;
            if (ks < C::KSTEPS - 1) read_step(bufc, ks + 1, cs ^ 1);
            mfmas(cs);
            if (ks < C::KSTEPS - 1) {
#pragma unroll
                for (int g = 0; g < C::TM * C::TN; ++g) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x100, NREAD - C::TM * C::TN, 0);
            }
        }
        __builtin_amdgcn_s_setprio(0);
    };
    int64_t kt = kbeg / BK;
    if (kt < nk) issue(kt, 0);
    for (; kt + 1 < nk; kt += 2) {
        slice(std::integral_constant<int, 0>{}, kt);
        slice(std::integral_constant<int, 1>{}, kt + 1);
    }
    if (kt < nk) slice(std::integral_constant<int, 0>{}, kt);
    __syncthreads();
#else
    (void)A, (void)lda, (void)B, (void)ldb, (void)M, (void)N, (void)kbeg, (void)K, (void)m0;
    (void)n0, (void)sm, (void)acc;
#endif
}

// The same for small tiles of four waves, of which three fit a compute unit, so that some multiply
// while others begin or store: slices of 32 through a ring of three buffers, every wave its own
// loads. Sums run over k in the same order. (128 x 256 in two a unit was the fastest of the three
// in 6 of 110 sizes, by 3%.)
using BwdSmall = Cfg<128, 128, 2, 2, 3, 32>;

template <class C, bool A_KMAJ>
__device__ __forceinline__ void gemm_tile_bwd_ring(const uint16_t* __restrict__ A, int64_t lda,
                                                   const uint16_t* __restrict__ B, int64_t ldb,
                                                   int64_t M, int64_t N, int64_t kbeg, int64_t K,
                                                   int64_t m0, int64_t n0, typename C::Smem& sm,
                                                   f32x16 (&acc)[C::TM][C::TN]) {
#if defined(__HIP_DEVICE_COMPILE__)
    static_assert(C::NS == 3 && C::WAVES == 4, "ring of three, four waves");
    constexpr int BK = C::BK, CH = C::CH;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wr = (wave / C::WN) * 32, wc = (wave % C::WN) * (C::BN / C::WN);
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int j = 0; j < C::TN; ++j)
#pragma unroll
            for (int v = 0; v < 16; ++v) acc[i][j][v] = 0.f;
    const int64_t nk = (K + BK - 1) / BK;
    constexpr uint32_t kNowhere = 0x80000000u;  // past any resource here: less than 2^31 bytes

    // Loads of a transposed operand, W elements wide: an instruction fills 512 / W rows, the
    // wave's q-th the rows (q * 4 + wave) * (512 / W) and on (a lane's row modulo 4, and so
    // its slot's chunk, is the same for every q).
    constexpr int RPA = 512 / C::BM, RPB = 512 / C::BN;      // rows an instruction
    constexpr int QA = A_KMAJ ? C::IA : BK / RPA / C::WAVES, QB = BK / RPB / C::WAVES;
    static_assert(QB * RPB * C::WAVES == BK && C::WAVES * RPB % 4 == 0, "transposed rows per wave");
    static_assert(A_KMAJ || (QA * RPA * C::WAVES == BK && C::WAVES * RPA % 4 == 0), "as above");
    uint32_t va, qa;
    if constexpr (A_KMAJ) {
        const int r = wave * C::LROWS + lane / CH;
        va = (uint32_t)((r * lda + (lane % CH ^ swz<CH>(r)) * 8) * 2);
        qa = (uint32_t)(C::WAVES * C::LROWS * lda * 2);
    } else {
        const int k = wave * RPA + lane / (C::BM / 8);
        va = (uint32_t)((k * lda + tr_slot(lane % (C::BM / 8), k) * 8) * 2);
        qa = (uint32_t)(C::WAVES * RPA * lda * 2);
    }
    const int kb = wave * RPB + lane / (C::BN / 8);
    const uint32_t vb = (uint32_t)((kb * ldb + tr_slot(lane % (C::BN / 8), kb) * 8) * 2);
    const uint32_t qb = (uint32_t)(C::WAVES * RPB * ldb * 2);
    const __amdgpu_buffer_rsrc_t rak =
        tile_rsrc(A + m0 * lda, A_KMAJ ? (M - m0 < C::BM ? M - m0 : C::BM) * lda * 2 : 0);
    // a transposed operand's slice: rows kt * BK .. K - 1 from column t0; none past the last
    auto tr_rsrc = [&](const uint16_t* X, int64_t ld, int64_t t0, int64_t len, int64_t kt) {
        const int64_t first = (kt < nk ? kt : 0) * BK * ld + t0;
        const int64_t end = (K - 1) * ld + (len + 7) / 8 * 8;
        return tile_rsrc(X + first, kt < nk ? (end - first) * 2 : 0);
    };
    auto issue = [&](int64_t kt, int buf) {
        if constexpr (A_KMAJ) {
            const uint32_t at = kt < nk ? (uint32_t)(kt * BK * 2) : 0u;
#pragma unroll
            for (uint32_t q = 0; q < QA; ++q)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    rak, lds_ptr(&sm.in.a[buf][0][0] + (q * C::WAVES + wave) * 512), 16,
                    kt < nk ? va : kNowhere, kt < nk ? at + q * qa : 0u, 0, 0);
        } else {
            const __amdgpu_buffer_rsrc_t ra = tr_rsrc(A, lda, m0, M, kt);
#pragma unroll
            for (uint32_t q = 0; q < QA; ++q)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    ra, lds_ptr(&sm.in.a[buf][0][0] + (q * C::WAVES + wave) * 512), 16, va, q * qa,
                    0, 0);
        }
        const __amdgpu_buffer_rsrc_t rb = tr_rsrc(B, ldb, n0, N, kt);
#pragma unroll
        for (uint32_t q = 0; q < QB; ++q)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rb, lds_ptr(&sm.in.b[buf][0][0] + (q * C::WAVES + wave) * 512), 16, vb, q * qb, 0, 0);
    };

    // operand offsets in a slice, as in gemm_tile_bwd; opaque, so that buffer, k-step and half
    // are the reads' immediates
    const char* const lds0 = reinterpret_cast<const char*>(&sm);
    const int kq = (lane >> 2) & 3, tr_row = 8 * (lane >> 5) + kq;
    const int tr_delta = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
    auto tr_off = [&](int mb, int width) -> uint32_t {
        const int slot = ((mb / 8) ^ (4 * kq)) | tr_delta;
        return (uint32_t)(tr_row * width * 2 + slot * 16 + 8 * (lane & 1));
    };
    uint32_t rda[A_KMAJ ? C::KSTEPS : C::TM], rdb[C::TN];
    if constexpr (A_KMAJ) {
#pragma unroll
        for (int ks = 0; ks < C::KSTEPS; ++ks) {
            const int c = ks * 2 + (lane >> 5), r = wr + (lane & 31);
            rda[ks] = (uint32_t)(r * BK + (c ^ swz<CH>(r)) * 8) * 2;
            asm volatile("" : "+v"(rda[ks]));
        }
    } else {
#pragma unroll
        for (int i = 0; i < C::TM; ++i) {
            rda[i] = tr_off(wr + i * C::RS, C::BM);
            asm volatile("" : "+v"(rda[i]));
        }
    }
    const uint32_t b_at = (uint32_t)(reinterpret_cast<const char*>(&sm.in.b[0][0][0]) - lds0);
#pragma unroll
    for (int j = 0; j < C::TN; ++j) {
        rdb[j] = b_at + tr_off(wc + j * 32, C::BN);
        asm volatile("" : "+v"(rdb[j]));
    }
    auto tr_pair = [&](uint32_t at, int width) -> bf16x8 {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(lds0 + at));
        const s16x4 hi =
            __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4_ptr)(lds0 + at + 4 * width * 2));
        typedef short s16x8 __attribute__((ext_vector_type(8)));
        const s16x8 v = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
        return __builtin_bit_cast(bf16x8, v);
    };
    bf16x8 af[2][C::TM], bfr[2][C::TN];
    auto read_step = [&](auto bufc, int ks, int set) {
        constexpr int buf = decltype(bufc)::value;
#pragma unroll
        for (int i = 0; i < C::TM; ++i) {
            if constexpr (A_KMAJ)
                af[set][i] = __builtin_bit_cast(
                    bf16x8, *reinterpret_cast<const u32x4*>(lds0 + rda[ks] + buf * C::BM * BK * 2 +
                                                            i * C::RS * BK * 2));
            else
                af[set][i] = tr_pair(rda[i] + buf * C::BM * BK * 2 + ks * 16 * C::BM * 2, C::BM);
        }
#pragma unroll
        for (int j = 0; j < C::TN; ++j)
            bfr[set][j] = tr_pair(rdb[j] + buf * C::BN * BK * 2 + ks * 16 * C::BN * 2, C::BN);
    };
    // k past K of a K-major A (also inside the chunk that straddles K) set to 0
    auto zero_tail = [&](int64_t kt, int buf) {
        const int kv = (int)(K - kt * BK);
        uint16_t* a = &sm.in.a[buf][0][0];
        for (int e = tid; e < BK * C::BM; e += C::THREADS) {
            const int r = e / BK, kk = ((e % BK / 8) ^ swz<CH>(r)) * 8 + e % 8;
            if (kk >= kv) a[e] = 0;
        }
    };
    auto slice = [&](auto bufc, int64_t kt) {
        constexpr int buf = decltype(bufc)::value;
        wait_vmcnt<QA + QB>();  // the loads of slice kt + 1
        lds_ring_barrier();
        if (A_KMAJ && (K % BK) && kt == nk - 1) {
            zero_tail(kt, buf);
            lds_ring_barrier();
        }
        issue(kt + 2, (buf + 2) % 3);
        __builtin_amdgcn_sched_barrier(0);
        read_step(bufc, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int ks = 0; ks < C::KSTEPS; ++ks) {
            if (ks + 1 < C::KSTEPS) read_step(bufc, ks + 1, (ks & 1) ^ 1);
#pragma unroll
            for (int i = 0; i < C::TM; ++i)
#pragma unroll
                for (int j = 0; j < C::TN; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bfr[ks & 1][j], af[ks & 1][i],
                                                                        acc[i][j], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
        // the products stay in their slice
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j) asm volatile("" : "+v"(acc[i][j]));
    };
    int64_t kt = kbeg / BK;
    if (kt < nk) {
        issue(kt, 0);
        issue(kt + 1, 1);
        for (; kt + 2 < nk; kt += 3) {
            slice(std::integral_constant<int, 0>{}, kt);
            slice(std::integral_constant<int, 1>{}, kt + 1);
            slice(std::integral_constant<int, 2>{}, kt + 2);
        }
        if (kt < nk) slice(std::integral_constant<int, 0>{}, kt);
        if (kt + 1 < nk) slice(std::integral_constant<int, 1>{}, kt + 1);
    }
    wait_vmcnt<0>();  // the zeros of slices past the last are in LDS
    __syncthreads();
#else
    (void)A, (void)lda, (void)B, (void)ldb, (void)M, (void)N, (void)kbeg, (void)K, (void)m0;
    (void)n0, (void)sm, (void)acc;
#endif
}

// One GEMM of the backward: C[M, N] (+)= A B with gemm_tile_bwd's operands,
// written to out [M, ldc] (fp32, or bf16 bits rounded to nearest even); vec:
// out 16-byte aligned and ldc a multiple of 16 bytes' worth of elements.
struct BwdGemm {
    const uint16_t* A;
    int64_t lda;
    const uint16_t* B;
    int64_t ldb;
    int64_t M, N, K;
    void* out;
    int64_t ldc;
    int vec;
    int64_t nmt, nnt;  // tiles
    // optional device row count: M (dyn_m) or K (dyn_k) is at most
    // *dyn - dyn_base (the grid covers the host values, the most there can be)
    const int32_t* dyn;
    int64_t dyn_base;
    bool dyn_m, dyn_k;
    // optional: row m of the result belongs at row map[m] of out
    const int32_t* map;
    // the sum over k in ksplit parts of kper (a multiple of BK), part i written
    // to out + i * part_stride elements
    int64_t ksplit, kper, part_stride;
    // optional: a factor of the result (device memory)
    const float* scale;
};

// Output modes of a backward GEMM: fp32 written, fp32 added to, bf16 written.
enum BwdOut { kOutF32 = 0, kOutF32Acc = 1, kOutBf16 = 2 };

// Logical tile of the workgroup with index b among the nb workgroups of one
// GEMM whose first workgroup sits on XCD 0 (workgroup i of a launch runs on
// XCD i % 8): each XCD takes a contiguous run of logical tiles, column tile
// fastest, so the tiles that share a row block of A run together on one XCD
// and read it from that XCD's L2.
__device__ __forceinline__ void tile_of_block_nfast(int64_t b, int64_t nmt, int64_t nnt,
                                                    int64_t& mt, int64_t& nt) {
    const int64_t nb = nmt * nnt, q = nb / 8, rr = nb % 8;
    const int64_t x = b % 8, sl = b / 8;
    const int64_t lg = x * q + min(x, rr) + sl;
    nt = lg % nnt;
    mt = lg / nnt;
}

// Tile b of GEMM g: the MFMA tile, then the result through LDS.
template <class C, bool A_KMAJ, int OUT>
__device__ __forceinline__ void bwd_gemm_tile(const BwdGemm& g, int64_t b, typename C::Smem& sm) {
    using OutT = typename std::conditional<OUT == kOutBf16, uint16_t, float>::type;
    constexpr bool ACC = OUT == kOutF32Acc;
    int64_t M = g.M, K = g.K, nmt = g.nmt, kbeg = 0;
    const int64_t N = g.N;
    if (g.dyn) {
        const int64_t live = (int64_t)*g.dyn - g.dyn_base;
        const int64_t lim = live > 0 ? live : 0;
        if (g.dyn_k && lim < K) K = lim;
        // no rows of this block to add: nothing to do
        if (K == 0 && ACC) return;
        if (g.dyn_m && lim < M) {
            // the tiles laid over the live rows' tiles (spread over every XCD)
            M = lim;
            nmt = (M + C::BM - 1) / C::BM;
            if (b >= nmt * g.nnt * g.ksplit) return;
        }
    }
    int64_t mt, nt;
    tile_of_block_nfast(b, nmt * g.ksplit, g.nnt, mt, nt);
    OutT* out = static_cast<OutT*>(g.out);
    if (g.ksplit > 1) {  // row tiles of part 0, then of part 1, ...
        const int64_t part = mt / nmt;
        mt -= part * nmt;
        out += part * g.part_stride;
        kbeg = part * g.kper;
        K = kbeg + g.kper < K ? kbeg + g.kper : K;
        if (kbeg >= K && ACC) return;
    }
    const int64_t m0 = mt * C::BM, n0 = nt * C::BN;
    const float f = g.scale ? *g.scale : 1.f;  // here, where its latency is hidden
    f32x16 acc[C::TM][C::TN];
    if constexpr (C::WAVES == 4)
        gemm_tile_bwd_ring<C, A_KMAJ>(g.A, g.lda, g.B, g.ldb, M, N, kbeg, K, m0, n0, sm, acc);
    else
        gemm_tile_bwd<C, A_KMAJ>(g.A, g.lda, g.B, g.ldb, M, N, kbeg, K, m0, n0, sm, acc);
    if (g.scale) {
#pragma unroll
        for (int i = 0; i < C::TM; ++i)
#pragma unroll
            for (int j = 0; j < C::TN; ++j)
#pragma unroll
                for (int v = 0; v < 16; ++v) acc[i][j][v] *= f;
    }

    // Pieces of 32 rows x 64 columns through the wave's own part of the LDS, without
    // barriers, as in lmhead_dlogits_tile: a row's piece leaves as 16-byte vectors (vec),
    // else one element at a time.
    constexpr int EPC = 16 / sizeof(OutT), CPR = 64 / EPC, RPI = 64 / CPR;  // a chunk, a row,
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;             // a store
    const int wr = (wave / C::WN) * 32, wc = (wave % C::WN) * (C::BN / C::WN);
    const int rr = lane / CPR, cc = lane % CPR * EPC;
#pragma unroll
    for (int i = 0; i < C::TM; ++i)
#pragma unroll
        for (int u = 0; u < C::TN / 2; ++u) {
            const OutT* src;  // the lane's chunk of the piece's first RPI rows
            int ld;
            lds_wave_order();  // fp32 pieces of every i share their rows of the LDS
            if constexpr (OUT == kOutBf16) {
                blocks_to_lds_bf16<C, 2>(&acc[i][2 * u], i, 2 * u, sm);
                src = &sm.c16[wr + i * C::RS + rr][wc + u * 64 + cc];
                ld = C::CROW16;
            } else {
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int v = 0; v < 16; v += 4) {
                        const f32x16& t = acc[i][2 * u + j];
                        const f32x4 x = {t[v], t[v + 1], t[v + 2], t[v + 3]};
                        *reinterpret_cast<f32x4*>(
                            &sm.c[wr + (lane & 31)]
                                 [wc + u * 64 + j * 32 + (v >> 2) * 8 + (lane >> 5) * 4]) = x;
                    }
                src = &sm.c[wr + rr][wc + u * 64 + cc];
                ld = C::CROW;
            }
            lds_wave_order();
            const int64_t m = m0 + wr + i * C::RS + rr, n = n0 + wc + u * 64 + cc;
            // the lane's q-th row of the piece, which is below M
            auto dst = [&](int q) {
                const int64_t r = m + q * RPI;
                return out + (g.map ? (int64_t)g.map[r] : r) * g.ldc + n;
            };
            if (g.vec && n + EPC <= N) {
                typedef typename std::conditional<ACC, f32x4, u32x4>::type Vec;
                Vec x[32 / RPI];
#pragma unroll
                for (int q = 0; q < 32 / RPI; ++q)
                    if constexpr (ACC)
                        if (m + q * RPI < M) x[q] = *reinterpret_cast<const Vec*>(dst(q));
#pragma unroll
                for (int q = 0; q < 32 / RPI; ++q) {
                    const Vec y = *reinterpret_cast<const Vec*>(src + q * RPI * ld);
                    if (m + q * RPI >= M) continue;
                    if constexpr (ACC)
                        x[q] += y;
                    else
                        x[q] = y;
                    *reinterpret_cast<Vec*>(dst(q)) = x[q];
                }
            } else {
                for (int q = 0; q < 32 / RPI && m + q * RPI < M; ++q) {
                    OutT* o = dst(q);
                    for (int e = 0; e < EPC && n + e < N; ++e) {
                        const OutT y = src[q * RPI * ld + e];
                        o[e] = ACC ? o[e] + y : y;
                    }
                }
            }
        }
}

// The two GEMMs of one backward block in one launch: dh = dz W (dz read
// along its rows) on the first n_dh workgroups (a multiple of 8; those past
// dh's tiles return at once), dW = dz^T h (dz read down its columns) on the
// rest. dh has few tiles with a long sum (a block's rows x d) and dW many
// with a short one, so dW's tiles fill the compute units that dh leaves
// free, and both start from the dz block just written.
template <class C, int DH_OUT, int DW_OUT>
__global__ void __launch_bounds__(C::THREADS, C::WAVES == 4 ? 3 : 1)
lmhead_bwd_gemms_kernel(BwdGemm dh, BwdGemm dw, int64_t n_dh) {
    __shared__ typename C::Smem sm;
    const int64_t b = blockIdx.x;
    if (b < n_dh) {
        if (b < dh.nmt * dh.nnt * dh.ksplit) bwd_gemm_tile<C, true, DH_OUT>(dh, b, sm);
    } else {
        bwd_gemm_tile<C, false, DW_OUT>(dw, b - n_dh, sm);
    }
}

// Whether row t takes part in the compact problem. Its dlogits are zeros when
// its coefficient is 0: by the caller's word under the skip flag (lse null),
// else where lse is finite (an infinity or a NaN in the row would give NaNs).
__device__ __forceinline__ bool row_counts(const float* __restrict__ coef,
                                           const float* __restrict__ lse, int64_t t) {
    return coef[t] != 0.f || (lse && !(fabsf(lse[t]) < INFINITY));
}

// The rows that count, in increasing order: map[0 .. n) and count[0] = n. One
// workgroup walks the rows 1024 at a time; the position of each kept row is its
// wave's ballot prefix plus the earlier waves' counts.
constexpr int kCompactThreads = 1024;
__global__ void __launch_bounds__(kCompactThreads)
compact_rows_kernel(const float* __restrict__ coef, const float* __restrict__ lse, int64_t T,
                    int32_t* __restrict__ map, int32_t* __restrict__ count) {
    __shared__ int wave_n[kCompactThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    int64_t base = 0;
    for (int64_t t0 = 0; t0 < T; t0 += kCompactThreads) {
        const int64_t t = t0 + tid;
        const bool keep = t < T && row_counts(coef, lse, t);
        const uint64_t ballot = __ballot(keep);
        const int before = __popcll(ballot & ((uint64_t(1) << lane) - 1));
        if (lane == 0) wave_n[wave] = __popcll(ballot);
        __syncthreads();
        int off = 0, total = 0;
        for (int w = 0; w < kCompactThreads / 64; ++w) {
            off += w < wave ? wave_n[w] : 0;
            total += wave_n[w];
        }
        if (keep) map[base + off + before] = (int32_t)t;
        base += total;
        __syncthreads();
    }
    if (tid == 0) count[0] = (int32_t)base;
}

// An element of a gradient output: fp32, or bf16 bits rounded to nearest even.
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(uint16_t* p, float v) { *p = bf16_bits(v); }

// Row i < count of the compact problem: hidden row map[i] and its per-row
// values; and row i of dh set to 0 where it does not count: one workgroup per row
// (grid-stride over the rows). lse_word: lse or null, as row_counts takes it.
template <class O>
__global__ void __launch_bounds__(128)
gather_rows_kernel(const int32_t* __restrict__ map, const int32_t* __restrict__ count, int64_t T,
                   const uint16_t* __restrict__ h, int64_t ld_h, int64_t d,
                   const int32_t* __restrict__ target, const float* __restrict__ lse,
                   const float* __restrict__ logp, const float* __restrict__ coef,
                   const float* __restrict__ lse_word, uint16_t* __restrict__ h_c,
                   int32_t* __restrict__ target_c, float* __restrict__ lse_c,
                   float* __restrict__ logp_c, float* __restrict__ coef_c, O* __restrict__ dh,
                   int64_t ld_dh) {
    const int64_t n = count[0];
    for (int64_t i = blockIdx.x; i < T; i += gridDim.x) {
        if (!row_counts(coef, lse_word, i))
            for (int64_t c = threadIdx.x; c < d; c += 128) put(dh + i * ld_dh + c, 0.f);
        if (i >= n) continue;
        const int64_t t = map[i];
        const u32x4* src = reinterpret_cast<const u32x4*>(h + t * ld_h);
        u32x4* dst = reinterpret_cast<u32x4*>(h_c + i * d);
        for (int64_t j = threadIdx.x; j < d / 8; j += 128) dst[j] = src[j];
        if (threadIdx.x == 0) {
            target_c[i] = target[t];
            lse_c[i] = lse[t];
            logp_c[i] = logp[t];
            coef_c[i] = coef[t];
        }
    }
}

// dst[r, c] = bf16(src[r, c]) for rows [0, rows), columns [0, cols).
__global__ void __launch_bounds__(256)
to_bf16_kernel(const float* __restrict__ src, int64_t ld_src, int64_t rows, int64_t cols,
               uint16_t* __restrict__ dst, int64_t ld_dst) {
    for (int64_t r = blockIdx.x; r < rows; r += gridDim.x)
        for (int64_t c = threadIdx.x; c < cols; c += 256)
            dst[r * ld_dst + c] = bf16_bits(src[r * ld_src + c]);
}

// The sum of the ksplit parts of dh (each [rows, d] fp32, part_stride elements
// apart) in part order, for rows [0, rows), with dyn_rows those below
// *dyn_rows - dyn_base; row r goes to row r of out, or (map, its first entry
// that of row 0) to row map[r]. Four columns a work-item at a time, grid-stride: all
// T rows at once (the compact rows of one sum) are more than a dispatch holds from
// T d = 2^34 on.
template <class O>
__global__ void __launch_bounds__(256)
sum_parts_kernel(const float* __restrict__ part, int64_t ksplit, int64_t part_stride, int64_t rows,
                 int64_t d, const int32_t* __restrict__ map, O* __restrict__ out, int64_t ld_out,
                 const int32_t* __restrict__ dyn_rows, int64_t dyn_base) {
    if (dyn_rows) {
        const int64_t live = (int64_t)*dyn_rows - dyn_base;
        rows = live < rows ? live : rows;
    }
    const int64_t step = (int64_t)gridDim.x * 256;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i * 4 < rows * d; i += step) {
        const f32x4* p = reinterpret_cast<const f32x4*>(part) + i;  // d % 8 == 0
        f32x4 x = p[0];
#pragma unroll 8
        for (int64_t k = 1; k < ksplit; ++k) x += p[k * (part_stride / 4)];
        const int64_t r = i * 4 / d;
        O* o = out + (map ? (int64_t)map[r] : r) * ld_out + (i * 4 - r * d);
#pragma unroll
        for (int q = 0; q < 4; ++q) put(o + q, x[q]);
    }
}

// Workgroups of the row kernels above: one per row (of the sum of parts: per 1024
// elements) up to this many.
constexpr int64_t kRowBlocks = 65536;

// Host-side argument rules shared by the LM-head entry points.
bool bad_lmhead_args(const void* hidden, int64_t T, int64_t d, int64_t ld_h, const void* weight,
                     int64_t V, int64_t ld_w) {
    if (!hidden || !weight) return true;
    if (T < 1 || V < 1 || d < 8 || T > 0x7FFFFFFFll || V > 0x7FFFFFFFll || d > 0x7FFFFFFFll)
        return true;
    if (d % 8 || ld_h < d || ld_w < d || ld_h % 8 || ld_w % 8) return true;
    return reinterpret_cast<uintptr_t>(hidden) % 16 || reinterpret_cast<uintptr_t>(weight) % 16;
}

dart_status_t launch_dlogits(const uint16_t* hidden, int64_t rows, int64_t d, int64_t ld_h,
                             const uint16_t* weight, int64_t V, int64_t ld_w,
                             const int32_t* target, const float* lse, const float* logp,
                             const float* coef, float scale, uint16_t* out, int64_t ld_out,
                             int64_t vbase, hipStream_t stream, const int32_t* dyn_rows = nullptr,
                             int64_t dyn_base = 0) {
    const int64_t nmt = (rows + LmCfg::BM - 1) / LmCfg::BM, nvt = vocab_tiles(V);
    if (!grid_fits(nmt * nvt, LmCfg::THREADS) || ld_h > kMaxLd || ld_w > kMaxLd)
        return DART_ERR_UNSUPPORTED;
    with_tile(tile_rows(rows, V, d <= 1024 ? 57 : 54), rows, V, [&](auto cfg) {
        using C = decltype(cfg);
        const int64_t nm = (rows + C::BM - 1) / C::BM;
        hipLaunchKernelGGL(lmhead_dlogits_kernel<C>, dim3((unsigned)(nm * nvt)), dim3(C::THREADS),
                           0, stream, hidden, rows, ld_h, weight, V, ld_w, d, target, lse, logp,
                           coef, scale, out, ld_out, vbase, nvt, dyn_rows, dyn_base);
    });
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

}  // namespace

extern "C" {

size_t dart_lmhead_stats_workspace_bytes(int64_t T, int64_t V) {
    if (T < 1 || V < 1 || T > 0x7FFFFFFFll || V > 0x7FFFFFFFll) return 0;
    return (size_t)T * (size_t)vocab_tiles(V) * sizeof(float4) + (size_t)T * sizeof(float);
}

dart_status_t dart_lmhead_tok_stats_ex(const void* hidden, int64_t T, int64_t d, int64_t ld_h,
                                       const void* weight, int64_t V, int64_t ld_w,
                                       const int32_t* target, float inv_temp, float* logp,
                                       float* entropy, float* lse, void* workspace,
                                       size_t workspace_bytes, hipStream_t stream) {
    if (bad_lmhead_args(hidden, T, d, ld_h, weight, V, ld_w)) return DART_ERR_INVALID_ARG;
    if (!(inv_temp > 0.f) || isinf(inv_temp)) return DART_ERR_INVALID_ARG;
    if (!target || !logp || !entropy || !lse || !workspace ||
        reinterpret_cast<uintptr_t>(workspace) % 16)
        return DART_ERR_INVALID_ARG;
    if (const dart_status_t ck = dart_check::run(
            stream, {{dart_check::Item::Ids, target, T, V}}); ck != DART_OK)
        return ck;

    if (workspace_bytes < dart_lmhead_stats_workspace_bytes(T, V)) return DART_ERR_INVALID_ARG;
    const int64_t nmt = (T + LmCfg::BM - 1) / LmCfg::BM, nvt = vocab_tiles(V);
    if (!grid_fits(nmt * nvt, LmCfg::THREADS) ||
        !grid_fits((T + kMergeWaves - 1) / kMergeWaves, kMergeWaves * 64) || ld_h > kMaxLd ||
        ld_w > kMaxLd)
        return DART_ERR_UNSUPPORTED;
    float4* part = static_cast<float4*>(workspace);
    float* z_y = reinterpret_cast<float*>(part + T * nvt);
    with_tile(tile_rows(T, V), T, V, [&](auto cfg) {
        using C = decltype(cfg);
        const int64_t nm = (T + C::BM - 1) / C::BM;
        hipLaunchKernelGGL(lmhead_stats_kernel<C>, dim3((unsigned)(nm * nvt)), dim3(C::THREADS), 0,
                           stream, static_cast<const uint16_t*>(hidden), T, ld_h,
                           static_cast<const uint16_t*>(weight), V, ld_w, d, target, inv_temp, nvt,
                           part, z_y);
    });
    hipLaunchKernelGGL(lmhead_merge_kernel, dim3((unsigned)((T + kMergeWaves - 1) / kMergeWaves)),
                       dim3(kMergeWaves * 64), 0, stream, part, z_y, T, nvt, V, target, logp,
                       entropy, lse);
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

dart_status_t dart_lmhead_tok_stats(const void* hidden, int64_t T, int64_t d, int64_t ld_h,
                                    const void* weight, int64_t V, int64_t ld_w,
                                    const int32_t* target, float* logp, float* entropy,
                                    float* lse, void* workspace, size_t workspace_bytes,
                                    hipStream_t stream) {
    return dart_lmhead_tok_stats_ex(hidden, T, d, ld_h, weight, V, ld_w, target, 1.f, logp,
                                    entropy, lse, workspace, workspace_bytes, stream);
}

dart_status_t dart_lmhead_dlogits_ex(const void* hidden, int64_t T, int64_t d, int64_t ld_h,
                                     const void* weight, int64_t V, int64_t ld_w,
                                     const int32_t* target, const float* lse, const float* logp,
                                     const float* tok_coef, float inv_temp, void* dlogits,
                                     int64_t ld_out, hipStream_t stream) {
    if (bad_lmhead_args(hidden, T, d, ld_h, weight, V, ld_w)) return DART_ERR_INVALID_ARG;
    if (!(inv_temp > 0.f) || isinf(inv_temp)) return DART_ERR_INVALID_ARG;
    if (!target || !lse || !logp || !tok_coef || !dlogits || ld_out < V || ld_out % 8 ||
        reinterpret_cast<uintptr_t>(dlogits) % 16)
        return DART_ERR_INVALID_ARG;
    if (const dart_status_t ck = dart_check::run(
            stream, {{dart_check::Item::Ids, target, T, V}}); ck != DART_OK)
        return ck;

    return launch_dlogits(static_cast<const uint16_t*>(hidden), T, d, ld_h,
                          static_cast<const uint16_t*>(weight), V, ld_w, target, lse, logp,
                          tok_coef, inv_temp, static_cast<uint16_t*>(dlogits), ld_out, 0, stream);
}

dart_status_t dart_lmhead_dlogits(const void* hidden, int64_t T, int64_t d, int64_t ld_h,
                                  const void* weight, int64_t V, int64_t ld_w,
                                  const int32_t* target, const float* lse, const float* logp,
                                  const float* tok_coef, void* dlogits, int64_t ld_out,
                                  hipStream_t stream) {
    return dart_lmhead_dlogits_ex(hidden, T, d, ld_h, weight, V, ld_w, target, lse, logp, tok_coef,
                                  1.f, dlogits, ld_out, stream);
}

size_t dart_lmhead_backward_workspace_bytes(int64_t chunk_rows, int64_t V) {
    if (chunk_rows < 1 || V < 1 || chunk_rows > 0x7FFFFFFFll || V > 0x7FFFFFFFll) return 0;
    return (size_t)chunk_rows * (size_t)((V + 7) / 8 * 8) * 2;
}

}  // extern "C"

namespace {

using lmhead::Grad;

constexpr uint32_t kBackwardFlags = DART_LMHEAD_SKIP_ZERO_ROWS | DART_LMHEAD_BF16_GRADS;

int64_t ceil8(int64_t x) { return (x + 7) / 8 * 8; }
size_t align256(size_t x) { return (x + 255) / 256 * 256; }

// How a backward call runs and where its parts sit in the workspace (byte
// offsets, each part 256-byte aligned; total is the end of the last part).
struct BackwardPlan {
    bool bf16, skip;
    int64_t rows, cols;  // block of rows x vocabulary entries, at most T x V
    bool acc_w;          // dW summed over row blocks into bf16: through fp32
    bool acc_h;          // dh summed over vocabulary blocks into bf16: through fp32
    size_t dz, accw, acch, h_c, dh_c, target_c, lse_c, logp_c, coef_c, map, count, total;
    // beyond total, used where the caller's workspace reaches split_total: dh's
    // sum over the vocabulary in ksplit parts (1: none), and room to leave out
    // rows with zero dlogits without being told to (compact)
    int64_t ksplit;
    bool compact;
    size_t parts, split_total;
};

// Whether a call that is not told to skip zero rows leaves them out all the
// same, as the gradient pass on logits does: where that is worth the kernels
// around it (finding the rows and copying them: 7 us at T = 1000, 20 at 2500, d = 3584,
// against the share of zero rows of a backward that takes at least 0.5 ms) and the
// compact rows fit 128 MiB. Few rows are bound by W and dW, not by their number.
// Measured at d = 3584, V = 152064, bf16 gradients: with 20% zero rows 2738 -> 2568
// us at T = 1000 and 10107 -> 8629 at 4096, with 50% 2668 -> 1658 and 9830 -> 5626;
// with none 2801 -> 2808 and 10475 -> 10490, at T = 2500 1425 -> 1442 (V = 32000) and
// 979 -> 990 (V = 20000). Below the line, at T = 1500, V = 14000, d = 1776 (3.7e10),
// leaving none out costs 3%.
bool leaves_zero_rows_out(int64_t T, int64_t d, int64_t V) {
    return T >= 256 && (double)T * (double)V * (double)d >= 1e11 &&
           (double)T * (double)(6 * d + 20) <= double(128 << 20);
}

// Parts of a block's dh sum. dh has rows / 256 x d / 256 tiles, each a sum over
// the block's whole vocabulary, and one launch holds them and dW's tiles, the
// same work in many short sums: while dh's tiles fill less than half of the
// compute units the launch waits for them (at 1000 rows, d = 3584, V = 152064:
// 56 tiles of 2376 slices, 3.62 ms; in 2, 4 or 9 parts 2.10, 1.95 or 2.02 ms, adding
// them up 7, 17 or 37 us more). So that at least half
// and at most all of the units have a part, none shorter than kMinPartSlices.
constexpr int64_t kMinPartSlices = 32;
int64_t dh_parts(int64_t rows, int64_t d, int64_t cols) {
    const int64_t tiles =
        ((rows + LmCfg::BM - 1) / LmCfg::BM) * ((d + LmCfg::BN - 1) / LmCfg::BN);
    const int64_t by_units = kUnits / tiles, by_k = cols / (LmCfg::BK * kMinPartSlices);
    const int64_t n = by_units < by_k ? by_units : by_k;
    return n > 1 ? n : 1;
}

// total = 0 when the sizes do not fit the address arithmetic.
BackwardPlan plan_backward(int64_t T, int64_t d, int64_t V, int64_t chunk_rows,
                           int64_t chunk_cols, uint32_t flags) {
    BackwardPlan P = {};
    P.bf16 = flags & DART_LMHEAD_BF16_GRADS;
    P.skip = flags & DART_LMHEAD_SKIP_ZERO_ROWS;
    P.rows = chunk_rows < T ? chunk_rows : T;
    P.cols = chunk_cols < V ? chunk_cols : V;
    // with rows skipped, dh is summed in the compact fp32 rows
    P.acc_w = P.bf16 && P.rows < T;
    P.acc_h = P.bf16 && P.cols < V && !P.skip;
    const double big = double(int64_t(1) << 60);
    if ((double)P.rows * (double)ceil8(P.cols) * 2 > big || (double)V * (double)d * 4 > big ||
        (double)T * (double)d * 6 > big)
        return P;
    size_t end = 0;
    auto take = [&](size_t bytes) {
        const size_t at = align256(end);
        end = at + bytes;
        return at;
    };
    P.dz = take((size_t)P.rows * (size_t)ceil8(P.cols) * 2);
    if (P.acc_w) P.accw = take((size_t)V * (size_t)d * 4);
    if (P.acc_h) P.acch = take((size_t)T * (size_t)d * 4);
    auto take_rows = [&] {
        P.h_c = take((size_t)T * (size_t)d * 2);
        P.dh_c = take((size_t)T * (size_t)d * 4);
        P.target_c = take((size_t)T * 4);
        P.lse_c = take((size_t)T * 4);
        P.logp_c = take((size_t)T * 4);
        P.coef_c = take((size_t)T * 4);
        P.map = take((size_t)T * 4);
        P.count = take(4);
    };
    if (P.skip) take_rows();
    P.total = end;
    P.ksplit = dh_parts(P.rows, d, P.cols);
    P.compact = !P.skip && leaves_zero_rows_out(T, d, V);
    if (P.compact) take_rows();
    if (P.ksplit > 1) P.parts = take((size_t)P.ksplit * (size_t)P.rows * (size_t)d * 4);
    P.split_total = end;
    return P;
}

// The GEMM description of one backward output (out.p at the block's first
// row); mode: kOutF32, kOutF32Acc or kOutBf16.
BwdGemm make_bwd_gemm(const uint16_t* A, int64_t lda, const uint16_t* B, int64_t ldb, int64_t M,
                      int64_t N, int64_t K, const Grad& out, int bm, int bn) {
    BwdGemm g;
    g.A = A, g.lda = lda, g.B = B, g.ldb = ldb, g.M = M, g.N = N, g.K = K;
    g.out = out.p, g.ldc = out.ld;
    const size_t esz = out.bf16 ? 2 : 4;
    g.vec = reinterpret_cast<uintptr_t>(out.p) % 16 == 0 && (out.ld * esz) % 16 == 0;
    g.nmt = (M + bm - 1) / bm;
    g.nnt = (N + bn - 1) / bn;
    g.dyn = nullptr, g.dyn_base = 0, g.dyn_m = g.dyn_k = false;
    g.map = nullptr, g.ksplit = 1, g.kper = K, g.part_stride = 0;
    g.scale = nullptr;
    return g;
}

int out_mode(const Grad& out, bool accumulate) {
    return out.bf16 ? kOutBf16 : accumulate ? kOutF32Acc : kOutF32;
}

template <class C, int DH, int DW>
void launch_bwd_gemms_t(const BwdGemm& dh, const BwdGemm& dw, int64_t n_dh, int64_t blocks,
                        hipStream_t stream) {
    hipLaunchKernelGGL((lmhead_bwd_gemms_kernel<C, DH, DW>), dim3((unsigned)blocks),
                       dim3(C::THREADS), 0, stream, dh, dw, n_dh);
}

template <class C, int DH>
void launch_bwd_gemms_dw(int dw_mode, const BwdGemm& dh, const BwdGemm& dw, int64_t n_dh,
                         int64_t blocks, hipStream_t stream) {
    if (dw_mode == kOutF32) launch_bwd_gemms_t<C, DH, kOutF32>(dh, dw, n_dh, blocks, stream);
    else if (dw_mode == kOutF32Acc) launch_bwd_gemms_t<C, DH, kOutF32Acc>(dh, dw, n_dh, blocks, stream);
    else launch_bwd_gemms_t<C, DH, kOutBf16>(dh, dw, n_dh, blocks, stream);
}

template <class C>
void launch_bwd_gemms_c(int dh_mode, int dw_mode, const BwdGemm& dh, const BwdGemm& dw, int64_t n_dh,
                        int64_t blocks, hipStream_t stream) {
    if (dh_mode == kOutF32) launch_bwd_gemms_dw<C, kOutF32>(dw_mode, dh, dw, n_dh, blocks, stream);
    else if (dh_mode == kOutBf16) launch_bwd_gemms_dw<C, kOutBf16>(dw_mode, dh, dw, n_dh, blocks, stream);
    else if constexpr (std::is_same<C, LmCfg>::value)
        launch_bwd_gemms_dw<C, kOutF32Acc>(dw_mode, dh, dw, n_dh, blocks, stream);
}

}  // namespace

dart_status_t lmhead::launch_bwd_gemms(const uint16_t* dz, int64_t ld_dz, int64_t rows, int64_t cols,
                                       const uint16_t* w, int64_t ld_w, const uint16_t* h, int64_t ld_h,
                                       int64_t d, const Grad& dh_out, bool dh_acc, int64_t ksplit,
                                       int64_t part_stride, const Grad& dw_out, bool dw_acc,
                                       hipStream_t stream, const int32_t* dh_map, const int32_t* dyn_rows,
                                       int64_t dyn_base, const float* scale, bool small) {
    if ((dh_out.bf16 && dh_acc) || (dw_out.bf16 && dw_acc) || (small && dh_acc))
        return DART_ERR_INVALID_ARG;
    if (ld_dz > kMaxLd || ld_w > kMaxLd || ld_h > kMaxLd || dh_out.ld > kMaxLd ||
        dw_out.ld > kMaxLd)
        return DART_ERR_UNSUPPORTED;
    const int bm = small ? BwdSmall::BM : LmCfg::BM, bn = small ? BwdSmall::BN : LmCfg::BN;
    BwdGemm dh = make_bwd_gemm(dz, ld_dz, w, ld_w, rows, d, cols, dh_out, bm, bn);
    BwdGemm dw = make_bwd_gemm(dz, ld_dz, h, ld_h, cols, d, rows, dw_out, bm, bn);
    // the block's rows are dh's M and dW's K
    dh.dyn = dw.dyn = dyn_rows;
    dh.dyn_base = dw.dyn_base = dyn_base;
    dh.dyn_m = dw.dyn_k = dyn_rows != nullptr;
    dh.map = dh_map;
    dh.scale = dw.scale = scale;
    if (ksplit > 1) {
        const int64_t nk = (cols + LmCfg::BK - 1) / LmCfg::BK;
        dh.ksplit = ksplit, dh.kper = (nk + ksplit - 1) / ksplit * LmCfg::BK;
        dh.part_stride = part_stride;
    }
    const int64_t n_dh = dh_out.p ? (dh.nmt * dh.nnt * ksplit + 7) / 8 * 8 : 0;
    const int64_t blocks = n_dh + (dw_out.p ? dw.nmt * dw.nnt : 0);
    if (blocks == 0) return DART_OK;
    if (!grid_fits(blocks, LmCfg::THREADS)) return DART_ERR_UNSUPPORTED;
    const int dhm = out_mode(dh_out, dh_acc), dwm = out_mode(dw_out, dw_acc);
    if (small)
        launch_bwd_gemms_c<BwdSmall>(dhm, dwm, dh, dw, n_dh, blocks, stream);
    else
        launch_bwd_gemms_c<LmCfg>(dhm, dwm, dh, dw, n_dh, blocks, stream);
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

void lmhead::launch_to_bf16(const float* src, int64_t rows, int64_t cols, const Grad& dst,
                    hipStream_t stream) {
    const unsigned blocks = (unsigned)(rows < kRowBlocks ? rows : kRowBlocks);
    hipLaunchKernelGGL(to_bf16_kernel, dim3(blocks), dim3(256), 0, stream, src, cols, rows, cols,
                       static_cast<uint16_t*>(dst.p), dst.ld);
}

namespace {

// The gradient pass over rows [0, T) of h in blocks of rows x vocabulary
// entries: per block, its dlogits into dz (bf16), then the block's share of
// dh (summed over the vocabulary blocks of its rows) and of dW (summed over
// the row blocks of its entries). A sum goes into its fp32 output directly,
// or, for a bf16 output that more than one block adds to, into acc_h ([T, d])
// or acc_w ([V, d]) and is rounded to bf16 once at the end; an output that
// one block writes is that GEMM's fp32 result rounded once. With dyn_rows, T
// is the most rows there can be and only the first *dyn_rows are formed (the
// count is read on the device: blocks past it have nothing to do, and the
// first row block writes dW even when it holds no rows). With parts (ksplit > 1),
// a row block's dh is summed there, [ksplit][R, d], and added up once its last
// vocabulary block is in. With map (and dyn_rows), the rows are compact ones and
// row i of dh belongs at row map[i]: the GEMM puts it there, unless its sum needs
// acc_h ([T, d]) or the parts, from where it is put there at the end. (With every sum
// in acc_h first, 2500 rows of V = 20000, d = 3584, none of them zero, took 1012 us
// with bf16 gradients and 1052 with fp32 ones, now 990 and 1022; 999 and 1006 where
// the rows are not looked at.)
dart_status_t backward_core(const uint16_t* h, int64_t T, int64_t d,
                            int64_t ld_h, const uint16_t* w, int64_t V, int64_t ld_w,
                            const int32_t* target, const float* lse, const float* logp,
                            const float* coef, float scale, const Grad& dh, const Grad& dw,
                            int64_t R,
                            int64_t C, uint16_t* dz, float* acc_h, float* acc_w, float* parts,
                            int64_t ksplit, hipStream_t stream, const int32_t* map = nullptr,
                            const int32_t* dyn_rows = nullptr) {
    if (R > T) R = T;
    if (C > V) C = V;
    const int64_t ld_dz = ceil8(C);
    const bool via_h = !parts && dh.bf16 && C < V, via_w = dw.bf16 && R < T;
    const bool put = map && !parts && !via_h;
    auto sum_parts = [&](const float* p, int64_t n, int64_t stride, int64_t r0, int64_t rows) {
        const int64_t blocks = (rows * d / 4 + 255) / 256;
        const dim3 grid((unsigned)(blocks < kRowBlocks ? blocks : kRowBlocks));
        const int32_t* m = map ? map + r0 : nullptr;
        void* out = map ? dh.p : dh.row(r0);
        if (dh.bf16)
            hipLaunchKernelGGL(sum_parts_kernel<uint16_t>, grid, dim3(256), 0, stream, p, n, stride,
                               rows, d, m, static_cast<uint16_t*>(out), dh.ld, dyn_rows, r0);
        else
            hipLaunchKernelGGL(sum_parts_kernel<float>, grid, dim3(256), 0, stream, p, n, stride,
                               rows, d, m, static_cast<float*>(out), dh.ld, dyn_rows, r0);
    };
    const Grad sum_h = via_h ? Grad{acc_h, d, false} : dh;
    const Grad sum_w = via_w ? Grad{acc_w, d, false} : dw;
    for (int64_t r0 = 0; r0 < T; r0 += R) {
        const int64_t rows = T - r0 < R ? T - r0 : R;
        const uint16_t* hr = h + r0 * ld_h;
        for (int64_t c0 = 0; c0 < V; c0 += C) {
            const int64_t cols = V - c0 < C ? V - c0 : C;
            const uint16_t* wc = w + c0 * ld_w;
            const dart_status_t st =
                launch_dlogits(hr, rows, d, ld_h, wc, cols, ld_w, target + r0, lse + r0,
                               logp + r0, coef + r0, scale, dz, ld_dz, c0, stream, dyn_rows, r0);
            if (st != DART_OK) return st;
            const dart_status_t sg = lmhead::launch_bwd_gemms(
                dz, ld_dz, rows, cols, wc, ld_w, hr, ld_h, d,
                parts ? Grad{parts, d, false}
                      : Grad{put ? sum_h.p : sum_h.row(r0), sum_h.ld, sum_h.bf16},
                c0 > 0, parts ? ksplit : 1, R * d, Grad{sum_w.row(c0), sum_w.ld, sum_w.bf16},
                r0 > 0, stream, put ? map + r0 : nullptr, dyn_rows, r0, nullptr, false);
            if (sg != DART_OK) return sg;
        }
        if (parts) sum_parts(parts, ksplit, R * d, r0, rows);
    }
    if (via_h && map)
        sum_parts(acc_h, 1, 0, 0, T);
    else if (via_h)
        lmhead::launch_to_bf16(acc_h, T, d, dh, stream);
    if (via_w) lmhead::launch_to_bf16(acc_w, V, d, dw, stream);
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

}  // namespace

extern "C" {

size_t dart_lmhead_backward_ex_workspace_bytes(int64_t T, int64_t d, int64_t V,
                                               int64_t chunk_rows, int64_t chunk_cols,
                                               uint32_t flags) {
    if (T < 1 || d < 1 || V < 1 || chunk_rows < 1 || chunk_cols < 1 || T > 0x7FFFFFFFll ||
        d > 0x7FFFFFFFll || V > 0x7FFFFFFFll || (flags & ~kBackwardFlags))
        return 0;
    return plan_backward(T, d, V, chunk_rows, chunk_cols, flags).total;
}

size_t dart_lmhead_backward_split_workspace_bytes(int64_t T, int64_t d, int64_t V,
                                                  int64_t chunk_rows, int64_t chunk_cols,
                                                  uint32_t flags) {
    if (dart_lmhead_backward_ex_workspace_bytes(T, d, V, chunk_rows, chunk_cols, flags) == 0)
        return 0;
    return plan_backward(T, d, V, chunk_rows, chunk_cols, flags).split_total;
}

dart_status_t dart_lmhead_backward_ex(const void* hidden, int64_t T, int64_t d, int64_t ld_h,
                                      const void* weight, int64_t V, int64_t ld_w,
                                      const int32_t* target, const float* lse, const float* logp,
                                      const float* tok_coef, float inv_temp, void* dhidden,
                                      int64_t ld_dh, void* dweight, int64_t ld_dw,
                                      int64_t chunk_rows, int64_t chunk_cols, uint32_t flags,
                                      void* workspace, size_t workspace_bytes,
                                      hipStream_t stream) {
    if (bad_lmhead_args(hidden, T, d, ld_h, weight, V, ld_w)) return DART_ERR_INVALID_ARG;
    if (!(inv_temp > 0.f) || isinf(inv_temp)) return DART_ERR_INVALID_ARG;
    if (!target || !lse || !logp || !tok_coef || !dhidden || !dweight || !workspace)
        return DART_ERR_INVALID_ARG;
    if (ld_dh < d || ld_dw < d || chunk_rows < 1 || chunk_cols < 1 ||
        (flags & ~kBackwardFlags) || reinterpret_cast<uintptr_t>(workspace) % 16)
        return DART_ERR_INVALID_ARG;
    // the MFMA tiles address rows by 32-bit offsets from a tile's first row
    if (ld_h > kMaxLd || ld_w > kMaxLd || ld_dh > kMaxLd || ld_dw > kMaxLd)
        return DART_ERR_UNSUPPORTED;
    const BackwardPlan P = plan_backward(T, d, V, chunk_rows, chunk_cols, flags);
    if (P.total == 0) return DART_ERR_UNSUPPORTED;
    if (workspace_bytes < P.total) return DART_ERR_INVALID_ARG;
    if (const dart_status_t ck = dart_check::run(
            stream, {{dart_check::Item::Ids, target, T, V}}); ck != DART_OK)
        return ck;

    const uint16_t* h = static_cast<const uint16_t*>(hidden);
    const uint16_t* w = static_cast<const uint16_t*>(weight);
    char* ws = static_cast<char*>(workspace);
    uint16_t* dz = reinterpret_cast<uint16_t*>(ws + P.dz);
    float* acc_w = P.acc_w ? reinterpret_cast<float*>(ws + P.accw) : nullptr;
    float* acc_h = P.acc_h ? reinterpret_cast<float*>(ws + P.acch) : nullptr;
    const bool split = P.ksplit > 1 && workspace_bytes >= P.split_total;
    float* parts = split ? reinterpret_cast<float*>(ws + P.parts) : nullptr;
    const Grad dh{dhidden, ld_dh, P.bf16}, dw{dweight, ld_dw, P.bf16};
    if (!P.skip && !(P.compact && workspace_bytes >= P.split_total))
        return backward_core(h, T, d, ld_h, w, V, ld_w, target, lse, logp, tok_coef, inv_temp, dh,
                             dw, P.rows, P.cols, dz, acc_h, acc_w, parts, P.ksplit, stream);

    // rows with a zero coefficient have dz = 0: they add nothing to dW and
    // their rows of dh are 0, so the GEMMs run over the other rows only
    int32_t* map = reinterpret_cast<int32_t*>(ws + P.map);
    int32_t* count = reinterpret_cast<int32_t*>(ws + P.count);
    uint16_t* h_c = reinterpret_cast<uint16_t*>(ws + P.h_c);
    float* dh_c = reinterpret_cast<float*>(ws + P.dh_c);
    int32_t* target_c = reinterpret_cast<int32_t*>(ws + P.target_c);
    float* lse_c = reinterpret_cast<float*>(ws + P.lse_c);
    float* logp_c = reinterpret_cast<float*>(ws + P.logp_c);
    float* coef_c = reinterpret_cast<float*>(ws + P.coef_c);
    const float* lse_word = P.skip ? nullptr : lse;
    hipLaunchKernelGGL(compact_rows_kernel, dim3(1), dim3(kCompactThreads), 0, stream, tok_coef,
                       lse_word, T, map, count);
    const dim3 row_blocks((unsigned)(T < kRowBlocks ? T : kRowBlocks));
    if (P.bf16)
        hipLaunchKernelGGL(gather_rows_kernel<uint16_t>, row_blocks, dim3(128), 0, stream, map,
                           count, T, h, ld_h, d, target, lse, logp, tok_coef, lse_word, h_c,
                           target_c, lse_c, logp_c, coef_c, static_cast<uint16_t*>(dhidden), ld_dh);
    else
        hipLaunchKernelGGL(gather_rows_kernel<float>, row_blocks, dim3(128), 0, stream, map, count,
                           T, h, ld_h, d, target, lse, logp, tok_coef, lse_word, h_c, target_c,
                           lse_c, logp_c, coef_c, static_cast<float*>(dhidden), ld_dh);
    if (hipGetLastError() != hipSuccess) return DART_ERR_HIP;
    // the kernels read the kept-row count on the device: T rows at most
    return backward_core(h_c, T, d, d, w, V, ld_w, target_c, lse_c, logp_c, coef_c, inv_temp, dh,
                         dw, P.rows, P.cols, dz, dh_c, acc_w, parts, P.ksplit, stream, map, count);
}

dart_status_t dart_lmhead_backward(const void* hidden, int64_t T, int64_t d, int64_t ld_h,
                                   const void* weight, int64_t V, int64_t ld_w,
                                   const int32_t* target, const float* lse, const float* logp,
                                   const float* tok_coef, float* dhidden, int64_t ld_dh,
                                   float* dweight, int64_t ld_dw, int64_t chunk_rows,
                                   void* workspace, size_t workspace_bytes, hipStream_t stream) {
    return dart_lmhead_backward_ex(hidden, T, d, ld_h, weight, V, ld_w, target, lse, logp,
                                   tok_coef, 1.f, dhidden, ld_dh, dweight, ld_dw, chunk_rows, V,
                                   0u, workspace, workspace_bytes, stream);
}

}  // extern "C"
