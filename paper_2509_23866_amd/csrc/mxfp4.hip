// libdart, four-bit part: matrices in MXFP4 (blocks of 32 values along a row, each value
// in E2M1, the block's scale a power of two in E8M0), their product on the matrix cores,
// and the token statistics of the LM head kept so.
//
// Paper: DART, arXiv 2509.23866. Its truncated importance weight (Sec. 4.4) corrects for
// a rollout policy that differs from the trainer's by quantisation; this part makes that
// policy's head (quantise), its logits (product) and its log-probs (statistics).
//
//   mxfp4_quantize_kernel    one workgroup per 32 rows x 256 columns: four lanes a block,
//                            their largest size by two exchanges, E2M1 by the hardware's
//                            conversion. Bound by memory.
//   mxfp4_dequantize_kernel  the same tile back.
//   mxfp4_matmul_kernel      gemm_tile on MXFP4 operands, the fp32 tile written in bf16 or
//                            fp32.
//   mxfp4_stats_kernel       gemm_tile and the epilogue of lmhead_stats_kernel: the
//                            logits are not written.
//
// Layout of a quantised R x K matrix, in slices of 256 columns (K padded with zeros to
// whole slices) and runs of 32 rows:
//   packed  row-major, slices * 128 bytes a row, value k in the low (k even) or high half
//           of byte k / 2;
//   scales  [slice][run][64] dwords: byte ks of dword half * 32 + r is the scale of block
//           half * 4 + ks (of the slice's 8) of row r (of the run's 32). So one dword holds
//           the scales of a lane's four MFMA operands in a slice, 64 lanes read 256 bytes in
//           a row, and one load instruction brings those of 128 rows.
#include "lmhead_tile.h"

namespace {

constexpr int64_t kSlice = 256;  // columns
constexpr int64_t kRun = 32;     // rows
constexpr int kQuantThreads = 256;

int64_t slices_of(int64_t K) { return (K + kSlice - 1) / kSlice; }
int64_t runs_of(int64_t R) { return (R + kRun - 1) / kRun; }
// a packed row in 16-bit elements
int64_t packed_ld(int64_t K) { return slices_of(K) * (kSlice / 4); }

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
mxfp4_quantize_kernel(const X* __restrict__ x, int64_t R, int64_t K, int64_t ld,
                      int64_t slices, int64_t runs, uint8_t* __restrict__ packed,
                      uint32_t* __restrict__ scales) {
    __shared__ uint32_t sc[64];
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
        const int64_t r = run * kRun + row;
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
        const uint32_t w = byte == 255u ? 0u : e2m1x8(v[p]);
        if (r < R)
            *reinterpret_cast<uint32_t*>(packed + (r * slices + slice) * 128 + c8 * 4) = w;
        const int c = c8 >> 2;
        if ((c8 & 3) == 0)
            reinterpret_cast<uint8_t*>(sc)[(c >> 2) * 128 + row * 4 + (c & 3)] = (uint8_t)byte;
    }
    __syncthreads();
    if (tid < 64) scales[(slice * runs + run) * 64 + tid] = sc[tid];
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
mxfp4_dequantize_kernel(const uint8_t* __restrict__ packed, const uint8_t* __restrict__ scales,
                        int64_t R, int64_t K, int64_t slices, int64_t runs,
                        X* __restrict__ out, int64_t ld) {
    const int64_t run = blockIdx.x / slices, slice = blockIdx.x % slices;
    const int tid = threadIdx.x, c8 = tid & 31, c = c8 >> 2;
    const int64_t k = slice * kSlice + c8 * 8;
    if (k >= K) return;
    uint32_t w[4], byte[4];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int row = p * 8 + (tid >> 5);
        const int64_t r = min(run * kRun + row, R - 1);
        w[p] = *reinterpret_cast<const uint32_t*>(packed + (r * slices + slice) * 128 + c8 * 4);
        byte[p] = scales[(slice * runs + run) * 256 + (c >> 2) * 128 + row * 4 + (c & 3)];
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        const int64_t r = run * kRun + p * 8 + (tid >> 5);
        if (r >= R) return;
        // the scale as fp32 (2^-127 is a denormal, byte 255 a NaN); a code's three bits
        // below the sign as the low exponent and high mantissa bits of an fp32, times
        // 2^126, are its size (0.5 from the denormal 2^-127)
        const float scale = byte[p] == 255u   ? __builtin_nanf("")
                            : byte[p] == 0u   ? __uint_as_float(0x00400000u)
                                              : __uint_as_float(byte[p] << 23);
        float v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t code = w[p] >> (4 * i);
            const float size = __uint_as_float((code & 7u) << 22) * 0x1p126f;
            v[i] = __uint_as_float(__float_as_uint(size) | (code & 8u) << 28) * scale;
        }
        store8(out + r * ld + k, K - k, v);
    }
}

// This wave's part of a result tile to out [M, ld] through the wave's own part of the
// LDS (its accesses run in order: no barrier), 32 rows at a time, as in
// lmhead_dlogits_tile: bf16 rows of the wave's columns, fp32 ones 64 columns at a time, in
// 16-byte vectors, which the hardware takes at any multiple of an element's size.
template <class C, class O>
__device__ __forceinline__ void store_tile(f32x16 (&acc)[C::TM][C::TN], int64_t M, int64_t N,
                                           O* __restrict__ out, int64_t ld, typename C::Smem& sm,
                                           int64_t m0, int64_t n0) {
    constexpr bool BF16 = sizeof(O) == 2;
    constexpr int NJ = BF16 ? C::TN : 2;                        // 32-column blocks a piece
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

// The operands of a product: packed matrices and their scales.
struct Mxfp4Pair {
    const uint16_t *a, *b;
    Mxfp4Scales scales;
    int64_t K4;  // columns in 16-bit elements: the row stride too
};

template <class C, class O>
__global__ void __launch_bounds__(C::THREADS)
mxfp4_matmul_kernel(Mxfp4Pair x, int64_t M, int64_t N, int64_t nnt, O* __restrict__ out,
                    int64_t ld) {
    with_row_tile<C>(M, nnt, [&](auto cfg, auto& sm, int64_t m0, int64_t nt) {
        using T = decltype(cfg);
        f32x16 acc[T::TM][T::TN];
        gemm_tile<T>(x.a, M, x.K4, x.b, N, x.K4, x.K4, m0, nt * T::BN, sm, acc, x.scales);
        store_tile<T, O>(acc, M, N, out, ld, sm, m0, nt * T::BN);
    });
}

template <class C>
__global__ void __launch_bounds__(C::THREADS)
mxfp4_stats_kernel(Mxfp4Pair x, int64_t T, int64_t V, const int32_t* __restrict__ target,
                   float scale, int64_t nvt, float4* __restrict__ part, float* __restrict__ z_y) {
    with_row_tile<C>(T, nvt, [&](auto cfg, auto& sm, int64_t m0, int64_t vt) {
        using R = decltype(cfg);
        stats_of_tile<R>(
            [&](int64_t n0, f32x16(&acc)[R::TM][R::TN]) {
                gemm_tile<R>(x.a, T, x.K4, x.b, V, x.K4, x.K4, m0, n0, sm, acc, x.scales);
            },
            T, V, target, scale, nvt, part, z_y, sm, m0, vt);
    });
}

bool bad_size(int64_t n) { return n < 1 || n > 0x7FFFFFFFll; }
bool misaligned(const void* p, size_t to) { return reinterpret_cast<uintptr_t>(p) % to != 0; }
bool bad_quantized(const void* packed, const void* scales, int64_t R, int64_t K) {
    return !packed || !scales || bad_size(R) || bad_size(K) || misaligned(packed, 16) ||
           misaligned(scales, 16);
}
size_t size_of(dart_dtype_t t) { return t == DART_BF16 ? 2 : 4; }
bool bad_dtype(dart_dtype_t t) { return t != DART_BF16 && t != DART_F32; }

Mxfp4Pair pair_of(const void* a, const void* as, int64_t M, const void* b, const void* bs,
                  int64_t N, int64_t K) {
    return {static_cast<const uint16_t*>(a), static_cast<const uint16_t*>(b),
            {static_cast<const uint32_t*>(as), static_cast<const uint32_t*>(bs), runs_of(M),
             runs_of(N)},
            packed_ld(K)};
}

}  // namespace

extern "C" {

size_t dart_mxfp4_packed_bytes(int64_t R, int64_t K) {
    if (bad_size(R) || bad_size(K)) return 0;
    return (size_t)R * (size_t)slices_of(K) * 128;
}

size_t dart_mxfp4_scales_bytes(int64_t R, int64_t K) {
    if (bad_size(R) || bad_size(K)) return 0;
    return (size_t)runs_of(R) * (size_t)slices_of(K) * 256;
}

dart_status_t dart_mxfp4_quantize(const void* x, dart_dtype_t dtype, int64_t R, int64_t K,
                                  int64_t ld, void* packed, void* scales, hipStream_t stream) {
    if (bad_dtype(dtype) || !x || ld < K || bad_quantized(packed, scales, R, K) ||
        misaligned(x, size_of(dtype)))
        return DART_ERR_INVALID_ARG;
    const int64_t blocks = runs_of(R) * slices_of(K);
    if (!grid_fits(blocks, kQuantThreads)) return DART_ERR_UNSUPPORTED;
    auto launch = [&](auto kernel, auto* p) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kQuantThreads), 0, stream, p, R, K,
                           ld, slices_of(K), runs_of(R), static_cast<uint8_t*>(packed),
                           static_cast<uint32_t*>(scales));
    };
    if (dtype == DART_BF16)
        launch(mxfp4_quantize_kernel<uint16_t>, static_cast<const uint16_t*>(x));
    else
        launch(mxfp4_quantize_kernel<float>, static_cast<const float*>(x));
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

dart_status_t dart_mxfp4_dequantize(const void* packed, const void* scales, int64_t R, int64_t K,
                                    dart_dtype_t dtype, void* out, int64_t ld_out,
                                    hipStream_t stream) {
    if (bad_dtype(dtype) || !out || ld_out < K || bad_quantized(packed, scales, R, K) ||
        misaligned(out, size_of(dtype)))
        return DART_ERR_INVALID_ARG;
    const int64_t blocks = runs_of(R) * slices_of(K);
    if (!grid_fits(blocks, kQuantThreads)) return DART_ERR_UNSUPPORTED;
    auto launch = [&](auto kernel, auto* p) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)blocks), dim3(kQuantThreads), 0, stream,
                           static_cast<const uint8_t*>(packed), static_cast<const uint8_t*>(scales),
                           R, K, slices_of(K), runs_of(R), p, ld_out);
    };
    if (dtype == DART_BF16)
        launch(mxfp4_dequantize_kernel<uint16_t>, static_cast<uint16_t*>(out));
    else
        launch(mxfp4_dequantize_kernel<float>, static_cast<float*>(out));
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

dart_status_t dart_mxfp4_matmul(const void* a_packed, const void* a_scales, int64_t M,
                                const void* b_packed, const void* b_scales, int64_t N, int64_t K,
                                dart_dtype_t dtype, void* out, int64_t ld_out, hipStream_t stream) {
    if (bad_dtype(dtype) || !out || ld_out < N || bad_quantized(a_packed, a_scales, M, K) ||
        bad_quantized(b_packed, b_scales, N, K) || misaligned(out, size_of(dtype)))
        return DART_ERR_INVALID_ARG;
    const int64_t nnt = vocab_tiles(N), nmt = (M + LmCfg::BM - 1) / LmCfg::BM;
    if (!grid_fits(nmt * nnt, LmCfg::THREADS) || packed_ld(K) > kMaxLd) return DART_ERR_UNSUPPORTED;
    const Mxfp4Pair x = pair_of(a_packed, a_scales, M, b_packed, b_scales, N, K);
    with_tile<true>(tile_rows(M, N), M, N, [&](auto cfg) {
        using C = decltype(cfg);
        const dim3 grid((unsigned)((M + C::BM - 1) / C::BM * nnt)), block(C::THREADS);
        if (dtype == DART_BF16)
            hipLaunchKernelGGL((mxfp4_matmul_kernel<C, uint16_t>), grid, block, 0, stream, x, M, N,
                               nnt, static_cast<uint16_t*>(out), ld_out);
        else
            hipLaunchKernelGGL((mxfp4_matmul_kernel<C, float>), grid, block, 0, stream, x, M, N,
                               nnt, static_cast<float*>(out), ld_out);
    });
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

dart_status_t dart_lmhead_mxfp4_tok_stats(const void* hidden_packed, const void* hidden_scales,
                                          int64_t T, const void* weight_packed,
                                          const void* weight_scales, int64_t V, int64_t d,
                                          const int32_t* target, float inv_temp, float* logp,
                                          float* entropy, float* lse, void* workspace,
                                          size_t workspace_bytes, hipStream_t stream) {
    if (bad_quantized(hidden_packed, hidden_scales, T, d) ||
        bad_quantized(weight_packed, weight_scales, V, d))
        return DART_ERR_INVALID_ARG;
    if (!(inv_temp > 0.f) || isinf(inv_temp)) return DART_ERR_INVALID_ARG;
    if (!target || !logp || !entropy || !lse || !workspace || misaligned(workspace, 16) ||
        workspace_bytes < dart_lmhead_stats_workspace_bytes(T, V))
        return DART_ERR_INVALID_ARG;
    const int64_t nvt = vocab_tiles(V), nmt = (T + LmCfg::BM - 1) / LmCfg::BM;
    if (!grid_fits(nmt * nvt, LmCfg::THREADS) ||
        !grid_fits((T + kMergeWaves - 1) / kMergeWaves, kMergeWaves * 64) || packed_ld(d) > kMaxLd)
        return DART_ERR_UNSUPPORTED;
    if (const dart_status_t ck = dart_check::run(
            stream, {{dart_check::Item::Ids, target, T, V}}); ck != DART_OK)
        return ck;
    const Mxfp4Pair x = pair_of(hidden_packed, hidden_scales, T, weight_packed, weight_scales, V, d);
    float4* part = static_cast<float4*>(workspace);
    float* z_y = reinterpret_cast<float*>(part + T * nvt);
    with_tile<true>(tile_rows(T, V), T, V, [&](auto cfg) {
        using C = decltype(cfg);
        hipLaunchKernelGGL(mxfp4_stats_kernel<C>, dim3((unsigned)((T + C::BM - 1) / C::BM * nvt)),
                           dim3(C::THREADS), 0, stream, x, T, V, target, inv_temp, nvt, part, z_y);
    });
    hipLaunchKernelGGL(lmhead_merge_kernel, dim3((unsigned)((T + kMergeWaves - 1) / kMergeWaves)),
                       dim3(kMergeWaves * 64), 0, stream, part, z_y, T, nvt, V, target, logp,
                       entropy, lse);
    return hipGetLastError() == hipSuccess ? DART_OK : DART_ERR_HIP;
}

}  // extern "C"
