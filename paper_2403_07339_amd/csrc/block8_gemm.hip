// Product of two tensors in 8-bit floating point with a power of two per row and block of 128 places of the contraction (block8.h):
//
//   out[m, n] = sum_k value_A[m, k] value_B[n, k] + bias[n]
//
// The codes with their power of two are numbers of bfloat16, so that products on v_mfma_f32_32x32x16_bf16 are exact and sums binary32's.
#include "block8.h"

namespace imu {
typedef float v16f32 __attribute__((ext_vector_type(16)));
typedef __bf16 v2bf16 __attribute__((ext_vector_type(2)));
typedef __bf16 v8bf16 __attribute__((ext_vector_type(8)));

struct GemmArgs {
    const uint8_t *a, *sa, *b, *sb;
    const float *bias;  // may be null
    void *out;
    int64_t lda, ldsa, ldb, ldsb, ldo;
    int m, n, kt;       // kt: blocks of the contraction
    int mtiles, ntiles;
};

// Eight codes times their power of two as bfloat16 (exact).
template <int FORMAT>
__device__ __forceinline__ v8bf16 widen(uint32_t lo, uint32_t hi, float scale) {
    v2bf16 p[4];
    if constexpr (FORMAT == IMUNPACK_E4M3) {
        p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
        p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    } else {
        p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, false), p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(lo, scale, true);
        p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, false), p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(hi, scale, true);
    }
    return v8bf16{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}

// 64 x 64 results to a workgroup, 32 x 32 to a wave, operands straight from memory.
template <int FA, int FB, class T>
__global__ __launch_bounds__(256) void block8_gemm_kernel(const GemmArgs g) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = lane & 31, half = lane >> 5;
    const int m = ((int)blockIdx.x % g.mtiles) * 64 + (wave >> 1) * 32 + row, n0 = ((int)blockIdx.x / g.mtiles) * 64 + (wave & 1) * 32;
    const int ma = min(m, g.m - 1), nb = min(n0 + row, g.n - 1);
    const uint8_t *a = g.a + ma * g.lda + half * 64, *b = g.b + nb * g.ldb + half * 64;
    v16f32 acc;
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[r] = 0.0f;
    for (int kt = 0; kt < g.kt; ++kt) {
        const float sa = block8_scale(g.sa[ma * g.ldsa + kt]), sb = block8_scale(g.sb[nb * g.ldsb + kt]);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint4 wa = *reinterpret_cast<const uint4 *>(a + kt * 128 + q * 16), wb = *reinterpret_cast<const uint4 *>(b + kt * 128 + q * 16);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen<FB>(wb.x, wb.y, sb), widen<FA>(wa.x, wa.y, sa), acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen<FB>(wb.z, wb.w, sb), widen<FA>(wa.z, wa.w, sa), acc, 0, 0, 0);
        }
    }
    // the lane's row of A with the columns 8 (r / 4) + 4 half + r % 4 of the wave's 32
    if (m >= g.m) return;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int n = n0 + q * 8 + half * 4;
        float f[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) f[r] = acc[q * 4 + r] + (g.bias && n + r < g.n ? g.bias[n + r] : 0.0f);
        if (n < g.n) store_upto<T, 4>((T *)g.out + m * g.ldo + n, f, g.n - n);
    }
}

static bool operand_fits(const Blocks8 &t, int64_t rows, int64_t cols, int format) {
    return blocks8_fit(t, cols) && rows >= 1 && (format == IMUNPACK_E4M3 || format == IMUNPACK_E5M2);
}
}  // namespace imu

using namespace imu;

constexpr int64_t kGemmRows = 1 << 24;

extern "C" int imunpack_block8_gemm_workspace(int64_t m, int64_t n, int64_t k, int dtype, size_t *bytes) {
    if (m < 0 || n < 0 || k < 1 || m > kGemmRows || n > kGemmRows || k > kBlock8Cols || (dtype != IMUNPACK_F32 && dtype != IMUNPACK_BF16) || !bytes) return IMUNPACK_EINVAL;
    *bytes = 0;
    return IMUNPACK_OK;
}

extern "C" int imunpack_block8_gemm(const void *a, int64_t lda, const void *a_scales, int64_t ldsa, int a_format, const void *b, int64_t ldb, const void *b_scales, int64_t ldsb,
                                    int b_format, int64_t m, int64_t n, int64_t k, const float *bias, void *out, int64_t ldo, int dtype, void *workspace, size_t workspace_bytes,
                                    imunpack_stream_t stream) {
    size_t need = 0;
    IMU_TRY(imunpack_block8_gemm_workspace(m, n, k, dtype, &need));
    if (m == 0 || n == 0) return IMUNPACK_OK;
    const Blocks8 A = {(uint8_t *)a, (uint8_t *)a_scales, lda, ldsa}, B = {(uint8_t *)b, (uint8_t *)b_scales, ldb, ldsb};
    if (!operand_fits(A, m, k, a_format) || !operand_fits(B, n, k, b_format) || !out || ldo < n) return IMUNPACK_EINVAL;
    if (need && (!workspace || ((uintptr_t)workspace & 15))) return IMUNPACK_EINVAL;
    if (workspace_bytes < need) return IMUNPACK_ESMALL;
    GemmArgs g = {A.codes, A.scales, B.codes, B.scales, bias, out, lda, ldsa, ldb, ldsb, ldo, (int)m, (int)n, (int)((k + kBlock8 - 1) / kBlock8), 0, 0};
    g.mtiles = (int)((m + 63) / 64);
    g.ntiles = (int)((n + 63) / 64);
    const int64_t groups = (int64_t)g.mtiles * g.ntiles;
    if (groups > (1 << 23)) return IMUNPACK_EINVAL;
    auto launch = [&](auto fa, auto fb, auto t) {
        hipLaunchKernelGGL((block8_gemm_kernel<decltype(fa)::value, decltype(fb)::value, decltype(t)>), dim3((unsigned)groups), dim3(256), 0, (hipStream_t)stream, g);
    };
    using E4 = std::integral_constant<int, IMUNPACK_E4M3>;
    using E5 = std::integral_constant<int, IMUNPACK_E5M2>;
    auto typed = [&](auto fa, auto fb) { dtype == IMUNPACK_F32 ? launch(fa, fb, 0.0f) : launch(fa, fb, (__bf16)0.0f); };
    if (a_format == IMUNPACK_E4M3) b_format == IMUNPACK_E4M3 ? typed(E4(), E4()) : typed(E4(), E5());
    else b_format == IMUNPACK_E4M3 ? typed(E5(), E4()) : typed(E5(), E5());
    return launch_status();
}
