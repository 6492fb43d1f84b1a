// Tensors in 8-bit floating point with a power of two for every block of 128 (a row's, or 128 x 128).
//
//   e = the smallest whole number >= -127 with  max |x| over the block <= top 2^e    (top = 448 for e4m3, 57344 for e5m2; 0 for a block of zeros)
//   code = x 2^-e rounded to nearest, ties to even;  value = code 2^e
//
// Why a power of two and not largest / top: the matrix instruction takes the byte e + 127 (e8m0) with its operands and scales by it at no cost;
// multiplying by it is exact, so that x 2^-e has no rounding of its own and equal inputs have equal codes however they are computed; and a
// value keeps its bits under another block's scale (turning a tensor loses only what falls below the smallest codes).  The price is up to one bit of
// range at the small end, none of the precision.
//
// Rows of codes are filled with zeros up to a whole block, so that a product needs no mask along the contraction: bases and pitches of codes and
// scales are multiples of 16 bytes, codes go over ceil(cols / 128) * 128 bytes of a row.
#pragma once
#include "common.h"
#include "elements.h"

namespace imu {
constexpr int kBlock8 = IMUNPACK_BLOCK8;
constexpr int64_t kBlock8Cols = 1 << 24, kBlock8Rows = 1ll << 31;  // sizes that are taken

// One tensor in 8 bits, as a call gives it.
struct Blocks8 {
    uint8_t *codes, *scales;
    int64_t ldc, lds;
};
inline bool blocks8_fit(const Blocks8 &t, int64_t cols) {
    return t.codes && t.scales && !((uintptr_t)t.codes & 15) && !((uintptr_t)t.scales & 15) && !(t.ldc & 15) && !(t.lds & 15) &&
           t.ldc >= (cols + kBlock8 - 1) / kBlock8 * kBlock8 && t.lds >= (cols + kBlock8 - 1) / kBlock8;
}

#if defined(__HIPCC__)
// The byte of a block whose largest finite magnitude has these bits (not negative).  One bit pattern decides: with E the exponent's field,
// x <= 1.75 2^(8 + e) is e >= E - 127 - 8, or one more where the fraction is above 0.75.
// UP: the bits are those of the magnitude times 2^-UP.
template <int FORMAT, int UP = 0>
__device__ __forceinline__ int block8_byte(int bits) {
    constexpr int up = FORMAT == IMUNPACK_E4M3 ? 8 : 15;
    const int e = (bits >> 23) - up + UP + ((bits & 0x7fffff) > 0x600000);
    return bits == 0 ? 127 : max(e, 0);
}
__device__ __forceinline__ float block8_scale(int byte) { return __int_as_float(byte ? byte << 23 : 0x400000); }  // 2^(byte - 127)
__device__ __forceinline__ float block8_inverse(int byte) { return __int_as_float((254 - byte) << 23); }          // (byte <= 253)
// The magnitude that counts for a block's scale: infinity and NaN do not, so that they cost their neighbours nothing.
__device__ __forceinline__ int finite_bits(float x) {
    const int b = __float_as_int(x) & 0x7fffffff;
    return b < 0x7f800000 ? b : 0;
}
// The largest over the 16 lanes of a row of lanes, in each of them.
__device__ __forceinline__ int max16(int v) {
    v = max(v, IMU_DPP(v, 0x128, 0xf, true));  // rotations by 8, 4, 2, 1
    v = max(v, IMU_DPP(v, 0x124, 0xf, true));
    v = max(v, IMU_DPP(v, 0x122, 0xf, true));
    return max(v, IMU_DPP(v, 0x121, 0xf, true));
}
template <int FORMAT>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
    if constexpr (FORMAT == IMUNPACK_E4M3) return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false), true);
    else return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(c, d, __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false), true);
}
template <int FORMAT>
__device__ __forceinline__ void decode4(uint32_t w, float scale, float *f) {
    typedef float v2 __attribute__((ext_vector_type(2)));
    v2 lo, hi;
    if constexpr (FORMAT == IMUNPACK_E4M3) lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    else lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)w, true);
    f[0] = lo[0] * scale; f[1] = lo[1] * scale; f[2] = hi[0] * scale; f[3] = hi[1] * scale;
}
template <int FORMAT>
__device__ __forceinline__ uint2 encode8(const float (&x)[8], float inverse) {
    return make_uint2(encode4<FORMAT>(x[0] * inverse, x[1] * inverse, x[2] * inverse, x[3] * inverse),
                      encode4<FORMAT>(x[4] * inverse, x[5] * inverse, x[6] * inverse, x[7] * inverse));
}
template <int FORMAT>
__device__ __forceinline__ void decode8(uint2 w, float scale, float (&f)[8]) {
    decode4<FORMAT>(w.x, scale, f);
    decode4<FORMAT>(w.y, scale, f + 4);
}
// The largest magnitude's bits of N values that count for a scale.  Infinity and NaN are looked for only where the plain maximum shows one.
template <int N>
__device__ __forceinline__ int top_bits(const float (&x)[N]) {
    int top = 0;
#pragma unroll
    for (int k = 0; k < N; ++k) top = max(top, __float_as_int(x[k]) & 0x7fffffff);
    if (top >= 0x7f800000) {
        top = 0;
#pragma unroll
        for (int k = 0; k < N; ++k) top = max(top, finite_bits(x[k]));
    }
    return top;
}
// Eight consecutive elements of a block to a lane, the block's 16 lanes together: its byte.
template <int FORMAT>
__device__ __forceinline__ int block8_of(const float (&x)[8]) {
    return block8_byte<FORMAT>(max16(top_bits<8>(x)));
}
#endif
}  // namespace imu
