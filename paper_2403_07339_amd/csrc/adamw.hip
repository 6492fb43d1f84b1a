// One AdamW step over many tensors.
//
//   m = beta1 m + (1 - beta1) g,   v = beta2 v + (1 - beta2) g^2
//   p = (1 - lr wd) p - lr / (1 - beta1^t) * m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// States in 32 bits, or in 8: m and sqrt(v) as e4m3 with a binary32 scale for every 256 elements (largest magnitude / 448).  The
// root is held, not v: with the same codes it covers twice the range in powers of two.  A code's step is 6 to 12 % of its value and a step of
// the average moves it by 0.1 %: rounded to nearest, nearly every state would stand still.  So codes are rounded up
// with the probability of what is left over (stochastic rounding), by 16 bits for each state of a hash of seed, step, tensor and
// element, so that a step can be repeated.  That leaves the means of m and of the root as they are; v, the root's square, comes out about 5 % too
// large where the gradients keep their size (for beta2 0.99 and 0.999 alike), and the root scatters by some 16 %.  A root that is not zero keeps the
// smallest code at least, 2^-18 of its block's largest: as zero it would leave eps alone below m in the next step.
//
// Bound by memory: 28 bytes an element with 32-bit states and gradients, 16 with 8-bit states.  More than the last-level cache holds is read and
// written past the caches (85 million elements: 464 -> 410 us with 32-bit states; 157 million 478 -> 455 with 8-bit ones, bfloat16 gradients and
// copies).  A wave takes 256 elements, four to a lane, which is a block of the 8-bit states; tensors come as a table in the kernel's
// arguments.  85 million elements with 32-bit states take 383 us, 6.2 TB/s, 157 million with 8-bit ones 448 us, 5.6 TB/s.
#include "common.h"
#include "elements.h"

#include <algorithm>
#include <cmath>

namespace imu {
constexpr int kAdamTensors = 48;      // to a launch: their table travels in the kernel's arguments (4 KiB)
constexpr int kAdamBlock = 256;       // elements that share a scale
constexpr int kAdamBlocks = 1;        // blocks of a wave (4: 85 million elements 383 -> 405 us, 0.27 million in 112 tensors 19 -> 25; 1, but written
                                      // without the loops over them: 390, the compiler then puts the loads of a tensor's last elements in line)
constexpr int kAdamChunk = 4 * kAdamBlocks * kAdamBlock;  // elements of a workgroup
constexpr int64_t kAdamGroups = (1 << 24) - 1;  // workgroups of a launch at most: 2^32 threads are more than a grid may have along an axis
constexpr float kE4m3Max = 448.0f, kNothing = 0x1p-96f;  // a block of no more than that is held as zeros

struct AdamArgs {
    float *p[kAdamTensors];
    const void *g[kAdamTensors];
    void *m[kAdamTensors], *v[kAdamTensors];
    float *ms[kAdamTensors], *vs[kAdamTensors];
    __bf16 *copy[kAdamTensors];
    int64_t n[kAdamTensors];
    int32_t first[kAdamTensors];  // workgroups before the tensor's
    int32_t count, base;          // tensors of this launch, and before it
    int64_t skip;                 // workgroups' worth of a tensor that is too large for one launch, before this one
    uint32_t key;
    float beta1, rest1, beta2, rest2, decay, rate, root_scale, eps;
};
static_assert(sizeof(AdamArgs) <= 4096, "kernel arguments");

__host__ __device__ __forceinline__ uint32_t mix32(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0xBB67AE85u;
    return x ^ (x >> 16);
}
constexpr uint32_t kGolden = 0x9E3779B1u;

// |x| (at most 448) to one of its two neighbours in e4m3: up where what is left over and u in [0, 1) reach a whole step; not
// below `least` steps unless it is zero.
__device__ __forceinline__ float round_e4m3(float x, float u, float least) {
    const float a = fabsf(x);
    const uint32_t e = max(__float_as_uint(a) & 0x7f800000u, 121u << 23);  // steps are 2^-9 below 2^-6
    const float n0 = floorf(a * __uint_as_float((257u << 23) - e) + u);
    const float n = a > 0.0f && n0 < least ? least : n0;
    const float v = n * __uint_as_float(e - (3u << 23));
    return copysignf(v > kE4m3Max ? kE4m3Max : v, x);
}
// The largest of 256 magnitudes, four to a lane, in every lane (NaN above infinity, as the bits have it).
__device__ __forceinline__ float block_max(const float (&x)[4]) {
    int b = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) b = max(b, (int)(__float_as_uint(x[k]) & 0x7fffffffu));
    return __uint_as_float((uint32_t)from_lane63(wave_max_nonneg_lane63(b)));
}
__device__ __forceinline__ void decode(uint32_t w, float scale, float (&f)[4]) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    f[0] = lo[0] * scale; f[1] = lo[1] * scale; f[2] = hi[0] * scale; f[3] = hi[1] * scale;
}
__device__ __forceinline__ uint32_t encode(const float (&f)[4]) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w, true);
}
template <bool ONCE>
__device__ __forceinline__ uint32_t load_codes(const void *p, int64_t at) {
    return __builtin_bit_cast(uint32_t, load_piece<uint8_t, 4, ONCE>((const uint8_t *)p + at, 4));
}
template <bool ONCE>
__device__ __forceinline__ void store_codes(void *p, int64_t at, uint32_t w) {
    piece_t<uint8_t, 4> *to = reinterpret_cast<piece_t<uint8_t, 4> *>((uint8_t *)p + at);
    if constexpr (ONCE) __builtin_nontemporal_store(__builtin_bit_cast(piece_t<uint8_t, 4>, w), to);
    else *to = __builtin_bit_cast(piece_t<uint8_t, 4>, w);
}

// (No sum is contracted into a fused multiply-add: a state near the edge between two codes would go one way here and another
// way where the same formula is written out elsewhere, and a step of a code is an eighth of its value.)
#pragma clang fp contract(off)
template <bool EIGHT, class G, bool ONCE>
__global__ __launch_bounds__(256) void adamw_kernel(const AdamArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // which tensor the workgroup belongs to: lane k looks at tensor k
    const int32_t mine = lane < a.count ? a.first[lane] : 0x7fffffff;
    const int k = __builtin_popcountll(__ballot(mine <= (int)blockIdx.x)) - 1;
    const int64_t n = a.n[k];
    float *p = a.p[k];
    const G *g = (const G *)a.g[k];
    __bf16 *copy = a.copy[k];
    const int64_t chunk = ((int)blockIdx.x - a.first[k] + a.skip) * kAdamChunk;
    const uint32_t key = mix32(a.key + (uint32_t)(a.base + k) * kGolden);
    const int64_t at0 = chunk + wave * kAdamBlock + lane * 4;
    float P[kAdamBlocks][4], M[kAdamBlocks][4], V[kAdamBlocks][4];
    piece_t<G, 4> g4[kAdamBlocks];
    uint32_t mw[kAdamBlocks], vw[kAdamBlocks];
    float msc[kAdamBlocks], vsc[kAdamBlocks];
#pragma unroll
    for (int i = 0; i < kAdamBlocks; ++i) {
        const int64_t at = at0 + i * 4 * kAdamBlock, block = at / kAdamBlock;
        const int have = (int)min((int64_t)4, n - at);
        to_floats<float, 4>(load_piece<float, 4, ONCE>(p + at, have), P[i]);
        g4[i] = load_piece<G, 4, ONCE>(g + at, have);
        if constexpr (EIGHT) {
            mw[i] = vw[i] = 0;
            msc[i] = vsc[i] = 0.0f;
            if (block * kAdamBlock < n) {  // the states go over whole blocks
                mw[i] = load_codes<ONCE>(a.m[k], at);
                vw[i] = load_codes<ONCE>(a.v[k], at);
                msc[i] = a.ms[k][block];
                vsc[i] = a.vs[k][block];
            }
        } else {
            to_floats<float, 4>(load_piece<float, 4, ONCE>((const float *)a.m[k] + at, have), M[i]);
            to_floats<float, 4>(load_piece<float, 4, ONCE>((const float *)a.v[k] + at, have), V[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kAdamBlocks; ++i) {
        const int64_t at = at0 + i * 4 * kAdamBlock, block = at / kAdamBlock;
        const int have = (int)min((int64_t)4, n - at);
        if (block * kAdamBlock >= n) break;  // the whole wave
        if constexpr (EIGHT) {
            decode(mw[i], msc[i], M[i]);
            decode(vw[i], vsc[i], V[i]);
#pragma unroll
            for (int j = 0; j < 4; ++j) V[i][j] *= V[i][j];
        }
        float root[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float gr = (float)g4[i][j];
            M[i][j] = a.beta1 * M[i][j] + a.rest1 * gr;
            V[i][j] = a.beta2 * V[i][j] + a.rest2 * (gr * gr);
            root[j] = sqrtf(V[i][j]);
            P[i][j] = P[i][j] * a.decay - a.rate * (M[i][j] / (root[j] * a.root_scale + a.eps));
        }
        store_upto<float, 4, ONCE>(p + at, P[i], have);
        if (copy) store_upto<__bf16, 4, ONCE>(copy + at, P[i], have);
        if constexpr (EIGHT) {
            const float mmax = block_max(M[i]), vmax = block_max(root);
            const float mi = mmax >= kNothing ? (1.0f / mmax) * kE4m3Max : mmax == mmax ? 0.0f : mmax;
            const float vi = vmax >= kNothing ? (1.0f / vmax) * kE4m3Max : vmax == vmax ? 0.0f : vmax;
            float mq[4], vq[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t bits = mix32((uint32_t)(at + j) * kGolden + key);
                mq[j] = round_e4m3(M[i][j] * mi, (float)(bits & 0xffffu) * 0x1p-16f, 0.0f);
                vq[j] = round_e4m3(root[j] * vi, (float)(bits >> 16) * 0x1p-16f, 1.0f);
            }
            store_codes<ONCE>(a.m[k], at, encode(mq));
            store_codes<ONCE>(a.v[k], at, encode(vq));
            if (lane == 0) {
                a.ms[k][block] = mmax >= kNothing || mmax != mmax ? mmax * (1.0f / kE4m3Max) : 0.0f;
                a.vs[k][block] = vmax >= kNothing || vmax != vmax ? vmax * (1.0f / kE4m3Max) : 0.0f;
            }
        } else {
            store_upto<float, 4, ONCE>((float *)a.m[k] + at, M[i], have);
            store_upto<float, 4, ONCE>((float *)a.v[k] + at, V[i], have);
        }
    }
}

template <bool EIGHT, class G>
static void launch_adamw(const AdamArgs &a, unsigned groups, bool once, hipStream_t st) {
    if (once) hipLaunchKernelGGL((adamw_kernel<EIGHT, G, true>), dim3(groups), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((adamw_kernel<EIGHT, G, false>), dim3(groups), dim3(256), 0, st, a);
}
}  // namespace imu

using namespace imu;

extern "C" int imunpack_adamw(int64_t count, float *const *params, const void *const *grads, void *const *exp_avg,
                              void *const *exp_avg_sq, float *const *m_scales, float *const *v_scales, void *const *copies,
                              const int64_t *numel, int grad_dtype, int state_bits, double lr, double beta1, double beta2,
                              double eps, double weight_decay, int64_t step, uint32_t seed, imunpack_stream_t stream) {
    if (count < 0 || (grad_dtype != IMUNPACK_F32 && grad_dtype != IMUNPACK_BF16) || (state_bits != 8 && state_bits != 32) || step < 1 ||
        !(lr >= 0.0) || !(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0) || !(weight_decay >= 0.0) ||
        !std::isfinite(lr) || !std::isfinite(eps) || !std::isfinite(weight_decay))
        return IMUNPACK_EINVAL;
    if (count > 0 && (!params || !grads || !exp_avg || !exp_avg_sq || !numel || (state_bits == 8 && (!m_scales || !v_scales)))) return IMUNPACK_EINVAL;
    int64_t total = 0;
    for (int64_t k = 0; k < count; ++k) {
        if (numel[k] < 0 || numel[k] > (int64_t)1 << 40) return IMUNPACK_EINVAL;
        if (numel[k] > 0 && (!params[k] || !grads[k] || !exp_avg[k] || !exp_avg_sq[k] || (state_bits == 8 && (!m_scales[k] || !v_scales[k])) || (copies && !copies[k])))
            return IMUNPACK_EINVAL;
        total += numel[k];
    }
    // bytes that are read, not counting the copies: what does not fit the caches is not brought into them
    const bool once = total * (4 + (grad_dtype == IMUNPACK_F32 ? 4 : 2) + (state_bits == 8 ? 2 : 8)) > kLastLevelCache;
    hipStream_t st = (hipStream_t)stream;
    AdamArgs a;
    a.key = mix32(seed + (uint32_t)step * kGolden);
    a.beta1 = (float)beta1; a.rest1 = (float)(1.0 - beta1);
    a.beta2 = (float)beta2; a.rest2 = (float)(1.0 - beta2);
    a.decay = (float)(1.0 - lr * weight_decay);
    a.rate = (float)(lr / (1.0 - std::pow(beta1, (double)step)));
    a.root_scale = (float)(1.0 / std::sqrt(1.0 - std::pow(beta2, (double)step)));
    a.eps = (float)eps;
    auto launch = [&](int64_t groups) {
        const bool bf16 = grad_dtype == IMUNPACK_BF16;
        if (state_bits == 8) bf16 ? launch_adamw<true, __bf16>(a, (unsigned)groups, once, st) : launch_adamw<true, float>(a, (unsigned)groups, once, st);
        else bf16 ? launch_adamw<false, __bf16>(a, (unsigned)groups, once, st) : launch_adamw<false, float>(a, (unsigned)groups, once, st);
        return launch_status();
    };
    for (int64_t k = 0; k < count;) {
        a.count = 0;
        a.base = (int32_t)k;
        int64_t groups = 0;
        for (; k < count && a.count < kAdamTensors; ++k) {
            const int i = a.count;
            const int64_t more = (numel[k] + kAdamChunk - 1) / kAdamChunk;
            if (i > 0 && groups + more > kAdamGroups) break;
            a.p[i] = params[k]; a.g[i] = grads[k]; a.m[i] = exp_avg[k]; a.v[i] = exp_avg_sq[k];
            a.ms[i] = state_bits == 8 ? m_scales[k] : nullptr;
            a.vs[i] = state_bits == 8 ? v_scales[k] : nullptr;
            a.copy[i] = copies ? (__bf16 *)copies[k] : nullptr;
            a.n[i] = numel[k];
            a.first[i] = (int32_t)groups;
            groups += more;
            ++a.count;
            if (groups > kAdamGroups) {  // a tensor by itself
                ++k;
                break;
            }
        }
        for (a.skip = 0; a.skip < groups; a.skip += kAdamGroups) IMU_TRY(launch(std::min(groups - a.skip, kAdamGroups)));
    }
    return IMUNPACK_OK;
}
