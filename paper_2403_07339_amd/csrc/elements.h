// Elements of fp32 and bfloat16 arrays sixteen bytes at a time, at any alignment of the element, and sums over workgroups
// (norm, loss and optimiser kernels).
#pragma once
#include "common.h"

namespace imu {
constexpr int64_t kLastLevelCache = 256ll << 20;  // bytes that the memory side's cache holds

#if defined(__HIPCC__)
template <class T>
constexpr int kVec = 16 / (int)sizeof(T);  // elements of one load

// N elements that lie at any multiple of their own size: one load or store where the hardware has it so wide (rows of odd
// length put every second row at such an address).  Vectors, not arrays: the compiler takes a store of an array apart where
// another path stores its first element too.
template <class T, int N>
struct Pieces {
    typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T))));
};

template <class T, int N>
using piece_t = typename Pieces<T, N>::type;

// A piece of a row of which `have` elements are left; those behind them are zero.  Pieces are asked for one after the other and
// turned into binary32 only then: each load stands in a branch of its own, and a conversion beside it would wait for it there.
// ONCE: the caches are not asked to keep it.
template <class T, int N, bool ONCE = false>
__device__ __forceinline__ piece_t<T, N> load_piece(const T *p, int have) {
    if (have >= N) {
        if constexpr (ONCE) return __builtin_nontemporal_load(reinterpret_cast<const piece_t<T, N> *>(p));
        else return *reinterpret_cast<const piece_t<T, N> *>(p);
    }
    piece_t<T, N> x;
#pragma unroll
    for (int k = 0; k < N; ++k) x[k] = k < have ? p[k] : (T)0;
    return x;
}
template <class T, int N>
__device__ __forceinline__ void to_floats(const piece_t<T, N> &x, float (&f)[N]) {
#pragma unroll
    for (int k = 0; k < N; ++k) f[k] = (float)x[k];
}
template <class T, int N>
__device__ __forceinline__ void load_upto(const T *p, float (&f)[N], int have) {
    to_floats<T, N>(load_piece<T, N>(p, have), f);
}
template <class T, int N, bool ONCE = false>
__device__ __forceinline__ void store_upto(T *p, const float (&f)[N], int have) {
    if (have >= N) {
        piece_t<T, N> x;
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = (T)f[k];
        if constexpr (ONCE) __builtin_nontemporal_store(x, reinterpret_cast<piece_t<T, N> *>(p));
        else *reinterpret_cast<piece_t<T, N> *>(p) = x;
        return;
    }
#pragma unroll
    for (int k = 0; k < N; ++k)
        if (k < have) p[k] = (T)f[k];
}
// Weights come as fp32 or bfloat16, whatever the rest is in.
template <int N>
__device__ __forceinline__ void load_weights(const void *w, bool bf16, int64_t at, float (&f)[N], int have) {
    if (bf16) load_upto<__bf16, N>((const __bf16 *)w + at, f, have);
    else load_upto<float, N>((const float *)w + at, f, have);
}

// Sum / maximum over the 64 lanes, in every lane.  The order of the additions is fixed.
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m);
    return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
    for (int m = 32; m; m >>= 1) v = fmaxf(v, __shfl_xor(v, m));
    return v;
}
// Over TPR threads (a wave, or a whole workgroup of TPR / 64 waves, through `lds` of TPR / 64 words, which the
// caller does not use again before another barrier).
template <int TPR, bool MAX>
__device__ __forceinline__ float reduce_threads(float v, float *lds) {
    v = MAX ? wave_max(v) : wave_sum(v);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        v = lds[0];
#pragma unroll
        for (int k = 1; k < TPR / 64; ++k) v = MAX ? fmaxf(v, lds[k]) : v + lds[k];
    }
    return v;
}
#endif
}  // namespace imu
