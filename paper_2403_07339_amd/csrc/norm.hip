// Root-mean-square norm over rows, with the addition of the residual stream in front of it, an output of b-bit integers with
// a scale per row for serving, and the backward pass.
//
//   h = x + residual                          (the residual stream, returned)
//   r = 1 / sqrt(mean_j h_j^2 + eps)
//   y_j = h_j r w_j
//   quantised: scale = max_j |y_j| / (2^(b-1) - 1), q_j = rint(y_j / scale), which no split of Alg. 1 to 5 has to touch: every
//   |q_j| is In-Bound for b
//   backward: gx_j = gh_j + r (gy_j w_j - h_j r^2 mean_k(gy_k w_k h_k)),  gw_j = sum over rows of gy_j h_j r
//
// Bound by memory: every array is read once and written once.  A row stays in the registers of one wave (up to 256 pieces of 16
// bytes: 12608 rows of 768 fp32, both passes, 56 us, of a workgroup 64), of a workgroup of 256 threads (up to 1024: 2000 rows of 4096 fp32
// 45.5 us, of 1024 threads 46.2) or of 1024 threads (up to 4096) between the sums over it and its use;
// longer rows are read again for each.  Results leave past the caches where a call moves as much as the last-level cache holds (8192 x 4096
// bfloat16, forward and backward: 121 -> 111 us; 12608 x 768 fp32, whose backward pass finds them there: 64, 69 that way).  Of 8192 x 4096
// bfloat16 the forward pass takes 42 us and the backward pass 50, 6.4 and 5.4 TB/s, where a copy of 1 GiB reaches 5.1.
// Sums, statistics and products are binary32; what is stored as bfloat16 is rounded once, from the binary32 value (y from the unrounded h).
#include "common.h"
#include "elements.h"

#include <algorithm>
#include <type_traits>

namespace imu {
constexpr int kNormThreads = 256;   // of a workgroup whose waves take a row each
constexpr int kNormGroups = 2048;   // workgroups at most: they walk over the rows
constexpr int kNormPartials = 512;  // workgroups of the backward pass at most: each leaves a row of partial sums of gw
constexpr int kNormFewRows = 256;   // up to so many rows other workgroups of the same launch read them again, column by column, for gw: no second
                                    // launch for the sums (256 rows of 1024 fp32, forward and backward: 14.3 us and 17.2 with one; 500 rows: 20.5 and 17.0)

struct NormArgs {
    const void *x, *res, *w;
    void *y, *h, *values;
    float *rstd, *scale;
    int8_t *q;
    int64_t ldx, ldres, ldy, ldh, ldq, ldv;
    int64_t rows;
    int d, w_bf16;
    float eps, qmax;  // qmax: 2^(b-1) - 1, or 0 where y itself is wanted
};

// What a row's integers count; NaN for a row that holds a NaN or an infinity, 1 for a row of zeros.
__device__ __forceinline__ float quant_scale(float amax, bool finite, float qmax) {
    float s = amax / qmax;
    // a step below 2^-126 has few bits: rounded down it would put the largest value beyond b bits, or be none
    if (s < 0x1p-126f && amax > 0.0f && (s == 0.0f || rintf(amax / s) > qmax)) s = __uint_as_float(__float_as_uint(s) + 1);
    return !finite ? __builtin_nanf("") : s > 0.0f ? s : 1.0f;
}
template <class T, int N, bool ONCE>
__device__ __forceinline__ void store_quantised(const NormArgs &a, int64_t row, int col, const float (&y)[N], float scale, int have) {
    float q[N], v[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
        q[k] = rintf(y[k] / scale);
        v[k] = q[k] * scale;
        if (!(fabsf(q[k]) <= 127.0f)) q[k] = 0.0f;  // a row with NaN or infinity: its scale says so
    }
    store_upto<int8_t, N, ONCE>(a.q + row * a.ldq + col, q, have);
    if (a.values) store_upto<T, N, ONCE>((T *)a.values + row * a.ldv + col, v, have);
}

template <class T, int TPR, int NV, bool QUANT, bool ONCE>
__global__ __launch_bounds__(TPR == 64 ? kNormThreads : TPR) void norm_kernel(const NormArgs a) {
    constexpr int N = kVec<T>, kRows = TPR == 64 ? kNormThreads / 64 : 1;
    __shared__ float lds[2][TPR / 64];
    const int t = TPR == 64 ? threadIdx.x & 63 : threadIdx.x;
    const int first = TPR == 64 ? threadIdx.x >> 6 : 0;
    float w[NV][N];
#pragma unroll
    for (int i = 0; i < NV; ++i) load_weights<N>(a.w, a.w_bf16, (i * TPR + t) * N, w[i], a.d - (i * TPR + t) * N);
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRows + first; row < a.rows; row += (int64_t)gridDim.x * kRows, turn ^= !QUANT) {
        const T *x = (const T *)a.x + row * a.ldx, *res = a.res ? (const T *)a.res + row * a.ldres : nullptr;
        float h[NV][N], sum = 0.0f;
        piece_t<T, N> px[NV], pr[NV];
#pragma unroll
        for (int i = 0; i < NV; ++i) px[i] = load_piece<T, N>(x + (i * TPR + t) * N, a.d - (i * TPR + t) * N);
        if (res) {
#pragma unroll
            for (int i = 0; i < NV; ++i) pr[i] = load_piece<T, N>(res + (i * TPR + t) * N, a.d - (i * TPR + t) * N);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            to_floats<T, N>(px[i], h[i]);
            if (!res) continue;
#pragma unroll
            for (int k = 0; k < N; ++k) h[i][k] += (float)pr[i][k];
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < N; ++k) sum += h[i][k] * h[i][k];
        sum = reduce_threads<TPR, false>(sum, lds[turn]);  // (two sets of words in turn: one barrier to a sum)
        const float r = 1.0f / sqrtf(sum / (float)a.d + a.eps);
        if (a.rstd && t == 0) a.rstd[row] = r;
        if (a.h) {
#pragma unroll
            for (int i = 0; i < NV; ++i) store_upto<T, N, ONCE>((T *)a.h + row * a.ldh + (i * TPR + t) * N, h[i], a.d - (i * TPR + t) * N);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < N; ++k) h[i][k] = h[i][k] * r * w[i][k];
        if constexpr (!QUANT) {
#pragma unroll
            for (int i = 0; i < NV; ++i) store_upto<T, N, ONCE>((T *)a.y + row * a.ldy + (i * TPR + t) * N, h[i], a.d - (i * TPR + t) * N);
        } else {
            float amax = 0.0f;  // infinity stands for NaN as well, which a maximum would lose
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int k = 0; k < N; ++k) amax = fmaxf(amax, h[i][k] == h[i][k] ? fabsf(h[i][k]) : __builtin_inff());
            amax = reduce_threads<TPR, true>(amax, lds[1]);
            const float scale = quant_scale(amax, amax < __builtin_inff(), a.qmax);
            if (t == 0) a.scale[row] = scale;
#pragma unroll
            for (int i = 0; i < NV; ++i) store_quantised<T, N, ONCE>(a, row, (i * TPR + t) * N, h[i], scale, a.d - (i * TPR + t) * N);
        }
    }
}

// Rows that no workgroup holds in registers: read once for each thing that is summed over them.
template <class T, bool QUANT>
__global__ __launch_bounds__(1024) void norm_long_kernel(const NormArgs a) {
    constexpr int N = kVec<T>, TPR = 1024;
    __shared__ float lds[2][TPR / 64];
    const int t = threadIdx.x;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.ldx, *res = a.res ? (const T *)a.res + row * a.ldres : nullptr;
        auto piece = [&](int col, float (&h)[N]) {
            load_upto<T, N>(x + col, h, a.d - col);
            if (!res) return;
            float f[N];
            load_upto<T, N>(res + col, f, a.d - col);
#pragma unroll
            for (int k = 0; k < N; ++k) h[k] += f[k];
        };
        float sum = 0.0f, amax = 0.0f;
        for (int col = t * N; col < a.d; col += TPR * N) {
            float h[N];
            piece(col, h);
#pragma unroll
            for (int k = 0; k < N; ++k) sum += h[k] * h[k];
        }
        sum = reduce_threads<TPR, false>(sum, lds[0]);
        const float r = 1.0f / sqrtf(sum / (float)a.d + a.eps);
        if (a.rstd && t == 0) a.rstd[row] = r;
        float scale = 1.0f;
        if constexpr (QUANT) {
            for (int col = t * N; col < a.d; col += TPR * N) {
                float h[N], w[N];
                piece(col, h);
                load_weights<N>(a.w, a.w_bf16, col, w, a.d - col);
#pragma unroll
                for (int k = 0; k < N; ++k) {
                    const float y = h[k] * r * w[k];
                    amax = fmaxf(amax, y == y ? fabsf(y) : __builtin_inff());
                }
            }
            amax = reduce_threads<TPR, true>(amax, lds[1]);
            scale = quant_scale(amax, amax < __builtin_inff(), a.qmax);
            if (t == 0) a.scale[row] = scale;
        }
        for (int col = t * N; col < a.d; col += TPR * N) {
            float h[N], w[N];
            piece(col, h);
            load_weights<N>(a.w, a.w_bf16, col, w, a.d - col);
            if (a.h) store_upto<T, N>((T *)a.h + row * a.ldh + col, h, a.d - col);
#pragma unroll
            for (int k = 0; k < N; ++k) h[k] = h[k] * r * w[k];
            if constexpr (QUANT) store_quantised<T, N, false>(a, row, col, h, scale, a.d - col);
            else store_upto<T, N>((T *)a.y + row * a.ldy + col, h, a.d - col);
        }
        __syncthreads();
    }
}

struct NormBackArgs {
    const void *gy, *x, *res, *gh, *w;
    const float *rstd;
    void *gx;
    void *gw;        // few rows: written by the workgroups from `groups` on
    float *partial;  // else [workgroups][d], or nullptr
    int64_t ldgy, ldx, ldres, ldgh, ldgx;
    int64_t rows;
    int d, w_bf16, groups;
};

// gw of 64 columns, a column to a lane, the rows shared by the waves.
template <class T, int THREADS>
__device__ __forceinline__ void norm_columns(const NormBackArgs &a, int block) {
    constexpr int kWaves = THREADS / 64, kAhead = 8;
    __shared__ float sums[kWaves][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = block * 64 + lane;
    float s = 0.0f;
    if (col < a.d)
        for (int64_t row0 = wave; row0 < a.rows; row0 += kWaves * kAhead) {
            T g[kAhead], x[kAhead], res[kAhead];
            float r[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int64_t row = min(row0 + k * kWaves, a.rows - 1);  // (those behind the last one count nothing)
                r[k] = row0 + k * kWaves < a.rows ? a.rstd[row] : 0.0f;
                g[k] = ((const T *)a.gy)[row * a.ldgy + col];
                x[k] = ((const T *)a.x)[row * a.ldx + col];
                res[k] = a.res ? ((const T *)a.res)[row * a.ldres + col] : (T)0.0f;
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (row0 + k * kWaves < a.rows) s += (float)g[k] * (((float)x[k] + (float)res[k]) * r[k]);
        }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave != 0 || col >= a.d) return;
#pragma unroll
    for (int k = 1; k < kWaves; ++k) s += sums[k][lane];
    if (a.w_bf16) ((__bf16 *)a.gw)[col] = (__bf16)s;
    else ((float *)a.gw)[col] = s;
}

// The same in a launch of its own, before the rows', where these write gx over what the columns read.
template <class T, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_columns_kernel(const NormBackArgs a) {
    norm_columns<T, THREADS>(a, blockIdx.x);
}

template <class T, int TPR, int NV, bool ONCE>
__global__ __launch_bounds__(TPR == 64 ? kNormThreads : TPR) void norm_back_kernel(const NormBackArgs a) {
    constexpr int N = kVec<T>, kRows = TPR == 64 ? kNormThreads / 64 : 1;
    if ((int)blockIdx.x >= a.groups) return norm_columns<T, TPR == 64 ? kNormThreads : TPR>(a, blockIdx.x - a.groups);
    __shared__ float lds[2][TPR / 64];
    __shared__ float fold[TPR == 64 ? kNormThreads * N : 1];
    const int t = TPR == 64 ? threadIdx.x & 63 : threadIdx.x;
    const int first = TPR == 64 ? threadIdx.x >> 6 : 0;
    float w[NV][N], gw[NV][N];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        load_weights<N>(a.w, a.w_bf16, (i * TPR + t) * N, w[i], a.d - (i * TPR + t) * N);
#pragma unroll
        for (int k = 0; k < N; ++k) gw[i][k] = 0.0f;
    }
    int turn = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRows + first; row < a.rows; row += (int64_t)a.groups * kRows, turn ^= 1) {
        float g[NV][N], h[NV][N], dot = 0.0f;
        piece_t<T, N> pg[NV], ph[NV], pr[NV], pgh[NV];
        const float r = a.rstd[row];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            pg[i] = load_piece<T, N>((const T *)a.gy + row * a.ldgy + (i * TPR + t) * N, a.d - (i * TPR + t) * N);
            ph[i] = load_piece<T, N>((const T *)a.x + row * a.ldx + (i * TPR + t) * N, a.d - (i * TPR + t) * N);
        }
        if (a.res) {
#pragma unroll
            for (int i = 0; i < NV; ++i) pr[i] = load_piece<T, N>((const T *)a.res + row * a.ldres + (i * TPR + t) * N, a.d - (i * TPR + t) * N);
        }
        if (a.gh) {
#pragma unroll
            for (int i = 0; i < NV; ++i) pgh[i] = load_piece<T, N>((const T *)a.gh + row * a.ldgh + (i * TPR + t) * N, a.d - (i * TPR + t) * N);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int k = 0; k < N; ++k) {
                g[i][k] = (float)pg[i][k];
                h[i][k] = (float)ph[i][k];
                if (a.res) h[i][k] += (float)pr[i][k];
                h[i][k] *= r;
                gw[i][k] += g[i][k] * h[i][k];
                g[i][k] *= w[i][k];
                dot += g[i][k] * h[i][k];
            }
        dot = reduce_threads<TPR, false>(dot, lds[turn]) / (float)a.d;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            float f[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float v = r * (g[i][k] - h[i][k] * dot);
                f[k] = a.gh ? (float)pgh[i][k] + v : v;
            }
            store_upto<T, N, ONCE>((T *)a.gx + row * a.ldgx + (i * TPR + t) * N, f, a.d - (i * TPR + t) * N);
        }
    }
    if (!a.partial) return;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int col = (i * TPR + t) * N;
        if constexpr (TPR == 64) {  // the waves' sums together
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k) fold[(first * 64 + t) * N + k] = gw[i][k];
            __syncthreads();
            if (first) continue;
#pragma unroll
            for (int k = 0; k < N; ++k)
                for (int v = 1; v < kRows; ++v) gw[i][k] += fold[(v * 64 + t) * N + k];
        }
        if (col < a.d) store_upto<float, N>(a.partial + (int64_t)blockIdx.x * a.d + col, gw[i], a.d - col);
    }
}

template <class T>
__global__ __launch_bounds__(1024) void norm_back_long_kernel(const NormBackArgs a) {
    constexpr int N = kVec<T>, TPR = 1024;
    if ((int)blockIdx.x >= a.groups) return norm_columns<T, 1024>(a, blockIdx.x - a.groups);
    __shared__ float lds[2][TPR / 64];
    const int t = threadIdx.x;
    float *part = a.partial ? a.partial + (int64_t)blockIdx.x * a.d : nullptr;
    int turn = 0;
    for (int64_t row = blockIdx.x; row < a.rows; row += a.groups, turn ^= 1) {
        const float r = a.rstd[row];
        const T *gy = (const T *)a.gy + row * a.ldgy, *x = (const T *)a.x + row * a.ldx, *res = a.res ? (const T *)a.res + row * a.ldres : nullptr;
        auto piece = [&](int col, float (&h)[N]) {
            load_upto<T, N>(x + col, h, a.d - col);
            if (!res) return;
            float f[N];
            load_upto<T, N>(res + col, f, a.d - col);
#pragma unroll
            for (int k = 0; k < N; ++k) h[k] += f[k];
        };
        float dot = 0.0f;
        for (int col = t * N; col < a.d; col += TPR * N) {
            float g[N], h[N], w[N];
            load_upto<T, N>(gy + col, g, a.d - col);
            piece(col, h);
            load_weights<N>(a.w, a.w_bf16, col, w, a.d - col);
#pragma unroll
            for (int k = 0; k < N; ++k) dot += g[k] * w[k] * (h[k] * r);
        }
        dot = reduce_threads<TPR, false>(dot, lds[turn]) / (float)a.d;
        for (int col = t * N; col < a.d; col += TPR * N) {
            float g[N], h[N], w[N], f[N], s[N];
            load_upto<T, N>(gy + col, g, a.d - col);
            piece(col, h);
            load_weights<N>(a.w, a.w_bf16, col, w, a.d - col);
            if (a.gh) load_upto<T, N>((const T *)a.gh + row * a.ldgh + col, f, a.d - col);
            if (part) {  // the thread's own columns, row after row
                load_upto<float, N>(part + col, s, row == blockIdx.x ? 0 : a.d - col);
#pragma unroll
                for (int k = 0; k < N; ++k) s[k] += g[k] * (h[k] * r);
                store_upto<float, N>(part + col, s, a.d - col);
            }
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const float v = r * (g[k] * w[k] - h[k] * r * dot);
                f[k] = a.gh ? f[k] + v : v;
            }
            store_upto<T, N>((T *)a.gx + row * a.ldgx + col, f, a.d - col);
        }
    }
}

// gw from the rows of partial sums: 32 columns and 32 rows at a time to a workgroup, in a fixed order.
__global__ __launch_bounds__(1024) void norm_fold_kernel(const float *partial, int parts, int d, void *gw, int bf16) {
    __shared__ float lds[32][33];
    const int c = threadIdx.x & 31, p = threadIdx.x >> 5, col = blockIdx.x * 32 + c;
    float s = 0.0f;
    if (col < d)
        for (int k0 = p; k0 < parts; k0 += 512) {  // sixteen loads at a time
            float f[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) f[k] = k0 + 32 * k < parts ? partial[(int64_t)(k0 + 32 * k) * d + col] : 0.0f;
#pragma unroll
            for (int k = 0; k < 16; ++k) s += f[k];
        }
    lds[p][c] = s;
    __syncthreads();
    if (p != 0 || col >= d) return;
#pragma unroll
    for (int k = 1; k < 32; ++k) s += lds[k][c];
    if (bf16) ((__bf16 *)gw)[col] = (__bf16)s;
    else ((float *)gw)[col] = s;
}

static int norm_pieces(int d, int dtype) { return dtype == IMUNPACK_F32 ? (d + 3) / 4 : (d + 7) / 8; }
static bool known_type(int t) { return t == IMUNPACK_F32 || t == IMUNPACK_BF16; }
// Workgroups of the backward pass, each of which leaves a row of partial sums.
static int back_groups(int64_t rows, int pieces) {
    const int64_t per = pieces <= 256 ? kNormThreads / 64 : 1;
    return (int)std::min<int64_t>((rows + per - 1) / per, kNormPartials);
}

template <class T, bool QUANT, bool ONCE>
static int launch_norm(const NormArgs &a, int pieces, hipStream_t st) {
    const int64_t groups = pieces <= 256 ? (a.rows + kNormThreads / 64 - 1) / (kNormThreads / 64) : a.rows;
    const dim3 grid((unsigned)std::min<int64_t>(groups, kNormGroups));
    auto go = [&](auto nv) {
        constexpr int NV = decltype(nv)::value;
        if (pieces <= 256) hipLaunchKernelGGL((norm_kernel<T, 64, NV, QUANT, ONCE>), grid, dim3(kNormThreads), 0, st, a);
        else if (pieces <= 1024) hipLaunchKernelGGL((norm_kernel<T, 256, NV, QUANT, ONCE>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((norm_kernel<T, 1024, NV, QUANT, ONCE>), grid, dim3(1024), 0, st, a);
    };
    const int tpr = pieces <= 256 ? 64 : pieces <= 1024 ? 256 : 1024;
    switch ((pieces + tpr - 1) / tpr) {
        case 1: go(std::integral_constant<int, 1>()); break;
        case 2: go(std::integral_constant<int, 2>()); break;
        case 3: go(std::integral_constant<int, 3>()); break;
        case 4: go(std::integral_constant<int, 4>()); break;
        default: hipLaunchKernelGGL((norm_long_kernel<T, QUANT>), grid, dim3(1024), 0, st, a);
    }
    return launch_status();
}

template <class T>
static int launch_norm_columns(const NormBackArgs &a, int pieces, hipStream_t st) {
    const dim3 grid((unsigned)((a.d + 63) / 64));
    if (pieces <= 1024) hipLaunchKernelGGL((norm_columns_kernel<T, kNormThreads>), grid, dim3(kNormThreads), 0, st, a);
    else hipLaunchKernelGGL((norm_columns_kernel<T, 1024>), grid, dim3(1024), 0, st, a);
    return launch_status();
}

template <class T, bool ONCE>
static int launch_norm_back(const NormBackArgs &a, int pieces, hipStream_t st) {
    const dim3 grid((unsigned)(a.groups + (a.gw ? (a.d + 63) / 64 : 0)));
    auto go = [&](auto nv) {
        constexpr int NV = decltype(nv)::value;
        if (pieces <= 256) hipLaunchKernelGGL((norm_back_kernel<T, 64, NV, ONCE>), grid, dim3(kNormThreads), 0, st, a);
        else if (pieces <= 1024) hipLaunchKernelGGL((norm_back_kernel<T, 256, NV, ONCE>), grid, dim3(256), 0, st, a);
        else if constexpr (NV * kVec<T> <= (kVec<T> == 4 ? 12 : 16)) hipLaunchKernelGGL((norm_back_kernel<T, 1024, NV, ONCE>), grid, dim3(1024), 0, st, a);
        else hipLaunchKernelGGL((norm_back_long_kernel<T>), grid, dim3(1024), 0, st, a);  // (more would not fit the 128 registers of a thread)
    };
    const int tpr = pieces <= 256 ? 64 : pieces <= 1024 ? 256 : 1024;
    switch ((pieces + tpr - 1) / tpr) {
        case 1: go(std::integral_constant<int, 1>()); break;
        case 2: go(std::integral_constant<int, 2>()); break;
        case 3: go(std::integral_constant<int, 3>()); break;
        case 4: go(std::integral_constant<int, 4>()); break;
        default: hipLaunchKernelGGL((norm_back_long_kernel<T>), grid, dim3(1024), 0, st, a);
    }
    return launch_status();
}
}  // namespace imu

using namespace imu;

// Sizes and strides that every call of this file takes.
static bool norm_sizes(int64_t rows, int64_t d, int dtype, int w_dtype) {
    return rows >= 0 && rows <= (int64_t)1 << 31 && d > 0 && d <= 1 << 24 && known_type(dtype) && known_type(w_dtype);
}

// Whether rows of d elements of two arrays share memory.
static bool rows_overlap(const void *p, int64_t ldp, const void *q, int64_t ldq, int64_t rows, int64_t d, int64_t size) {
    if (!p || !q || rows == 0) return false;
    const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
    return a < b + (uintptr_t)(((rows - 1) * ldq + d) * size) && b < a + (uintptr_t)(((rows - 1) * ldp + d) * size);
}

static int norm_forward(NormArgs &a, int64_t d, int dtype, int w_dtype, hipStream_t st) {
    if (a.rows == 0) return IMUNPACK_OK;
    a.d = (int)d;
    a.w_bf16 = w_dtype == IMUNPACK_BF16;
    const int pieces = norm_pieces(a.d, dtype);
    const int64_t size = dtype == IMUNPACK_F32 ? 4 : 2;
    const int64_t moved = a.rows * d * (size * (1 + (a.res != nullptr) + (a.y != nullptr) + (a.h != nullptr) + (a.values != nullptr)) + (a.q != nullptr));
    const bool once = moved >= kLastLevelCache;
    auto go = [&](auto type, auto quant) {
        using T = decltype(type);
        constexpr bool QUANT = decltype(quant)::value;
        return once ? launch_norm<T, QUANT, true>(a, pieces, st) : launch_norm<T, QUANT, false>(a, pieces, st);
    };
    if (dtype == IMUNPACK_F32) return a.qmax > 0.0f ? go(float(), std::true_type()) : go(float(), std::false_type());
    return a.qmax > 0.0f ? go(__bf16(), std::true_type()) : go(__bf16(), std::false_type());
}

extern "C" int imunpack_rmsnorm(const void *x, int64_t ldx, const void *residual, int64_t ldres, const void *weight,
                                int64_t rows, int64_t d, int dtype, int weight_dtype, float eps, void *y, int64_t ldy,
                                void *h, int64_t ldh, float *rstd, imunpack_stream_t stream) {
    if (!norm_sizes(rows, d, dtype, weight_dtype) || !(eps >= 0.0f) || ldx < d || ldy < d || (residual && ldres < d) || (h && ldh < d))
        return IMUNPACK_EINVAL;
    if (rows > 0 && (!x || !weight || !y)) return IMUNPACK_EINVAL;
    NormArgs a = {};
    a.x = x; a.res = residual; a.w = weight; a.y = y; a.h = h; a.rstd = rstd;
    a.ldx = ldx; a.ldres = ldres; a.ldy = ldy; a.ldh = ldh;
    a.rows = rows; a.eps = eps;
    return norm_forward(a, d, dtype, weight_dtype, (hipStream_t)stream);
}

extern "C" int imunpack_rmsnorm_quantize(const void *x, int64_t ldx, const void *residual, int64_t ldres, const void *weight,
                                         int64_t rows, int64_t d, int dtype, int weight_dtype, float eps, int b, int8_t *q,
                                         int64_t ldq, float *scale, void *values, int64_t ldv, void *h, int64_t ldh,
                                         imunpack_stream_t stream) {
    if (!norm_sizes(rows, d, dtype, weight_dtype) || !(eps >= 0.0f) || b < 2 || b > 8 || ldx < d || ldq < d || (residual && ldres < d) ||
        (values && ldv < d) || (h && ldh < d))
        return IMUNPACK_EINVAL;
    if (rows > 0 && (!x || !weight || !q || !scale)) return IMUNPACK_EINVAL;
    NormArgs a = {};
    a.x = x; a.res = residual; a.w = weight; a.h = h; a.q = q; a.scale = scale; a.values = values;
    a.ldx = ldx; a.ldres = ldres; a.ldh = ldh; a.ldq = ldq; a.ldv = ldv;
    a.rows = rows; a.eps = eps;
    a.qmax = (float)((1 << (b - 1)) - 1);
    return norm_forward(a, d, dtype, weight_dtype, (hipStream_t)stream);
}

extern "C" int imunpack_rmsnorm_backward_workspace(int64_t rows, int64_t d, int dtype, size_t *bytes) {
    if (!norm_sizes(rows, d, dtype, IMUNPACK_F32) || !bytes) return IMUNPACK_EINVAL;
    *bytes = rows <= kNormFewRows ? 0 : (size_t)back_groups(rows, norm_pieces((int)d, dtype)) * (size_t)d * sizeof(float);
    return IMUNPACK_OK;
}

extern "C" int imunpack_rmsnorm_backward(const void *gy, int64_t ldgy, const void *x, int64_t ldx, const void *residual, int64_t ldres,
                                         const void *gh, int64_t ldgh, const void *weight, const float *rstd, int64_t rows, int64_t d, int dtype, int weight_dtype,
                                         void *gx, int64_t ldgx, void *gweight, void *workspace, size_t workspace_bytes,
                                         imunpack_stream_t stream) {
    if (!norm_sizes(rows, d, dtype, weight_dtype) || ldgy < d || ldx < d || (residual && ldres < d) || (gh && ldgh < d) || ldgx < d) return IMUNPACK_EINVAL;
    if (rows > 0 && (!gy || !x || !weight || !rstd || !gx)) return IMUNPACK_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    const int pieces = norm_pieces((int)d, dtype), groups = back_groups(rows, pieces);
    const bool few = rows <= kNormFewRows;
    if (gweight && !few) {
        if (!workspace) return IMUNPACK_EINVAL;
        if (workspace_bytes < (size_t)groups * (size_t)d * sizeof(float)) return IMUNPACK_ESMALL;
    }
    NormBackArgs a = {};
    a.gy = gy; a.x = x; a.res = residual; a.gh = gh; a.w = weight; a.rstd = rstd; a.gx = gx;
    a.partial = gweight && !few ? (float *)workspace : nullptr;
    a.gw = few ? gweight : nullptr;
    a.groups = groups;
    a.ldgy = ldgy; a.ldx = ldx; a.ldres = ldres; a.ldgh = ldgh; a.ldgx = ldgx;
    a.rows = rows; a.d = (int)d; a.w_bf16 = weight_dtype == IMUNPACK_BF16;
    if (rows > 0) {
        const int64_t size = dtype == IMUNPACK_F32 ? 4 : 2;
        // gx may lie where gy does, of which the columns' workgroups read every row: they are done first then
        if (a.gw && (rows_overlap(gx, ldgx, gy, ldgy, rows, d, size) || rows_overlap(gx, ldgx, x, ldx, rows, d, size) || rows_overlap(gx, ldgx, residual, ldres, rows, d, size))) {
            IMU_TRY(dtype == IMUNPACK_F32 ? launch_norm_columns<float>(a, pieces, st) : launch_norm_columns<__bf16>(a, pieces, st));
            a.gw = nullptr;
        }
        const bool once = rows * d * size * (3 + (residual != nullptr) + (gh != nullptr)) >= kLastLevelCache;
        if (dtype == IMUNPACK_F32) IMU_TRY((once ? launch_norm_back<float, true> : launch_norm_back<float, false>)(a, pieces, st));
        else IMU_TRY((once ? launch_norm_back<__bf16, true> : launch_norm_back<__bf16, false>)(a, pieces, st));
    }
    if (gweight && (!few || rows == 0)) {  // (no rows: zeros)
        hipLaunchKernelGGL(norm_fold_kernel, dim3((unsigned)((d + 31) / 32)), dim3(1024), 0, st, a.partial, groups, (int)d, gweight, a.w_bf16);
        return launch_status();
    }
    return IMUNPACK_OK;
}
