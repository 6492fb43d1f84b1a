// Softmax cross entropy of x W^T over a vocabulary, and its gradients, without keeping the logits.
//
//   l[t, v] = sum_k x[t, k] W[v, k],   lse[t] = log sum_v exp l[t, v],   loss[t] = lse[t] - l[t, target[t]]
//   G[t, v] = (exp(l[t, v] - lse[t]) - [v = target[t]]) g[t],   gx = G W,   gW = G^T x            (g: the gradient of loss[t])
//
// Rows without a target take no part: those with one are gathered first, and how many there are is known on the device alone.
// Forward: a tile of the product keeps, per row t, the largest logit and the sum of exponentials of its part of the vocabulary, and a
// small kernel joins them.  Backward: a tile is made again and G leaves it in 16 bits, both ways round, for one piece of the vocabulary at a
// time (at most kPieceBytes); gx and the piece's rows of gW are products of it.  8 T V d operations in all, all on the matrix cores.
//
// bfloat16 operands: products in bfloat16, G rounded to bfloat16.  fp32 operands: each value is the sum of two binary16 numbers
// (22 bits of it; scaled by a power of two so that the operand's largest lies below 2^15) and a product is three of them, which is within
// the rounding of a binary32 sum; three times the instructions at eight times and more the rate of the binary32 ones.
#include "common.h"
#include "elements.h"
#include "product.h"

#include <algorithm>
#include <atomic>

namespace imu {
constexpr int64_t kPieceBytes = 1ll << 30;  // G of a piece of the vocabulary, both ways round, at most (or 256 columns)
constexpr int kTop = 14;                    // the largest magnitude of a scaled operand is below 2^(kTop + 1)
constexpr int kXentSlots = 256;             // parts of the tiles of gx that go at a time: one to a CU

struct XentHeader {
    int32_t count;    // rows with a target
    int32_t bad;      // rows whose target is outside the vocabulary
    uint32_t amax[2]; // bits of the largest magnitude of x (rows with a target) and of W
    int32_t gexp;     // exponent of the largest gradient of a row
    int32_t pad[59];
};
static_assert(sizeof(XentHeader) == 256, "header");

// What 2 to its power an operand is multiplied by before it is split.
__device__ __forceinline__ int scale_exponent(uint32_t amax) { return min(kTop - ((int)(amax >> 23) - 127), 126); }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Rows with a target in order, their targets, and for every row its place among them (-1: none, -2: a target outside the vocabulary).
__global__ __launch_bounds__(1024) void xent_rows_kernel(const int64_t *target, int rows, int64_t vocab, int64_t ignore, XentHeader *hdr, int32_t *source,
                                                         int32_t *place, int32_t *wanted, float *loss) {
    __shared__ int32_t sums[2][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int base = 0, bad = 0, turn = 0;
    for (int t0 = 0; t0 < rows; t0 += 1024, turn ^= 1) {
        const int t = t0 + threadIdx.x;
        const int64_t v = t < rows ? target[t] : ignore;
        const bool inside = v >= 0 && v < vocab && v != ignore, outside = !inside && v != ignore;
        const uint64_t mask = __ballot(inside);
        bad |= __ballot(outside) != 0;
        if (lane == 0) sums[turn][wave] = __builtin_popcountll(mask);
        __syncthreads();
        int before = base, all = 0;
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            before += w < wave ? sums[turn][w] : 0;
            all += sums[turn][w];
        }
        const int at = before + __builtin_popcountll(mask & ((1ull << lane) - 1));
        if (inside) {
            source[at] = t;
            wanted[at] = (int)v;
        }
        if (t < rows) {
            place[t] = inside ? at : outside ? -2 : -1;
            if (loss && !inside) loss[t] = outside ? __builtin_nanf("") : 0.0f;
        }
        base += all;
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) {
        hdr->count = base;
        hdr->bad = bad;
        hdr->amax[0] = hdr->amax[1] = 0;
    }
}

// Largest magnitudes of x (rows with a target) and W.
__global__ __launch_bounds__(256) void xent_amax_kernel(const float *x, int64_t ldx, const float *w, int64_t ldw, int d, int64_t vocab, XentHeader *hdr,
                                                        const int32_t *source, int xgroups) {
    __shared__ float lds[4];
    const bool isX = (int)blockIdx.x < xgroups;
    const int64_t rows = isX ? hdr->count : vocab, step = isX ? xgroups : gridDim.x - xgroups;
    float m = 0.0f;
    for (int64_t row = isX ? blockIdx.x : blockIdx.x - xgroups; row < rows; row += step) {
        const float *p = isX ? x + (int64_t)source[row] * ldx : w + row * ldw;
        for (int col = threadIdx.x * 4; col < d; col += 1024) {
            float f[4];
            load_upto<float, 4>(p + col, f, d - col);
#pragma unroll
            for (int k = 0; k < 4; ++k) m = fmaxf(m, fabsf(f[k]));
        }
    }
    m = reduce_threads<256, true>(m, lds);
    if (threadIdx.x == 0 && m > 0.0f) atomicMax(&hdr->amax[isX ? 0 : 1], __float_as_uint(m));
}

struct PrepareArgs {
    const void *x, *w;
    int64_t ldx, ldw;
    const XentHeader *hdr;
    const int32_t *source;
    char *px, *pw, *tx, *tw;               // rows and columns of x and W in 16 bits; nullptr: not wanted
    int64_t px2, pw2, tx2, tw2;            // from the first piece of a value to the second, bytes
    int64_t pitch_p, pitch_tx, pitch_tw;   // bytes from row to row
    int64_t vocab;
    int d, xtiles;
};
// 64 rows by 64 columns of x (gathered) or W: in 16 bits, one or two numbers to a value, row by row and transposed; zeros around.
template <class T>
__global__ __launch_bounds__(256) void xent_prepare_kernel(const PrepareArgs a) {
    constexpr bool SPLIT = sizeof(T) == 4;
    __shared__ uint32_t tile[64][65];
    const bool isX = (int)blockIdx.x < a.xtiles;
    const int64_t rows = isX ? a.hdr->count : a.vocab, row0 = (int64_t)(isX ? blockIdx.x : blockIdx.x - a.xtiles) * 64;
    if (row0 >= rows) return;
    const int col0 = blockIdx.y * 64, r = threadIdx.x >> 2, c = (threadIdx.x & 3) * 16;
    const float scale = SPLIT ? power_of_two(scale_exponent(a.hdr->amax[isX ? 0 : 1])) : 1.0f;
    const int64_t row = row0 + r;
    const T *p = isX ? (const T *)a.x + (row < rows ? (int64_t)a.source[row] : 0) * a.ldx : (const T *)a.w + row * a.ldw;
    const int have = row < rows ? a.d - (col0 + c) : 0;
    uint32_t q[16];
    if constexpr (SPLIT) {
        piece_t<float, 4> f[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = load_piece<float, 4>(p + col0 + c + 4 * k, have - 4 * k);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
            const float v = f[k >> 2][k & 3] * scale;
            const _Float16 h = (_Float16)v, l = (_Float16)(v - (float)h);
            q[k] = (uint32_t)__builtin_bit_cast(uint16_t, h) | (uint32_t)__builtin_bit_cast(uint16_t, l) << 16;
        }
    } else {
        piece_t<__bf16, 8> f[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) f[k] = load_piece<__bf16, 8>(p + col0 + c + 8 * k, have - 8 * k);
#pragma unroll
        for (int k = 0; k < 16; ++k) q[k] = __builtin_bit_cast(uint16_t, (__bf16)f[k >> 3][k & 7]);
    }
    auto put = [&](char *to, const uint32_t (&v)[16], bool second) {
        v4i32 s[2];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t lo = second ? v[2 * k] >> 16 : v[2 * k] & 0xffffu, hi = second ? v[2 * k + 1] & 0xffff0000u : v[2 * k + 1] << 16;
            s[k >> 2][k & 3] = (int)(lo | hi);
        }
        *reinterpret_cast<v4i32 *>(to) = s[0];
        *reinterpret_cast<v4i32 *>(to + 16) = s[1];
    };
    char *out = isX ? a.px : a.pw;
    if (out && (isX || row < rows)) {  // (rows of zeros behind the last of x; there is no room behind W's)
        char *to = out + row * a.pitch_p + (col0 + c) * 2;
        put(to, q, false);
        if (SPLIT) put(to + (isX ? a.px2 : a.pw2), q, true);
    }
    out = isX ? a.tx : a.tw;
    if (!out) return;
#pragma unroll
    for (int k = 0; k < 16; ++k) tile[r][c + k] = q[k];
    __syncthreads();
    if (col0 + r >= a.d) return;
#pragma unroll
    for (int k = 0; k < 16; ++k) q[k] = tile[c + k][r];
    char *to = out + (int64_t)(col0 + r) * (isX ? a.pitch_tx : a.pitch_tw) + (row0 + c) * 2;
    put(to, q, false);
    if (SPLIT) put(to + (isX ? a.tx2 : a.tw2), q, true);
}

struct LogitArgs {
    Operand w, x;             // rows of the vocabulary (of this piece) and of x
    const XentHeader *hdr;
    const int32_t *wanted;
    float *stats, *hit;       // forward: [part of the vocabulary][row] largest logit and sum; the target's logit
    const float *lse, *g;     // backward
    char *G, *GT;             // [row][vocabulary of the piece] and [vocabulary of the piece][row]
    int64_t G2, GT2, pitch_G, pitch_GT;
    int64_t stride;           // rows there is room for
    int v0, ktiles;           // first column of the piece
    int vlimit;               // columns of the piece, rounded up to whole k-tiles (what is stored of G)
};
constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// A tile of logits, vocabulary down, rows of x across: a lane holds one row of x per column block, so that the sums over the
// vocabulary are sums over its registers and one exchange between the halves of the wave.
template <bool F16, int T, bool BACK>
__global__ __launch_bounds__(kProductThreads, T == 4 ? 1 : 2) void xent_logits_kernel(const LogitArgs a) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    constexpr int kEdge = 64 * T;
    const int count = a.hdr->count, vocab = a.w.rows, mtiles = (vocab + kEdge - 1) / kEdge, ntiles = (count + kEdge - 1) / kEdge;
    if ((int)blockIdx.x >= mtiles * ntiles) return;
    int tm, tn;
    tile_at(blockIdx.x, mtiles, ntiles, tm, tn);
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
    Operand x = a.x;
    x.rows = count;
    v16f32 acc[T][T];
    product_tile<F16, T, T, F16 ? 3 : 1>(a.w, x, tm * kEdge, tn * kEdge, 0, a.ktiles, smem, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, lrow = lane & 31, lhalf = lane >> 5;
    const int vbase = tm * kEdge + (wave >> 1) * 32 * T + 4 * lhalf, tbase = tn * kEdge + (wave & 1) * 32 * T + lrow;
    const int down = F16 ? -(scale_exponent(a.hdr->amax[0]) + scale_exponent(a.hdr->amax[1])) : 0;
#pragma unroll
    for (int j = 0; j < T; ++j) {
        const int t = tbase + 32 * j;
        const int target = t < count ? a.wanted[t] - a.v0 : -1;  // in columns of the piece
        if constexpr (!BACK) {
            float top = -__builtin_inff(), sum = 0.0f, hit = 0.0f;
#pragma unroll
            for (int i = 0; i < T; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int v = vbase + 32 * i + (r >> 2) * 8 + (r & 3);
                    if (F16) acc[i][j][r] = ldexpf(acc[i][j][r], down);
                    if (v < vocab) top = fmaxf(top, acc[i][j][r]);
                    if (v == target) hit = acc[i][j][r];
                }
            top = fmaxf(top, __shfl_xor(top, 32));
            const float from = top == -__builtin_inff() ? 0.0f : top;  // (nothing of the vocabulary in this part)
#pragma unroll
            for (int i = 0; i < T; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int v = vbase + 32 * i + (r >> 2) * 8 + (r & 3);
                    sum += v < vocab ? fast_exp(acc[i][j][r] - from) : 0.0f;
                }
            sum += __shfl_xor(sum, 32);
            if (t >= count) continue;
            if (lhalf == 0) {
                float *to = a.stats + ((int64_t)(2 * tm + (wave >> 1)) * a.stride + t) * 2;
                to[0] = top;
                to[1] = sum;
            }
            const int in = target - vbase + 4 * lhalf;  // of the wave's columns
            if (in >= 0 && in < 32 * T && ((in >> 2) & 1) == lhalf) a.hit[t] = hit;
        } else {
            const float lse = t < count ? a.lse[t] : 0.0f, g = t < count ? a.g[t] : 0.0f, scaled = F16 ? g * power_of_two(kTop) : g;
#pragma unroll
            for (int i = 0; i < T; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int v = vbase + 32 * i + 8 * q;
                    uint16_t hi[4], lo[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        float l = acc[i][j][4 * q + k];
                        if (F16) l = ldexpf(l, down);
                        float p = fast_exp(l - lse) - (v + k == target ? 1.0f : 0.0f);
                        p = v + k < vocab && t < count ? p * scaled : 0.0f;
                        if constexpr (F16) {
                            const _Float16 h = (_Float16)p;
                            hi[k] = __builtin_bit_cast(uint16_t, h);
                            lo[k] = __builtin_bit_cast(uint16_t, (_Float16)(p - (float)h));
                        } else {
                            hi[k] = __builtin_bit_cast(uint16_t, (__bf16)p);
                            lo[k] = 0;
                        }
                    }
                    auto put = [&](const uint16_t (&e)[4], int64_t offG, int64_t offGT) {
                        if (t < count && v < a.vlimit)
                            *reinterpret_cast<uint2 *>(a.G + offG + t * a.pitch_G + v * 2) =
                                make_uint2((uint32_t)e[0] | (uint32_t)e[1] << 16, (uint32_t)e[2] | (uint32_t)e[3] << 16);
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (v + k < vocab && t < (count + 63) / 64 * 64) *reinterpret_cast<uint16_t *>(a.GT + offGT + (v + k) * a.pitch_GT + t * 2) = e[k];
                    };
                    put(hi, 0, 0);
                    if (F16) put(lo, a.G2, a.GT2);
                }
        }
    }
}

// lse and loss of 32 rows from the parts of the vocabulary, eight threads to a row.
__global__ __launch_bounds__(256) void xent_join_kernel(const float *stats, const float *hit, int parts, int64_t stride, const XentHeader *hdr, const int32_t *source,
                                                        float *lse, float *row_loss, float *loss) {
    __shared__ float tops[8][32], sums[8][32];
    const int r = threadIdx.x & 31, g = threadIdx.x >> 5, t = blockIdx.x * 32 + r, count = hdr->count;
    if ((int)blockIdx.x * 32 >= count) return;
    float top = -__builtin_inff(), sum = 0.0f;
    if (t < count)
        for (int k = g; k < parts; k += 8) {
            const float2 s = *reinterpret_cast<const float2 *>(stats + ((int64_t)k * stride + t) * 2);
            const float next = fmaxf(top, s.x);
            if (next > -__builtin_inff()) sum = sum * fast_exp(top - next) + s.y * fast_exp(s.x - next);
            else sum += s.y;  // (NaN stays)
            top = next;
        }
    tops[g][r] = top;
    sums[g][r] = sum;
    __syncthreads();
    if (g != 0 || t >= count) return;
#pragma unroll
    for (int k = 1; k < 8; ++k) top = fmaxf(top, tops[k][r]);
    sum = 0.0f;
    const float from = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
    for (int k = 0; k < 8; ++k) sum += sums[k][r] * fast_exp(tops[k][r] - from);
    const float l = from + logf(sum);
    lse[t] = l;
    const float v = l - hit[t];
    row_loss[t] = v;
    if (loss) loss[source[t]] = v;
}

// The sum (mean) over the rows with a target, in a fixed order.
__global__ __launch_bounds__(1024) void xent_sum_kernel(const float *row_loss, const XentHeader *hdr, int mean, float *loss) {
    __shared__ float lds[16];
    const int count = hdr->count;
    float s = 0.0f;
    for (int t = threadIdx.x; t < count; t += 1024) s += row_loss[t];
    s = reduce_threads<1024, false>(s, lds);
    if (threadIdx.x == 0) *loss = hdr->bad ? __builtin_nanf("") : mean && count > 0 ? s / (float)count : s;
}

// The gradient of each row's loss, divided by a power of two that the results are multiplied with at the end.
__global__ __launch_bounds__(1024) void xent_factor_kernel(const float *grad, int reduction, XentHeader *hdr, const int32_t *source, float *g) {
    __shared__ float lds[16];
    const int count = hdr->count;
    const float one = reduction == IMUNPACK_NONE ? 0.0f : reduction == IMUNPACK_MEAN ? *grad / (float)max(count, 1) : *grad;
    float m = fabsf(one);
    if (reduction == IMUNPACK_NONE)
        for (int t = threadIdx.x; t < count; t += 1024) m = fmaxf(m, fabsf(grad[source[t]]));
    m = reduce_threads<1024, true>(m, lds);
    const int e = m > 0.0f ? (int)(__float_as_uint(m) >> 23) - 127 : 0;
    if (threadIdx.x == 0) hdr->gexp = e;
    for (int t = threadIdx.x; t < count; t += 1024) g[t] = ldexpf(reduction == IMUNPACK_NONE ? grad[source[t]] : one, -e);
}

// How the tiles of gx are cut along the vocabulary, so that every CU has a part.
__device__ __forceinline__ int gx_parts(int tiles, int slots) { return tiles > 0 ? max(1, slots / tiles) : 1; }

struct GradXArgs {
    Operand G, wt;     // [row][vocabulary of the piece], [feature][vocabulary of the piece]
    const XentHeader *hdr;
    float *parts;      // [slot][tile]
    int ktiles, slots, first;
};
template <bool F16, int T>
__global__ __launch_bounds__(kProductThreads, T == 4 ? 1 : 2) void xent_grad_x_kernel(const GradXArgs a) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    constexpr int kEdge = 64 * T;
    const int count = a.hdr->count, mtiles = (count + kEdge - 1) / kEdge, ntiles = (a.wt.rows + kEdge - 1) / kEdge, tiles = mtiles * ntiles;
    const int parts = gx_parts(tiles, a.slots);
    if ((int)blockIdx.x >= tiles * parts) return;
    // workgroups of an XCD: consecutive tiles of one part of the vocabulary
    const int xcd = blockIdx.x & 7, idx = blockIdx.x >> 3, per = tiles * parts >> 3, rem = (tiles * parts) & 7;
    const int slot = __builtin_amdgcn_readfirstlane(xcd * per + min(xcd, rem) + idx);
    const int part = slot / tiles, tile = slot - part * tiles, tn = tile / mtiles, tm = tile - tn * mtiles;
    Operand G = a.G;
    G.rows = count;
    v16f32 acc[T][T];
    const int k0 = (int)((int64_t)a.ktiles * part / parts), k1 = (int)((int64_t)a.ktiles * (part + 1) / parts);
    product_tile<F16, T, T, F16 ? 3 : 1>(G, a.wt, tm * kEdge, tn * kEdge, k0, k1, smem, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float *to = a.parts + (int64_t)slot * kEdge * kEdge + ((wave >> 1) * 32 * T + 4 * (lane >> 5)) * kEdge + (wave & 1) * 32 * T + (lane & 31);
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int j = 0; j < T; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                float *p = to + (32 * i + (r >> 2) * 8 + (r & 3)) * kEdge + 32 * j;
                *p = a.first ? acc[i][j][r] : *p + acc[i][j][r];
            }
}

// Rows of gx from the parts of its tiles; zeros for rows without a target.
template <class T>
__global__ __launch_bounds__(256) void xent_fold_x_kernel(const float *parts, const XentHeader *hdr, const int32_t *place, int d, int edge, int slots, T *gx, int64_t ldgx) {
    const int64_t row = blockIdx.x;
    const int col = (blockIdx.y * 256 + threadIdx.x) * 4, at = place[row];
    if (col >= d) return;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (at >= 0) {
        const int mtiles = (hdr->count + edge - 1) / edge, ntiles = (d + edge - 1) / edge, tiles = mtiles * ntiles, n = gx_parts(tiles, slots);
        const int tile = col / edge * mtiles + at / edge;
        const float *p = parts + (int64_t)tile * edge * edge + (at % edge) * edge + col % edge;
        for (int k = 0; k < n; ++k) {
            const float4 f = *reinterpret_cast<const float4 *>(p + (int64_t)k * tiles * edge * edge);
            s[0] += f.x; s[1] += f.y; s[2] += f.z; s[3] += f.w;
        }
        const int e = hdr->gexp - (sizeof(T) == 4 ? kTop + scale_exponent(hdr->amax[1]) : 0);
#pragma unroll
        for (int k = 0; k < 4; ++k) s[k] = ldexpf(s[k], e);
    }
    store_upto<T, 4>(gx + row * ldgx + col, s, d - col);
}

struct GradWArgs {
    Operand GT, xt;    // [vocabulary of the piece][row], [feature][row]
    const XentHeader *hdr;
    void *gw;          // the piece's first row
    int64_t ldgw;
};
template <bool F16, int T>
__global__ __launch_bounds__(kProductThreads, T == 4 ? 1 : 2) void xent_grad_w_kernel(const GradWArgs a) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    constexpr int kEdge = 64 * T;
    const int mtiles = (a.GT.rows + kEdge - 1) / kEdge, ntiles = (a.xt.rows + kEdge - 1) / kEdge;
    int tm, tn;
    tile_at(blockIdx.x, mtiles, ntiles, tm, tn);
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
    v16f32 acc[T][T];
    product_tile<F16, T, T, F16 ? 3 : 1>(a.GT, a.xt, tm * kEdge, tn * kEdge, 0, (a.hdr->count + kStageCols - 1) / kStageCols, smem, acc);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int v0 = tm * kEdge + (wave >> 1) * 32 * T + 4 * (lane >> 5), c0 = tn * kEdge + (wave & 1) * 32 * T + (lane & 31);
    const int e = a.hdr->gexp - (F16 ? kTop + scale_exponent(a.hdr->amax[0]) : 0);
    using Out = std::conditional_t<F16, float, __bf16>;
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int j = 0; j < T; ++j) {
            const int col = c0 + 32 * j;
            if (col >= a.xt.rows) continue;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int64_t v = v0 + 32 * i + (r >> 2) * 8 + (r & 3);
                if (v < a.GT.rows) ((Out *)a.gw)[v * a.ldgw + col] = (Out)ldexpf(acc[i][j][r], e);
            }
        }
}

static int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Where everything lies in the forward pass's buffer, which the backward pass reads, and in the backward pass's own.
struct XentLayout {
    int64_t dp, tp, vp;           // features, rows, vocabulary rounded up to what the products read
    bool split, direct;           // two numbers to a value; W read in place
    int64_t pitch_p, pitch_tx, pitch_tw;
    size_t source, place, wanted, lse, row_loss, hit, stats, px, pw, tx, tw, bytes;
    size_t px2, pw2, tx2, tw2;
    int edge_l, edge_x, edge_w;   // tile edges of the three products
    int parts_v;                  // parts of the vocabulary whose sums are joined
    int64_t piece, pieces;        // columns of the vocabulary to a piece
    int slots;
    size_t g, G, GT, G2, GT2, gparts, back_bytes;
    int64_t pitch_G, pitch_GT;
};
// Large tiles where they fill the CUs.
static int tile_edge(int64_t m, int64_t n) {
    const int64_t large = up(m, 256) / 256 * (up(n, 256) / 256);
    return large >= 128 ? 256 : 128;
}
static XentLayout xent_layout(const void *w, int64_t ldw, int64_t rows, int64_t d, int64_t vocab, int dtype, bool grad) {
    XentLayout l = {};
    l.split = dtype == IMUNPACK_F32;
    l.dp = up(d, kStageCols);
    l.tp = up(std::max<int64_t>(rows, 1), 256);
    l.vp = up(vocab, 256);
    l.direct = !l.split && d % kStageCols == 0 && ldw % 8 == 0 && (size_t)w % 16 == 0;
    l.edge_l = tile_edge(vocab, rows);
    l.edge_x = tile_edge(rows, d) == 256 || rows * d * vocab >= 1ll << 33 ? 256 : 128;
    l.edge_w = tile_edge(vocab, d);
    l.parts_v = (int)(2 * (up(vocab, l.edge_l) / l.edge_l));
    size_t at = sizeof(XentHeader);
    auto take = [&](int64_t bytes) { const size_t here = at; at = (at + (size_t)bytes + 255) & ~(size_t)255; return here; };
    l.source = take(rows * 4); l.place = take(rows * 4); l.wanted = take(rows * 4);
    l.lse = take(rows * 4); l.row_loss = take(rows * 4); l.hit = take(rows * 4);
    l.stats = take((int64_t)l.parts_v * l.tp * 8);
    const int pieces = l.split ? 2 : 1;
    l.pitch_p = l.dp * 2;
    l.px2 = (size_t)(l.tp * l.pitch_p);
    l.px = take((int64_t)l.px2 * pieces);
    l.pw2 = (size_t)up(vocab * l.pitch_p, 256);
    l.pw = take(l.direct ? 0 : (int64_t)l.pw2 * pieces);
    l.pitch_tx = l.tp * 2;
    l.pitch_tw = l.vp * 2;
    l.tx2 = (size_t)(d * l.pitch_tx);
    l.tx = take(grad ? (int64_t)l.tx2 * pieces : 0);
    l.tw2 = (size_t)(d * l.pitch_tw);
    l.tw = take(grad ? (int64_t)l.tw2 * pieces : 0);
    l.bytes = at;
    // backward
    const int64_t column = l.tp * 2 * 2 * pieces;  // bytes of a column of G
    l.piece = std::min(l.vp, std::max<int64_t>(256, kPieceBytes / column / 256 * 256));
    l.pieces = (vocab + l.piece - 1) / l.piece;
    l.pitch_G = l.piece * 2;
    l.pitch_GT = l.tp * 2;
    at = 0;
    l.g = take(rows * 4);
    l.G2 = (size_t)(l.tp * l.pitch_G);
    l.G = take((int64_t)l.G2 * pieces);
    l.GT2 = (size_t)(l.piece * l.pitch_GT);
    l.GT = take((int64_t)l.GT2 * pieces);
    const int64_t tiles = up(rows, l.edge_x) / l.edge_x * (up(d, l.edge_x) / l.edge_x);
    l.slots = (int)std::max<int64_t>(tiles, kXentSlots);
    l.gparts = take((int64_t)l.slots * l.edge_x * l.edge_x * 4);
    l.back_bytes = at;
    return l;
}

static bool xent_sizes(int64_t rows, int64_t d, int64_t vocab, int dtype) {
    return rows >= 0 && rows <= 1 << 22 && d > 0 && d <= 1 << 20 && vocab > 0 && vocab <= 1 << 22 && (dtype == IMUNPACK_F32 || dtype == IMUNPACK_BF16);
}

// Kernels whose tiles take more LDS than a launch may have by default.
template <class K>
static int more_lds(K kernel, int bytes) {
    IMU_HIP(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes));
    return IMUNPACK_OK;
}
template <bool F16, int T>
static int xent_lds() {
    IMU_TRY(more_lds(xent_logits_kernel<F16, T, false>, product_lds(T, T)));
    IMU_TRY(more_lds(xent_logits_kernel<F16, T, true>, product_lds(T, T)));
    IMU_TRY(more_lds(xent_grad_x_kernel<F16, T>, product_lds(T, T)));
    return more_lds(xent_grad_w_kernel<F16, T>, product_lds(T, T));
}
static int xent_lds_opt_in() {
    static std::atomic<int> done{0};  // (the attribute is idempotent: two threads set the same)
    if (done.load(std::memory_order_acquire)) return IMUNPACK_OK;
    IMU_TRY((xent_lds<false, 4>()));
    IMU_TRY((xent_lds<false, 2>()));
    IMU_TRY((xent_lds<true, 4>()));
    IMU_TRY((xent_lds<true, 2>()));
    done.store(1, std::memory_order_release);
    return IMUNPACK_OK;
}

template <bool F16, int T>
static void launch_logits(const LogitArgs &a, bool back, int64_t rows, hipStream_t st) {
    const dim3 grid((unsigned)(up(a.w.rows, 64 * T) / (64 * T) * (up(rows, 64 * T) / (64 * T))));
    if (back) hipLaunchKernelGGL((xent_logits_kernel<F16, T, true>), grid, dim3(kProductThreads), product_lds(T, T), st, a);
    else hipLaunchKernelGGL((xent_logits_kernel<F16, T, false>), grid, dim3(kProductThreads), product_lds(T, T), st, a);
}
static int logits(const LogitArgs &a, bool f16, int edge, bool back, int64_t rows, hipStream_t st) {
    if (f16) edge == 256 ? launch_logits<true, 4>(a, back, rows, st) : launch_logits<true, 2>(a, back, rows, st);
    else edge == 256 ? launch_logits<false, 4>(a, back, rows, st) : launch_logits<false, 2>(a, back, rows, st);
    return launch_status();
}
}  // namespace imu

using namespace imu;

extern "C" int imunpack_xent_workspace(const void *w, int64_t ldw, int64_t rows, int64_t d, int64_t vocab, int dtype, int want_grad, size_t *saved_bytes,
                                       size_t *backward_bytes) {
    if (!xent_sizes(rows, d, vocab, dtype) || ldw < d || !saved_bytes) return IMUNPACK_EINVAL;
    const XentLayout l = xent_layout(w, ldw, rows, d, vocab, dtype, want_grad != 0);
    *saved_bytes = l.bytes;
    if (backward_bytes) *backward_bytes = l.back_bytes;
    return IMUNPACK_OK;
}

extern "C" int imunpack_xent(const void *x, int64_t ldx, const void *w, int64_t ldw, const int64_t *target, int64_t rows, int64_t d, int64_t vocab,
                             int dtype, int64_t ignore_index, int reduction, int want_grad, float *loss, void *saved, size_t saved_bytes,
                             imunpack_stream_t stream) {
    if (!xent_sizes(rows, d, vocab, dtype) || ldx < d || ldw < d || reduction < IMUNPACK_NONE || reduction > IMUNPACK_MEAN || !w || !saved || (size_t)saved % 16 ||
        (rows > 0 && (!x || !target)) || (!loss && (rows > 0 || reduction != IMUNPACK_NONE)))
        return IMUNPACK_EINVAL;
    const XentLayout l = xent_layout(w, ldw, rows, d, vocab, dtype, want_grad != 0);
    if (saved_bytes < l.bytes) return IMUNPACK_ESMALL;
    IMU_TRY(xent_lds_opt_in());
    hipStream_t st = (hipStream_t)stream;
    char *s = (char *)saved;
    XentHeader *hdr = (XentHeader *)s;
    int32_t *source = (int32_t *)(s + l.source), *place = (int32_t *)(s + l.place), *wanted = (int32_t *)(s + l.wanted);
    hipLaunchKernelGGL(xent_rows_kernel, dim3(1), dim3(1024), 0, st, target, (int)rows, vocab, ignore_index, hdr, source, place, wanted,
                       reduction == IMUNPACK_NONE ? loss : nullptr);
    if (rows > 0) {
        if (l.split) {
            const int xg = (int)std::min<int64_t>(rows, 256), wg = (int)std::min<int64_t>(vocab, 1024);
            hipLaunchKernelGGL(xent_amax_kernel, dim3(xg + wg), dim3(256), 0, st, (const float *)x, ldx, (const float *)w, ldw, (int)d, vocab, hdr, source, xg);
        }
        PrepareArgs p = {};
        p.x = x; p.w = w; p.ldx = ldx; p.ldw = ldw; p.hdr = hdr; p.source = source;
        p.px = s + l.px; p.px2 = l.px2;
        p.pw = l.direct ? nullptr : s + l.pw; p.pw2 = l.pw2;
        if (want_grad) { p.tx = s + l.tx; p.tx2 = l.tx2; p.tw = s + l.tw; p.tw2 = l.tw2; }
        p.pitch_p = l.pitch_p; p.pitch_tx = l.pitch_tx; p.pitch_tw = l.pitch_tw;
        p.vocab = vocab; p.d = (int)d; p.xtiles = (int)(up(rows, 64) / 64);
        const unsigned wtiles = p.pw || p.tw ? (unsigned)(up(vocab, 64) / 64) : 0;
        const dim3 grid(p.xtiles + wtiles, (unsigned)(l.dp / 64));
        if (l.split) hipLaunchKernelGGL(xent_prepare_kernel<float>, grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL(xent_prepare_kernel<__bf16>, grid, dim3(256), 0, st, p);
        LogitArgs a = {};
        a.w = {l.direct ? (const char *)w : s + l.pw, l.direct ? ldw * 2 : l.pitch_p, (int64_t)l.pw2, (int)vocab};
        a.x = {s + l.px, l.pitch_p, (int64_t)l.px2, 0};
        a.hdr = hdr; a.wanted = wanted;
        a.stats = (float *)(s + l.stats); a.hit = (float *)(s + l.hit);
        a.stride = l.tp; a.ktiles = (int)(l.dp / kStageCols);
        IMU_TRY(logits(a, l.split, l.edge_l, false, rows, st));
        hipLaunchKernelGGL(xent_join_kernel, dim3((unsigned)(up(rows, 32) / 32)), dim3(256), 0, st, (const float *)a.stats, (const float *)a.hit, l.parts_v, l.tp, hdr, source,
                           (float *)(s + l.lse), (float *)(s + l.row_loss), reduction == IMUNPACK_NONE ? loss : nullptr);
    }
    if (reduction != IMUNPACK_NONE)
        hipLaunchKernelGGL(xent_sum_kernel, dim3(1), dim3(1024), 0, st, (const float *)(s + l.row_loss), hdr, reduction == IMUNPACK_MEAN, loss);
    return launch_status();
}

extern "C" int imunpack_xent_backward(const void *w, int64_t ldw, int64_t rows, int64_t d, int64_t vocab, int dtype, int reduction, const float *grad, void *saved,
                                      size_t saved_bytes, void *gx, int64_t ldgx, void *gw, int64_t ldgw, void *workspace, size_t workspace_bytes,
                                      imunpack_stream_t stream) {
    if (!xent_sizes(rows, d, vocab, dtype) || ldw < d || (gx && ldgx < d) || (gw && ldgw < d) || reduction < IMUNPACK_NONE || reduction > IMUNPACK_MEAN || !w || !saved ||
        !workspace || (size_t)saved % 16 || (size_t)workspace % 16 || (!grad && (rows > 0 || reduction != IMUNPACK_NONE)))
        return IMUNPACK_EINVAL;
    const XentLayout l = xent_layout(w, ldw, rows, d, vocab, dtype, true);
    if (saved_bytes < l.bytes || workspace_bytes < l.back_bytes) return IMUNPACK_ESMALL;
    if (!gx && !gw) return IMUNPACK_OK;
    IMU_TRY(xent_lds_opt_in());
    hipStream_t st = (hipStream_t)stream;
    char *s = (char *)saved, *b = (char *)workspace;
    XentHeader *hdr = (XentHeader *)s;
    const int32_t *source = (const int32_t *)(s + l.source), *place = (const int32_t *)(s + l.place);
    float *g = (float *)(b + l.g), *parts = (float *)(b + l.gparts);
    hipLaunchKernelGGL(xent_factor_kernel, dim3(1), dim3(1024), 0, st, grad, reduction, hdr, source, g);
    for (int64_t p = 0; p < l.pieces; ++p) {
        const int64_t v0 = p * l.piece, n = std::min(l.piece, vocab - v0);
        const int ktiles = (int)(up(n, kStageCols) / kStageCols);
        if (rows > 0) {
            LogitArgs a = {};
            a.w = {l.direct ? (const char *)w + v0 * ldw * 2 : s + l.pw + v0 * l.pitch_p, l.direct ? ldw * 2 : l.pitch_p, (int64_t)l.pw2, (int)n};
            a.x = {s + l.px, l.pitch_p, (int64_t)l.px2, 0};
            a.hdr = hdr; a.wanted = (const int32_t *)(s + l.wanted);
            a.lse = (const float *)(s + l.lse); a.g = g;
            a.G = b + l.G; a.GT = b + l.GT; a.G2 = l.G2; a.GT2 = l.GT2;
            a.pitch_G = l.pitch_G; a.pitch_GT = l.pitch_GT;
            a.v0 = (int)v0; a.ktiles = (int)(l.dp / kStageCols); a.vlimit = ktiles * kStageCols;
            IMU_TRY(logits(a, l.split, l.edge_l, true, rows, st));
        }
        if (gx && rows > 0) {
            GradXArgs a = {};
            a.G = {b + l.G, l.pitch_G, (int64_t)l.G2, 0};
            a.wt = {s + l.tw + v0 * 2, l.pitch_tw, (int64_t)l.tw2, (int)d};
            a.hdr = hdr; a.parts = parts; a.ktiles = ktiles; a.slots = l.slots; a.first = p == 0;
            const dim3 grid((unsigned)l.slots), block(kProductThreads);
            const int lds = product_lds(l.edge_x / 64, l.edge_x / 64);
            if (l.split) {
                if (l.edge_x == 256) hipLaunchKernelGGL((xent_grad_x_kernel<true, 4>), grid, block, lds, st, a);
                else hipLaunchKernelGGL((xent_grad_x_kernel<true, 2>), grid, block, lds, st, a);
            } else {
                if (l.edge_x == 256) hipLaunchKernelGGL((xent_grad_x_kernel<false, 4>), grid, block, lds, st, a);
                else hipLaunchKernelGGL((xent_grad_x_kernel<false, 2>), grid, block, lds, st, a);
            }
            IMU_TRY(launch_status());
        }
        if (gw) {
            GradWArgs a = {};
            a.GT = {b + l.GT, l.pitch_GT, (int64_t)l.GT2, (int)n};
            a.xt = {s + l.tx, l.pitch_tx, (int64_t)l.tx2, (int)d};
            a.hdr = hdr; a.gw = (char *)gw + v0 * ldgw * (l.split ? 4 : 2); a.ldgw = ldgw;
            const int edge = l.edge_w;
            const dim3 grid((unsigned)(up(n, edge) / edge * (up(d, edge) / edge))), block(kProductThreads);
            const int lds = product_lds(edge / 64, edge / 64);
            if (l.split) {
                if (edge == 256) hipLaunchKernelGGL((xent_grad_w_kernel<true, 4>), grid, block, lds, st, a);
                else hipLaunchKernelGGL((xent_grad_w_kernel<true, 2>), grid, block, lds, st, a);
            } else {
                if (edge == 256) hipLaunchKernelGGL((xent_grad_w_kernel<false, 4>), grid, block, lds, st, a);
                else hipLaunchKernelGGL((xent_grad_w_kernel<false, 2>), grid, block, lds, st, a);
            }
            IMU_TRY(launch_status());
        }
    }
    if (gx && rows > 0) {
        const dim3 grid((unsigned)rows, (unsigned)(up(d, 1024) / 1024));
        if (l.split) hipLaunchKernelGGL(xent_fold_x_kernel<float>, grid, dim3(256), 0, st, parts, hdr, place, (int)d, l.edge_x, l.slots, (float *)gx, ldgx);
        else hipLaunchKernelGGL(xent_fold_x_kernel<__bf16>, grid, dim3(256), 0, st, parts, hdr, place, (int)d, l.edge_x, l.slots, (__bf16 *)gx, ldgx);
    }
    return launch_status();
}
