// Softmax cross entropy of x W^T over a vocabulary, and its gradients, without keeping the logits.
//
//   l[t, v] = sum_k x[t, k] W[v, k],   lse[t] = log sum_v exp l[t, v],   loss[t] = lse[t] - l[t, target[t]]
//   G[t, v] = (exp(l[t, v] - lse[t]) - [v = target[t]]) g[t],   gx = G W,   gW = G^T x            (g: the gradient of loss[t])
//
// Rows without a target take no part: those with one are gathered first, and how many there are is known on the device alone.
// A tile of the product l keeps, per row t, the largest logit and the sum of exponentials of its part of the vocabulary, and a small kernel
// joins them to lse: for the loss alone nothing else of l is left.  For the gradients the rows go through in pieces (as many as kPieceBytes
// allows): the tiles leave their exponentials in 16 bits, relative to the largest of the row and part; once lse stands they become G where
// they lie; gx and gW are products of it, and the next piece takes the same memory.  So l is made once: 6 T V d operations,
// all on the matrix cores, and what is held of l does not grow with the rows beyond a piece (for the loss alone kPieceBytes bounds what the tiles keep).
//
// bfloat16 operands: products in bfloat16, G rounded to bfloat16.  fp32 operands: each value is the sum of two binary16 numbers
// (22 bits of it, and no finer than 2^-25 under a scale) and a
// product is three of them, which is within the rounding of a binary32 sum; three times the instructions at eight times and more the rate of the binary32 ones.
// The scale, a power of two, puts the largest finite magnitude below 2^15: the operand's where its rows are much alike, else (kSpan) each row's own, so
// that a huge or infinite row costs its neighbours nothing.  A sum over the rows of an operand needs one scale for all: where they have
// their own, the operand is split again in between, W for gx = G W and x for gW = G^T x.  What is then lost lies 2^-39 below the operand's largest value.  With a
// gradient to each row's loss that goes to x for gW (which is split again with it) and to the finished rows of gx, so that a
// row's own gradient is no coarser for a neighbour's.
#include "common.h"
#include "elements.h"
#include "product.h"

#include <algorithm>
#include <atomic>
#include <type_traits>

namespace imu {
constexpr int64_t kPieceBytes = 2ll << 30;  // G of a piece of the rows at most (or 256 rows); for the loss alone, the parts' largest logits and sums
constexpr int kTop = 14;                    // the largest magnitude of a scaled operand is below 2^(kTop + 1)
constexpr int kSpan = 8;                    // powers of two between the rows' largest magnitudes beyond which each row has a scale of its own (up to
                                            // there what one scale rounds off lies 2^-31 below the largest value of the row)
constexpr unsigned kCus = 256;
constexpr int kXentSlots = 256;             // parts of the tiles of a gradient that go at a time: one to a CU
constexpr int kPartTiles = 2;               // k-tiles of a part at least (1: as fast; 4: 100 x 1024 by 16000 bf16 58.0 -> 59.5 us)
constexpr int kScanGroups = 512, kScanX = 64;  // workgroups that look for the largest magnitudes, those of x first
constexpr int kJoinRows = 8;
constexpr int64_t kJoinReads = 1 << 22;     // parts read, by every workgroup of a row, up to which those join them that turn the exponentials
constexpr int kLargeRows = 1024;            // rows from which the logits may go in large tiles

// The largest finite magnitude in some rows (its bits) and the largest exponent of a row's scale (rows of zeros have none) plus kFinest.
struct Largest {
    int32_t top, finest;
    __device__ void with(const Largest &o) {
        top = max(top, o.top);
        finest = max(finest, o.finest);
    }
};
constexpr int kFinest = 1024;
struct XentHeader {
    int32_t count;    // rows with a target
    int32_t bad;      // rows whose target is outside the vocabulary
    uint32_t amax[2]; // bits of the largest finite magnitude of x (rows with a target) and of W
    int32_t wide[2];  // rows of x, of W have scales of their own in the logits
    int32_t gexp;     // where each row has a gradient: exponent of the largest (bfloat16), of the scale of x times them (fp32)
    uint32_t joined;  // workgroups that have left the losses of their rows
    int32_t pad[56];
    Largest found[kScanGroups];  // as the workgroups found them
};
static_assert(sizeof(XentHeader) == 256 + 8 * kScanGroups, "header");
// Rows of the piece that begins at row `first` and has room for `room`.
__device__ __forceinline__ int rows_of(const XentHeader *hdr, int first, int room) { return max(0, min(hdr->count - first, room)); }

// Edges of the tiles of the logits and of the gradients, from the rows of a piece: 256, which reads each operand half as often, where the rows
// fill such tiles and the tiles fill the CUs.  The loss of 4096 x 2048 by 16000 columns: 260 us with edges of 128, 233 with 256 (bf16; fp32 721
// and 678); of 200 rows: 40 and 60.  With its gradients, 868 and 783 (2176 and 2033); of 640 rows 188 and 204 (473 and 521).  Only the
// device knows how many rows have a target: where both are possible both are launched, and one of them finds nothing to do.
__host__ __device__ __forceinline__ int logits_edge(int rows, int d, int vocab) {
    return rows >= kLargeRows && d >= 512 && (rows + 255) / 256 * ((vocab + 255) / 256) >= (int)kCus ? 256 : 128;
}
__host__ __device__ __forceinline__ int grads_edge(int rows, int d, int vocab) { return rows >= 1536 && (int64_t)vocab * d >= 1 << 23 ? 256 : 128; }
__device__ __forceinline__ int rows_at_most(const XentHeader *hdr, int room) { return min(hdr->count, room); }

// What 2 to its power an operand is multiplied by before it is split.
__device__ __forceinline__ int scale_exponent(uint32_t amax) { return min(kTop - ((int)(amax >> 23) - 127), 126); }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// Where column col of a row lies, in 16 bits or as the first of two numbers, the second one kSecond bytes behind it (blocks of 32, see product.h).
template <bool PAIRS>
__host__ __device__ __forceinline__ int64_t byte_of(int64_t col) { return PAIRS ? (col / 32 * 64 + col % 32) * 2 : col * 2; }
constexpr int kSecond = 64;

struct ScanArgs {
    const int64_t *target;
    int64_t vocab, ignore;
    XentHeader *hdr;
    int32_t *source, *place, *wanted;
    float *loss;                 // where each row has a loss of its own
    const float *x, *w;          // fp32: whose largest magnitudes are wanted
    int64_t ldx, ldw;
    int32_t *own_x, *own_w;      // exponents of the rows' own scales
    int rows, d, nx;             // nx: workgroups that look at x
};
__device__ __forceinline__ bool has_target(const ScanArgs &a, int64_t v) { return v >= 0 && v < a.vocab && v != a.ignore; }

// What `largest` finds in rows first, first + step, ... of a matrix, and the exponent of each row's scale; x: of those with a target.  A wave takes
// four rows at a time; all of its lanes have the results.
__device__ __forceinline__ int over_wave(int v) { return from_lane63(wave_max_nonneg_lane63(v)); }
template <bool X>
__device__ __forceinline__ Largest largest(const ScanArgs &a, const float *m, int64_t ld, int64_t rows, int first, int step, int32_t *own) {
    const int lane = threadIdx.x & 63;
    Largest l = {0, 0};
    for (int64_t row = (int64_t)first * 4; row < rows; row += (int64_t)step * 4) {
        int n[4];
        float top[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int r = 0; r < 4; ++r) n[r] = row + r < rows && (!X || has_target(a, a.target[row + r])) ? a.d : 0;
        for (int col = lane * 4; col < a.d; col += 256) {
            piece_t<float, 4> f[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) f[r] = load_piece<float, 4>(m + (row + r) * ld + col, n[r] - col);
#pragma unroll
            for (int r = 0; r < 4; ++r)
#pragma unroll
                for (int k = 0; k < 4; ++k) top[r] = fmaxf(top[r], fabsf(f[r][k]));
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            if (n[r] == 0) continue;
            float t = __uint_as_float((uint32_t)over_wave((int)__float_as_uint(top[r])));
            if (t == __builtin_inff()) {  // (the whole wave) once more, without what is infinite
                t = 0.0f;
                for (int col = lane; col < a.d; col += 64) {
                    const float v = fabsf(m[(row + r) * ld + col]);
                    t = v < __builtin_inff() ? fmaxf(t, v) : t;
                }
                t = __uint_as_float((uint32_t)over_wave((int)__float_as_uint(t)));
            }
            const int e = scale_exponent(__float_as_uint(t));
            if (lane == 0) own[row + r] = e;
            l.with({(int)__float_as_uint(t), t > 0.0f ? e + kFinest : 0});
        }
    }
    return l;
}

// Rows with a target in order (also in `own`), their targets, and for every row its place among them (-1: none, -2: a target outside the
// vocabulary).  A workgroup of 1024 threads; returns how many there are, to be left by the one that writes.
__device__ __forceinline__ int scan_rows(const ScanArgs &a, int32_t (*sums)[16], int32_t *own, bool write) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int base = 0, bad = 0, turn = 0;
    for (int t0 = 0; t0 < a.rows; t0 += 1024, turn ^= 1) {
        const int t = t0 + threadIdx.x;
        const int64_t v = t < a.rows ? a.target[t] : a.ignore;
        const bool inside = has_target(a, v), outside = !inside && v != a.ignore;
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
        if (own && inside) own[at] = t;
        if (write) {
            if (inside) {
                a.source[at] = t;
                a.wanted[at] = (int)v;
            }
            if (t < a.rows) {
                a.place[t] = inside ? at : outside ? -2 : -1;
                if (a.loss && !inside) a.loss[t] = outside ? __builtin_nanf("") : 0.0f;
            }
        }
        base += all;
    }
    bad = __syncthreads_or(bad);
    if (write && threadIdx.x == 0) {
        a.hdr->count = base;
        a.hdr->bad = bad;
        a.hdr->joined = 0;
    }
    return base;
}

// Workgroup 0: the rows.  The others (fp32): the largest magnitudes of x and W (50265 x 768: 38 us, 4.1 TB/s).
__global__ __launch_bounds__(1024) void xent_scan_kernel(const ScanArgs a) {
    __shared__ int32_t sums[2][16];
    __shared__ Largest found[16];
    if (blockIdx.x > 0) {
        const int wave = threadIdx.x >> 6;
        const int g = blockIdx.x - 1, nx = a.nx;
        Largest l = g < nx ? largest<true>(a, a.x, a.ldx, a.rows, g * 16 + wave, nx * 16, a.own_x)
                                 : largest<false>(a, a.w, a.ldw, a.vocab, (g - nx) * 16 + wave, ((int)gridDim.x - 1 - nx) * 16, a.own_w);
        if ((threadIdx.x & 63) == 0) found[wave] = l;
        __syncthreads();
        if (threadIdx.x == 0) {
#pragma unroll
            for (int w = 1; w < 16; ++w) l.with(found[w]);
            a.hdr->found[g] = l;
        }
        return;
    }
    scan_rows(a, sums, nullptr, true);
}

template <class E>
__device__ __forceinline__ uint32_t pack(E a, E b) {
    return (uint32_t)__builtin_bit_cast(uint16_t, a) | (uint32_t)__builtin_bit_cast(uint16_t, b) << 16;
}

struct PrepareArgs {
    ScanArgs scan;
    const void *x, *w;
    int64_t ldx, ldw;
    XentHeader *hdr;
    const int32_t *source;
    char *px, *pw;            // x (gathered) and W in 16 bits, rows of `pieces` times 16 bytes
    int64_t xrows, wrows;     // rows there is room for; rows of W that are wanted
    int d, pieces, xgroups, nx, nw;  // workgroups that work on x; nx, nw: workgroups that looked for the largest magnitudes
    const int32_t *own_x;     // fp32: exponents of the scales of the rows of x before they are gathered
    int32_t *ex, *ew;         // what 2 to their power a row of x, of W is multiplied with; ew: the rows' own before
};
// Eight columns of a row as two binary16 numbers each.
__device__ __forceinline__ void store_split(char *to, const float (&f)[8]) {
    uint32_t hi[4], lo[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const _Float16 h0 = (_Float16)f[2 * k], h1 = (_Float16)f[2 * k + 1];
        hi[k] = pack(h0, h1);
        lo[k] = pack((_Float16)(f[2 * k] - (float)h0), (_Float16)(f[2 * k + 1] - (float)h1));
    }
    *reinterpret_cast<v4i32 *>(to) = v4i32{(int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
    *reinterpret_cast<v4i32 *>(to + kSecond) = v4i32{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3]};
}
constexpr int kPrepareTurns = 4, kScanHere = 1024;
// Eight columns of a row at a time: binary32 as two binary16 numbers, bfloat16 as it is; zeros behind the last column and, to a whole
// k-tile, behind the last row of x.  Bound by memory: 50265 x 768 fp32 59 us, 5.2 TB/s (what it reads is in the
// last-level cache).  SCAN: up to kScanHere rows, among which every workgroup finds those with a target itself (one launch less: 197 x 256
// by 1000, loss alone: 21.5 -> 18.3 us).
template <class T, bool SCAN>
__global__ __launch_bounds__(SCAN ? 1024 : 256) void xent_prepare_kernel(const PrepareArgs a) {
    constexpr bool SPLIT = sizeof(T) == 4;
    constexpr int kThreads = SCAN ? 1024 : 256;
    __shared__ Largest found[4];
    __shared__ int32_t sums[2][16], own[SCAN ? kScanHere : 1];
    const bool isX = (int)blockIdx.x < a.xgroups;
    const int group = isX ? blockIdx.x : blockIdx.x - a.xgroups;
    int64_t count = a.wrows;
    if (isX) {
        if constexpr (SCAN) {
            count = scan_rows(a.scan, sums, own, group == 0);
            __syncthreads();
        } else {
            count = a.hdr->count;
        }
    }
    const int64_t rows = isX ? min((count + kStageCols - 1) / kStageCols * kStageCols, a.xrows) : count;
    int common = 0;
    bool wide = false;
    if constexpr (SPLIT) {  // the first workgroup of either operand leaves what was found for the kernels behind
        Largest l = {0, 0}, some[kScanGroups / 256];
#pragma unroll
        for (int i = 0; i < kScanGroups / 256; ++i) {
            const int k = threadIdx.x + 256 * i;
            some[i] = k < (isX ? a.nx : a.nw) ? a.hdr->found[isX ? k : a.nx + k] : Largest{0, 0};
        }
#pragma unroll
        for (int i = 0; i < kScanGroups / 256; ++i) l.with(some[i]);
        l = {over_wave(l.top), over_wave(l.finest)};
        if ((threadIdx.x & 63) == 0) found[threadIdx.x >> 6] = l;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < 4; ++w) l.with(found[w]);
        common = scale_exponent((uint32_t)l.top);
        wide = l.finest - kFinest - common > kSpan;
        if (threadIdx.x == 0 && group == 0) {
            a.hdr->amax[isX ? 0 : 1] = (uint32_t)l.top;
            a.hdr->wide[isX ? 0 : 1] = wide;
        }
    }
    const int64_t at0 = (int64_t)group * kThreads * kPrepareTurns + threadIdx.x;
    int64_t row[kPrepareTurns];
    int col[kPrepareTurns];
    piece_t<T, 4> f[kPrepareTurns][2];
#pragma unroll
    for (int i = 0; i < kPrepareTurns; ++i) {
        const int64_t at = at0 + kThreads * i;
        row[i] = at / a.pieces;
        col[i] = (int)(at - row[i] * a.pieces) * 8;
        const T *p = isX ? (const T *)a.x + (row[i] < count ? (int64_t)(SCAN ? own[row[i]] : a.source[row[i]]) : 0) * a.ldx : (const T *)a.w + row[i] * a.ldw;
        const int have = row[i] < count ? a.d - col[i] : 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) f[i][k] = load_piece<T, 4>(p + col[i] + 4 * k, have - 4 * k);
    }
#pragma unroll
    for (int i = 0; i < kPrepareTurns; ++i) {
        if (row[i] >= rows) continue;
        char *to = (isX ? a.px : a.pw) + row[i] * a.pieces * (SPLIT ? 32 : 16) + byte_of<SPLIT>(col[i]);
        if constexpr (SPLIT) {
            int e = common;
            if (wide && row[i] < count) e = isX ? a.own_x[a.source[row[i]]] : a.ew[row[i]];
            if (col[i] == 0 && row[i] < count && (isX || !wide)) (isX ? a.ex : a.ew)[row[i]] = e;
            const float scale = power_of_two(e);
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = f[i][k >> 2][k & 3] * scale;
            store_split(to, v);
        } else {
            uint32_t q[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) q[k] = pack(f[i][k >> 1][2 * (k & 1)], f[i][k >> 1][2 * (k & 1) + 1]);
            *reinterpret_cast<v4i32 *>(to) = v4i32{(int)q[0], (int)q[1], (int)q[2], (int)q[3]};
        }
    }
}

// The gradient of each row's loss.  One for all: the results are multiplied with it (a factor between -2 and 2 and a power of two), and G is without: a row's
// largest entry is the target's, next to -1, where bfloat16 has its finest steps (with the factor of a mean over 614 rows in it, gx and gW were off by up to 2.3 times
// what the rounding of the results makes, and 1.1 times without).  One for each row: G has them under one power of two (bfloat16), or not at all (fp32: gx
// and x have them, see below).
struct Upstream {
    const float *grad, *g;  // grad: nullptr for 1; g: bfloat16, the rows' factors where each has a gradient of its own, else nullptr
    int mean, rows;         // rows: fp32, each row has a gradient of its own
    __device__ __forceinline__ float whole(const XentHeader *hdr) const {
        const float one = grad ? *grad : 1.0f;
        return mean ? one / (float)max(hdr->count, 1) : one;
    }
    __device__ __forceinline__ static int exponent_of(float m) { return fabsf(m) > 0.0f ? (int)(__float_as_uint(fabsf(m)) >> 23) - 127 : 0; }
    __device__ __forceinline__ int exponent(const XentHeader *hdr) const { return rows ? 0 : g ? hdr->gexp : exponent_of(whole(hdr)); }
    __device__ __forceinline__ float factor(const XentHeader *hdr) const { return rows || g || hdr->count == 0 ? 1.0f : ldexpf(whole(hdr), -exponent_of(whole(hdr))); }
    // Of the scale of x in gW's product.
    __device__ __forceinline__ int scale_x(const XentHeader *hdr) const { return rows ? hdr->gexp : scale_exponent(hdr->amax[0]); }
};

// fp32: the operands of the gradients' products whose rows have scales of their own are split again under one scale: W for gx, and x, with the rows'
// gradients where each has one, for gW.  (Else nothing: the logits' operands are these.)  By all workgroups of a launch.
struct AlignArgs {
    const float *x, *w;       // nullptr: not wanted
    int64_t ldx, ldw, pitch;
    char *px, *pw;
    const int32_t *source, *own_x, *ew;
    int d, vocab;
};
template <class S>
__device__ __forceinline__ void split_rows(const float *m, int64_t ld, char *to, int64_t pitch, int64_t rows, int d, S &&scaled) {
    const int pieces = (int)(pitch / 32);  // (two numbers of eight columns)
    for (int64_t at = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; at < rows * pieces; at += (int64_t)gridDim.x * blockDim.x) {
        const int64_t row = at / pieces;
        const int col = (int)(at - row * pieces) * 8;
        const int64_t from = scaled.row(row);
        float f[8];
        load_upto<float, 8>(m + from * ld + col, f, d - col);
#pragma unroll
        for (int k = 0; k < 8; ++k) f[k] = scaled(f[k], row, from);
        store_split(to + row * pitch + byte_of<true>(col), f);
    }
}
struct ScaledWeights {
    const int32_t *ew;  // nullptr: one scale
    int common;
    __device__ int64_t row(int64_t v) const { return v; }
    __device__ float operator()(float x, int64_t v, int64_t) const { return x * power_of_two(ew ? ew[v] : common); }
};
struct ScaledInputs {
    const int32_t *source, *own;
    const float *grad;  // nullptr: without
    int common;
    __device__ int64_t row(int64_t t) const { return source[t]; }
    __device__ float operator()(float x, int64_t, int64_t t) const {
        if (!grad) return x * power_of_two(common);
        const int e = own[t], eg = Upstream::exponent_of(grad[t]);  // (neither factor nor their product leaves binary32's range; what the last step rounds is below 2^-39 of the largest)
        return ldexpf(x * power_of_two(e) * ldexpf(grad[t], -eg), common - e + eg);
    }
};
__device__ __forceinline__ void align_operands(const AlignArgs &a, const XentHeader *hdr, bool wide_x, bool wide_w, const Upstream &up, int first, int rows) {
    if (a.w && wide_w) split_rows(a.w, a.ldw, a.pw, a.pitch, a.vocab, a.d, ScaledWeights{nullptr, scale_exponent(hdr->amax[1])});
    if (a.x && (wide_x || up.rows))
        split_rows(a.x, a.ldx, a.px + first * a.pitch, a.pitch, rows, a.d, ScaledInputs{a.source + first, a.own_x, up.rows ? up.grad : nullptr, up.scale_x(hdr)});
}
// Back to the rows' own scales, for the logits of the next piece.
__global__ __launch_bounds__(256) void xent_weights_kernel(const AlignArgs a, const XentHeader *hdr) {
    if (hdr->wide[1]) split_rows(a.w, a.ldw, a.pw, a.pitch, a.vocab, a.d, ScaledWeights{a.ew, 0});
}

// The same row by row, for the loss alone: each row by its own largest magnitude, which no other kernel has to look for.  A wave to a row,
// which it reads twice (the second time out of a cache).  32003 x 1031 60 us, 4.5 TB/s.
struct PrepareRowsArgs {
    const float *x, *w;
    int64_t ldx, ldw;
    const XentHeader *hdr;
    const int32_t *source;
    char *px, *pw;
    int64_t pitch, wrows;
    int32_t *ex, *ew;
    int d, xgroups;
};
__global__ __launch_bounds__(256) void xent_prepare_rows_kernel(const PrepareRowsArgs a) {
    const bool isX = (int)blockIdx.x < a.xgroups;
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)(isX ? blockIdx.x : blockIdx.x - a.xgroups) * 4 + (threadIdx.x >> 6), rows = isX ? a.hdr->count : a.wrows;
    if (row >= rows) return;
    const float *p = isX ? a.x + (int64_t)a.source[row] * a.ldx : a.w + row * a.ldw;
    float m = 0.0f;
    for (int col = lane * 8; col < a.d; col += 2048) {
        piece_t<float, 4> f[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) f[i][k] = load_piece<float, 4>(p + col + 512 * i + 4 * k, a.d - (col + 512 * i + 4 * k));
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < 8; ++k) m = fmaxf(m, fabsf(f[i][k >> 2][k & 3]));
    }
    m = wave_max(m);
    const int e = scale_exponent(__float_as_uint(m));
    const float scale = power_of_two(e);
    if (lane == 0) (isX ? a.ex : a.ew)[row] = e;
    char *to = (isX ? a.px : a.pw) + row * a.pitch;
    for (int col = lane * 8; col < a.pitch / 4; col += 2048) {
        piece_t<float, 4> f[4][2];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int k = 0; k < 2; ++k) f[i][k] = load_piece<float, 4>(p + col + 512 * i + 4 * k, a.d - (col + 512 * i + 4 * k));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (col + 512 * i >= a.pitch / 4) break;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = f[i][k >> 2][k & 3] * scale;
            store_split(to + byte_of<true>(col + 512 * i), v);
        }
    }
}

struct LogitArgs {
    Operand w, x;             // rows of the vocabulary and of the piece
    const XentHeader *hdr;
    const int32_t *wanted;
    const int32_t *ex, *ew;   // fp32: exponents of the rows' scales
    float *stats, *hit;       // [part of the vocabulary][row of the piece] largest logit and sum; the target's logit
    char *P;                  // [row of the piece][vocabulary] exponentials, relative to the largest of the row and part, times 2^kTop where they are binary16
    int64_t pitch_P;
    int first, room;          // the piece's first row, and for how many there is room
    int d, ktiles;
};
constexpr float kLog2e = 1.44269504088896340736f;
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// Four lanes hold a row of four 16-bit elements each (lo: 0 and 1, hi: 2 and 3); afterwards lane k of them holds element k of all four.
__device__ __forceinline__ void quad_transpose(uint32_t &lo, uint32_t &hi, int lane) {
    const uint32_t pick = lane & 1 ? 0x03020706u : 0x05040100u;  // odd: the neighbour's upper half below one's own; even: one's own lower half below the neighbour's
    const uint32_t nlo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)lo, 0xB1, 0xf, 0xf, true), nhi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)hi, 0xB1, 0xf, 0xf, true);
    const uint32_t a = __builtin_amdgcn_perm(nlo, lo, pick), b = __builtin_amdgcn_perm(nhi, hi, pick);
    const bool upper = lane & 2;
    const uint32_t r = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(upper ? a : b), 0x4E, 0xf, 0xf, true);
    lo = upper ? r : a;
    hi = upper ? b : r;
}

// A tile of logits, vocabulary down, rows of x across: a lane holds one row of x per column block, so that the sums over the
// vocabulary are sums over its registers and one exchange between the halves of the wave.  Bound by the matrix cores: 4096 x 4096 by 32000
// bfloat16 836 us, 1.28 PFLOP/s, where a library's product of 8192^3 reaches 1.37 (busy 75 % of the cycles at the clock that its power allows); 614 x 768
// by 50265 fp32 160 us, 0.89 PFLOP/s of binary16 (busy 58 %: the contraction is short, and the exponentials are made
// and stored behind it).
template <bool F16, int T, bool KEEP>
__global__ __launch_bounds__(kProductThreads, T == 4 ? 1 : 2) void xent_logits_kernel(const LogitArgs a) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    constexpr int kEdge = 64 * T;
    const int count = rows_of(a.hdr, a.first, a.room), vocab = a.w.rows, mtiles = (vocab + kEdge - 1) / kEdge, ntiles = (count + kEdge - 1) / kEdge;
    if ((int)blockIdx.x >= mtiles * ntiles || logits_edge(rows_at_most(a.hdr, a.room), a.d, vocab) != kEdge) return;
    int tm, tn;
    tile_at(blockIdx.x, mtiles, ntiles, tm, tn);
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
    Operand x = a.x;
    x.rows = count;
    v16f32 acc[T][T];
    product_tile<F16, T, T, false, false>(a.w, x, tm * kEdge, tn * kEdge, 0, a.ktiles, smem, acc);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lrow = lane & 31, lhalf = lane >> 5;
    const int vwave = tm * kEdge + (wave >> 1) * 32 * T, twave = tn * kEdge + (wave & 1) * 32 * T;  // the wave's first column and row of the piece
    const bool own_scales = F16 && KEEP && (a.hdr->wide[0] || a.hdr->wide[1]);
    const int down = F16 && KEEP ? -(scale_exponent(a.hdr->amax[0]) + scale_exponent(a.hdr->amax[1])) : 0;  // (of one scale for each operand)
    // FULL: no column behind the vocabulary and no row behind the last one in the wave's part (nothing to compare)
    auto finish = [&](auto full) __attribute__((always_inline)) {
        constexpr bool FULL = decltype(full)::value;
#pragma unroll
        for (int j = 0; j < T; ++j) {
            const int t = twave + 32 * j + lrow;
            const bool in_rows = FULL || t < count;
            const int hit_at = in_rows ? a.wanted[a.first + t] - vwave : -1;   // the target among the wave's columns
            const bool hits = hit_at >= 0 && hit_at < 32 * T;
            const int left = vocab - vwave - 4 * lhalf, own = hit_at - 4 * lhalf;  // the lane has columns 32 i + 8 q + k
            float top = -__builtin_inff(), sum = 0.0f;
            if constexpr (F16) {
                if (KEEP && !own_scales) {
#pragma unroll
                    for (int i = 0; i < T; ++i)
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[i][j][r] = ldexpf(acc[i][j][r], down);
                } else {
                    const int ex = in_rows ? a.ex[a.first + t] : 0;
#pragma unroll
                    for (int i = 0; i < T; ++i)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const v4i32 ew = *reinterpret_cast<const v4i32 *>(a.ew + vwave + 32 * i + 8 * q + 4 * lhalf);  // (room for whole tiles)
#pragma unroll
                            for (int k = 0; k < 4; ++k) acc[i][j][4 * q + k] = ldexpf(acc[i][j][4 * q + k], -ex - ew[k]);
                        }
                }
            }
#pragma unroll
            for (int i = 0; i < T; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (FULL || 32 * i + (r >> 2) * 8 + (r & 3) < left) top = fmaxf(top, acc[i][j][r]);
            top = fmaxf(top, __shfl_xor(top, 32));
            const float from = top == -__builtin_inff() ? 0.0f : top;  // (nothing of the vocabulary in this part)
            if (__ballot(hits) != 0) {
                float hit = 0.0f;
#pragma unroll
                for (int i = 0; i < T; ++i)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        if (32 * i + (r >> 2) * 8 + (r & 3) == own) hit = acc[i][j][r];
                if (hits && ((hit_at >> 2) & 1) == lhalf) a.hit[a.first + t] = hit;
            }
            char *to = a.P + t * a.pitch_P + byte_of<F16>(vwave) + 16 * lhalf;
#pragma unroll
            for (int i = 0; i < T; ++i) {
                float p[16];
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    p[r] = fast_exp(acc[i][j][r] - from);  // (not log2 e of either: of large logits the difference of the rounded products is none)
                    if (FULL || 32 * i + (r >> 2) * 8 + (r & 3) < left) sum += p[r];
                }
                if constexpr (KEEP) {
                    // columns 8 q .. 8 q + 7 lie in both halves of the wave; the halves trade, and each has eight in a row: 16 bytes to a store
                    auto put = [&](const uint32_t (&w)[8], int off) __attribute__((always_inline)) {
#pragma unroll
                        for (int q = 0; q < 4; q += 2) {
                            const auto x = __builtin_amdgcn_permlane32_swap(w[2 * q], w[2 * q + 2], false, false);
                            const auto y = __builtin_amdgcn_permlane32_swap(w[2 * q + 1], w[2 * q + 3], false, false);
                            if (FULL || in_rows)
                                *reinterpret_cast<v4i32 *>(to + off + byte_of<F16>(32 * i + 8 * q)) = v4i32{(int)x[0], (int)y[0], (int)x[1], (int)y[1]};
                        }
                    };
                    uint32_t w[8];
                    if constexpr (F16) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) {
                            const float p0 = p[2 * k] * power_of_two(kTop), p1 = p[2 * k + 1] * power_of_two(kTop);
                            const _Float16 h0 = (_Float16)p0, h1 = (_Float16)p1;
                            w[k] = pack(h0, h1);
                            p[2 * k] = p0 - (float)h0;
                            p[2 * k + 1] = p1 - (float)h1;
                        }
                        put(w, 0);
#pragma unroll
                        for (int k = 0; k < 8; ++k) w[k] = pack((_Float16)p[2 * k], (_Float16)p[2 * k + 1]);
                        put(w, kSecond);
                    } else {
#pragma unroll
                        for (int k = 0; k < 8; ++k) w[k] = pack((__bf16)p[2 * k], (__bf16)p[2 * k + 1]);
                        put(w, 0);
                    }
                }
            }
            sum += __shfl_xor(sum, 32);
            if (in_rows && lhalf == 0)
                *reinterpret_cast<float2 *>(a.stats + ((int64_t)(2 * tm + (wave >> 1)) * a.room + t) * 2) = make_float2(top, sum);
        }
    };
    if (vwave + 32 * T <= vocab && twave + 32 * T <= count) finish(std::true_type());
    else finish(std::false_type());
}

struct FewArgs {
    const float *x, *w;
    int64_t ldx, ldw;
    const XentHeader *hdr;
    const int32_t *source, *wanted;
    float *stats, *hit;
    int room, d, vocab;
};
constexpr int kFewRows = 8;
// The loss alone of up to eight fp32 rows over weights that the last-level cache does not hold: W is read once, as it is, where splitting
// it would move it three times.  64 columns (a part of a tile of 128) to a workgroup, eight at a time to a wave, sums in binary32.  Bound by
// memory: 8 x 4096 by 32000 123 us (split: 412), by 128000 381 us (1386), 4.3 and 5.5 TB/s.  Weights that the cache holds go the way of all others.
__global__ __launch_bounds__(256) void xent_few_kernel(const FewArgs a) {
    __shared__ float logits[64][kFewRows];
    const int count = a.hdr->count, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (count == 0) return;
    const float *x[kFewRows];
#pragma unroll
    for (int r = 0; r < kFewRows; ++r) x[r] = a.x + (int64_t)a.source[min(r, count - 1)] * a.ldx;
    for (int c0 = wave * 16; c0 < wave * 16 + 16; c0 += 8) {
        const float *w[8];
        float sum[8][kFewRows];
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            w[c] = a.w + (int64_t)min((int)blockIdx.x * 64 + c0 + c, a.vocab - 1) * a.ldw;
#pragma unroll
            for (int r = 0; r < kFewRows; ++r) sum[c][r] = 0.0f;
        }
        for (int k0 = 0; k0 < a.d; k0 += 256) {
            const int k = k0 + lane * 4;
            piece_t<float, 4> fw[8], fx[kFewRows];
#pragma unroll
            for (int c = 0; c < 8; ++c) fw[c] = load_piece<float, 4, true>(w[c] + k, a.d - k);
#pragma unroll
            for (int r = 0; r < kFewRows; ++r) fx[r] = load_piece<float, 4>(x[r] + k, a.d - k);
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int r = 0; r < kFewRows; ++r)
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[c][r] = fmaf(fw[c][e], fx[r][e], sum[c][r]);
        }
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int r = 0; r < kFewRows; ++r) {
                const float l = wave_sum(sum[c][r]);
                if (lane == 0) logits[c0 + c][r] = l;
            }
    }
    __syncthreads();
    const int r = threadIdx.x >> 5, j = threadIdx.x & 31, v0 = (int)blockIdx.x * 64;  // 32 lanes to a row, two columns to a lane
    if (r >= count) return;
    const float l0 = v0 + j < a.vocab ? logits[j][r] : -__builtin_inff(), l1 = v0 + j + 32 < a.vocab ? logits[j + 32][r] : -__builtin_inff();
    float top = fmaxf(l0, l1);
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) top = fmaxf(top, __shfl_xor(top, m));
    const float from = top == -__builtin_inff() ? 0.0f : top;
    float s = fast_exp(l0 - from) + fast_exp(l1 - from);
#pragma unroll
    for (int m = 16; m > 0; m >>= 1) s += __shfl_xor(s, m);
    const int own = a.wanted[r] - v0;
    if (own == j || own == j + 32) a.hit[r] = own == j ? l0 : l1;
    if (j == 0) *reinterpret_cast<float2 *>(a.stats + ((int64_t)blockIdx.x * a.room + r) * 2) = make_float2(top, s);
}

struct JoinArgs {
    const float *stats, *hit;
    int d, vocab, how, first, room;
    XentHeader *hdr;
    const int32_t *source;
    float *lse, *row_loss, *loss;
};
struct JoinShared {
    float tops[32][kJoinRows], sums[32][kJoinRows], lds[4];
    int last;
};
// lse of eight rows from the parts of the vocabulary, 32 threads to a row, in the first of them.
__device__ __forceinline__ float join_rows(const JoinArgs &a, int group, JoinShared &sh) {
    const int r = threadIdx.x % kJoinRows, g = threadIdx.x / kJoinRows, at = group * kJoinRows + r, t = a.first + at, count = a.hdr->count;
    const int edge = logits_edge(rows_at_most(a.hdr, a.room), a.d, a.vocab), parts = (a.vocab + edge - 1) / edge * 2;
    float top = -__builtin_inff(), sum = 0.0f;
    if (t < count)
        for (int k0 = g; k0 < parts; k0 += 128) {
            float2 s[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                s[k] = k0 + 32 * k < parts ? *reinterpret_cast<const float2 *>(a.stats + ((int64_t)(k0 + 32 * k) * a.room + at) * 2) : make_float2(-__builtin_inff(), 0.0f);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float next = fmaxf(top, s[k].x);
                if (next > -__builtin_inff()) sum = sum * fast_exp(top - next) + s[k].y * fast_exp(s[k].x - next);
                else sum += s[k].y;  // (NaN stays)
                top = next;
            }
        }
    sh.tops[g][r] = top;
    sh.sums[g][r] = sum;
    __syncthreads();
    if (g > 0 || t >= count) return 0.0f;
#pragma unroll
    for (int k = 1; k < 32; ++k) top = fmaxf(top, sh.tops[k][r]);
    sum = 0.0f;
    const float from = top == -__builtin_inff() ? 0.0f : top;
#pragma unroll
    for (int k = 0; k < 32; ++k) sum += sh.sums[k][r] * fast_exp(sh.tops[k][r] - from);
    return from + logf(sum);
}
// Their losses.  Where one value is wanted, the workgroup that comes last adds the rows' losses, in a fixed order.
__device__ __forceinline__ void rows_losses(const JoinArgs &a, int group, float lse, JoinShared &sh) {
    const int t = a.first + group * kJoinRows + (int)threadIdx.x, count = a.hdr->count;
    const int groups = max(1, (count + kJoinRows - 1) / kJoinRows);  // of all pieces
    if (threadIdx.x < kJoinRows && t < count) {
        const float v = lse - a.hit[t];
        __hip_atomic_store(a.row_loss + t, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // (past this XCD's cache: no fence has to write it back)
        if (a.how == IMUNPACK_NONE && a.loss) a.loss[a.source[t]] = v;
    }
    if (a.how == IMUNPACK_NONE) return;
    stores_done();
    __syncthreads();
    if (threadIdx.x == 0) sh.last = atomicAdd(&a.hdr->joined, 1u) == (unsigned)groups - 1;
    __syncthreads();
    if (!sh.last) return;
    float s = 0.0f;
    for (int k = threadIdx.x; k < count; k += 256) s += __hip_atomic_load(a.row_loss + k, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    s = reduce_threads<256, false>(s, sh.lds);
    if (threadIdx.x == 0) *a.loss = a.hdr->bad ? __builtin_nanf("") : a.how == IMUNPACK_MEAN && count > 0 ? s / (float)count : s;
}
__global__ __launch_bounds__(256) void xent_join_kernel(const JoinArgs a) {
    __shared__ JoinShared sh;
    const int count = a.hdr->count, t = a.first + blockIdx.x * kJoinRows + threadIdx.x;
    if ((int)blockIdx.x + a.first / kJoinRows >= max(1, (count + kJoinRows - 1) / kJoinRows)) return;
    const float l = join_rows(a, blockIdx.x, sh);
    if (threadIdx.x < kJoinRows && t < count) a.lse[t] = l;
    rows_losses(a, blockIdx.x, l, sh);
}

// Factors of the rows' own gradients (bfloat16) and their exponent, or that of the scale of x times them (fp32: each below 2^(kTop + 1)).  Gradients that are
// infinite or NaN do not count: they would make zeros of the others.
template <bool F16>
__global__ __launch_bounds__(1024) void xent_factor_kernel(const float *grad, XentHeader *hdr, const int32_t *source, const int32_t *own_x, float *g) {
    __shared__ float lds[16];
    const int count = hdr->count;
    float top = -1024.0f;
    for (int t = threadIdx.x; t < count; t += 1024) {
        const int s = source[t];
        const float m = fabsf(grad[s]);
        if (m > 0.0f && m < __builtin_inff()) top = fmaxf(top, (float)(Upstream::exponent_of(m) - (F16 ? own_x[s] : 0)));
    }
    top = reduce_threads<1024, true>(top, lds);
    const int e = top > -1024.0f ? (int)top : 0;
    if (threadIdx.x == 0) hdr->gexp = F16 ? -1 - e : e;
    if constexpr (!F16)
        for (int t = threadIdx.x; t < count; t += 1024) g[t] = ldexpf(grad[source[t]], -e);
}

struct TurnArgs {
    JoinArgs join;
    const int32_t *wanted;
    Upstream up;
    AlignArgs align;
    char *P;
    int64_t pitch_P;
};
// Exponentials become G where they lie, 256 columns of ROWS rows to a workgroup, eight columns to a lane: zeros behind the vocabulary and, to a
// whole k-tile, behind the last row.  614 x 50265 in binary16 pairs 55 us, 248 MB read and written.  32 rows, or eight where that leaves CUs
// without a workgroup (500 x 512 by 8000 fp32, both passes: 83.6 us and 81.8).  JOIN: those join the parts of their rows themselves, as the
// kernel above does, which saves its launch (both passes, fp32: 200 x 256 by 1000 43.3 -> 40.6 us, 50 x 256 by 16000 55.3 -> 51.8, 20 x 64 by
// 50000 65.3 -> 61.5; but 300 x 768 by 16000 bf16 69.2 -> 70.4).  fp32: what the gradients' products read is split again here where it has to be (see
// AlignArgs; 50265 x 768 for one huge row 38 us).
template <bool F16, int ROWS, bool JOIN>
__global__ __launch_bounds__(256) void xent_turn_kernel(const TurnArgs a) {
    static_assert(!JOIN || ROWS == kJoinRows, "the rows of a workgroup");
    const JoinArgs &j = a.join;
    const int across = (j.vocab + 255) / 256, group_y = blockIdx.x / across, group_x = blockIdx.x - group_y * across;  // (rows can be too many for a grid's second axis)
    const bool wide_x = F16 && j.hdr->wide[0], wide_w = F16 && j.hdr->wide[1];
    const int rows = rows_of(j.hdr, j.first, j.room), last = (rows + kStageCols - 1) / kStageCols * kStageCols;
    if constexpr (F16) align_operands(a.align, j.hdr, wide_x, wide_w, a.up, j.first, rows);
    const int row0 = group_y * ROWS + (threadIdx.x >> 5), v0 = group_x * 256 + (threadIdx.x & 31) * 8, left = j.vocab - v0;
    const bool losses = JOIN && group_x == 0 && group_y < max(1, (rows + ROWS - 1) / ROWS);
    if (group_y * ROWS >= last && !losses) return;
    if (!JOIN && v0 >= (j.vocab + kStageCols - 1) / kStageCols * kStageCols) return;
    const int part = v0 / (logits_edge(rows_at_most(j.hdr, j.room), j.d, j.vocab) / 2);  // whose columns share a largest logit
    constexpr int kTurns = ROWS / 8;
    v4i32 hi[kTurns], lo[kTurns];
    char *const p0 = a.P + byte_of<F16>(v0);
    const int end = JOIN && v0 >= (j.vocab + kStageCols - 1) / kStageCols * kStageCols ? 0 : last, some = min(rows, end);  // rows of this lane's columns
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int t = row0 + 8 * i;
        if (t >= some) continue;
        hi[i] = *reinterpret_cast<const v4i32 *>(p0 + t * a.pitch_P);
        if (F16) lo[i] = *reinterpret_cast<const v4i32 *>(p0 + t * a.pitch_P + kSecond);
    }
    __shared__ JoinShared sh;
    __shared__ float lse[kJoinRows];
    float own_lse = 0.0f;
    if constexpr (JOIN) {
        own_lse = join_rows(j, group_y, sh);
        if (threadIdx.x < kJoinRows) lse[threadIdx.x] = own_lse;
        __syncthreads();
    }
#pragma unroll
    for (int i = 0; i < kTurns; ++i) {
        const int t = row0 + 8 * i;
        if (t >= end) continue;
        uint32_t qh[4] = {0, 0, 0, 0}, ql[4] = {0, 0, 0, 0};
        if (t < rows) {
            const float top = j.stats[((int64_t)part * j.room + t) * 2];
            const float g = a.up.g ? a.up.g[j.first + t] : 1.0f, l = JOIN ? lse[threadIdx.x >> 5] : j.lse[j.first + t];
            const float down = __builtin_amdgcn_exp2f((top - l) * kLog2e) * g, one = F16 ? g * power_of_two(kTop) : g;
            const int own = a.wanted[j.first + t] - v0;
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint16_t h = (uint16_t)((uint32_t)hi[i][k >> 1] >> (16 * (k & 1)));
                if constexpr (F16) v[k] = (float)__builtin_bit_cast(_Float16, h) + (float)__builtin_bit_cast(_Float16, (uint16_t)((uint32_t)lo[i][k >> 1] >> (16 * (k & 1))));
                else v[k] = (float)__builtin_bit_cast(__bf16, h);
                v[k] = k < left ? v[k] * down - (k == own ? one : 0.0f) : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (F16) {
                    const _Float16 h0 = (_Float16)v[2 * k], h1 = (_Float16)v[2 * k + 1];
                    qh[k] = pack(h0, h1);
                    ql[k] = pack((_Float16)(v[2 * k] - (float)h0), (_Float16)(v[2 * k + 1] - (float)h1));
                } else {
                    qh[k] = pack((__bf16)v[2 * k], (__bf16)v[2 * k + 1]);
                }
            }
        }
        *reinterpret_cast<v4i32 *>(p0 + t * a.pitch_P) = v4i32{(int)qh[0], (int)qh[1], (int)qh[2], (int)qh[3]};
        if (F16) *reinterpret_cast<v4i32 *>(p0 + t * a.pitch_P + kSecond) = v4i32{(int)ql[0], (int)ql[1], (int)ql[2], (int)ql[3]};
    }
    if constexpr (JOIN)
        if (losses) rows_losses(j, group_y, own_lse, sh);
}

// Into how many parts the tiles of a gradient are cut along the contraction, so that every CU has one.
__host__ __device__ __forceinline__ int parts_of(int tiles, int slots, int ktiles) {
    const int most = tiles > 0 ? slots / tiles : 1, able = ktiles / kPartTiles;
    const int n = most < able ? most : able;
    return n > 1 ? n : 1;
}

// How the gradients are cut with tiles of one size.
struct Cut {
    int xslots, xgroups, wcut;  // parts of tiles of gx that go at a time, and as many as there can be of this problem; parts of the tiles of gW
    bool through;               // gW goes through sums in fp32
};
struct GradArgs {
    Operand G, w, x;   // [row of the piece][vocabulary], [vocabulary][feature], [row of the piece][feature]
    const XentHeader *hdr;
    Upstream up;
    float *xparts, *wparts;  // [slot][tile]; wparts: where the tiles of gW are cut, or are sums over several pieces
    void *gw;
    int64_t ldgw;
    int d, ktiles, first, room;  // ktiles: of gx's contraction
    Cut cut;
};
// A tile (or part of one) of gx = G W, with W across, or of gW = G^T x, both across and with rows of zeros to whole k-tiles.
template <bool F16, int T, bool X>
__device__ __forceinline__ void grad_tile(const GradArgs &a, int wg, char *smem) {
    constexpr int kEdge = 64 * T;
    const int count = rows_of(a.hdr, a.first, a.room);
    if (!X && count == 0 && a.first > 0) return;  // (the first piece writes zeros)
    const int height = X ? count : a.w.rows, width = a.d;  // of the gradient
    const int mtiles = (height + kEdge - 1) / kEdge, ntiles = (width + kEdge - 1) / kEdge, tiles = mtiles * ntiles;
    constexpr int R = kPlaces<F16>;
    const int rtiles = (count + R - 1) / R, ktiles = X ? a.ktiles : rtiles, parts = X ? parts_of(tiles, a.cut.xslots, a.ktiles) : a.cut.wcut;
    if (wg >= tiles * parts) return;
    int tm, tn, part = 0, slot = 0;
    if (parts == 1) {
        tile_at(wg, mtiles, ntiles, tm, tn);
        slot = tn * mtiles + tm;
    } else {  // workgroups of an XCD: consecutive tiles of one part of the contraction
        const int xcd = wg & 7, idx = wg >> 3, per = tiles * parts >> 3, rem = (tiles * parts) & 7;
        slot = xcd * per + min(xcd, rem) + idx;
        part = slot / tiles;
        const int tile = slot - part * tiles;
        tn = tile / mtiles;
        tm = tile - tn * mtiles;
    }
    tm = __builtin_amdgcn_readfirstlane(tm);
    tn = __builtin_amdgcn_readfirstlane(tn);
    const int k0 = __builtin_amdgcn_readfirstlane((int)((int64_t)ktiles * part / parts)), k1 = __builtin_amdgcn_readfirstlane((int)((int64_t)ktiles * (part + 1) / parts));
    Operand G = a.G, x = a.x;
    G.rows = X ? count : rtiles * R;
    if (X) G.cols = ktiles * kStageCols;  // (zeros behind the vocabulary)
    x.rows = rtiles * R;
    v16f32 acc[T][T];
    product_tile<F16, T, T, !X, true>(G, X ? a.w : x, tm * kEdge, tn * kEdge, k0, k1, smem, acc);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r0 = (wave >> 1) * 32 * T, rl = 4 * (lane >> 5), c0 = (wave & 1) * 32 * T + (lane & 31);
    if (X || a.cut.through) {
        float *to = (X ? a.xparts : a.wparts) + (int64_t)slot * kEdge * kEdge + r0 * kEdge;
        const bool add = !X && a.first > 0;
#pragma unroll
        for (int i = 0; i < T; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r)
#pragma unroll
                for (int j = 0; j < T; ++j) {
                    float *p = to + (32 * i + (r >> 2) * 8 + (r & 3)) * kEdge + (rl * kEdge + c0 + 32 * j);
                    *p = add ? *p + acc[i][j][r] : acc[i][j][r];
                }
        return;
    }
    const int e = a.up.exponent(a.hdr) - (F16 ? kTop + a.up.scale_x(a.hdr) : 0);
    const float factor = a.up.factor(a.hdr);
    auto done = [&](float v) __attribute__((always_inline)) { return ldexpf(v * factor, e); };
    const int v0 = tm * kEdge + r0, f0 = tn * kEdge + c0;
#pragma unroll
    for (int i = 0; i < T; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if constexpr (F16) {
                float *to = (float *)a.gw + (int64_t)(v0 + 32 * i + 8 * q) * a.ldgw;  // (the lane's row is rl further)
#pragma unroll
                for (int k = 0; k < 4; ++k)
#pragma unroll
                    for (int j = 0; j < T; ++j)
                        if (v0 + 32 * i + 8 * q + rl + k < height && f0 + 32 * j < width) to[(rl + k) * a.ldgw + f0 + 32 * j] = done(acc[i][j][4 * q + k]);
            } else {  // four rows by four columns trade places among four lanes: 8 bytes to a store
                const int v = v0 + 32 * i + 8 * q + rl + (lane & 3);
                uint16_t *to = (uint16_t *)a.gw + (int64_t)v * a.ldgw;
#pragma unroll
                for (int j = 0; j < T; ++j) {
                    uint32_t lo = pack((__bf16)done(acc[i][j][4 * q]), (__bf16)done(acc[i][j][4 * q + 1]));
                    uint32_t hi = pack((__bf16)done(acc[i][j][4 * q + 2]), (__bf16)done(acc[i][j][4 * q + 3]));
                    quad_transpose(lo, hi, lane);
                    const int f = (f0 & ~3) + 32 * j;
                    if (v >= height) continue;
                    const piece_t<uint16_t, 4> x4 = __builtin_bit_cast(piece_t<uint16_t, 4>, make_uint2(lo, hi));
                    if (f + 4 <= width) *reinterpret_cast<piece_t<uint16_t, 4> *>(to + f) = x4;
                    else
                        for (int k = 0; k < 4; ++k)
                            if (f + k < width) to[f + k] = x4[k];
                }
            }
        }
}
// Both gradients from a piece of the rows: the first xgroups workgroups take parts of the tiles of gx, those behind them tiles of gW (parts of
// them, where there are few), so that neither waits for the other's last ones.  4096 x 4096 by 32000 bfloat16 1700 us, 1.26 PFLOP/s; 614 x 768
// by 50265 fp32 291 us, 0.98 of binary16.
template <bool F16, int T>
__global__ __launch_bounds__(kProductThreads, T == 4 ? 1 : 2) void xent_grads_kernel(const GradArgs a) {
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    if (grads_edge(rows_at_most(a.hdr, a.room), a.d, a.w.rows) != 64 * T) return;
    if ((int)blockIdx.x < a.cut.xgroups) grad_tile<F16, T, true>(a, blockIdx.x, smem);
    else grad_tile<F16, T, false>(a, blockIdx.x - a.cut.xgroups, smem);
}

struct FoldArgs {
    const float *xparts, *wparts;
    const XentHeader *hdr;
    Upstream up;
    const int32_t *place;
    void *gx, *gw;
    int64_t ldgx, ldgw, xrows, wrows;  // rows of gx and gW that are made here
    int d, vocab, ktiles, first, room;
    Cut cut[2];               // with tiles of 128 and of 256
};
// Rows of gx that belong to the piece (the first: zeros for those without a target) and of gW from the parts of their tiles, 256 columns to a
// workgroup, four to a lane.  ROWS = 4: a row to a wave; 1: a row to the workgroup, a quarter of the parts to a wave, so that as many loads
// are under way where there are many parts (76 parts of 74 rows of 168 columns: 22 us and 5; 2 of 8192 rows of 768 columns, bf16: 103 and 39).
template <class T, int ROWS>
__global__ __launch_bounds__(256) void xent_fold_kernel(const FoldArgs a) {
    __shared__ float4 sums[4][64];
    const int64_t xgroups = (a.xrows + ROWS - 1) / ROWS;
    const bool isX = (int64_t)blockIdx.x < xgroups;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = (blockIdx.y * 64 + lane) * 4;
    const int64_t row = (isX ? blockIdx.x : blockIdx.x - xgroups) * ROWS + (ROWS == 4 ? wave : 0);
    const int edge = grads_edge(rows_at_most(a.hdr, a.room), a.d, a.vocab);
    const Cut cut = a.cut[edge / 256];
    if (row >= (isX ? a.xrows : a.wrows) || (!isX && !cut.through)) return;
    const int place = isX ? a.place[row] : (int)row, rows = isX ? rows_of(a.hdr, a.first, a.room) : (int)a.wrows, at = place < 0 ? place : isX ? place - a.first : place;
    if (place < 0 ? a.first > 0 : at < 0 || at >= rows) return;
    const int mtiles = (rows + edge - 1) / edge, ntiles = (a.d + edge - 1) / edge, tiles = mtiles * ntiles;
    const int n = place < 0 ? 0 : isX ? parts_of(tiles, cut.xslots, a.ktiles) : cut.wcut, last = ROWS == 4 ? n : n * (wave + 1) / 4;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (col < a.d) {
        const float *p = (isX ? a.xparts : a.wparts) + (int64_t)(col / edge * mtiles + at / edge) * edge * edge + at % edge * edge + col % edge;
        const int64_t step = (int64_t)tiles * edge * edge;
        for (int k0 = ROWS == 4 ? 0 : n * wave / 4; k0 < last; k0 += 4) {
            float4 f[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) f[k] = k0 + k < last ? *reinterpret_cast<const float4 *>(p + (k0 + k) * step) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < 4; ++k) { s[0] += f[k].x; s[1] += f[k].y; s[2] += f[k].z; s[3] += f[k].w; }
        }
    }
    if constexpr (ROWS == 1) {
        sums[wave][lane] = make_float4(s[0], s[1], s[2], s[3]);
        __syncthreads();
        if (wave > 0) return;
#pragma unroll
        for (int w = 1; w < 4; ++w) { s[0] += sums[w][lane].x; s[1] += sums[w][lane].y; s[2] += sums[w][lane].z; s[3] += sums[w][lane].w; }
    }
    if (col >= a.d) return;
    int e = a.up.exponent(a.hdr) - (sizeof(T) == 4 ? kTop + (isX ? scale_exponent(a.hdr->amax[1]) : a.up.scale_x(a.hdr)) : 0);
    float factor = place < 0 ? 1.0f : a.up.factor(a.hdr);  // (zeros stay zeros)
    if (sizeof(T) == 4 && a.up.rows && isX && place >= 0) {  // the row's own gradient
        const float g = a.up.grad[row];
        const int eg = Upstream::exponent_of(g);
        e += eg;
        factor = ldexpf(g, -eg);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) s[k] = ldexpf(s[k] * factor, e);
    store_upto<T, 4>((T *)(isX ? a.gx : a.gw) + row * (isX ? a.ldgx : a.ldgw) + col, s, a.d - col);
}

// What the gradients, which may have been made for a gradient of 1, are multiplied with.  bfloat16 ones are rounded a second time (a scale of the loss
// is a power of two as a rule, which rounds nothing); only a second pass over the products would save that.
template <class T>
__global__ __launch_bounds__(256) void xent_rescale_kernel(const float *grad, T *gx, int64_t nx, T *gw, int64_t nw) {
    const float g = *grad;
    if (g == 1.0f) return;
    constexpr int N = kVec<T>;
    for (int64_t k = ((int64_t)blockIdx.x * 256 + threadIdx.x) * N; k < nx + nw; k += (int64_t)gridDim.x * 256 * N) {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const int64_t at = k + e;
            if (at >= nx + nw) break;
            T *p = at < nx ? gx + at : gw + (at - nx);
            *p = (T)((float)*p * g);
        }
    }
}

static int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

// Where everything lies in the workspace.
struct XentLayout {
    int64_t places;               // of a contraction in a k-tile
    int64_t dp, tp, vp;           // features, rows, vocabulary rounded up to what the products read
    bool split, direct;           // two numbers to a value; W read in place
    int64_t pitch_p, pitch_P;     // bytes from row to row of x and W in 16 bits, and of G
    int edge_l, edge_g;           // largest tile edges that the rows allow, of the logits and of the gradients
    int64_t room, pieces;         // rows to a piece, pieces
    Cut cut[2];                   // of the gradients, with tiles of 128 and of 256
    bool few;                     // W is read as it is
    bool by_rows;                 // each row of x and W has a scale of its own
    size_t source, place, wanted, lse, row_loss, hit, g, ex, ew, own_x, stats, px, pw, P, xparts, wparts, bytes;
};
static XentLayout xent_layout(const void *w, int64_t ldw, int64_t rows, int64_t d, int64_t vocab, int dtype, bool grad) {
    XentLayout l = {};
    l.split = dtype == IMUNPACK_F32;
    const int64_t numbers = l.split ? 2 : 1;
    l.places = l.split ? kPlaces<true> : kPlaces<false>;
    l.dp = up(d, kStageCols);
    l.tp = up(std::max<int64_t>(rows, 1), 256);
    l.vp = up(vocab, 256);
    l.direct = !l.split && d % 8 == 0 && ldw % 8 == 0 && ldw <= 1 << 22 && (size_t)w % 16 == 0;  // (a tile's rows lie within 32 bits)
    // (for the loss alone that is 2^34 logits, whose tiles are few enough for a grid: with 2^38 its threads would pass 32 bits)
    const int64_t row_bytes = grad ? 2 * numbers * l.vp : up(vocab, 128) / 64 * 8;
    l.room = std::min(l.tp, std::max<int64_t>(256, kPieceBytes / row_bytes / 256 * 256));
    l.pieces = (l.tp + l.room - 1) / l.room;
    l.edge_l = logits_edge((int)std::min(rows, l.room), (int)d, (int)vocab);
    l.edge_g = grads_edge((int)std::min(rows, l.room), (int)d, (int)vocab);
    size_t at = sizeof(XentHeader);
    auto take = [&](int64_t bytes) { const size_t here = at; at = (at + (size_t)bytes + 255) & ~(size_t)255; return here; };
    l.source = take(rows * 4); l.place = take(rows * 4); l.wanted = take(rows * 4);
    l.lse = take(rows * 4); l.row_loss = take(rows * 4); l.hit = take(rows * 4); l.g = take(rows * 4);
    // (a wave to a row: 1418 x 1031 by 32003 rows 83 -> 60 us for both passes over the operands, but 64 x 85 by 16360 10 -> 16)
    l.few = l.split && !grad && rows <= kFewRows && vocab * d * 4 > kLastLevelCache;
    l.by_rows = l.split && !grad && !l.few && d >= 512;
    l.ex = take(l.split ? rows * 4 : 0); l.ew = take(l.split ? l.vp * 4 : 0); l.own_x = take(l.split ? rows * 4 : 0);
    l.stats = take(2 * (up(vocab, 128) / 128) * l.room * 8);  // (two parts to a tile)
    l.pitch_p = l.dp * 2 * numbers;
    l.px = take(l.tp * l.pitch_p);
    l.pw = take(l.direct || l.few ? 0 : vocab * l.pitch_p);
    if (grad) {
        l.pitch_P = l.vp * 2 * numbers;
        l.P = take(l.room * l.pitch_P);
        int64_t xbytes = 0, wbytes = 0;
        for (int64_t edge = 128; edge <= l.edge_g; edge *= 2) {
            Cut &c = l.cut[edge / 256];
            const int64_t xtiles = up(l.room, edge) / edge * (up(d, edge) / edge), wtiles = up(vocab, edge) / edge * (up(d, edge) / edge);
            c.xslots = (int)std::max<int64_t>(xtiles, kXentSlots);
            const int64_t able = std::max<int64_t>(1, up(vocab, l.places) / l.places / kPartTiles);  // (as parts_of; a multiple of the XCDs)
            c.xgroups = (int)up(std::max(xtiles, std::min<int64_t>(c.xslots, xtiles * able)), 8);
            c.wcut = l.pieces == 1 && wtiles <= kXentSlots / 2 ? parts_of((int)wtiles, kXentSlots, (int)(up(rows, l.places) / l.places)) : 1;
            c.through = c.wcut > 1 || l.pieces > 1;
            xbytes = std::max(xbytes, (int64_t)c.xgroups * edge * edge * 4);
            wbytes = std::max(wbytes, c.through ? c.wcut * wtiles * edge * edge * 4 : 0);
        }
        l.xparts = take(xbytes);
        l.wparts = take(wbytes);
    }
    l.bytes = at;
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
    return more_lds(xent_grads_kernel<F16, T>, product_lds(T, T));
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
static void launch_logits(const LogitArgs &a, bool keep, unsigned groups, hipStream_t st) {
    if (keep) hipLaunchKernelGGL((xent_logits_kernel<F16, T, true>), dim3(groups), dim3(kProductThreads), product_lds(T, T), st, a);
    else hipLaunchKernelGGL((xent_logits_kernel<F16, T, false>), dim3(groups), dim3(kProductThreads), product_lds(T, T), st, a);
}
template <bool F16>
static void launch_logits(const LogitArgs &a, int edge, bool keep, int64_t rows, hipStream_t st) {
    auto groups = [&](int64_t edge) { return (unsigned)(up(a.w.rows, edge) / edge * (up(rows, edge) / edge)); };
    if (edge == 256) {  // (a workgroup that finds nothing to do takes its time too: no more of them than would have something)
        launch_logits<F16, 4>(a, keep, groups(256), st);
        if (logits_edge(kLargeRows, a.d, a.w.rows) == 256) rows = std::min<int64_t>(rows, kLargeRows);
    }
    launch_logits<F16, 2>(a, keep, groups(128), st);
}
template <bool F16, int T>
static void launch_grads(const GradArgs &a, unsigned groups, hipStream_t st) {
    hipLaunchKernelGGL((xent_grads_kernel<F16, T>), dim3(groups), dim3(kProductThreads), product_lds(T, T), st, a);
}
template <bool F16>
static void launch_grads(GradArgs a, const XentLayout &l, bool x, bool w, hipStream_t st) {
    for (int edge = l.edge_g; edge >= 128; edge /= 2) {
        a.cut = l.cut[edge / 256];
        if (!x) a.cut.xgroups = 0;
        const unsigned groups = (unsigned)(a.cut.xgroups + (w ? up(a.w.rows, edge) / edge * (up(a.d, edge) / edge) * a.cut.wcut : 0));
        if (groups == 0) continue;
        if (edge == 256) launch_grads<F16, 4>(a, groups, st);
        else launch_grads<F16, 2>(a, groups, st);
    }
}
}  // namespace imu

using namespace imu;

extern "C" int imunpack_xent_workspace(const void *w, int64_t ldw, int64_t rows, int64_t d, int64_t vocab, int dtype, int want_grad, size_t *bytes) {
    if (!xent_sizes(rows, d, vocab, dtype) || ldw < d || !bytes) return IMUNPACK_EINVAL;
    *bytes = xent_layout(w, ldw, rows, d, vocab, dtype, want_grad != 0).bytes;
    return IMUNPACK_OK;
}

extern "C" int imunpack_xent(const void *x, int64_t ldx, const void *w, int64_t ldw, const int64_t *target, int64_t rows, int64_t d, int64_t vocab,
                             int dtype, int64_t ignore_index, int reduction, float *loss, const float *grad, void *gx, int64_t ldgx, void *gw,
                             int64_t ldgw, void *workspace, size_t workspace_bytes, imunpack_stream_t stream) {
    if (!xent_sizes(rows, d, vocab, dtype) || ldx < d || ldw < d || reduction < IMUNPACK_NONE || reduction > IMUNPACK_MEAN || !w || !workspace ||
        (size_t)workspace % 16 || (gx && ldgx < d) || (gw && ldgw < d) || (rows > 0 && (!x || !target)) || (!loss && !gx && !gw && rows > 0) ||
        ((gx || gw) && !grad && rows > 0 && reduction == IMUNPACK_NONE))
        return IMUNPACK_EINVAL;
    const bool back = gx || gw;
    const XentLayout l = xent_layout(w, ldw, rows, d, vocab, dtype, back);
    if (workspace_bytes < l.bytes) return IMUNPACK_ESMALL;
    IMU_TRY(xent_lds_opt_in());
    hipStream_t st = (hipStream_t)stream;
    char *s = (char *)workspace;
    XentHeader *hdr = (XentHeader *)s;
    int32_t *source = (int32_t *)(s + l.source), *place = (int32_t *)(s + l.place), *wanted = (int32_t *)(s + l.wanted);
    ScanArgs c = {};
    c.target = target; c.vocab = vocab; c.ignore = ignore_index; c.hdr = hdr; c.source = source; c.place = place; c.wanted = wanted;
    c.loss = reduction == IMUNPACK_NONE ? loss : nullptr;
    c.x = (const float *)x; c.w = (const float *)w; c.ldx = ldx; c.ldw = ldw; c.rows = (int)rows; c.d = (int)d;
    c.own_x = (int32_t *)(s + l.own_x); c.own_w = (int32_t *)(s + l.ew);
    // (workgroups of 16 waves, a wave to four rows)
    const int nx = (int)std::min<int64_t>(up(rows, 64) / 64, kScanX), nw = (int)std::min<int64_t>(up(vocab, 64) / 64, kScanGroups - kScanX);
    c.nx = nx;
    const bool scans = !l.split && rows > 0 && rows <= kScanHere;  // the kernel that gathers x does it
    if (!scans) hipLaunchKernelGGL(xent_scan_kernel, dim3(l.split && !l.by_rows && !l.few && rows > 0 ? 1 + nx + nw : 1), dim3(1024), 0, st, c);
    if (rows > 0 && l.by_rows) {
        PrepareRowsArgs p = {};
        p.x = (const float *)x; p.w = (const float *)w; p.ldx = ldx; p.ldw = ldw; p.hdr = hdr; p.source = source;
        p.px = s + l.px; p.pw = s + l.pw; p.pitch = l.pitch_p; p.wrows = vocab;
        p.ex = (int32_t *)(s + l.ex); p.ew = (int32_t *)(s + l.ew); p.d = (int)d; p.xgroups = (int)(up(rows, 4) / 4);
        hipLaunchKernelGGL(xent_prepare_rows_kernel, dim3((unsigned)(p.xgroups + up(vocab, 4) / 4)), dim3(256), 0, st, p);
    } else if (rows > 0 && !l.few) {
        PrepareArgs p = {};
        p.scan = c;
        p.x = x; p.w = w; p.ldx = ldx; p.ldw = ldw; p.hdr = hdr; p.source = source;
        p.px = s + l.px; p.pw = s + l.pw;
        p.xrows = l.tp; p.wrows = l.direct ? 0 : vocab; p.d = (int)d; p.pieces = (int)(l.dp / 8); p.nx = nx; p.nw = nw;
        p.own_x = c.own_x; p.ex = (int32_t *)(s + l.ex); p.ew = (int32_t *)(s + l.ew);
        const int64_t threads = scans ? 1024 : 256, per = threads * kPrepareTurns;
        p.xgroups = (int)((up(rows, kStageCols) * p.pieces + per - 1) / per);
        const dim3 grid((unsigned)(p.xgroups + (p.wrows * p.pieces + per - 1) / per));
        if (l.split) hipLaunchKernelGGL((xent_prepare_kernel<float, false>), grid, dim3(256), 0, st, p);
        else hipLaunchKernelGGL((scans ? xent_prepare_kernel<__bf16, true> : xent_prepare_kernel<__bf16, false>), grid, dim3((unsigned)threads), 0, st, p);
    }
    Upstream upstream = {grad, nullptr, reduction == IMUNPACK_MEAN, l.split && reduction == IMUNPACK_NONE};
    if (back && reduction == IMUNPACK_NONE) {
        if (!l.split) upstream.g = (const float *)(s + l.g);
        hipLaunchKernelGGL((l.split ? xent_factor_kernel<true> : xent_factor_kernel<false>), dim3(1), dim3(1024), 0, st, grad, hdr, source, c.own_x, (float *)(s + l.g));
    }
    const AlignArgs align = {gw ? (const float *)x : nullptr, gx ? (const float *)w : nullptr, ldx, ldw, l.pitch_p, s + l.px, s + l.pw, source, c.own_x,
                             (const int32_t *)(s + l.ew), (int)d, (int)vocab};
    for (int64_t piece = 0; piece < l.pieces; ++piece) {
        const int64_t first = piece * l.room, n = std::min(l.room, rows - first);  // rows of the piece at most
        const int held = (int)(l.pitch_p / 2);  // (zeros behind the features)
        const Operand whole = {l.direct ? (const char *)w : s + l.pw, l.direct ? ldw * 2 : l.pitch_p, (int)vocab, l.direct ? (int)d : held};
        const Operand part = {s + l.px + first * l.pitch_p, l.pitch_p, 0, held};
        if (n > 0 && l.few) {
            FewArgs a = {(const float *)x, (const float *)w, ldx, ldw, hdr, source, wanted, (float *)(s + l.stats), (float *)(s + l.hit), (int)l.room, (int)d, (int)vocab};
            hipLaunchKernelGGL(xent_few_kernel, dim3((unsigned)(2 * (up(vocab, 128) / 128))), dim3(256), 0, st, a);
        } else if (n > 0) {
            if (l.split && gx && piece > 0) hipLaunchKernelGGL(xent_weights_kernel, dim3(4 * kCus), dim3(256), 0, st, align, hdr);
            LogitArgs a = {};
            a.w = whole; a.x = part;
            a.ex = (const int32_t *)(s + l.ex); a.ew = (const int32_t *)(s + l.ew);
            a.hdr = hdr; a.wanted = wanted; a.stats = (float *)(s + l.stats); a.hit = (float *)(s + l.hit);
            a.P = s + l.P; a.pitch_P = l.pitch_P;
            a.first = (int)first; a.room = (int)l.room; a.d = (int)d; a.ktiles = (int)(up(d, l.places) / l.places);
            l.split ? launch_logits<true>(a, l.edge_l, back, n, st) : launch_logits<false>(a, l.edge_l, back, n, st);
        }
        const unsigned across = (unsigned)(up(vocab, 256) / 256), down = (unsigned)up(n, kStageCols);
        const bool few = across * down / 32 < 4 * kCus, joins = back && n > 0 && few && l.pieces == 1 && (int64_t)across * n * (up(vocab, 128) / 64) <= kJoinReads;
        JoinArgs j = {};
        j.stats = (const float *)(s + l.stats); j.hit = (const float *)(s + l.hit); j.d = (int)d; j.vocab = (int)vocab; j.first = (int)first; j.room = (int)l.room;
        j.how = loss ? reduction : IMUNPACK_NONE;
        j.hdr = hdr; j.source = source; j.lse = (float *)(s + l.lse); j.row_loss = (float *)(s + l.row_loss); j.loss = loss;
        if (!joins && (n > 0 || (loss && reduction != IMUNPACK_NONE)))
            hipLaunchKernelGGL(xent_join_kernel, dim3((unsigned)(up(std::max<int64_t>(n, 1), kJoinRows) / kJoinRows)), dim3(256), 0, st, j);
        if (!back) continue;
        if (n > 0) {
            TurnArgs t = {};
            t.join = j; t.wanted = wanted; t.up = upstream; t.align = align; t.P = s + l.P; t.pitch_P = l.pitch_P;
            const dim3 grid(across * (down / (few ? 8 : 32)));
            if (l.split) hipLaunchKernelGGL((joins ? xent_turn_kernel<true, 8, true> : few ? xent_turn_kernel<true, 8, false> : xent_turn_kernel<true, 32, false>), grid, dim3(256), 0, st, t);
            else hipLaunchKernelGGL((joins ? xent_turn_kernel<false, 8, true> : few ? xent_turn_kernel<false, 8, false> : xent_turn_kernel<false, 32, false>), grid, dim3(256), 0, st, t);
        }
        GradArgs a = {};
        a.G = {s + l.P, l.pitch_P, 0, (int)(l.pitch_P / 2)};
        a.w = whole; a.x = part;
        a.hdr = hdr; a.up = upstream; a.xparts = (float *)(s + l.xparts); a.wparts = (float *)(s + l.wparts);
        a.gw = gw; a.ldgw = ldgw; a.d = (int)d; a.ktiles = (int)(up(vocab, l.places) / l.places);
        a.first = (int)first; a.room = (int)l.room;
        l.split ? launch_grads<true>(a, l, gx && n > 0, gw, st) : launch_grads<false>(a, l, gx && n > 0, gw, st);
        FoldArgs f = {};
        f.xparts = a.xparts; f.wparts = a.wparts; f.hdr = hdr; f.up = upstream; f.place = place;
        f.gx = gx; f.gw = gw; f.ldgx = ldgx; f.ldgw = ldgw; f.cut[0] = l.cut[0]; f.cut[1] = l.cut[1];
        f.xrows = gx && n > 0 ? rows : 0; f.wrows = gw && (l.cut[0].through || l.cut[1].through) && piece + 1 == l.pieces ? vocab : 0;
        f.d = (int)d; f.vocab = (int)vocab; f.ktiles = a.ktiles; f.first = a.first; f.room = a.room;
        if (f.xrows + f.wrows > 0) {
            const int64_t xtiles = up(std::min(rows, l.room), 128) / 128 * (up(d, 128) / 128);
            const bool many = std::max(f.wrows > 0 ? l.cut[0].wcut : 0, f.xrows > 0 ? parts_of((int)xtiles, l.cut[0].xslots, a.ktiles) : 0) >= 8;
            const int64_t each = many ? 1 : 4;
            const dim3 grid((unsigned)(up(f.xrows, each) / each + up(f.wrows, each) / each), (unsigned)(up(d, 256) / 256));
            if (l.split) hipLaunchKernelGGL((many ? xent_fold_kernel<float, 1> : xent_fold_kernel<float, 4>), grid, dim3(256), 0, st, f);
            else hipLaunchKernelGGL((many ? xent_fold_kernel<__bf16, 1> : xent_fold_kernel<__bf16, 4>), grid, dim3(256), 0, st, f);
        }
    }
    return launch_status();
}

extern "C" int imunpack_xent_rescale(const float *grad, void *gx, int64_t nx, void *gw, int64_t nw, int dtype, imunpack_stream_t stream) {
    if (!grad || nx < 0 || nw < 0 || (nx > 0 && !gx) || (nw > 0 && !gw) || (dtype != IMUNPACK_F32 && dtype != IMUNPACK_BF16)) return IMUNPACK_EINVAL;
    if (nx + nw == 0) return IMUNPACK_OK;
    const int64_t pieces = (nx + nw + 1023) / 1024;
    const dim3 grid((unsigned)std::min<int64_t>(pieces, 2048));
    hipStream_t st = (hipStream_t)stream;
    if (dtype == IMUNPACK_F32) hipLaunchKernelGGL(xent_rescale_kernel<float>, grid, dim3(256), 0, st, grad, (float *)gx, nx, (float *)gw, nw);
    else hipLaunchKernelGGL(xent_rescale_kernel<__bf16>, grid, dim3(256), 0, st, grad, (__bf16 *)gx, nx, (__bf16 *)gw, nw);
    return launch_status();
}
