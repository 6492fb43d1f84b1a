// Tensors into 8-bit floating point with a power of two per block (block8.h says how), back, turned; activation functions whose input is kept that way.
//
// All of it is bound by memory.  Along rows, sixteen lanes hold a block (eight elements each), so that its largest magnitude is a maximum over
// registers and four rotations within a row of lanes, nothing goes through LDS, and the blocks of a matrix of any width fill whole waves.
// For the turned tensor (codes of x^T with blocks along x's columns), a workgroup holds 128 x 128 elements in registers, four rows by eight columns a
// lane; column maxima meet in LDS, and so do the codes, four rows of a column at a time.
// 4096 x 11008 bfloat16: along rows 21 us (6.4 TB/s), both ways 36 (5.1), codes turned 21 (4.4); gated SiLU that keeps its input and gives its result in 8 bits 74 (5.5), its
// gradient 59 (6.1).
#include "block8.h"

namespace imu {
constexpr int kLaunchBlocks = 1 << 26;  // blocks of a launch: far below 2^32 threads, indexes in 32 bits

// ---- along rows -------------------------------------------------------------------------------------------------------------
struct RowsArgs {
    const void *x;
    uint8_t *codes, *scales;
    int64_t ldx, ldc, lds;
    int rows, cols, kb;
};
constexpr int kRowsUnroll = 4;  // blocks of 16 lanes, one after the other

// GROUPS of 16 lanes to a workgroup.
template <class T, int FORMAT, int GROUPS>
__device__ __forceinline__ void rows_into(const RowsArgs &a, int group) {
    const int total = a.rows * a.kb, lane16 = threadIdx.x & 15;
    const int first = group * (GROUPS * kRowsUnroll) + (threadIdx.x >> 4);
    int row[kRowsUnroll], kb[kRowsUnroll];
    piece_t<T, 8> in[kRowsUnroll];
#pragma unroll
    for (int u = 0; u < kRowsUnroll; ++u) {
        const int block = min(first + GROUPS * u, total - 1);
        row[u] = block / a.kb;
        kb[u] = block - row[u] * a.kb;
        const int col = kb[u] * kBlock8 + lane16 * 8;
        in[u] = load_piece<T, 8>((const T *)a.x + row[u] * a.ldx + col, a.cols - col);
    }
#pragma unroll
    for (int u = 0; u < kRowsUnroll; ++u) {
        if (first + GROUPS * u >= total) break;
        float x[8];
        to_floats<T, 8>(in[u], x);
        const int byte = block8_of<FORMAT>(x);
        *reinterpret_cast<uint2 *>(a.codes + row[u] * a.ldc + kb[u] * kBlock8 + lane16 * 8) = encode8<FORMAT>(x, block8_inverse(byte));
        if (lane16 == 0) a.scales[row[u] * a.lds + kb[u]] = (uint8_t)byte;
    }
}
template <class T, int FORMAT>
__global__ __launch_bounds__(256) void block8_rows_kernel(const RowsArgs a) {
    rows_into<T, FORMAT, 16>(a, (int)blockIdx.x);
}

// ---- both ways, or turned alone -----------------------------------------------------------------------------------------------
struct TileArgs {
    const void *x;                // T, or codes with their scales
    const uint8_t *xs;
    uint8_t *codes, *scales;      // may be null
    uint8_t *turned, *tscales;
    int64_t ldx, ldxs, ldc, lds, ldt, ldts;
    int64_t rows;
    int cols, kb, square;
};

// Where the four codes of rows 4 p .. 4 p + 3 of column c lie in LDS: sixteen bytes at a time at places that turn with the column, so that the
// sixteen lanes of a row of lanes, eight columns apart, fall on different banks.
__device__ __forceinline__ int turned_at(int c, int p) { return c * 128 + ((((p >> 2) ^ (c >> 3)) & 7) << 4) + (p & 3) * 4; }

// T: float, __bf16, or uint8_t for codes in FORMAT (turned alone).  128 x 128 elements to a workgroup of eight waves, four rows by eight columns to a lane
// (eight rows by eight columns to one of four waves needed 200 registers: 4096 x 4096 bfloat16 both ways 21.5 us).
constexpr int kTileWaves = 8;
struct TileShared {
    __attribute__((aligned(16))) uint8_t tile[128 * 128];
    __attribute__((aligned(16))) int tops[kTileWaves][128];
    __attribute__((aligned(16))) uint8_t columns[128];
};
template <class T, int FORMAT>
__device__ __forceinline__ void tile_into(const TileArgs &a, unsigned which, TileShared &shared) {
    constexpr bool kCodes = std::is_same<T, uint8_t>::value;
    constexpr int R = 4;
    // (Codes are held as half their values: binary32's largest rounds up to a code of 2^128.)
    constexpr int kHalved = kCodes ? 1 : 0;
    auto &tile = shared.tile;
    auto &tops = shared.tops;
    auto &columns = shared.columns;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, group = lane >> 4, l16 = lane & 15;
    const int kb = (int)(which % a.kb);
    const int64_t rb = which / a.kb, row0 = rb * 128 + wave * 16 + group * R;
    const int col = kb * 128 + l16 * 8, have = a.cols - col;
    float x[R][8];
    {
        const T *p = (const T *)a.x + row0 * a.ldx + col;
        piece_t<T, 8> in[R];
        if (rb * 128 + 128 <= a.rows && kb * 128 + 128 <= a.cols) {
#pragma unroll
            for (int i = 0; i < R; ++i) in[i] = load_piece<T, 8>(p + i * a.ldx, 8);
        } else {
#pragma unroll
            for (int i = 0; i < R; ++i) in[i] = load_piece<T, 8>(p + i * a.ldx, row0 + i < a.rows ? have : 0);
        }
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if constexpr (kCodes) {
                const int byte = row0 + i < a.rows ? a.xs[(row0 + i) * a.ldxs + kb] : 127;
                decode8<FORMAT>(__builtin_bit_cast(uint2, in[i]), block8_scale(byte) * 0.5f, x[i]);
            } else {
                to_floats<T, 8>(in[i], x[i]);
            }
        }
    }
    // the columns' maxima (or the square's)
    int top[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const float column[R] = {x[0][j], x[1][j], x[2][j], x[3][j]};
        top[j] = top_bits<R>(column);
        const auto far = __builtin_amdgcn_permlane32_swap(top[j], top[j], false, false);  // (either half's in both)
        top[j] = max((int)far[0], (int)far[1]);
        const auto next = __builtin_amdgcn_permlane16_swap(top[j], top[j], false, false);
        top[j] = max((int)next[0], (int)next[1]);
    }
    if (lane < 16) {
        *reinterpret_cast<int4 *>(&tops[wave][lane * 8]) = make_int4(top[0], top[1], top[2], top[3]);
        *reinterpret_cast<int4 *>(&tops[wave][lane * 8 + 4]) = make_int4(top[4], top[5], top[6], top[7]);
    }
    __syncthreads();
    int bytes[8];
    {
        int all = 0;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            int4 t = make_int4(0, 0, 0, 0);
#pragma unroll
            for (int w = 0; w < kTileWaves; ++w) {
                const int4 v = *reinterpret_cast<const int4 *>(&tops[w][l16 * 8 + 4 * h]);
                t.x = max(t.x, v.x), t.y = max(t.y, v.y), t.z = max(t.z, v.z), t.w = max(t.w, v.w);
            }
            top[4 * h] = t.x, top[4 * h + 1] = t.y, top[4 * h + 2] = t.z, top[4 * h + 3] = t.w;
            all = max(all, max(max(t.x, t.y), max(t.z, t.w)));
        }
        if (a.square) {
            all = max16(all);
#pragma unroll
            for (int j = 0; j < 8; ++j) top[j] = all;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) bytes[j] = block8_byte<FORMAT, kHalved>(top[j]);
    }
    if constexpr (!kCodes) {
        if (a.codes) {
#pragma unroll
            for (int i = 0; i < R; ++i) {
                const int byte = a.square ? bytes[0] : block8_of<FORMAT>(x[i]);
                if (row0 + i < a.rows) {
                    *reinterpret_cast<uint2 *>(a.codes + (row0 + i) * a.ldc + col) = encode8<FORMAT>(x[i], block8_inverse(byte));
                    if (l16 == 0) a.scales[(row0 + i) * a.lds + kb] = (uint8_t)byte;
                }
            }
        }
    }
    if (!a.turned) return;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        uint32_t &to = *reinterpret_cast<uint32_t *>(tile + turned_at(l16 * 8 + j, wave * 4 + group));
        if constexpr (kCodes) {  // (a factor of 2^128, of half a value in a block of byte 0, is no number of binary32)
            const int up = 127 + kHalved - bytes[j];
            to = encode4<FORMAT>(__builtin_ldexpf(x[0][j], up), __builtin_ldexpf(x[1][j], up), __builtin_ldexpf(x[2][j], up), __builtin_ldexpf(x[3][j], up));
        } else {
            const float inverse = block8_inverse(bytes[j]);
            to = encode4<FORMAT>(x[0][j] * inverse, x[1][j] * inverse, x[2][j] * inverse, x[3][j] * inverse);
        }
    }
    if (threadIdx.x < 16)
        *reinterpret_cast<uint2 *>(columns + l16 * 8) = make_uint2(bytes[0] | bytes[1] << 8 | bytes[2] << 16 | (unsigned)bytes[3] << 24, bytes[4] | bytes[5] << 8 | bytes[6] << 16 | (unsigned)bytes[7] << 24);
    __syncthreads();
    if (threadIdx.x < 128 && kb * 128 + (int)threadIdx.x < a.cols) a.tscales[(int64_t)(kb * 128 + threadIdx.x) * a.ldts + rb] = columns[threadIdx.x];
#pragma unroll
    for (int u = 0; u < 2; ++u) {  // sixteen rows of a column to a thread
        const int c = u * 64 + (threadIdx.x >> 3), p = (threadIdx.x & 7) * 4;
        if (kb * 128 + c < a.cols)
            *reinterpret_cast<uint4 *>(a.turned + (int64_t)(kb * 128 + c) * a.ldt + rb * 128 + p * 4) = *reinterpret_cast<const uint4 *>(tile + turned_at(c, p));
    }
}
template <class T, int FORMAT>
__global__ __launch_bounds__(64 * kTileWaves) void block8_tile_kernel(const TileArgs a) {
    __shared__ TileShared shared;
    tile_into<T, FORMAT>(a, blockIdx.x, shared);
}

// ---- several tensors in one launch ------------------------------------------------------------------------------------------------
// What a step brings into 8 bits at one time: the workgroups of one tensor behind those of another.  For small tensors a launch is most of the time, and large ones fill the device while
// the others end.  Microseconds on the device, two launches and one, for x with weights both ways and for a gradient both ways with x turned: 197 x 256 by 1000 fp32 8.1, 5.6 and 10.1, 6.0;
// 12608 x 768 by 768 fp32 14.0, 11.7 and 22.6, 19.0; 16384 x 4096 by 4096 bfloat16 46.7, 45.0 and 92.9, 90.2.
enum JobKind { kRowsF32, kRowsBf16, kTileF32, kTileBf16, kTileCodes };
struct ManyArgs {
    TileArgs job[IMUNPACK_BLOCK8_MANY];
    int kind[IMUNPACK_BLOCK8_MANY], end[IMUNPACK_BLOCK8_MANY];  // where the workgroups of a tensor end
};
template <int FORMAT>
__global__ __launch_bounds__(64 * kTileWaves) void block8_many_kernel(const ManyArgs a) {
    __shared__ TileShared shared;
    const int at = (int)blockIdx.x;
    int j = 0;
#pragma unroll
    for (int k = 0; k + 1 < IMUNPACK_BLOCK8_MANY; ++k) j += at >= a.end[k];
    const TileArgs &t = a.job[j];
    const int group = at - (j ? a.end[j - 1] : 0), kind = a.kind[j];
    if (kind <= kRowsBf16) {
        const RowsArgs r = {t.x, t.codes, t.scales, t.ldx, t.ldc, t.lds, (int)t.rows, t.cols, t.kb};
        if (kind == kRowsF32) rows_into<float, FORMAT, 4 * kTileWaves>(r, group);
        else rows_into<__bf16, FORMAT, 4 * kTileWaves>(r, group);
    } else if (kind == kTileF32) {
        tile_into<float, FORMAT>(t, (unsigned)group, shared);
    } else if (kind == kTileBf16) {
        tile_into<__bf16, FORMAT>(t, (unsigned)group, shared);
    } else {
        tile_into<uint8_t, FORMAT>(t, (unsigned)group, shared);
    }
}

// ---- values -------------------------------------------------------------------------------------------------------------------
struct ValuesArgs {
    const uint8_t *codes, *scales;
    void *out;
    int64_t ldc, lds, ldo;
    int rows, cols, kb;
};
template <class T, int FORMAT>
__global__ __launch_bounds__(256) void block8_values_kernel(const ValuesArgs a) {
    const int block = (int)blockIdx.x * 16 + (threadIdx.x >> 4);
    if (block >= a.rows * a.kb) return;
    const int row = block / a.kb, kb = block - row * a.kb, col = kb * kBlock8 + (threadIdx.x & 15) * 8;
    float f[8];
    decode8<FORMAT>(*reinterpret_cast<const uint2 *>(a.codes + row * a.ldc + col), block8_scale(a.scales[row * a.lds + kb]), f);
    if (col < a.cols) store_upto<T, 8>((T *)a.out + row * a.ldo + col, f, a.cols - col);
}

// ---- activation functions -------------------------------------------------------------------------------------------------------
// f(u) and f'(u).  GELU: u Phi(u), Phi + u phi; SiLU: u sig(u), sig (1 + u (1 - sig)).
// Phi(-x) = phi(x) R(x) for x >= 0 with Mills' ratio R = (1 - Phi) / phi, and 1 - that above 0: as (1 + erf) / 2 it cancels where u is negative (at -4 1e-3 of the value was wrong, at -6 nothing
// right, and a block of such inputs has a power of two of its own).  R(x) = t P(1 - t), t = 1 / (1 + 0.35 x), with the P of degree 8 whose largest relative error up to x = 14.5, where phi
// leaves binary32, is the least: 3.2e-8, in binary32 with its roundings 7 2^-24 (a P(t) 7.5, most of it where x is small).  phi's exponent leaves it off by u^2 2^-24 more; below 2^-126 it is 0.
// 4096 x 11008 bfloat16, forward and backward, gated 63 + 55 us, plain 41 + 41; by erff 62 + 67 and 44 + 55, by erfcf 83 + 95 and 63 + 82.
struct Normal {
    float below, density;  // Phi(u), phi(u)
};
__device__ __forceinline__ Normal normal_of(float u) {
    const float t = __builtin_amdgcn_rcpf(fmaf(0.35f, fabsf(u), 1.0f)), w = 1.0f - t, density = __builtin_amdgcn_exp2f(u * u * -0.72134752f) * 0.39894228f;
    float p = -0.073087960f;
    p = fmaf(p, w, 0.22367178f), p = fmaf(p, w, -0.16053279f), p = fmaf(p, w, -0.040340196f), p = fmaf(p, w, -0.16084722f), p = fmaf(p, w, 0.25727892f), p = fmaf(p, w, 0.65434307f);
    p = fmaf(p, w, -1.6038210f), p = fmaf(p, w, 1.2533141f);
    const float tail = density * (p * t);
    return {u < 0.0f ? tail : 1.0f - tail, density};
}
template <int ACT>
__device__ __forceinline__ float act_value(float u) {
    if constexpr (ACT == IMUNPACK_GELU) return u * normal_of(u).below;
    else return u / (1.0f + expf(-u));
}
template <int ACT>
__device__ __forceinline__ float act_slope(float u, float &value) {
    if constexpr (ACT == IMUNPACK_GELU) {
        const Normal n = normal_of(u);
        value = u * n.below;
        return fmaf(u, n.density, n.below);
    } else {
        const float sig = 1.0f / (1.0f + expf(-u));
        value = u * sig;
        return sig * fmaf(u, 1.0f - sig, 1.0f);
    }
}

struct ActArgs {
    const void *u;
    void *y;
    Blocks8 yq, kept, kept2;  // codes may be null
    int64_t ldu, ldy;
    int rows, cols, kb;
};
constexpr int kActBlocks = 2;  // blocks of 16 lanes, one after the other, all loads before the first is used
template <class T, int ACT, bool GATED, bool ONCE>
__global__ __launch_bounds__(256) void act8_kernel(const ActArgs a) {
    constexpr int F = IMUNPACK_E4M3;
    const int total = a.rows * a.kb, l16 = threadIdx.x & 15, first = (int)blockIdx.x * (16 * kActBlocks) + (threadIdx.x >> 4);
    piece_t<T, 8> in[kActBlocks], in2[kActBlocks];
    int rows[kActBlocks], kbs[kActBlocks];
#pragma unroll
    for (int v = 0; v < kActBlocks; ++v) {
        const int block = min(first + 16 * v, total - 1);
        rows[v] = block / a.kb;
        kbs[v] = block - rows[v] * a.kb;
        const int col = kbs[v] * kBlock8 + l16 * 8;
        const T *u = (const T *)a.u + rows[v] * a.ldu + col;
        in[v] = load_piece<T, 8, ONCE>(u, a.cols - col);
        if constexpr (GATED) in2[v] = load_piece<T, 8, ONCE>(u + a.cols, a.cols - col);
    }
#pragma unroll
    for (int v = 0; v < kActBlocks; ++v) {
        if (first + 16 * v >= total) return;
        const int row = rows[v], kb = kbs[v], col = kb * kBlock8 + l16 * 8, have = a.cols - col;
        float x[8], x2[8], y[8];
        to_floats<T, 8>(in[v], x);
        if constexpr (GATED) to_floats<T, 8>(in2[v], x2);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            y[k] = act_value<ACT>(x[k]);
            if constexpr (GATED) y[k] *= x2[k];
        }
        auto keep = [&](const Blocks8 &to, const float (&f)[8]) __attribute__((always_inline)) {
            const int byte = block8_of<F>(f);
            const uint2 w = encode8<F>(f, block8_inverse(byte));
            *reinterpret_cast<uint2 *>(to.codes + row * to.ldc + col) = w;
            if (l16 == 0) to.scales[row * to.lds + kb] = (uint8_t)byte;
            return make_uint3(w.x, w.y, (uint32_t)byte);
        };
        if (a.kept.codes) {
            keep(a.kept, x);
            if constexpr (GATED) keep(a.kept2, x2);
        }
        if (a.yq.codes) {
            const uint3 w = keep(a.yq, y);
            decode8<F>(make_uint2(w.x, w.y), block8_scale((int)w.z), y);
        }
        if (a.y && have > 0) store_upto<T, 8, ONCE>((T *)a.y + row * a.ldy + col, y, have);
    }
}

struct ActBackArgs {
    const void *g;
    void *gu;
    Blocks8 kept, kept2;
    int64_t ldg, ldgu;
    int rows, cols, kb;
};
template <class T, int ACT, bool GATED, bool ONCE>
__global__ __launch_bounds__(256) void act8_back_kernel(const ActBackArgs a) {
    constexpr int F = IMUNPACK_E4M3;
    const int total = a.rows * a.kb, l16 = threadIdx.x & 15, first = (int)blockIdx.x * (16 * kActBlocks) + (threadIdx.x >> 4);
    piece_t<T, 8> in[kActBlocks];
    uint2 codes[kActBlocks], codes2[kActBlocks];
    int rows[kActBlocks], kbs[kActBlocks], byte[kActBlocks], byte2[kActBlocks];
#pragma unroll
    for (int v = 0; v < kActBlocks; ++v) {
        const int block = min(first + 16 * v, total - 1);
        rows[v] = block / a.kb;
        kbs[v] = block - rows[v] * a.kb;
        const int row = rows[v], kb = kbs[v], col = kb * kBlock8 + l16 * 8;
        in[v] = load_piece<T, 8, ONCE>((const T *)a.g + row * a.ldg + col, a.cols - col);
        codes[v] = *reinterpret_cast<const uint2 *>(a.kept.codes + row * a.kept.ldc + col);
        byte[v] = a.kept.scales[row * a.kept.lds + kb];
        if constexpr (GATED) {
            codes2[v] = *reinterpret_cast<const uint2 *>(a.kept2.codes + row * a.kept2.ldc + col);
            byte2[v] = a.kept2.scales[row * a.kept2.lds + kb];
        }
    }
#pragma unroll
    for (int v = 0; v < kActBlocks; ++v) {
        if (first + 16 * v >= total) return;
        const int row = rows[v], col = kbs[v] * kBlock8 + l16 * 8, have = a.cols - col;
        float g[8], u[8], u2[8];
        decode8<F>(codes[v], block8_scale(byte[v]), u);
        if constexpr (GATED) decode8<F>(codes2[v], block8_scale(byte2[v]), u2);
        to_floats<T, 8>(in[v], g);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            float value;
            const float slope = act_slope<ACT>(u[k], value);
            if constexpr (GATED) {
                const float one = g[k] * slope * u2[k];
                u2[k] = g[k] * value;
                u[k] = one;
            } else {
                u[k] = g[k] * slope;
            }
        }
        if (have <= 0) continue;
        T *gu = (T *)a.gu + row * a.ldgu + col;
        store_upto<T, 8, ONCE>(gu, u, have);
        if constexpr (GATED) store_upto<T, 8, ONCE>(gu + a.cols, u2, have);
    }
}

// ---- entry points ---------------------------------------------------------------------------------------------------------------
static bool sizes_fit(int64_t rows, int64_t cols) { return rows >= 0 && rows <= kBlock8Rows && cols >= 1 && cols <= kBlock8Cols; }
static bool type_fits(int dtype) { return dtype == IMUNPACK_F32 || dtype == IMUNPACK_BF16; }
static bool format_fits(int format) { return format == IMUNPACK_E4M3 || format == IMUNPACK_E5M2; }
static int64_t element(int dtype) { return dtype == IMUNPACK_F32 ? 4 : 2; }
static int blocks_of(int64_t cols) { return (int)((cols + kBlock8 - 1) / kBlock8); }

constexpr int kManyGroups = 1 << 20;  // workgroups up to which several tensors share a launch

// launch(first row, rows) for pieces of the rows that a launch takes.
template <class L>
static int in_pieces(int64_t rows, int kb, int64_t whole, L launch) {
    const int64_t most = std::max<int64_t>(kLaunchBlocks / kb / whole * whole, whole);
    for (int64_t r = 0; r < rows; r += most) {
        launch(r, std::min(most, rows - r));
        IMU_TRY(launch_status());
    }
    return IMUNPACK_OK;
}
// f(float or __bf16, format) by what the call says.
template <class F>
static auto by_type(int dtype, int format, F f) {
    using E4 = std::integral_constant<int, IMUNPACK_E4M3>;
    using E5 = std::integral_constant<int, IMUNPACK_E5M2>;
    if (dtype == IMUNPACK_F32) return format == IMUNPACK_E4M3 ? f(0.0f, E4()) : f(0.0f, E5());
    return format == IMUNPACK_E4M3 ? f((__bf16)0.0f, E4()) : f((__bf16)0.0f, E5());
}

static int tiles(const TileArgs &whole, int dtype, int format, bool codes, hipStream_t st) {
    return in_pieces(whole.rows, whole.kb, 128, [&](int64_t r, int64_t n) {
        TileArgs a = whole;
        a.rows = n;
        a.x = (const char *)a.x + r * a.ldx * (codes ? 1 : element(dtype));
        if (a.xs) a.xs += r * a.ldxs;
        if (a.codes) a.codes += r * a.ldc, a.scales += r * a.lds;
        if (a.turned) a.turned += r, a.tscales += r / 128;
        const dim3 grid((unsigned)((n + 127) / 128 * a.kb));
        if (codes) {
            if (format == IMUNPACK_E4M3) hipLaunchKernelGGL((block8_tile_kernel<uint8_t, IMUNPACK_E4M3>), grid, dim3(64 * kTileWaves), 0, st, a);
            else hipLaunchKernelGGL((block8_tile_kernel<uint8_t, IMUNPACK_E5M2>), grid, dim3(64 * kTileWaves), 0, st, a);
        } else {
            by_type(dtype, format, [&](auto t, auto f) { hipLaunchKernelGGL((block8_tile_kernel<decltype(t), decltype(f)::value>), grid, dim3(64 * kTileWaves), 0, st, a); });
        }
    });
}
}  // namespace imu

using namespace imu;

extern "C" int imunpack_block8_quantize(const void *x, int64_t ldx, int64_t rows, int64_t cols, int dtype, int format, int square, void *codes, int64_t ldc, void *scales,
                                        int64_t lds, void *turned, int64_t ldt, void *turned_scales, int64_t ldts, imunpack_stream_t stream) {
    if (!sizes_fit(rows, cols) || !type_fits(dtype) || !format_fits(format) || ldx < cols) return IMUNPACK_EINVAL;
    if (turned && rows > kBlock8Cols) return IMUNPACK_EINVAL;
    if (rows == 0) return IMUNPACK_OK;
    const Blocks8 q = {(uint8_t *)codes, (uint8_t *)scales, ldc, lds}, t = {(uint8_t *)turned, (uint8_t *)turned_scales, ldt, ldts};
    if (!x || (!codes && !turned) || (codes && !blocks8_fit(q, cols)) || (turned && !blocks8_fit(t, rows))) return IMUNPACK_EINVAL;
    const hipStream_t st = (hipStream_t)stream;
    const int kb = blocks_of(cols);
    if (turned || square) return tiles({x, nullptr, q.codes, q.scales, t.codes, t.scales, ldx, 0, ldc, lds, ldt, ldts, rows, (int)cols, kb, square}, dtype, format, false, st);
    return in_pieces(rows, kb, 1, [&](int64_t r, int64_t n) {
        const RowsArgs a = {(const char *)x + r * ldx * element(dtype), q.codes + r * ldc, q.scales + r * lds, ldx, ldc, lds, (int)n, (int)cols, kb};
        const dim3 grid((unsigned)((n * kb + 16 * kRowsUnroll - 1) / (16 * kRowsUnroll)));
        by_type(dtype, format, [&](auto e, auto f) { hipLaunchKernelGGL((block8_rows_kernel<decltype(e), decltype(f)::value>), grid, dim3(256), 0, st, a); });
    });
}

extern "C" int imunpack_block8_turn(const void *codes, int64_t ldc, const void *scales, int64_t lds, int64_t rows, int64_t cols, int format, void *turned, int64_t ldt,
                                    void *turned_scales, int64_t ldts, imunpack_stream_t stream) {
    if (!sizes_fit(rows, cols) || rows > kBlock8Cols || !format_fits(format)) return IMUNPACK_EINVAL;
    if (rows == 0) return IMUNPACK_OK;
    const Blocks8 q = {(uint8_t *)codes, (uint8_t *)scales, ldc, lds}, t = {(uint8_t *)turned, (uint8_t *)turned_scales, ldt, ldts};
    if (!blocks8_fit(q, cols) || !blocks8_fit(t, rows)) return IMUNPACK_EINVAL;
    return tiles({q.codes, q.scales, nullptr, nullptr, t.codes, t.scales, ldc, lds, 0, 0, ldt, ldts, rows, (int)cols, blocks_of(cols), 0}, IMUNPACK_F32, format, true,
                 (hipStream_t)stream);
}

extern "C" int imunpack_block8_many(int count, const imunpack_block8_job *jobs, int format, imunpack_stream_t stream) {
    if (count < 1 || count > IMUNPACK_BLOCK8_MANY || !jobs || !format_fits(format)) return IMUNPACK_EINVAL;
    ManyArgs a = {};
    int64_t groups = 0;
    int kinds = 0;
    for (int k = 0; k < count; ++k) {  // (all of them before anything is launched)
        const imunpack_block8_job &j = jobs[k];
        const Blocks8 q = {(uint8_t *)j.codes, (uint8_t *)j.scales, j.ldc, j.lds}, t = {(uint8_t *)j.turned, (uint8_t *)j.turned_scales, j.ldt, j.ldts};
        const bool codes = j.x_scales != nullptr;
        if (!sizes_fit(j.rows, j.cols) || (!codes && (!type_fits(j.dtype) || j.ldx < j.cols)) || (t.codes && j.rows > kBlock8Cols)) return IMUNPACK_EINVAL;
        if (codes && (q.codes || !t.codes || j.square)) return IMUNPACK_EINVAL;
        if (j.rows == 0) continue;
        if (!j.x || (!q.codes && !t.codes) || (q.codes && !blocks8_fit(q, j.cols)) || (t.codes && !blocks8_fit(t, j.rows))) return IMUNPACK_EINVAL;
        if (codes && !blocks8_fit({(uint8_t *)j.x, (uint8_t *)j.x_scales, j.ldx, j.ldxs}, j.cols)) return IMUNPACK_EINVAL;
        const int kb = blocks_of(j.cols);
        const bool rows = !codes && !t.codes && !j.square;
        groups += rows ? (j.rows * kb + 4 * kTileWaves * kRowsUnroll - 1) / (4 * kTileWaves * kRowsUnroll) : (j.rows + 127) / 128 * kb;
        if (j.rows * kb > kLaunchBlocks) groups = kLaunchBlocks;  // (more than one launch takes)
        groups = std::min<int64_t>(groups, kLaunchBlocks);
        a.job[kinds] = {j.x, (const uint8_t *)j.x_scales, q.codes, q.scales, t.codes, t.scales, j.ldx, j.ldxs, j.ldc, j.lds, j.ldt, j.ldts, j.rows, (int)j.cols, kb, j.square};
        a.kind[kinds] = codes ? kTileCodes : (rows ? kRowsF32 : kTileF32) + (j.dtype == IMUNPACK_F32 ? 0 : 1);
        a.end[kinds++] = (int)groups;
    }
    if (kinds == 0) return IMUNPACK_OK;
    if (kinds == 1 || groups > kManyGroups) {
        for (int k = 0; k < count; ++k) {
            const imunpack_block8_job &j = jobs[k];
            if (j.x_scales) IMU_TRY(imunpack_block8_turn(j.x, j.ldx, j.x_scales, j.ldxs, j.rows, j.cols, format, j.turned, j.ldt, j.turned_scales, j.ldts, stream));
            else IMU_TRY(imunpack_block8_quantize(j.x, j.ldx, j.rows, j.cols, j.dtype, format, j.square, j.codes, j.ldc, j.scales, j.lds, j.turned, j.ldt, j.turned_scales, j.ldts, stream));
        }
        return IMUNPACK_OK;
    }
    for (int k = kinds; k < IMUNPACK_BLOCK8_MANY; ++k) a.end[k] = (int)groups;
    if (format == IMUNPACK_E4M3) hipLaunchKernelGGL(block8_many_kernel<IMUNPACK_E4M3>, dim3((unsigned)groups), dim3(64 * kTileWaves), 0, (hipStream_t)stream, a);
    else hipLaunchKernelGGL(block8_many_kernel<IMUNPACK_E5M2>, dim3((unsigned)groups), dim3(64 * kTileWaves), 0, (hipStream_t)stream, a);
    return launch_status();
}

extern "C" int imunpack_block8_values(const void *codes, int64_t ldc, const void *scales, int64_t lds, int64_t rows, int64_t cols, int format, void *out, int64_t ldo, int dtype,
                                      imunpack_stream_t stream) {
    if (!sizes_fit(rows, cols) || !type_fits(dtype) || !format_fits(format) || ldo < cols) return IMUNPACK_EINVAL;
    if (rows == 0) return IMUNPACK_OK;
    const Blocks8 q = {(uint8_t *)codes, (uint8_t *)scales, ldc, lds};
    if (!out || !blocks8_fit(q, cols)) return IMUNPACK_EINVAL;
    const int kb = blocks_of(cols);
    return in_pieces(rows, kb, 1, [&](int64_t r, int64_t n) {
        const ValuesArgs a = {q.codes + r * ldc, q.scales + r * lds, (char *)out + r * ldo * element(dtype), ldc, lds, ldo, (int)n, (int)cols, kb};
        const dim3 grid((unsigned)((n * kb + 15) / 16));
        by_type(dtype, format, [&](auto e, auto f) { hipLaunchKernelGGL((block8_values_kernel<decltype(e), decltype(f)::value>), grid, dim3(256), 0, (hipStream_t)stream, a); });
    });
}

// f(float or __bf16, function, gated or not) by what the call says.
template <class F>
static void by_act(int dtype, int act, int gated, F f) {
    auto typed = [&](auto t) {
        using G = std::integral_constant<int, IMUNPACK_GELU>;
        using S = std::integral_constant<int, IMUNPACK_SILU>;
        if (act == IMUNPACK_GELU) gated ? f(t, G(), std::true_type()) : f(t, G(), std::false_type());
        else gated ? f(t, S(), std::true_type()) : f(t, S(), std::false_type());
    };
    if (dtype == IMUNPACK_F32) typed(0.0f);
    else typed((__bf16)0.0f);
}
static bool act_fits(int64_t rows, int64_t cols, int dtype, int act) {
    return sizes_fit(rows, cols) && type_fits(dtype) && (act == IMUNPACK_GELU || act == IMUNPACK_SILU);
}

extern "C" int imunpack_act8(const void *u, int64_t ldu, int64_t rows, int64_t cols, int dtype, int act, int gated, void *y, int64_t ldy, void *y_codes, int64_t ldyc,
                             void *y_scales, int64_t ldys, void *kept, void *kept2, int64_t ldk, void *kept_scales, void *kept2_scales, int64_t ldks, imunpack_stream_t stream) {
    if (!act_fits(rows, cols, dtype, act) || ldu < cols * (gated ? 2 : 1) || (y && ldy < cols)) return IMUNPACK_EINVAL;
    if (rows == 0) return IMUNPACK_OK;
    const Blocks8 q = {(uint8_t *)y_codes, (uint8_t *)y_scales, ldyc, ldys}, k = {(uint8_t *)kept, (uint8_t *)kept_scales, ldk, ldks},
                  k2 = {(uint8_t *)kept2, (uint8_t *)kept2_scales, ldk, ldks};
    if (!u || (!y && !y_codes) || (y_codes && !blocks8_fit(q, cols)) || (kept && !blocks8_fit(k, cols)) || (kept && gated && !blocks8_fit(k2, cols))) return IMUNPACK_EINVAL;
    const int kb = blocks_of(cols);
    const bool once = rows * cols * element(dtype) * (gated ? 3 : 2) >= kLastLevelCache;  // u, y and what is kept, or their gradients
    auto from = [](Blocks8 t, int64_t r) { return t.codes ? Blocks8{t.codes + r * t.ldc, t.scales + r * t.lds, t.ldc, t.lds} : t; };
    return in_pieces(rows, kb, 1, [&](int64_t r, int64_t n) {
        const int64_t size = element(dtype);
        const ActArgs a = {(const char *)u + r * ldu * size, y ? (char *)y + r * ldy * size : nullptr, from(q, r), from(k, r), from(k2, r), ldu, ldy, (int)n, (int)cols, kb};
        const dim3 grid((unsigned)((n * kb + 16 * kActBlocks - 1) / (16 * kActBlocks)));
        by_act(dtype, act, gated, [&](auto t, auto f, auto g) {
            using T = decltype(t);
            constexpr int A = decltype(f)::value;
            constexpr bool G = decltype(g)::value;
            hipLaunchKernelGGL((once ? act8_kernel<T, A, G, true> : act8_kernel<T, A, G, false>), grid, dim3(256), 0, (hipStream_t)stream, a);
        });
    });
}

extern "C" int imunpack_act8_backward(const void *g, int64_t ldg, int64_t rows, int64_t cols, int dtype, int act, int gated, const void *kept, const void *kept2, int64_t ldk,
                                      const void *kept_scales, const void *kept2_scales, int64_t ldks, void *gu, int64_t ldgu, imunpack_stream_t stream) {
    if (!act_fits(rows, cols, dtype, act) || ldg < cols || ldgu < cols * (gated ? 2 : 1)) return IMUNPACK_EINVAL;
    if (rows == 0) return IMUNPACK_OK;
    const Blocks8 k = {(uint8_t *)kept, (uint8_t *)kept_scales, ldk, ldks}, k2 = {(uint8_t *)kept2, (uint8_t *)kept2_scales, ldk, ldks};
    if (!g || !gu || !blocks8_fit(k, cols) || (gated && !blocks8_fit(k2, cols))) return IMUNPACK_EINVAL;
    const int kb = blocks_of(cols);
    const bool once = rows * cols * element(dtype) * (gated ? 3 : 2) >= kLastLevelCache;  // u, y and what is kept, or their gradients
    auto from = [](Blocks8 t, int64_t r) { return t.codes ? Blocks8{t.codes + r * t.ldc, t.scales + r * t.lds, t.ldc, t.lds} : t; };
    return in_pieces(rows, kb, 1, [&](int64_t r, int64_t n) {
        const int64_t size = element(dtype);
        const ActBackArgs a = {(const char *)g + r * ldg * size, (char *)gu + r * ldgu * size, from(k, r), from(k2, r), ldg, ldgu, (int)n, (int)cols, kb};
        const dim3 grid((unsigned)((n * kb + 16 * kActBlocks - 1) / (16 * kActBlocks)));
        by_act(dtype, act, gated, [&](auto t, auto f, auto gt) {
            using T = decltype(t);
            constexpr int A = decltype(f)::value;
            constexpr bool G = decltype(gt)::value;
            hipLaunchKernelGGL((once ? act8_back_kernel<T, A, G, true> : act8_back_kernel<T, A, G, false>), grid, dim3(256), 0, (hipStream_t)stream, a);
        });
    });
}
