// Product of two 16-bit operands, C = A B^T, accumulated in binary32 on v_mfma_f32_32x32x16: the loop that the
// loss over a vocabulary is made of.  Tiles of (64 TM) x (64 TN), 2 x 2 waves of (32 TM) x (32 TN) each.
//
// Either operand may lie with the contraction contiguous (a row of memory is a row of the operand) or across (a row of memory is one
// place of the contraction, the operand's rows side by side): in the second case the fragments come out of LDS through ds_read_b64_tr_b16, whose
// sixteen lanes read four rows of sixteen elements and get a column of four each.  So no operand is ever transposed in memory.
//
// The walk over the contraction is that of the int8 GEMM, whose fragments have the same bytes: k-tiles of 64 places (128 bytes of a row, or 64
// rows), loaded straight into LDS, a ring of five half-stages (A and B of a k-tile in slots of their own), one barrier to a k-tile, loads two
// k-tiles ahead (four, where a product has so few tiles that a CU has a small one to itself, took as long: 100 x 1024 by 4000 fp32 62 us).
// 16-byte piece c of row r lies at slot c ^ ((r >> 1) & 7) of the row (contraction contiguous: the 32 rows of a fragment fall on different banks)
// or c ^ ((r & 3) << 2) (across: the four rows of a read do).
//
// binary32 values are held as sums of two binary16 numbers, A = A_0 + A_1 and B = B_0 + B_1: three products, A_1 B_0, A_0 B_1 and A_0 B_0
// (A_1 B_1 lies below the last bit), the small ones first.  A row of memory then holds 32 first numbers, the 32 second ones that go with them, and so
// on, so that all of the above stays as it is: a k-tile is 32 places with both numbers of each, and a k-step is three products of its fragments.
#pragma once
#include "common.h"

#include <type_traits>

namespace imu {
#if defined(__HIPCC__)
typedef float v16f32 __attribute__((ext_vector_type(16)));
typedef _Float16 v8f16 __attribute__((ext_vector_type(8)));
typedef __bf16 v8bf16 __attribute__((ext_vector_type(8)));
typedef int v4i32 __attribute__((ext_vector_type(4)));
typedef int v2i32 __attribute__((ext_vector_type(2)));
typedef short v4i16 __attribute__((ext_vector_type(4)));

constexpr int kStageBytes = 128;   // of a row and k-tile
constexpr int kStageCols = 64;     // 16-bit elements of it
template <bool F16>
constexpr int kPlaces = F16 ? 32 : 64;  // places of the contraction in a k-tile
constexpr int kProductThreads = 256;
constexpr int kRing = 5;           // slots
constexpr int product_lds(int tm, int tn) { return kRing * 64 * (tm > tn ? tm : tn) * kStageBytes; }

// One operand: rows of memory of 16-bit elements, `pitch` bytes apart (a multiple of 16, as is the base).  Rows from `rows` on are not read, nor
// pieces of 16 bytes that hold nothing of the first `cols` elements of a row: the last one is, in their place.  (Where that is along the
// contraction, the other operand has zeros there.)
struct Operand {
    const char *base;
    int64_t pitch;
    int rows, cols;
};

template <bool F16>
__device__ __forceinline__ void mfma16(const v4i32 &a, const v4i32 &b, v16f32 &c) {
    if constexpr (F16) c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8f16, a), __builtin_bit_cast(v8f16, b), c, 0, 0, 0);
    else c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8bf16, a), __builtin_bit_cast(v8bf16, b), c, 0, 0, 0);
}

// Every lane fetches 16 bytes from base + off; the wave's kilobyte lands at LDS byte `lds` (lane l at lds + 16 l).
__device__ __forceinline__ void fetch_to_lds(unsigned lds, unsigned off, const char *base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ const char *uniform_address(const char *p) {
    const uint64_t v = (uint64_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);  // (unsigned: the builtin's int would be extended by its sign)
    const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
    return (const char *)(((uint64_t)hi << 32) | lo);
}

// XCD-aware order of tiles: workgroups are dealt to the 8 XCDs in turn, those of an XCD get consecutive tiles, which walk bands of
// four tile rows so that an XCD's workgroups share operands in its L2.
__device__ __forceinline__ void tile_at(int wg, int mtiles, int ntiles, int &tm, int &tn) {
    const int total = mtiles * ntiles, xcd = wg & 7, idx = wg >> 3, per = total >> 3, rem = total & 7;
    const int at = xcd * per + min(xcd, rem) + idx, size = 4 * ntiles, band = at / size, first = band * 4;
    const int rows = min(4, mtiles - first), in = at - band * size;
    tm = first + in % rows;
    tn = in / rows;
}

// acc[i][j] of the wave: register r of lane l is the sum at row 32 i + (r / 4) * 8 + (l / 32) * 4 + r % 4 and column 32 j + l % 32 of the
// wave's part of the tile.  k-tiles [k0, k1) of the contraction.  XA, XB: the operand lies across.
template <bool F16, int TM, int TN, bool XA, bool XB>
__device__ __forceinline__ void product_tile(const Operand &A, const Operand &B, int m0, int n0, int k0, int k1, char *smem, v16f32 (&acc)[TM][TN]) {
    constexpr int N = F16 ? 2 : 1, R = kPlaces<F16>, kSteps = R / 16;  // numbers of a value; places and k-steps of a k-tile
    constexpr int kSlot = 64 * (TM > TN ? TM : TN) * kStageBytes;  // bytes of a slot of the ring
    constexpr int LA = 2 * TM, LB = 2 * TN;                        // loads of a wave for its share of a half-stage: 16 TM (16 TN) rows
    constexpr int NF = N * (TM + TN), NM = TM * TN * (F16 ? 3 : 1);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    const int total = k1 - k0;
    if (total <= 0) return;
    const unsigned lds0 = (unsigned)(size_t)smem;
    // what lane l of the wave fetches with its load u: contiguous, eight rows of 128 bytes; across, 1 KiB / (128 N T) rows
    unsigned offA[LA], offB[LB], colA[4], colB[4];  // by row and, the same for every fourth load, within it
    auto offsets = [&](auto &off, auto &col, auto across, auto t, const Operand &op, int first) __attribute__((always_inline)) {
        constexpr int T = decltype(t)::value, L = 2 * T, kPieces = 8 * N * T, kRows = 64 / kPieces;  // pieces of a row of memory, rows to a load
#pragma unroll
        for (int u = 0; u < L; ++u) {
            if constexpr (decltype(across)::value) {
                const int row = R / 4 * wave + kRows * u + lane / kPieces;
                off[u] = (unsigned)(row * op.pitch);
                if (u < 4) col[u] = (unsigned)(min((lane % kPieces) ^ ((row & 3) << 2), (op.cols * 2 - 1) / 16 - first * N / 8) * 16);
            } else {
                const int row = 16 * T * wave + 8 * u + (lane >> 3);
                off[u] = (unsigned)(min(row, op.rows - 1 - first) * op.pitch);
                if (u < 4) col[u] = (unsigned)(((lane & 7) ^ ((row >> 1) & 7)) * 16);
            }
        }
    };
    offsets(offA, colA, std::bool_constant<XA>(), std::integral_constant<int, TM>(), A, m0);
    offsets(offB, colB, std::bool_constant<XB>(), std::integral_constant<int, TN>(), B, n0);
    const int64_t stepA = XA ? R * A.pitch : kStageBytes, stepB = XB ? R * B.pitch : kStageBytes;
    const char *gA = A.base + (XA ? m0 * 2 * N : m0 * A.pitch) + k0 * stepA, *gB = B.base + (XB ? n0 * 2 * N : n0 * B.pitch) + k0 * stepB;
    auto ring = [](int slot, int k) { slot += k; return slot >= kRing ? slot - kRing : slot; };
    const char *pg = nullptr;
    unsigned dl = 0, last = 0;
    // k-tile kt (past the last one it is loaded again, into a slot that is not read) of A or B into a slot
    auto setup = [&](bool isA, int kt, int slot) {
        const int k = min(kt, total - 1);
        pg = uniform_address((isA ? gA : gB) + k * (isA ? stepA : stepB));
        const Operand &op = isA ? A : B;
        if (isA ? XA : XB) last = __builtin_amdgcn_readfirstlane((unsigned)(min(op.rows - 1 - (k0 + k) * R, R) * op.pitch));
        else last = __builtin_amdgcn_readfirstlane((unsigned)(min((op.cols * 2 - 1) / 16 - (k0 + k) * 8, 7) * 16));
        dl = __builtin_amdgcn_readfirstlane(lds0 + (unsigned)(slot * kSlot) + (unsigned)(wave * (isA ? LA : LB) * 1024));
    };
    auto fetch = [&](bool isA, int u) __attribute__((always_inline)) {
        const unsigned row = isA ? offA[u] : offB[u], col = isA ? colA[u & 3] : colB[u & 3];
        fetch_to_lds(dl + u * 1024, (isA ? XA : XB) ? min(row, last) + col : row + min(col, last), pg);
    };

    const int lrow = lane & 31, lhalf = lane >> 5, swz = (lrow >> 1) & 7;
    const unsigned baseA = (unsigned)((wm * 32 * TM + lrow) * kStageBytes), baseB = (unsigned)((wn * 32 * TN + lrow) * kStageBytes);
    unsigned piece[4];
#pragma unroll
    for (int ks = 0; ks < 4; ++ks) piece[ks] = (unsigned)(((2 * ks + lhalf) ^ swz) << 4);
    v4i32 fa[2][N][TM], fb[2][N][TN];
    // across: the lane's row of four and its 8 bytes within a block of 32 columns; blocks trade places by the row
    const int xrow = (lane >> 2) & 3, xlane = ((lane >> 5) * 8 + xrow), xcol = ((lane >> 4) & 1) * 32 + (lane & 3) * 8;
    unsigned acrossA[TM], acrossB[TN];
    if constexpr (XA)
#pragma unroll
        for (int i = 0; i < TM; ++i) acrossA[i] = (unsigned)(xlane * 128 * N * TM + ((N * (wm * TM + i)) ^ xrow) * 64 + xcol);
    if constexpr (XB)
#pragma unroll
        for (int j = 0; j < TN; ++j) acrossB[j] = (unsigned)(xlane * 128 * N * TN + ((N * (wn * TN + j)) ^ xrow) * 64 + xcol);
    auto turned = [&](const char *p, int ks, int row) __attribute__((always_inline)) {  // places 16 ks + 0 .. 7 (8 .. 15) of the lane's row of the operand
        const v2i32 lo = __builtin_bit_cast(v2i32, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16 *)(p + ks * 16 * row)));
        const v2i32 hi = __builtin_bit_cast(v2i32, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4i16 *)(p + (ks * 16 + 4) * row)));
        return v4i32{lo[0], lo[1], hi[0], hi[1]};
    };
    // fragment q of a k-step, in the order in which the products need them (of pairs: A_1 and B_0, then A_0 and B_1)
    auto fragment = [&](const char *sa, const char *sb, int ks, int buf, int q) __attribute__((always_inline)) {
        constexpr int isA4[8] = {1, 0, 0, 1, 0, 0, 1, 1}, idx4[8] = {0, 0, 1, 1, 2, 3, 2, 3};
        const int at = q % (TM + TN), later = q / (TM + TN);
        const bool isA = (TM == 4 && TN == 4) ? isA4[at] : at == 0 || at > TN;
        const int idx = (TM == 4 && TN == 4) ? idx4[at] : at == 0 ? 0 : at > TN ? at - TN : at - 1;
        const int n = N == 2 && later != isA;  // which number
        if (isA) {
            if constexpr (XA) fa[buf][n][idx] = turned(sa + (acrossA[idx] ^ (n * 64)), ks, 128 * N * TM);
            else fa[buf][n][idx] = *reinterpret_cast<const v4i32 *>(sa + baseA + idx * 32 * kStageBytes + piece[n * kSteps + ks]);
        } else {
            if constexpr (XB) fb[buf][n][idx] = turned(sb + (acrossB[idx] ^ (n * 64)), ks, 128 * N * TN);
            else fb[buf][n][idx] = *reinterpret_cast<const v4i32 *>(sb + baseB + idx * 32 * kStageBytes + piece[n * kSteps + ks]);
        }
    };
    auto multiply = [&](int buf, int m) __attribute__((always_inline)) {
        constexpr int mi4[16] = {0, 0, 1, 1, 0, 0, 1, 1, 2, 2, 3, 3, 2, 2, 3, 3}, mj4[16] = {0, 1, 0, 1, 2, 3, 2, 3, 0, 1, 0, 1, 2, 3, 2, 3};
        const int product = m / (TM * TN), at = m % (TM * TN);
        const int i = (TM == 4 && TN == 4) ? mi4[at] : at / TN, j = (TM == 4 && TN == 4) ? mj4[at] : at % TN;
        mfma16<F16>(fa[buf][N == 2 && product == 0][i], fb[buf][N == 2 && product == 1][j], acc[i][j]);
    };
    // the products of a k-step, the fragments of the next one and `count` loads from number `from` on among them
    auto step = [&](int cur, const char *sa, const char *sb, int next_ks, bool isA, int from, int count) {
#pragma unroll
        for (int q = 0; q < NF; ++q) {
            fragment(sa, sb, next_ks, cur ^ 1, q);
#pragma unroll
            for (int m = q * NM / NF; m < (q + 1) * NM / NF; ++m) {
                multiply(cur, m);
                if (m == q * NM / NF && q < count) fetch(isA, from + q);
            }
            if (NM < NF && q * NM / NF == (q + 1) * NM / NF && q < count) fetch(isA, from + q);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // k-tile 0 landed, the next ones on their way
#pragma unroll
    for (int p = 0; p < 2; ++p) {
        setup(true, p, 2 * p);
#pragma unroll
        for (int u = 0; u < LA; ++u) fetch(true, u);
        setup(false, p, 2 * p + 1);
#pragma unroll
        for (int u = 0; u < LB; ++u) fetch(false, u);
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"i"(LA + LB) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
#pragma unroll
    for (int q = 0; q < NF; ++q) fragment(smem, smem + kSlot, 0, 0, q);
    // The steps before the last load A(kt + 2) into the slot that is free.  Behind them every fragment of k-tile kt has been read and this
    // wave's parts of k-tile kt + 1 have landed (all but the newest loads); past the barrier that holds for all waves, so that the last step may read
    // k-tile kt + 1 and load B(kt + 2) into the slot of A(kt).
    constexpr int c0 = (LA + 2) / 3, c1 = (LA - c0 + 1) / 2, c2 = LA - c0 - c1;
    int sa = 0;
    for (int kt = 0; kt < total; ++kt) {
        const char *stA = smem + sa * kSlot, *stB = smem + ring(sa, 1) * kSlot;
        const char *stA1 = smem + ring(sa, 2) * kSlot, *stB1 = smem + ring(sa, 3) * kSlot;
        setup(true, kt + 2, ring(sa, 4));
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (F16) {
            step(0, stA, stB, 1, true, 0, LA);
        } else {
            step(0, stA, stB, 1, true, 0, c0);
            step(1, stA, stB, 2, true, c0, c1);
            step(0, stA, stB, 3, true, c0 + c1, c2);
        }
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"(LA) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        setup(false, kt + 2, sa);
        __builtin_amdgcn_sched_barrier(0);
        step(1, stA1, stB1, 0, false, 0, LB);
        sa = ring(sa, 2);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing may land in LDS any more
    __syncthreads();
}
#endif
}  // namespace imu
