// Product of two tensors in 8-bit floating point with a power of two per row and block of 128 places of the contraction (block8.h):
//
//   out[m, n] = sum_k value_A[m, k] value_B[n, k] + bias[n]
//
// bfloat16 results: codes and powers of two as the scaled 8-bit matrix instruction takes them.  fp32 results: the codes with their power of two are numbers of bfloat16 (but at the ends of its
// range, which `Ends` watches for), so that products on its matrix instruction are exact and sums binary32's.
#include "block8.h"
#include "product.h"

#include <algorithm>
#include <atomic>

namespace imu {
typedef __bf16 v2bf16 __attribute__((ext_vector_type(2)));
typedef int v8i32 __attribute__((ext_vector_type(8)));

struct GemmArgs {
    const uint8_t *a, *sa, *b, *sb;
    const float *bias;  // may be null
    void *out;
    int64_t lda, ldsa, ldb, ldsb, ldo;
    int m, n, kt;       // kt: blocks of the contraction
    int mtiles, ntiles;
    int parts, per;     // of the contraction, blocks of each; with several, `out` is the workspace: fp32, m x n for each
};

// Eight codes times their power of two as bfloat16 (exact where the byte lies within Span).
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

// Bytes whose codes times their power of two are all numbers of bfloat16 (2^-133 to below 2^128, subnormals among them, which the instruction takes as they are): from `low` to `high`.
// What is lost of an operand below that is at most 2^-134, which counts (2^-126 and more in a product) only beside one that may reach 2^8, whose byte is `weighty` or above.
template <int FORMAT>
struct Span {
    static constexpr int low = FORMAT == IMUNPACK_E4M3 ? 3 : 10, high = FORMAT == IMUNPACK_E4M3 ? 246 : 239, weighty = FORMAT == IMUNPACK_E4M3 ? 127 : 120;
};
// What a lane has seen of its rows' bytes beyond the span: top bits of `odd`, four bytes at a time (x - n borrows from a byte's top bit).  Five operations for four blocks of a row; whether the
// products are wrong for it is found out behind the walk, by `counts`.
struct Ends {
    unsigned odd = 0;
    template <int FORMAT>
    __device__ __forceinline__ void look(unsigned w) {
        odd |= (w - Span<FORMAT>::low * 0x01010101u) & ~w;
        odd |= (Span<FORMAT>::high * 0x01010101u - w) & w;
    }
    __device__ __forceinline__ bool any() const { return __builtin_amdgcn_ballot_w64((odd & 0x80808080u) != 0) != 0; }  // in the wave
};
// Whether what a wave's products have lost counts: from the bytes of its 32 TM rows of A and 32 TN of B.
template <int FA, int FB, int TM, int TN>
__device__ __forceinline__ bool counts(const uint8_t *sa, const uint8_t *sb, const unsigned (&rowA)[TM], const unsigned (&rowB)[TN], int total) {
    int lowA = 255, lowB = 255, highA = 0, highB = 0;
#pragma unroll 1
    for (int kt = 0; kt < total; ++kt) {
#pragma unroll
        for (int i = 0; i < TM; ++i) lowA = min(lowA, (int)sa[rowA[i] + kt]), highA = max(highA, (int)sa[rowA[i] + kt]);
#pragma unroll
        for (int j = 0; j < TN; ++j) lowB = min(lowB, (int)sb[rowB[j] + kt]), highB = max(highB, (int)sb[rowB[j] + kt]);
    }
    auto some = [](bool x) { return __builtin_amdgcn_ballot_w64(x) != 0; };
    return some(highA > Span<FA>::high || highB > Span<FB>::high) || (some(lowA < Span<FA>::low) && some(highB >= Span<FB>::weighty)) ||
           (some(lowB < Span<FB>::low) && some(highA >= Span<FA>::weighty));
}

// ---- large products: tiles of (64 TM) x (64 TN), 2 x 2 waves of (32 TM) x (32 TN) -------------------------------------------------
// The walk over the contraction is that of product.h, whose k-tiles of 128 bytes are blocks of 128 places here: loads straight into LDS, a ring of five
// half-stages (A and B of a k-tile in slots of their own), one barrier to a k-tile, loads two k-tiles ahead; 16-byte piece c of row r at slot c ^ ((r >> 1) & 7).
// 8192^3: 381 us (2.9 PFLOP/s; a library product in 8 bits 2.8) and for fp32 results 765 (1.4; a library product in bfloat16 1.3), 4096^3 54 and 110: filling and emptying the one
// tile of a CU takes 11 us, a block 1.4.
// Powers of two are bytes beside the codes: a lane holds those of its rows for 4 G k-tiles, loaded ahead.
//
// NATIVE: v_mfma_scale_f32_32x32x64_f8f6f4, which takes codes and bytes as they are.  It adds eight products at a time and cuts each of them below 2^-13 of the
// largest's power of two, so that a result of random operands is off by 1.5e-5 of its size: a hundredth of what rounding it to bfloat16 leaves, too much for fp32.
// Otherwise codes become bfloat16 numbers times their power of two between LDS and the matrix instruction (exact), at half the rate.
// Returns whether the wave's results are right as they are (NATIVE: always).
template <bool NATIVE, int FA, int FB, int TM, int TN, int G>
__device__ __forceinline__ bool product8_tile(const GemmArgs &g, int m0, int n0, int k0, int k1, char *smem, v16f32 (&acc)[TM][TN]) {
    constexpr int kSlot = 64 * (TM > TN ? TM : TN) * kStageBytes, LA = 2 * TM, LB = 2 * TN, NF = TM + TN, NM = TM * TN, kSteps = NATIVE ? 2 : 4;
    constexpr bool kFour = TM == 4 && TN == 4;
    typedef int wide_t __attribute__((ext_vector_type(G)));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.0f;
    const int total = k1 - k0, lrow = lane & 31, lhalf = lane >> 5;
    const unsigned lds0 = (unsigned)(size_t)smem;
    // where the lane's part of load 0 lies; load u is 8 u rows on, the last row at most (offsets stay below 2^32: a pitch is 2^24 at most)
    const unsigned offA = (unsigned)(16 * TM * wave + (lane >> 3)) * (unsigned)g.lda, offB = (unsigned)(16 * TN * wave + (lane >> 3)) * (unsigned)g.ldb;
    const unsigned lastA = (unsigned)(min(g.m - 1 - m0, 64 * TM - 1)) * (unsigned)g.lda, lastB = (unsigned)(min(g.n - 1 - n0, 64 * TN - 1)) * (unsigned)g.ldb;
    unsigned col[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) col[u] = (unsigned)(((lane & 7) ^ (((8 * u + (lane >> 3)) >> 1) & 7)) * 16);  // (rows 16 apart have the same)
    const char *gA = (const char *)g.a + m0 * g.lda + k0 * 128, *gB = (const char *)g.b + n0 * g.ldb + k0 * 128;
    // the bytes of the lane's rows
    const uint8_t *tileA = g.sa + m0 * g.ldsa + k0, *tileB = g.sb + n0 * g.ldsb + k0;
    unsigned rowA[TM], rowB[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) rowA[i] = (unsigned)min(32 * (TM * wm + i) + lrow, g.m - 1 - m0) * (unsigned)g.ldsa;
#pragma unroll
    for (int j = 0; j < TN; ++j) rowB[j] = (unsigned)min(32 * (TN * wn + j) + lrow, g.n - 1 - n0) * (unsigned)g.ldsb;
    wide_t nextA[TM], nextB[TN];
    int sA[TM], sB[TN];
    auto shift = [](wide_t &w) __attribute__((always_inline)) {
        const int x = w[0];
#pragma unroll
        for (int d = 1; d < G; ++d) w[d - 1] = w[d];
        return x;
    };
    auto load_bytes = [&](int kt) __attribute__((always_inline)) {
        const int at = min(kt, (total - 1) / (4 * G) * (4 * G));
        const char *pA = uniform_address((const char *)tileA + at), *pB = uniform_address((const char *)tileB + at);
        // (the row's offset is made opaque here: widened to 64 bits outside the loop it took two registers and an addition)
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            unsigned r = rowA[i];
            asm volatile("" : "+v"(r));
            nextA[i] = *(const __attribute__((address_space(1))) wide_t *)(pA + r);
        }
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            unsigned r = rowB[j];
            asm volatile("" : "+v"(r));
            nextB[j] = *(const __attribute__((address_space(1))) wide_t *)(pB + r);
        }
    };
    load_bytes(0);

    auto ring = [](int slot, int k) { slot += k; return slot >= kRing ? slot - kRing : slot; };
    const char *pg = nullptr;
    unsigned dl = 0;
    auto setup = [&](bool isA, int kt, int slot) {  // (past the last k-tile it is loaded again, into a slot that is not read)
        pg = uniform_address((isA ? gA : gB) + min(kt, total - 1) * 128);
        dl = __builtin_amdgcn_readfirstlane(lds0 + (unsigned)(slot * kSlot) + (unsigned)(wave * (isA ? LA : LB) * 1024));
    };
    auto fetch = [&](bool isA, int u) __attribute__((always_inline)) { fetch_to_lds(dl + u * 1024, (isA ? min(offA + (unsigned)u * 8u * (unsigned)g.lda, lastA) : min(offB + (unsigned)u * 8u * (unsigned)g.ldb, lastB)) + col[u & 1], pg); };

    const int swz = (lrow >> 1) & 7;
    const unsigned baseA = (unsigned)((wm * 32 * TM + lrow) * kStageBytes), baseB = (unsigned)((wn * 32 * TN + lrow) * kStageBytes);
    auto piece = [&](int c) { return (unsigned)((c ^ swz) << 4); };
    v4i32 fa[2][TM][NATIVE ? 2 : 1], fb[2][TN][NATIVE ? 2 : 1];
    constexpr int isA4[8] = {1, 0, 0, 1, 0, 0, 1, 1}, idx4[8] = {0, 0, 1, 1, 2, 3, 2, 3};
    auto which = [&](int q, bool &isA, int &idx) __attribute__((always_inline)) {  // fragment q in the order in which the products need them
        isA = kFour ? isA4[q] : q == 0 || q > TN;
        idx = kFour ? idx4[q] : q == 0 ? 0 : q > TN ? q - TN : q - 1;
    };
    auto fragment = [&](const char *sa, const char *sb, int ks, int buf, int q) __attribute__((always_inline)) {
        bool isA;
        int idx;
        which(q, isA, idx);
        const char *p = isA ? sa + baseA + idx * 32 * kStageBytes : sb + baseB + idx * 32 * kStageBytes;
        auto &f = isA ? fa[buf][idx] : fb[buf][idx];
        if constexpr (NATIVE) {
            f[0] = *reinterpret_cast<const v4i32 *>(p + piece(4 * ks + 2 * lhalf));
            f[1] = *reinterpret_cast<const v4i32 *>(p + piece(4 * ks + 2 * lhalf + 1));
        } else {
            f[0] = *reinterpret_cast<const v4i32 *>(p + piece(2 * ks + lhalf));
        }
    };
    v8bf16 ca[NATIVE ? 1 : TM][2], cb[NATIVE ? 1 : TN][2];
    auto convert = [&](int buf, int q) __attribute__((always_inline)) {
        if constexpr (!NATIVE) {
            bool isA;
            int idx;
            which(q, isA, idx);
            if (isA) {
                const float s = __int_as_float((sA[idx] & 255) << 23);
                const v4i32 w = fa[buf][idx][0];
                ca[idx][0] = widen<FA>(w[0], w[1], s), ca[idx][1] = widen<FA>(w[2], w[3], s);
            } else {
                const float s = __int_as_float((sB[idx] & 255) << 23);
                const v4i32 w = fb[buf][idx][0];
                cb[idx][0] = widen<FB>(w[0], w[1], s), cb[idx][1] = widen<FB>(w[2], w[3], s);
            }
        }
    };
    auto multiply = [&](int buf, int m) __attribute__((always_inline)) {
        constexpr int mi4[16] = {0, 0, 1, 1, 0, 0, 1, 1, 2, 2, 3, 3, 2, 2, 3, 3}, mj4[16] = {0, 1, 0, 1, 2, 3, 2, 3, 0, 1, 0, 1, 2, 3, 2, 3};
        const int i = kFour ? mi4[m] : m / TN, j = kFour ? mj4[m] : m % TN;
        if constexpr (NATIVE) {
            const v4i32 a0 = fa[buf][i][0], a1 = fa[buf][i][1], b0 = fb[buf][j][0], b1 = fb[buf][j][1];
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(v8i32{b0[0], b0[1], b0[2], b0[3], b1[0], b1[1], b1[2], b1[3]},
                                                                v8i32{a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]}, acc[i][j], FB, FA, 0, sB[j], 0, sA[i]);
        } else {
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cb[j][0], ca[i][0], acc[i][j], 0, 0, 0);
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(cb[j][1], ca[i][1], acc[i][j], 0, 0, 0);
        }
    };
    // the products of a k-step, the fragments of the next one and `count` loads from number `from` on among them
    auto step = [&](int cur, const char *sa, const char *sb, int next_ks, bool isA, int from, int count) {
        constexpr int kFirst = NM / NF >= 2 ? 3 : 2;  // fragments that the first products need
        if constexpr (!NATIVE) {
#pragma unroll
            for (int q = 0; q < kFirst; ++q) convert(cur, q);
        }
#pragma unroll
        for (int q = 0; q < NF; ++q) {
            fragment(sa, sb, next_ks, cur ^ 1, q);
            if constexpr (!NATIVE) {
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (kFirst + 2 * q + c < NF) convert(cur, kFirst + 2 * q + c);
            }
#pragma unroll
            for (int m = q * NM / NF; m < (q + 1) * NM / NF; ++m) multiply(cur, m);
#pragma unroll
            for (int u = q * count / NF; u < (q + 1) * count / NF; ++u) fetch(isA, from + u);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
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
    // Before the last step of a k-tile every fragment of it has been read and this wave's parts of the next one have landed (all but the newest loads); past the
    // barrier that holds for all waves, so that the last step may read k-tile kt + 1 and load B(kt + 2) into the slot of A(kt).
    // (The bytes are taken in loops of their own around the k-tiles: a branch among the products lets the compiler move them behind it, and a load in one copies what
    // it loads, which waits for it at once.  Taking them waits for the k-tiles on their way as well, which is why a group is as long as registers allow.)
    int sa = 0;
    Ends ends;
    for (int group = 0; group < total; group += 4 * G) {
        wide_t nowA[TM], nowB[TN];
#pragma unroll
        for (int i = 0; i < TM; ++i) nowA[i] = nextA[i];
#pragma unroll
        for (int j = 0; j < TN; ++j) nowB[j] = nextB[j];
        if constexpr (!NATIVE) {  // (taken before the next are asked for: a wait behind that waits for them too)
            auto take = [](wide_t &w) __attribute__((always_inline)) {
#pragma unroll
                for (int d = 0; d < G; ++d) {
                    int x = w[d];
                    asm volatile("" : "+v"(x));
                    w[d] = x;
                }
            };
#pragma unroll
            for (int i = 0; i < TM; ++i) take(nowA[i]);
#pragma unroll
            for (int j = 0; j < TN; ++j) take(nowB[j]);
        }
        load_bytes(group + 4 * G);
        for (int four = group; four < min(group + 4 * G, total); four += 4) {
#pragma unroll
            for (int i = 0; i < TM; ++i) sA[i] = shift(nowA[i]);
#pragma unroll
            for (int j = 0; j < TN; ++j) sB[j] = shift(nowB[j]);
            if constexpr (!NATIVE) {  // (bytes behind the last block are anything: 64 in their place)
                const unsigned there = total - four >= 4 ? ~0u : (1u << 8 * (total - four)) - 1;
#pragma unroll
                for (int i = 0; i < TM; ++i) ends.look<FA>(((unsigned)sA[i] & there) | (0x40404040u & ~there));
#pragma unroll
                for (int j = 0; j < TN; ++j) ends.look<FB>(((unsigned)sB[j] & there) | (0x40404040u & ~there));
            }
            for (int kt = four; kt < min(four + 4, total); ++kt) {
                const char *stA = smem + sa * kSlot, *stB = smem + ring(sa, 1) * kSlot;
                const char *stA1 = smem + ring(sa, 2) * kSlot, *stB1 = smem + ring(sa, 3) * kSlot;
                setup(true, kt + 2, ring(sa, 4));
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (NATIVE) {
                    step(0, stA, stB, 1, true, 0, LA);
                } else {
                    constexpr int c0 = (LA + 2) / 3, c1 = (LA - c0 + 1) / 2;
                    step(0, stA, stB, 1, true, 0, c0);
                    step(1, stA, stB, 2, true, c0, c1);
                    step(0, stA, stB, 3, true, c0 + c1, LA - c0 - c1);
                }
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"i"(LA) : "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                setup(false, kt + 2, sa);
                __builtin_amdgcn_sched_barrier(0);
                step((kSteps - 1) & 1, stA1, stB1, 0, false, 0, LB);
                sa = ring(sa, 2);
#pragma unroll
                for (int i = 0; i < TM; ++i) sA[i] = (int)((unsigned)sA[i] >> 8);
#pragma unroll
                for (int j = 0; j < TN; ++j) sB[j] = (int)((unsigned)sB[j] >> 8);
            }
        }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // nothing may land in LDS any more
    __syncthreads();
    return NATIVE || !ends.any() || !counts<FA, FB, TM, TN>(tileA, tileB, rowA, rowB, total);
}

// The sums of 32 T x 32 T results of a wave with codes as they are: each block's products are added up first and multiplied by both powers of two together, which no exponent is too far for.  Straight from
// memory, 32 x 32 results at a time: up to nine times as long as the walk above (4096^3 with such a block in every row 979 us instead of 112, in one row 825: the others of its tile wait for
// it), for operands that no training or serving step should have; blocks beyond the span that do not count cost their look through the bytes (134).
template <int FA, int FB, int T>
__device__ __forceinline__ void careful_tile(const GemmArgs &g, int m0, int n0, int k0, int k1, const float *bias, float *out, int64_t ldo) {
    const int lane = threadIdx.x & 63, lrow = lane & 31, lhalf = lane >> 5;
#pragma unroll 1
    for (int at = 0; at < T * T; ++at) {
        const int m = m0 + 32 * (at / T), n = n0 + 32 * (at % T);
        if (m >= g.m || n >= g.n) continue;
        const int ma = min(m + lrow, g.m - 1), nb = min(n + lrow, g.n - 1);
        const uint8_t *a = g.a + ma * g.lda + lhalf * 16, *sa = g.sa + ma * g.ldsa, *b = g.b + nb * g.ldb + lhalf * 16, *sb = g.sb + nb * g.ldsb;
        float sum[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) sum[r] = 0.0f;
#pragma unroll 1
        for (int kb = k0; kb < k1; ++kb) {
            v16f32 block;
#pragma unroll
            for (int r = 0; r < 16; ++r) block[r] = 0.0f;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const v4i32 x = *reinterpret_cast<const v4i32 *>(a + (int64_t)kb * 128 + q * 32), y = *reinterpret_cast<const v4i32 *>(b + (int64_t)kb * 128 + q * 32);
                block = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen<FB>(y[0], y[1], 1.0f), widen<FA>(x[0], x[1], 1.0f), block, 0, 0, 0);
                block = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen<FB>(y[2], y[3], 1.0f), widen<FA>(x[2], x[3], 1.0f), block, 0, 0, 0);
            }
            const int ea = sa[kb], eb = sb[kb];
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[r] += __builtin_ldexpf(block[r], ea + __shfl(eb, (r >> 2) * 8 + lhalf * 4 + (r & 3)) - 254);
        }
        if (m + lrow >= g.m) continue;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int col = n + 8 * q + 4 * lhalf;
            if (col >= g.n) continue;
            float f[4] = {sum[4 * q], sum[4 * q + 1], sum[4 * q + 2], sum[4 * q + 3]}, add[4];
            if (bias) {
                load_upto<float, 4>(bias + col, add, g.n - col);
#pragma unroll
                for (int r = 0; r < 4; ++r) f[r] += add[r];
            }
            store_upto<float, 4>(out + (int64_t)(m + lrow) * ldo + col, f, g.n - col);
        }
    }
}

// A wave's results, 32 T x 32 T, to memory: a lane holds four neighbours at a time of 32 rows, so they go through LDS (the wave's own 32 T rows of 256 bytes; piece c of
// row r at slot c ^ r) and leave in whole rows of it.  Straight from the registers 4096 x 4096 results took 8 us more.
template <bool HALF, int T>
__device__ __forceinline__ void store_tile(const v16f32 (&acc)[T][T], char *lds, int m0, int n0, int m, int n, const float *bias, void *out, int64_t ldo) {
    using E = std::conditional_t<HALF, __bf16, float>;
    constexpr int kWide = 32 * T * (int)sizeof(E), kRow = kWide < 256 ? kWide : 256, kPieces = kRow / 16, kPasses = kWide / kRow, kCols = T / kPasses, kEach = 16 / (int)sizeof(E);
    const int lane = threadIdx.x & 63, lrow = lane & 31, lhalf = lane >> 5;
    // (what a lane writes is read by another of its wave: in order for the hardware, and told to the compiler)
    auto written = []() __attribute__((always_inline)) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
#pragma unroll
    for (int pass = 0; pass < kPasses; ++pass) {
        if (pass) written();
#pragma unroll
        for (int jj = 0; jj < kCols; ++jj)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int j = pass * kCols + jj, col = n0 + 32 * j + 8 * q + 4 * lhalf;
                float b[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (bias && col < n) load_upto<float, 4>(bias + col, b, n - col);
                const int piece = HALF ? 4 * jj + q : 8 * jj + 2 * q + lhalf;
#pragma unroll
                for (int i = 0; i < T; ++i) {
                    const int row = 32 * i + lrow;
                    piece_t<E, 4> v;
#pragma unroll
                    for (int r = 0; r < 4; ++r) v[r] = (E)(acc[i][j][q * 4 + r] + b[r]);
                    typedef E aligned_t __attribute__((ext_vector_type(4)));
                    *reinterpret_cast<aligned_t *>(lds + row * kRow + ((piece ^ row) & (kPieces - 1)) * 16 + (HALF ? lhalf * 8 : 0)) = v;
                }
            }
        written();
        const int piece = lane & (kPieces - 1), col = n0 + pass * 32 * kCols + piece * kEach;
#pragma unroll 4
        for (int r = 0; r < 32 * T * kPieces / 64; ++r) {
            const int row = r * (64 / kPieces) + lane / kPieces;
            typedef E aligned_t __attribute__((ext_vector_type(kEach)));
            const aligned_t v = *reinterpret_cast<const aligned_t *>(lds + row * kRow + ((piece ^ row) & (kPieces - 1)) * 16);
            if (m0 + row >= m || col >= n) continue;
            E *to = (E *)out + (int64_t)(m0 + row) * ldo + col;
            if (n - col >= kEach) {
                *reinterpret_cast<piece_t<E, kEach> *>(to) = v;
            } else {
#pragma unroll
                for (int k = 0; k < kEach; ++k)
                    if (k < n - col) to[k] = v[k];
            }
        }
    }
}

template <bool NATIVE, int FA, int FB, int T>
__global__ __launch_bounds__(kProductThreads, T == 4 ? 1 : T == 2 ? 2 : 4) void block8_tile_gemm_kernel(const GemmArgs g) {
    extern __shared__ __attribute__((aligned(16))) char smem[];
    const int tiles = g.mtiles * g.ntiles, part = (int)blockIdx.x / tiles;
    int tm, tn;
    tile_at((int)blockIdx.x - part * tiles, g.mtiles, g.ntiles, tm, tn);
    v16f32 acc[T][T];
    const int k0 = part * g.per, k1 = min((part + 1) * g.per, g.kt);
    const bool right = product8_tile<NATIVE, FA, FB, T, T, T == 4 ? 4 : 1>(g, tm * 64 * T, tn * 64 * T, k0, k1, smem, acc);
    const int wave = threadIdx.x >> 6;
    const int m0 = tm * 64 * T + (wave >> 1) * 32 * T, n0 = tn * 64 * T + (wave & 1) * 32 * T;
    char *own = smem + wave * 32 * T * 256;
    float *sums = (float *)g.out + (int64_t)part * g.m * g.n;
    if (!NATIVE && !right) {
        careful_tile<FA, FB, T>(g, m0, n0, k0, k1, g.parts > 1 ? nullptr : g.bias, g.parts > 1 ? sums : (float *)g.out, g.parts > 1 ? g.n : g.ldo);
        return;
    }
    if (g.parts > 1) store_tile<false, T>(acc, own, m0, n0, g.m, g.n, nullptr, sums, g.n);
    else store_tile<NATIVE, T>(acc, own, m0, n0, g.m, g.n, g.bias, g.out, g.ldo);
}

// The sum of the parts in their order, four columns to a thread.
template <class T>
__global__ __launch_bounds__(256) void block8_fold_kernel(const float *__restrict__ sums, const float *__restrict__ bias, T *__restrict__ out, int64_t ldo, int parts, int m, int n) {
    const int across = (n + 3) / 4;
    const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, row = at / across;
    const int col = (int)(at - row * across) * 4;
    if (row >= m) return;
    float f[4], s[4];
    load_upto<float, 4>(sums + row * n + col, f, n - col);
    for (int p = 1; p < parts; ++p) {
        load_upto<float, 4>(sums + ((int64_t)p * m + row) * n + col, s, n - col);
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] += s[k];
    }
    if (bias) {
        load_upto<float, 4>(bias + col, s, n - col);
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] += s[k];
    }
    store_upto<T, 4>(out + row * ldo + col, f, n - col);
}

// ---- up to sixteen rows: the contraction is dealt to a workgroup's waves -----------------------------------------------------------------
// What counts is that B is read once, at once: a wave takes every eighth block of 16 rows of B straight into registers (four lanes to a row, a quarter of its
// block's first half and of its second to each, so that a load takes 64 bytes of every row), four blocks ahead of the products, with the blocks of A's rows, which the
// caches hold.  The waves' sums meet in LDS.  16 x 4096 by 4096: 7.5 us a call, fp32 results 7.7; the kernel 7.8 by the profiler's clock, 7.1 also where it is one workgroup alone (by 16), 1.6 where that has
// one block: the way of a wave's loads and what comes behind them bounds it, not bytes (2.7 at 6.5 TB/s).  32 rows of B to a workgroup were slower (10.2), a second set of registers under way as well (16 x 4096 by 11008: 18.0, 19.5).
constexpr int kFewRows = 16, kFewWaves = 8, kFewAhead = 4;
template <bool NATIVE, int FA, int FB>
__global__ __launch_bounds__(64 * kFewWaves) void block8_few_kernel(const GemmArgs g) {
    typedef float v4f32 __attribute__((ext_vector_type(4)));
    __shared__ __attribute__((aligned(16))) float sums[kFewWaves][64][4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), row = lane & 15, quarter = lane >> 4;
    const int n0 = (int)blockIdx.x * 16, ma = min(row, g.m - 1), nb = min(n0 + row, g.n - 1);
    const uint8_t *a = g.a + ma * g.lda + quarter * 16, *sa = g.sa + ma * g.ldsa, *b = g.b + nb * g.ldb + quarter * 16, *sb = g.sb + nb * g.ldsb;
    v4f32 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    Ends ends;
    for (int first = wave; first < g.kt; first += kFewWaves * kFewAhead) {
        v4i32 xa[kFewAhead][2], xb[kFewAhead][2];
        int ea[kFewAhead], eb[kFewAhead];
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u) {
            const int kb = min(first + u * kFewWaves, g.kt - 1);
            xb[u][0] = *reinterpret_cast<const v4i32 *>(b + kb * 128), xb[u][1] = *reinterpret_cast<const v4i32 *>(b + kb * 128 + 64);
            xa[u][0] = *reinterpret_cast<const v4i32 *>(a + kb * 128), xa[u][1] = *reinterpret_cast<const v4i32 *>(a + kb * 128 + 64);
            eb[u] = sb[kb], ea[u] = sa[kb];
        }
#pragma unroll
        for (int u = 0; u < kFewAhead; ++u) {
            if (first + u * kFewWaves >= g.kt) break;
            const v4i32 a0 = xa[u][0], a1 = xa[u][1], b0 = xb[u][0], b1 = xb[u][1];
            if constexpr (NATIVE) {
                acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(v8i32{b0[0], b0[1], b0[2], b0[3], b1[0], b1[1], b1[2], b1[3]},
                                                                       v8i32{a0[0], a0[1], a0[2], a0[3], a1[0], a1[1], a1[2], a1[3]}, acc, FB, FA, 0, eb[u], 0, ea[u]);
            } else {
                ends.look<FA>((unsigned)ea[u] | 0x40404000u), ends.look<FB>((unsigned)eb[u] | 0x40404000u);
                const float pb = __int_as_float(eb[u] << 23), pa = __int_as_float(ea[u] << 23);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FB>(b0[0], b0[1], pb), widen<FA>(a0[0], a0[1], pa), acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FB>(b0[2], b0[3], pb), widen<FA>(a0[2], a0[3], pa), acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FB>(b1[0], b1[1], pb), widen<FA>(a1[0], a1[1], pa), acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FB>(b1[2], b1[3], pb), widen<FA>(a1[2], a1[3], pa), acc, 0, 0, 0);
            }
        }
    }
    if (!NATIVE && ends.any()) {  // codes as they are, a block's sum times both powers of two
        acc = v4f32{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
        for (int kb = wave; kb < g.kt; kb += kFewWaves) {
            v4f32 block = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const v4i32 x = *reinterpret_cast<const v4i32 *>(a + kb * 128 + h * 64), y = *reinterpret_cast<const v4i32 *>(b + kb * 128 + h * 64);
                block = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FB>(y[0], y[1], 1.0f), widen<FA>(x[0], x[1], 1.0f), block, 0, 0, 0);
                block = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen<FB>(y[2], y[3], 1.0f), widen<FA>(x[2], x[3], 1.0f), block, 0, 0, 0);
            }
            const int ea = sa[kb], eb = sb[kb];
#pragma unroll
            for (int r = 0; r < 4; ++r) acc[r] += __builtin_ldexpf(block[r], ea + __shfl(eb, 4 * quarter + r) - 254);
        }
    }
    *reinterpret_cast<v4f32 *>(sums[wave][lane]) = acc;
    __syncthreads();
    // lane l holds row l % 16 of A with the columns 4 (l / 16) .. + 3; the waves' sums in their order
    if (threadIdx.x >= 64) return;
    const int n = n0 + 4 * quarter;
    if (row >= g.m || n >= g.n) return;
    float f[4], bias[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = sums[0][lane][k];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w)
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] += sums[w][lane][k];
    if (g.bias) {
        load_upto<float, 4>(g.bias + n, bias, g.n - n);
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] += bias[k];
    }
    if (NATIVE) store_upto<__bf16, 4>((__bf16 *)g.out + row * g.ldo + n, f, g.n - n);
    else store_upto<float, 4>((float *)g.out + row * g.ldo + n, f, g.n - n);
}

// How a product is cut: tiles of 64 T (T = 0: the kernel for few rows), the contraction in parts of `per` blocks, multiples of what a tile's bytes are taken in.
struct Cut {
    int tile, parts, per;
};
// The cut that should take the least time, in nanoseconds, from what the kernels were seen to take: a workgroup costs `fixed` and `each` for every block, a CU works on one after
// the other (or on several at once, no faster in all); with no more workgroups than CUs small tiles wait for their loads (`alone`; longer still with one row of tiles, where nobody else has
// fetched B).  Parts cost a launch and their sums' way to memory and back.  Microseconds, bfloat16 / fp32 results, by tiles of 64, 128 and 256:
//   1024^3 5.8, 7.4, 17.3 / 7.2, 12.1, 30.2;  2048^3 17.9, 12.6, 26.9 / 23.9, 22.6, 49.2;  256 x 4096 by 4096 12.7, 18.3, 39.4 / 18.4, 32.4, -;
//   12608 x 768 by 768 20.2, 16.4, 18.7 / 25.2, 24.3, 31.2;  4096^3 -, -, 54 / -, -, 110;  768 x 12608 by 768 in 4 parts of 64 24.3 / 26.9, in 7 of 128 22.3 / 27.3, in 2 of 128 36 / 54;
//   64 x 4096 by 4096 in 1, 2 and 4 parts of 64 12.1, 11.1, 10.4 / 16.9, 13.2, 11.4
// Up to 16 rows, the kernel for few rows and 1, 2, 4 and 8 parts of 64: 16 x 4096 by 5120 12.4 and 10.7, 9.5, 9.4, 10.6 / 12.6 and 17.1, 12.5, 11.2, 11.8;  by 11008 17.8 and 16.8, 13.5, 12.8, 15.8 /
//   17.9 and 19.5, 16.1, 13.9, 16.4;  1 x 4096 by 11008 11.8 and 16.5, 13.1, 12.0, 14.5 / 11.8 and 19.4, 15.6, 13.3, 15.5;  16 x 4096 by 4096 7.3 and 10.7, 9.5, 8.8, 9.8 / 7.7 and 17.2, 12.5, 9.9, 10.7.
// A CU takes its workgroups of 16 columns one after the other, and those behind the first (more than 4096 columns) have A's rows to wait for as well: 101 and 4 for each row, a block.
static Cut cut_of(int64_t m, int64_t n, int64_t kt, bool native) {
    struct Cost {
        int tile, whole, fixed, alone, first, each;
    };
    static const Cost costs[2][3] = {{{1, 4, 200, 420, 420, 310}, {2, 4, 500, 1020, 1020, 1020}, {4, 16, 10000, 2750, 2750, 2750}},
                                     {{1, 4, 200, 240, 370, 210}, {2, 4, 500, 550, 550, 550}, {4, 16, 8000, 1300, 1300, 1300}}};
    Cut best = {0, 1, (int)kt};
    const double rounds = (double)((n + 4095) / 4096);
    double least = m <= kFewRows ? rounds * 300.0 + (115.0 + (rounds - 1.0) * (101.0 + 4.0 * (double)m)) * (double)kt : 1e30;
    for (const Cost &c : costs[native]) {
        const int64_t edge = 64 * c.tile, down = (m + edge - 1) / edge, tiles = down * ((n + edge - 1) / edge);
        for (int64_t p = 1, last = 0; p <= 64 && (p == 1 || p * c.whole <= kt); ++p) {
            const int64_t per = ((kt + p - 1) / p + c.whole - 1) / c.whole * c.whole, parts = (kt + per - 1) / per, groups = tiles * parts;
            if (parts == last) continue;
            last = parts;
            const int64_t block = groups > 256 ? c.each : down > 1 ? c.alone : c.first;
            const double walk = (double)((groups + 255) / 256) * (double)(c.fixed + std::min(per, kt) * block);
            const double time = walk + (parts > 1 ? 3500.0 + (double)parts * (double)m * (double)n * 8.0 / 6000.0 : 0.0);
            if (time < least) best = {c.tile, (int)parts, (int)per}, least = time;
            if (groups > 2048) break;
        }
    }
    return best;
}

template <bool NATIVE, int FA, int FB, int T>
static int launch_tiles(const GemmArgs &g, hipStream_t st) {
    const auto kernel = block8_tile_gemm_kernel<NATIVE, FA, FB, T>;
    static std::atomic<int> done{0};  // (the attribute is idempotent: two threads set the same)
    if (!done.load(std::memory_order_acquire)) {
        IMU_HIP(hipFuncSetAttribute((const void *)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, product_lds(T, T)));
        done.store(1, std::memory_order_release);
    }
    hipLaunchKernelGGL(kernel, dim3((unsigned)((int64_t)g.mtiles * g.ntiles * g.parts)), dim3(kProductThreads), product_lds(T, T), st, g);
    return launch_status();
}

constexpr int64_t kPitch = 1 << 24;  // bytes from row to row at most, of codes and scales: offsets within a tile have 32 bits
static bool operand_fits(const Blocks8 &t, int64_t rows, int64_t cols, int format) {
    return blocks8_fit(t, cols) && rows >= 1 && t.ldc <= kPitch && t.lds <= kPitch && (format == IMUNPACK_E4M3 || format == IMUNPACK_E5M2);
}
}  // namespace imu

using namespace imu;

constexpr int64_t kGemmRows = 1 << 24;

static bool gemm_sizes(int64_t m, int64_t n, int64_t k, int dtype) {
    return m >= 0 && n >= 0 && k >= 1 && m <= kGemmRows && n <= kGemmRows && k <= kBlock8Cols && (dtype == IMUNPACK_F32 || dtype == IMUNPACK_BF16);
}

extern "C" int imunpack_block8_gemm_workspace(int64_t m, int64_t n, int64_t k, int dtype, size_t *bytes) {
    if (!gemm_sizes(m, n, k, dtype) || !bytes) return IMUNPACK_EINVAL;
    const Cut c = cut_of(m, n, (k + kBlock8 - 1) / kBlock8, dtype == IMUNPACK_BF16);
    *bytes = c.parts > 1 ? (size_t)c.parts * (size_t)m * (size_t)n * sizeof(float) : 0;
    return IMUNPACK_OK;
}

extern "C" int imunpack_diag_block8_cut(int64_t m, int64_t n, int64_t k, int dtype, int *tile, int *parts) {
    if (!gemm_sizes(m, n, k, dtype) || !tile || !parts) return IMUNPACK_EINVAL;
    const Cut c = cut_of(m, n, (k + kBlock8 - 1) / kBlock8, dtype == IMUNPACK_BF16);
    *tile = c.tile, *parts = c.parts;
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
    const int kt = (int)((k + kBlock8 - 1) / kBlock8);
    const Cut c = cut_of(m, n, kt, dtype == IMUNPACK_BF16);
    const hipStream_t st = (hipStream_t)stream;
    GemmArgs g = {A.codes, A.scales, B.codes, B.scales, bias, c.parts > 1 ? workspace : out, lda, ldsa, ldb, ldsb, ldo, (int)m, (int)n, kt, 0, 0, c.parts, c.per};
    const int64_t tall = c.tile ? 64 * c.tile : kFewRows, wide = c.tile ? 64 * c.tile : 16;
    g.mtiles = (int)((m + tall - 1) / tall);
    g.ntiles = (int)((n + wide - 1) / wide);
    if ((int64_t)g.mtiles * g.ntiles * g.parts > (1 << 23)) return IMUNPACK_EINVAL;
    const bool native = dtype == IMUNPACK_BF16;
    auto launch = [&](auto fa, auto fb) {
        constexpr int FA = decltype(fa)::value, FB = decltype(fb)::value;
        if (c.tile == 4) return native ? launch_tiles<true, FA, FB, 4>(g, st) : launch_tiles<false, FA, FB, 4>(g, st);
        if (c.tile == 2) return native ? launch_tiles<true, FA, FB, 2>(g, st) : launch_tiles<false, FA, FB, 2>(g, st);
        if (c.tile == 1) return native ? launch_tiles<true, FA, FB, 1>(g, st) : launch_tiles<false, FA, FB, 1>(g, st);
        if (native) hipLaunchKernelGGL((block8_few_kernel<true, FA, FB>), dim3((unsigned)g.ntiles), dim3(64 * kFewWaves), 0, st, g);
        else hipLaunchKernelGGL((block8_few_kernel<false, FA, FB>), dim3((unsigned)g.ntiles), dim3(64 * kFewWaves), 0, st, g);
        return launch_status();
    };
    using E4 = std::integral_constant<int, IMUNPACK_E4M3>;
    using E5 = std::integral_constant<int, IMUNPACK_E5M2>;
    if (a_format == IMUNPACK_E4M3) IMU_TRY(b_format == IMUNPACK_E4M3 ? launch(E4(), E4()) : launch(E4(), E5()));
    else IMU_TRY(b_format == IMUNPACK_E4M3 ? launch(E5(), E4()) : launch(E5(), E5()));
    if (g.parts == 1) return IMUNPACK_OK;
    const int64_t threads = m * ((n + 3) / 4);
    const dim3 grid((unsigned)((threads + 255) / 256));
    if (native) hipLaunchKernelGGL(block8_fold_kernel<__bf16>, grid, dim3(256), 0, st, (const float *)workspace, bias, (__bf16 *)out, ldo, c.parts, (int)m, (int)n);
    else hipLaunchKernelGGL(block8_fold_kernel<float>, grid, dim3(256), 0, st, (const float *)workspace, bias, (float *)out, ldo, c.parts, (int)m, (int)n);
    return launch_status();
}
