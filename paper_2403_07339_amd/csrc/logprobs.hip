// Log probabilities of given tokens, entropy and the largest alternatives of rows of logits, and their gradient.
//
//   m = max l,  S = sum exp(l - m),  A = sum exp(l - m) (l - m)       lse = m + log S,   entropy = log S - A / S
//   gl_v = sum_j g_j ([v = t_j] - p_v) - g_H p_v (l_v - lse + H)
//
// Forward: one pass over the row with the running maximum of a thread; where it moves by d <= 0, S -> S e^d, A -> e^d (A + d S).  Exponents are kept in
// units of log 2.  Few rows are cut into parts, a workgroup to each, which a second launch joins.
// The largest `top`: a wave gathers in LDS what may be among them.  The top-th largest of the lanes' maxima so far (found bit by bit) is a bound, which
// at least `top` elements reach and, but for ties, no more than `top` lanes' worth; chunks whose maximum stays below it are passed over, which is nearly every one after the
// first few.  64 gathered elements are sorted, one to a lane, and merged with the wave's best 64, whose top-th is the next bound; mostly that happens once, for what the workgroup's waves
// gathered together.  An element is a number that grows with the logit and falls with the place.  -infinity (and NaN) is never gathered: where fewer than `top` others exist, the
// lowest of the remaining places follow them.
// Bound by memory where rows are many: 4096 x 32000 bfloat16 47 us without alternatives (5.6 TB/s), 67 with 8, its gradient 80 (6.6 TB/s, past the last-level cache: what it
// left there dirty was written back while the next call read, 167 -> 136 us for both).
#include "common.h"
#include "elements.h"

#include <algorithm>

namespace imu {
constexpr int64_t kLogprobRows = 1 << 22;  // of a launch
constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;
constexpr int kScanPieces = 4;             // pieces of 16 bytes that a thread loads at a time
constexpr int kMostParts = 64;

struct LogprobArgs {
    const void *l;
    const int64_t *tokens;
    float *logp, *lse, *stats, *entropy, *top_logp;
    int64_t *top_index;
    float *part_stats;        // several parts: three numbers and `top` keys of each
    uint64_t *part_keys;
    int64_t ldl, ignore;
    int vocab, count, top, parts, per;
};

__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }

// Maximum m, S and A / log 2 of a part of a row.  Exponents are x log2(e) - M with M = m log2(e) rounded, one operation; S and A are relative to M, of which every step
// takes the rounded value (products and differences of it are not contracted), and what its rounding left is given back to log S at the end.  That is at most 1 / 16 where
// |m| < 2^20; beyond it (a row of a mask's number) exponents are (x - m) log2(e).
struct Moments {
    float m = -__builtin_inff(), s = 0.0f, a = 0.0f;
    __device__ __forceinline__ static bool plain(float m) { return fabsf(m) < 0x1p20f; }
    __device__ __forceinline__ static float base(float m) {
#pragma clang fp contract(off)
        return m * kLog2e;
    }
    __device__ __forceinline__ static float left(float m) { return plain(m) ? -fmaf(m, kLog2e, -base(m)) : 0.0f; }  // M - m log2(e)
    __device__ __forceinline__ void rebase(float to) {  // to >= m
#pragma clang fp contract(off)
        const float d = m == to ? 0.0f : plain(m) && plain(to) ? base(m) - base(to) : (m - to) * kLog2e + (left(m) - left(to));  // (m == to: both may be infinite)
        const float e = exp2_of(d);
        a = e > 0.0f ? e * fmaf(d, s, a) : 0.0f;
        s *= e;
        m = to;
    }
    template <int N>
    __device__ __forceinline__ void add(const float (&x)[N]) {  // x <= m, m > -infinity
        auto one = [&](float t) __attribute__((always_inline)) {
            const float e = exp2_of(t);
            s += e;
            a = fmaf(e, fmaxf(t, -1e4f), a);  // (e is 0 there; t may be -infinity)
        };
        if (plain(m)) {
            const float up = base(m);
#pragma unroll
            for (int k = 0; k < N; ++k) one(fmaf(x[k], kLog2e, -up));
        } else {
            for (int k = 0; k < N; ++k) one((x[k] - m) * kLog2e);
        }
    }
    __device__ __forceinline__ void join(Moments o) {
        const float to = fmaxf(m, o.m);
        rebase(to);
        o.rebase(to);
        s += o.s;
        a += o.a;
    }
};
// The value of the lane whose number differs by MASK, on the vector ALU's lane moves: within a row of 16 lanes permutations of four, a rotation by half, mirrors (7 - i and then 3 - i is
// i ^ 4); across rows and halves the swap of registers, of which each side keeps what it has not.  (Through LDS a step of a sort waits for it.)
template <int MASK>
__device__ __forceinline__ uint32_t other_lane(uint32_t v, int lane) {
    if constexpr (MASK == 1) return (uint32_t)IMU_DPP(v, 0xb1, 0xf, true);
    if constexpr (MASK == 2) return (uint32_t)IMU_DPP(v, 0x4e, 0xf, true);
    if constexpr (MASK == 4) return (uint32_t)IMU_DPP(IMU_DPP(v, 0x141, 0xf, true), 0x1b, 0xf, true);
    if constexpr (MASK == 8) return (uint32_t)IMU_DPP(v, 0x128, 0xf, true);
    if constexpr (MASK == 15) return (uint32_t)IMU_DPP(v, 0x140, 0xf, true);
    if constexpr (MASK == 16) {
        const auto both = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return lane & 16 ? both[0] : both[1];
    }
    if constexpr (MASK == 32) {
        const auto both = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return lane & 32 ? both[0] : both[1];
    }
    if constexpr (MASK == 63) return other_lane<32>(other_lane<16>(other_lane<15>(v, lane), lane), lane);
}
template <int MASK>
__device__ __forceinline__ uint64_t other_lane(uint64_t k, int lane) {
    return (uint64_t)other_lane<MASK>((uint32_t)(k >> 32), lane) << 32 | other_lane<MASK>((uint32_t)k, lane);
}

template <int MASK>
__device__ __forceinline__ void join_lanes(Moments &v, int lane) {
    Moments o;
    o.m = __uint_as_float(other_lane<MASK>(__float_as_uint(v.m), lane));
    o.s = __uint_as_float(other_lane<MASK>(__float_as_uint(v.s), lane));
    o.a = __uint_as_float(other_lane<MASK>(__float_as_uint(v.a), lane));
    v.join(o);
}
__device__ __forceinline__ Moments wave_join(Moments v, int lane) {
    join_lanes<32>(v, lane), join_lanes<16>(v, lane), join_lanes<8>(v, lane), join_lanes<4>(v, lane), join_lanes<2>(v, lane), join_lanes<1>(v, lane);
    return v;
}

// The order of a logit among a row's: larger first, then the lower place.  0 is below all.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b >> 31 ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint64_t key) {
    const uint32_t b = (uint32_t)(key >> 32);
    return __uint_as_float(b >> 31 ? b & 0x7fffffffu : ~b);
}
__device__ __forceinline__ uint64_t key_of(float x, int place) { return ((uint64_t)order_of(x) << 32) | (uint32_t)~place; }
// A wave's best 64, largest in lane 0.
struct Best {
    uint64_t key = 0;
    template <int MASK>
    __device__ __forceinline__ static uint64_t step(uint64_t k, int lane, bool down) {
        const uint64_t o = other_lane<MASK>(k, lane);
        return (((lane & MASK) == 0) == down) == (k > o) ? k : o;
    }
    template <int MASK>
    __device__ __forceinline__ static uint64_t steps(uint64_t k, int lane, bool down) {  // MASK, MASK / 2, ... 1
        k = step<MASK>(k, lane, down);
        if constexpr (MASK > 1) k = steps<MASK / 2>(k, lane, down);
        return k;
    }
    // the keys of the lanes in order, largest first; behind lane `n` there are none (0)
    __device__ __forceinline__ static uint64_t sorted(uint64_t k, int lane, int n) {
        k = steps<1>(k, lane, (lane & 2) == 0);
        k = steps<2>(k, lane, (lane & 4) == 0);
        k = steps<4>(k, lane, (lane & 8) == 0);
        k = steps<8>(k, lane, (lane & 16) == 0);
        if (n <= 16) return k;
        k = steps<16>(k, lane, (lane & 32) == 0);
        return steps<32>(k, lane, true);
    }
    __device__ __forceinline__ void merge(uint64_t other, int lane) {  // other in order too
        const uint64_t o = other_lane<63>(other, lane);
        key = steps<32>(key > o ? key : o, lane, true);
    }
};

// Token j of a row, and its logit (of one that is none: 0).
struct Given {
    int64_t t = -1;
    float x = 0.0f;
};
__device__ __forceinline__ Given given_of(const LogprobArgs &a, int64_t row, const void *l, bool bf16, int j) {
    Given k;
    if (j >= a.count) return k;
    k.t = a.tokens[row * a.count + j];
    if (k.t >= 0 && k.t < a.vocab) k.x = bf16 ? (float)((const __bf16 *)l)[k.t] : ((const float *)l)[k.t];
    return k;
}
// What a row's outputs are made of, by one workgroup (or wave): threads `at` of `of`, each with its first token.
__device__ __forceinline__ void logprob_outputs(const LogprobArgs &a, int64_t row, const void *l, bool bf16, const Moments &all, int at, int of, const Given &own, uint64_t key, bool lists) {
    const bool none = all.m == -__builtin_inff() && all.s == 0.0f;
    // (log p = (l - m) - log S: m may be so large that log S is lost beside it)
    const float sum = none ? 0.0f : logf(all.s), logs = none ? 0.0f : fmaf(kLn2, Moments::left(all.m), sum);
    auto logp = [&](float x) { return none ? all.m : (x - all.m) - logs; };
    if (at == 0) {
        if (a.lse) a.lse[row] = all.m + logs;
        if (a.stats) a.stats[2 * row] = all.m, a.stats[2 * row + 1] = logs;
        if (a.entropy) a.entropy[row] = none ? 0.0f : sum - kLn2 * (all.a / all.s);  // (both relative to M)
    }
    for (int j = at; j < a.count; j += of) {
        const Given k = j == at ? own : given_of(a, row, l, bf16, j);
        a.logp[row * a.count + j] = k.t == a.ignore ? 0.0f : k.t < 0 || k.t >= a.vocab ? __builtin_nanf("") : logp(k.x);
    }
    if (!lists) return;  // (a whole wave that holds the largest, in order)
    const int some = __builtin_popcountll(__ballot(key != 0));
    int place = (int)~(uint32_t)key;
    if (some < a.top) {  // the lowest places that are not among them: fewer than 64 are, so they lie below 128
        uint64_t low = 0, high = 0;
        for (int k = 0; k < some; ++k) {
            const int p = __shfl(place, k);
            if (p < 64) low |= 1ull << p;
            else if (p < 128) high |= 1ull << (p - 64);
        }
        int skip = at - some, found = 0;  // the skip-th free place, from 0
        for (int p = 0; p < 128; ++p) {
            const bool taken = ((p < 64 ? low >> p : high >> (p - 64)) & 1) != 0;
            if (!taken && skip-- == 0) found = p;
        }
        if (at >= some) place = found;
    }
    if (at < a.top) {
        a.top_index[row * a.top + at] = place;
        a.top_logp[row * a.top + at] = key ? logp(logit_of(key)) : logp(-__builtin_inff());
    }
}

template <class T, bool TOP, bool ONCE>
__global__ __launch_bounds__(256) void logprobs_kernel(const LogprobArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float part[4][3];
    __shared__ uint64_t gathered[4][TOP ? 128 : 1], lists[4][TOP ? 64 : 1];
    __shared__ int counts[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x / a.parts;
    const int which = (int)((int64_t)blockIdx.x - row * a.parts), from = which * a.per, to = min(a.vocab, from + a.per);
    const T *l = (const T *)a.l + row * a.ldl;
    Moments mine;
    Best best;
    float reach = -__FLT_MAX__;  // what an element has to reach to be gathered
    bool flushed = false;
    int held = 0;                // in `gathered`
    // (What a lane wrote is read by another of its wave: in order for the hardware, and here for the compiler, which moved loads over stores of other lanes' words
    // where a loop stood around them.)
    auto written = []() __attribute__((always_inline)) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    auto flush = [&](int n) __attribute__((always_inline)) {
        written();
        best.merge(Best::sorted(lane < n ? gathered[wave][lane] : 0, lane, n), lane);
        flushed = true;
    };
    // a chunk, a whole one without a look at the row's end
    auto scan = [&](int base, auto whole) __attribute__((always_inline)) {
        constexpr bool kWhole = decltype(whole)::value;
        constexpr int P = kScanPieces, E = V * P;
        piece_t<T, V> in[P];
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const int at = base + (u * 256 + (int)threadIdx.x) * V;
            in[u] = load_piece<T, V, ONCE>(l + at, kWhole ? V : to - at);
        }
        float x[E];
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const int have = to - (base + (u * 256 + (int)threadIdx.x) * V);
#pragma unroll
            for (int k = 0; k < V; ++k) x[u * V + k] = kWhole || k < have ? (float)in[u][k] : -__builtin_inff();
        }
        float highs[P], high;  // (NaN is passed over, unless all are)
#pragma unroll
        for (int u = 0; u < P; ++u) {
            highs[u] = x[u * V];
#pragma unroll
            for (int k = 1; k < V; ++k) highs[u] = fmaxf(highs[u], x[u * V + k]);
            high = u ? fmaxf(high, highs[u]) : highs[u];
        }
        if (high > mine.m) mine.rebase(high);
        if (mine.m > -__builtin_inff()) {
            mine.add(x);
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) mine.s += x[e] == x[e] ? 0.0f : x[e];
        }
        if constexpr (TOP) {
            auto wanted = [&](float v) { return v >= reach; };
            if (__ballot(wanted(high))) {
                {  // what at least `top` lanes have seen (the upper half of the order's bits will do)
                    const uint32_t own = mine.m > -__builtin_inff() ? order_of(mine.m) >> 16 : 0;
                    uint32_t bound = 0;
#pragma unroll 1
                    for (uint32_t bit = 0x8000u; bit; bit >>= 1)
                        if (__builtin_popcountll(__ballot(own >= (bound | bit))) >= a.top) bound |= bit;
                    const float all = logit_of((uint64_t)bound << 48);
                    if (bound && all > reach) reach = all;
                }
                const int first = base + (int)threadIdx.x * V;
                bool sorted = false;
#pragma unroll
                for (int u = 0; u < P; ++u) {
                    if (__ballot(wanted(highs[u])) == 0) continue;
#pragma unroll
                    for (int k = 0; k < V; ++k) {
                        const float v = x[u * V + k];
                        const uint64_t who = __ballot(wanted(v));  // (places behind the row's end hold -infinity)
                        if (who == 0) continue;
                        if (wanted(v)) gathered[wave][held + __builtin_popcountll(who & ((1ull << lane) - 1))] = key_of(v, first + u * 256 * V + k);
                        held += __builtin_popcountll(who);
                        if (held < 64) continue;
                        written();
                        const uint64_t rest = gathered[wave][64 + lane];
                        flush(64);
                        held -= 64;
                        written();
                        if (lane < held) gathered[wave][lane] = rest;
                        written();
                        sorted = true;
                    }
                }
                // (only now: of this chunk what equals the list's last may have a lower place; later ones have to exceed it)
                if (sorted) {
                    const uint64_t k = (uint64_t)__shfl((unsigned long long)best.key, a.top - 1);
                    const float above = logit_of(k + (1ull << 32));
                    if (k && above > reach) reach = above;
                }
            }
        }
    };
    int base = from;
    for (; base + 256 * V * kScanPieces <= to; base += 256 * V * kScanPieces) scan(base, std::true_type());
    if (base < to) scan(base, std::false_type());
    mine = wave_join(mine, lane);
    if (lane == 0) part[wave][0] = mine.m, part[wave][1] = mine.s, part[wave][2] = mine.a;
    if constexpr (TOP) {
        lists[wave][lane] = best.key;
        if (lane == 0) counts[wave] = flushed ? held | 0x1000 : held;
    }
    __syncthreads();
    Moments all;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        Moments o;
        o.m = part[w][0], o.s = part[w][1], o.a = part[w][2];
        all.join(o);
    }
    if constexpr (TOP) {
        if (wave == 0) {  // the waves' lists, where there are any, and what they gathered last, 64 at a time
            int before[5] = {0, 0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                before[w + 1] = before[w] + (counts[w] & 0xfff);
                if (w && counts[w] & 0x1000) best.merge(lists[w][lane], lane);
            }
            for (int i = 0; i < before[4]; i += 64) {
                const int at = i + lane, w = (at >= before[1]) + (at >= before[2]) + (at >= before[3]);
                const uint64_t k = at < before[4] ? gathered[w][at - (w == 0 ? 0 : w == 1 ? before[1] : w == 2 ? before[2] : before[3])] : 0;
                best.merge(Best::sorted(k, lane, before[4] - i), lane);
            }
        }
    }
    if (a.parts == 1) {
        logprob_outputs(a, row, l, std::is_same<T, __bf16>::value, all, (int)threadIdx.x, 256, given_of(a, row, l, std::is_same<T, __bf16>::value, (int)threadIdx.x), best.key, TOP && wave == 0);
        return;
    }
    if (threadIdx.x == 0) {
        float *p = a.part_stats + (row * a.parts + which) * 3;
        p[0] = all.m, p[1] = all.s, p[2] = all.a;
    }
    if (TOP && wave == 0 && lane < a.top) a.part_keys[(row * a.parts + which) * a.top + lane] = best.key;
}

// The parts of a row, a wave to a row.
template <class T>
__global__ __launch_bounds__(64) void logprobs_join_kernel(const LogprobArgs a) {
    constexpr bool kHalf = std::is_same<T, __bf16>::value;
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x;
    const T *l = (const T *)a.l + row * a.ldl;
    // (every load is asked for before anything waits)
    auto keys = [&](int p) { return lane < a.top && p < a.parts ? a.part_keys[(row * a.parts + p) * a.top + lane] : 0; };
    uint64_t k[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) k[u] = keys(u);
    Moments all;
    if (lane < a.parts) {
        const float *p = a.part_stats + (row * a.parts + lane) * 3;
        all.m = p[0], all.s = p[1], all.a = p[2];
    }
    const Given own = given_of(a, row, l, kHalf, lane);
    all = wave_join(all, lane);
    Best best;
    if (a.top) {
#pragma unroll 1
        for (int p = 0; p < a.parts; p += 8) {
            uint64_t next[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) next[u] = keys(p + 8 + u);
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (p + u < a.parts) best.merge(k[u], lane);
#pragma unroll
            for (int u = 0; u < 8; ++u) k[u] = next[u];
        }
    }
    logprob_outputs(a, row, l, kHalf, all, lane, 64, own, best.key, true);
}

struct LogprobBackArgs {
    const void *l;
    const int64_t *tokens, *top_index;
    const float *stats, *entropy, *g_logp, *g_entropy, *g_top;
    void *gl;
    int64_t ldl, ldg, ignore;
    int vocab, count, top, parts, per;
};

template <class T, bool ONCE>
__global__ __launch_bounds__(256) void logprobs_back_kernel(const LogprobBackArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float part[4];
    const int64_t row = (int64_t)blockIdx.x / a.parts;
    const int which = (int)((int64_t)blockIdx.x - row * a.parts), from = which * a.per, to = min(a.vocab, from + a.per);
    const T *l = (const T *)a.l + row * a.ldl;
    T *gl = (T *)a.gl + row * a.ldg;
    const float m = a.stats[2 * row], logs = a.stats[2 * row + 1], gh = a.g_entropy ? a.g_entropy[row] : 0.0f, h = a.g_entropy ? a.entropy[row] : 0.0f;
    const int listed = (a.g_logp ? a.count : 0) + (a.g_top ? a.top : 0), given = a.g_logp ? a.count : 0;
    // token j of both lists: its place (-1: none) and gradient
    auto token = [&](int j, float &g) {
        const bool asked = j < given;
        const int64_t t = asked ? a.tokens[row * a.count + j] : a.top_index[row * a.top + j - given];
        g = asked ? a.g_logp[row * a.count + j] : a.g_top[row * a.top + j - given];
        return (asked && t == a.ignore) || t < 0 || t >= a.vocab ? -1 : (int)t;
    };
    float sum = 0.0f;
    for (int j = threadIdx.x; j < listed; j += 256) {
        float g;
        if (token(j, g) >= 0) sum += g;
    }
    sum = reduce_threads<256, false>(sum, part);
    const bool none = m == -__builtin_inff() && logs == 0.0f;
    const float constant = -fmaf(gh, h, sum), slope = -gh;
    // (p from d as it is, so that NaN goes through; beside it d is kept finite: p is 0 there)
    auto dense = [&](float x) {
        const float d = (x - m) - logs;
        return exp2_of(d * kLog2e) * fmaf(slope, fmaxf(d, -1e4f), constant);
    };
    // the tokens' own logits before anything is overwritten (up to 1088 of them), then the row, then the tokens
    constexpr int kEach = (1024 + IMUNPACK_LOGPROBS_TOP + 255) / 256;
    float own[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int j = threadIdx.x + 256 * u;
        float g;
        const int t = j < listed ? token(j, g) : -1;
        own[u] = t >= from && t < to ? (float)l[t] : 0.0f;
    }
    __syncthreads();
    auto turn = [&](int base, auto pieces, auto whole) __attribute__((always_inline)) {
        constexpr bool kWhole = decltype(whole)::value;
        constexpr int P = decltype(pieces)::value;
        piece_t<T, V> in[P];
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const int at = base + (u * 256 + (int)threadIdx.x) * V;
            in[u] = load_piece<T, V, ONCE>(l + at, kWhole ? V : to - at);
        }
#pragma unroll
        for (int u = 0; u < P; ++u) {
            const int at = base + (u * 256 + (int)threadIdx.x) * V;
            float f[V];
#pragma unroll
            for (int k = 0; k < V; ++k) f[k] = none ? 0.0f : dense((float)in[u][k]);
            if (kWhole || at < to) store_upto<T, V, ONCE>(gl + at, f, kWhole ? V : to - at);
        }
    };
    int base = from;
    using Some = std::integral_constant<int, kScanPieces>;
    using One = std::integral_constant<int, 1>;
    for (; base + 256 * V * kScanPieces <= to; base += 256 * V * kScanPieces) turn(base, Some(), std::true_type());
    for (; base + 256 * V <= to; base += 256 * V) turn(base, One(), std::true_type());
    if (base < to) turn(base, One(), std::false_type());
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int j = threadIdx.x + 256 * u;
        float g;
        const int t = j < listed ? token(j, g) : -1;
        if (t < from || t >= to || none) continue;
        bool first = true;
        float add = 0.0f;
        for (int i = 0; i < listed; ++i) {  // all gradients of one token, in the lists' order
            float gi;
            if (token(i, gi) != t) continue;
            if (i < j) first = false;
            add += gi;
        }
        if (first) gl[t] = (T)(dense(own[u]) + add);
    }
}

static bool logprob_sizes(int64_t rows, int64_t vocab, int64_t count, int64_t top, int dtype) {
    return rows >= 0 && rows < (1ll << 31) && vocab >= 1 && vocab <= (1 << 30) && count >= 0 && count <= 1024 && top >= 0 && top <= IMUNPACK_LOGPROBS_TOP && top <= vocab &&
           (dtype == IMUNPACK_F32 || dtype == IMUNPACK_BF16);
}
// How many workgroups share a row, and how much of it each takes (whole pieces).  Forward a part costs its own bound and sort, and what is in one part needs no join: 1024 workgroups, four to a
// CU, were the best of 512, 768, 1024, 1536 and 2048 (microseconds with five alternatives, 1024 and 2048: 130 x 128000 bfloat16 25, 31; 256 x 128000 28.5, 31.3; 614 x 50265 fp32 34.5, 39.4;
// 1000 x 32000 bfloat16 23.6, 29.7; 700 x 128000 50.6, 50.0).  Backward a part costs nothing: 2048 (614 x 50265 fp32 54.6, in 1024 59.5).
constexpr int kForwardGroups = 1024, kBackwardGroups = 2048;
struct Parts {
    int parts, per;
};
static Parts parts_of(int64_t rows, int64_t vocab, int dtype, int groups) {
    const int64_t piece = 256 * (dtype == IMUNPACK_F32 ? 4 : 8), pieces = (vocab + piece - 1) / piece;
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>((pieces + kScanPieces - 1) / kScanPieces, kMostParts), groups / std::max<int64_t>(rows, 1)));
    const int64_t each = (pieces + parts - 1) / parts;
    return {(int)((pieces + each - 1) / each), (int)std::min(each * piece, vocab)};
}
}  // namespace imu

using namespace imu;

extern "C" int imunpack_logprobs_workspace(int64_t rows, int64_t vocab, int64_t count, int64_t top, int dtype, size_t *bytes) {
    if (!logprob_sizes(rows, vocab, count, top, dtype) || !bytes) return IMUNPACK_EINVAL;
    const int64_t parts = parts_of(rows, vocab, dtype, kForwardGroups).parts;
    *bytes = parts == 1 ? 0 : (size_t)rows * (size_t)parts * ((size_t)top * sizeof(uint64_t) + 3 * sizeof(float));
    return IMUNPACK_OK;
}

extern "C" int imunpack_logprobs(const void *logits, int64_t ldl, int64_t rows, int64_t vocab, int dtype, const int64_t *tokens, int64_t count, int64_t ignore_index, int64_t top,
                                 float *logp, float *lse, float *stats, float *entropy, float *top_logp, int64_t *top_index, void *workspace, size_t workspace_bytes, imunpack_stream_t stream) {
    size_t need = 0;
    IMU_TRY(imunpack_logprobs_workspace(rows, vocab, count, top, dtype, &need));
    if (ldl < vocab) return IMUNPACK_EINVAL;
    if (rows == 0) return IMUNPACK_OK;
    if (!logits || (count && (!tokens || !logp)) || (top && (!top_logp || !top_index))) return IMUNPACK_EINVAL;
    if (need && (!workspace || ((uintptr_t)workspace & 15))) return IMUNPACK_EINVAL;
    if (workspace_bytes < need) return IMUNPACK_ESMALL;
    const int64_t size = dtype == IMUNPACK_F32 ? 4 : 2;
    const Parts p = parts_of(rows, vocab, dtype, kForwardGroups);
    const bool once = rows * vocab * size >= kLastLevelCache;
    const hipStream_t st = (hipStream_t)stream;
    for (int64_t r = 0; r < rows; r += kLogprobRows) {  // (one launch wherever a row has parts)
        const LogprobArgs a = {(const char *)logits + r * ldl * size, tokens ? tokens + r * count : nullptr, logp ? logp + r * count : nullptr, lse ? lse + r : nullptr,
                               stats ? stats + 2 * r : nullptr, entropy ? entropy + r : nullptr, top_logp ? top_logp + r * top : nullptr, top_index ? top_index + r * top : nullptr,
                               (float *)((uint64_t *)workspace + rows * p.parts * top), (uint64_t *)workspace, ldl, ignore_index, (int)vocab, (int)count, (int)top, p.parts, p.per};
        const int64_t some = std::min(kLogprobRows, rows - r);
        const dim3 grid((unsigned)(some * p.parts));
        auto typed = [&](auto t) {
            using T = decltype(t);
            if (top) hipLaunchKernelGGL((once ? logprobs_kernel<T, true, true> : logprobs_kernel<T, true, false>), grid, dim3(256), 0, st, a);
            else hipLaunchKernelGGL((once ? logprobs_kernel<T, false, true> : logprobs_kernel<T, false, false>), grid, dim3(256), 0, st, a);
            if (p.parts > 1) hipLaunchKernelGGL(logprobs_join_kernel<T>, dim3((unsigned)some), dim3(64), 0, st, a);
        };
        if (dtype == IMUNPACK_F32) typed(0.0f);
        else typed((__bf16)0.0f);
        IMU_TRY(launch_status());
    }
    return IMUNPACK_OK;
}

extern "C" int imunpack_logprobs_backward(const void *logits, int64_t ldl, int64_t rows, int64_t vocab, int dtype, const int64_t *tokens, int64_t count, int64_t ignore_index,
                                          int64_t top, const int64_t *top_index, const float *stats, const float *entropy, const float *g_logp, const float *g_entropy,
                                          const float *g_top, void *gl, int64_t ldg, imunpack_stream_t stream) {
    if (!logprob_sizes(rows, vocab, count, top, dtype) || ldl < vocab || ldg < vocab) return IMUNPACK_EINVAL;
    if (rows == 0) return IMUNPACK_OK;
    if (!logits || !stats || !gl || (g_logp && count && !tokens) || (g_entropy && !entropy) || (g_top && top && !top_index) || (gl == logits && ldg != ldl)) return IMUNPACK_EINVAL;
    const int64_t size = dtype == IMUNPACK_F32 ? 4 : 2;
    auto at = [](auto *p, int64_t k) { return p ? p + k : p; };
    const Parts p = parts_of(rows, vocab, dtype, kBackwardGroups);
    const bool once = 2 * rows * vocab * size >= kLastLevelCache * 3 / 4;
    for (int64_t r = 0; r < rows; r += kLogprobRows) {
        const LogprobBackArgs a = {(const char *)logits + r * ldl * size, at(tokens, r * count), at(top_index, r * top), stats + 2 * r, at(entropy, r), count ? at(g_logp, r * count) : nullptr,
                                   at(g_entropy, r), top ? at(g_top, r * top) : nullptr, (char *)gl + r * ldg * size, ldl, ldg, ignore_index, (int)vocab, (int)count, (int)top, p.parts, p.per};
        const dim3 grid((unsigned)(std::min(kLogprobRows, rows - r) * p.parts));
        if (dtype == IMUNPACK_F32) hipLaunchKernelGGL((once ? logprobs_back_kernel<float, true> : logprobs_back_kernel<float, false>), grid, dim3(256), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL((once ? logprobs_back_kernel<__bf16, true> : logprobs_back_kernel<__bf16, false>), grid, dim3(256), 0, (hipStream_t)stream, a);
        IMU_TRY(launch_status());
    }
    return IMUNPACK_OK;
}
