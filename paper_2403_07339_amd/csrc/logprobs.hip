// Log probabilities of given tokens, entropy and the largest alternatives of rows of logits, and their gradient.
//
//   m = max l,  S = sum exp(l - m),  A = sum exp(l - m) (l - m)       lse = m + log S,   entropy = log S - A / S
//   gl_v = sum_j g_j ([v = t_j] - p_v) - g_H p_v (l_v - lse + H)
//
// One pass over the row with the running maximum; where it moves by d <= 0, S -> S e^d, A -> e^d (A + d S).
#include "common.h"
#include "elements.h"

#include <algorithm>

namespace imu {
constexpr int64_t kLogprobRows = 1 << 22;  // of a launch

struct LogprobArgs {
    const void *l;
    const int64_t *tokens;
    float *logp, *lse, *stats, *entropy, *top_logp;
    int64_t *top_index;
    int64_t ldl, ignore;
    int vocab, count, top;
};

// Maximum, S and A of a part of a row.
struct Moments {
    float m = -__builtin_inff(), s = 0.0f, a = 0.0f;
    __device__ __forceinline__ void add(float x) {
        if (x == -__builtin_inff()) return;
        if (x > m) rebase(x);
        const float d = x - m, e = expf(d);
        s += e;
        if (e > 0.0f) a += e * d;  // (d may be -infinity: a logit of the type's lowest value)
    }
    __device__ __forceinline__ void rebase(float to) {
        const float d = m - to, e = expf(d);
        a = e > 0.0f ? e * fmaf(d, s, a) : 0.0f;
        s = e * s;
        m = to;
    }
    __device__ __forceinline__ void join(Moments o) {
        const float to = fmaxf(m, o.m);
        if (to == -__builtin_inff()) {  // (nothing, or NaN in s)
            s += o.s;
            a += o.a;
            return;
        }
        if (m < to) m == -__builtin_inff() ? (void)(m = to) : rebase(to);
        if (o.m < to) o.m == -__builtin_inff() ? (void)(o.m = to) : o.rebase(to);
        s += o.s;
        a += o.a;
    }
};
// The order of a logit among a row's: larger first, then the lower place.  NaN stands with -infinity.
__device__ __forceinline__ uint64_t order_of(float x, int place) {
    const uint32_t b = x == x ? __float_as_uint(x + 0.0f) : 0xff800000u;
    return ((uint64_t)(b >> 31 ? ~b : b | 0x80000000u) << 32) | (uint32_t)~place;
}

template <class T>
__global__ __launch_bounds__(256) void logprobs_kernel(const LogprobArgs a) {
    __shared__ float part[4][3];
    __shared__ uint64_t best[4];
    const int64_t row = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T *l = (const T *)a.l + row * a.ldl;
    Moments mine;
    for (int v = threadIdx.x; v < a.vocab; v += 256) mine.add((float)l[v]);
#pragma unroll
    for (int k = 32; k; k >>= 1) {
        Moments o;
        o.m = __shfl_xor(mine.m, k), o.s = __shfl_xor(mine.s, k), o.a = __shfl_xor(mine.a, k);
        mine.join(o);
    }
    if (lane == 0) part[wave][0] = mine.m, part[wave][1] = mine.s, part[wave][2] = mine.a;
    __syncthreads();
    Moments all;
    for (int w = 0; w < 4; ++w) {
        Moments o;
        o.m = part[w][0], o.s = part[w][1], o.a = part[w][2];
        all.join(o);
    }
    const bool none = all.m == -__builtin_inff() && all.s == 0.0f;
    // (log p = (l - m) - log S: m may be so large that log S is lost beside it)
    const float logs = none ? 0.0f : logf(all.s);
    auto logp = [&](int64_t v) { return none ? all.m : ((float)l[v] - all.m) - logs; };
    if (threadIdx.x == 0) {
        if (a.lse) a.lse[row] = all.m + logs;
        if (a.stats) a.stats[2 * row] = all.m, a.stats[2 * row + 1] = logs;
        if (a.entropy) a.entropy[row] = none ? 0.0f : logs - all.a / all.s;
    }
    for (int j = threadIdx.x; j < a.count; j += 256) {
        const int64_t t = a.tokens[row * a.count + j];
        a.logp[row * a.count + j] = t == a.ignore ? 0.0f : t < 0 || t >= a.vocab ? __builtin_nanf("") : logp(t);
    }
    uint64_t last = ~0ull;
    for (int k = 0; k < a.top; ++k) {
        uint64_t found = 0;
        for (int v = threadIdx.x; v < a.vocab; v += 256) {
            const uint64_t o = order_of((float)l[v], v);
            if (o < last && o > found) found = o;
        }
#pragma unroll
        for (int d = 32; d; d >>= 1) found = max(found, (uint64_t)__shfl_xor((unsigned long long)found, d));
        if (lane == 0) best[wave] = found;
        __syncthreads();
        last = max(max(best[0], best[1]), max(best[2], best[3]));
        __syncthreads();
        if (threadIdx.x == 0) {
            const int v = (int)~(uint32_t)last;
            a.top_index[row * a.top + k] = v;
            a.top_logp[row * a.top + k] = logp(v);
        }
    }
}

struct LogprobBackArgs {
    const void *l;
    const int64_t *tokens, *top_index;
    const float *stats, *entropy, *g_logp, *g_entropy, *g_top;
    void *gl;
    int64_t ldl, ldg, ignore;
    int vocab, count, top;
};

template <class T>
__global__ __launch_bounds__(256) void logprobs_back_kernel(const LogprobBackArgs a) {
    __shared__ float part[4];
    const int64_t row = blockIdx.x;
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
    auto dense = [&](float x) {
        const float d = (x - m) - logs, p = expf(d);
        return none || p == 0.0f ? 0.0f : -p * (sum + (a.g_entropy ? gh * (d + h) : 0.0f));
    };
    // the tokens' own logits before anything is overwritten (up to 1088 of them), then the row, then the tokens
    constexpr int kEach = (1024 + IMUNPACK_LOGPROBS_TOP + 255) / 256;
    float own[kEach];
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int j = threadIdx.x + 256 * u;
        float g;
        const int t = j < listed ? token(j, g) : -1;
        own[u] = t >= 0 ? (float)l[t] : 0.0f;
    }
    __syncthreads();
    for (int v = threadIdx.x; v < a.vocab; v += 256) gl[v] = (T)dense((float)l[v]);
    __syncthreads();
#pragma unroll
    for (int u = 0; u < kEach; ++u) {
        const int j = threadIdx.x + 256 * u;
        float g;
        const int t = j < listed ? token(j, g) : -1;
        if (t < 0 || none) continue;
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
}  // namespace imu

using namespace imu;

extern "C" int imunpack_logprobs_workspace(int64_t rows, int64_t vocab, int64_t count, int64_t top, int dtype, size_t *bytes) {
    if (!logprob_sizes(rows, vocab, count, top, dtype) || !bytes) return IMUNPACK_EINVAL;
    *bytes = 0;
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
    for (int64_t r = 0; r < rows; r += kLogprobRows) {
        const LogprobArgs a = {(const char *)logits + r * ldl * size, tokens ? tokens + r * count : nullptr, logp ? logp + r * count : nullptr, lse ? lse + r : nullptr, stats ? stats + 2 * r : nullptr,
                               entropy ? entropy + r : nullptr, top_logp ? top_logp + r * top : nullptr, top_index ? top_index + r * top : nullptr, ldl, ignore_index,
                               (int)vocab, (int)count, (int)top};
        const dim3 grid((unsigned)std::min(kLogprobRows, rows - r));
        if (dtype == IMUNPACK_F32) hipLaunchKernelGGL(logprobs_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL(logprobs_kernel<__bf16>, grid, dim3(256), 0, (hipStream_t)stream, a);
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
    for (int64_t r = 0; r < rows; r += kLogprobRows) {
        const LogprobBackArgs a = {(const char *)logits + r * ldl * size, at(tokens, r * count), at(top_index, r * top), stats + 2 * r, at(entropy, r), count ? at(g_logp, r * count) : nullptr,
                                   at(g_entropy, r), top ? at(g_top, r * top) : nullptr, (char *)gl + r * ldg * size, ldl, ldg, ignore_index, (int)vocab, (int)count, (int)top};
        const dim3 grid((unsigned)std::min(kLogprobRows, rows - r));
        if (dtype == IMUNPACK_F32) hipLaunchKernelGGL(logprobs_back_kernel<float>, grid, dim3(256), 0, (hipStream_t)stream, a);
        else hipLaunchKernelGGL(logprobs_back_kernel<__bf16>, grid, dim3(256), 0, (hipStream_t)stream, a);
        IMU_TRY(launch_status());
    }
    return IMUNPACK_OK;
}
