// Sums of a matrix's columns in fp32, what a bias adds to every row of an output has for its gradient.
//
//   out_c = sum_r x_rc
//
// Sixteen lanes take 256 bytes of a row, a workgroup's sixteen groups every sixteenth row of a part, which meet in LDS; the parts' sums are a matrix of few rows, and the
// same kernel adds them.  The order depends on the sizes alone, and nothing has to be cleared beforehand (a library's sum over many workgroups clears a counter, which in a
// captured graph went wrong on the second replay).
// Bound by memory; with few elements by the two launches.  12608 x 768 fp32 10.1 us (3.8 TB/s; a library sum 21.8), 2048 x 256 7.0 (11.0).
#include "common.h"
#include "elements.h"

#include <algorithm>

namespace imu {
constexpr int kSumParts = 256, kSumRows = 64, kSumGroups = 1024;  // parts at most, rows of a part at least, workgroups that fill the device

struct SumsArgs {
    const void *x;
    float *out;  // a row for each part
    int64_t ldx, rows, per;
    int cols, strips;
};

template <class T>
__global__ __launch_bounds__(256) void column_sums_kernel(const SumsArgs a) {
    constexpr int V = kVec<T>, U = 4;
    __shared__ __attribute__((aligned(16))) float sums[16][16 * V];
    const int l16 = threadIdx.x & 15, group = threadIdx.x >> 4, part = (int)blockIdx.x / a.strips, strip = (int)blockIdx.x - part * a.strips;
    const int col = (strip * 16 + l16) * V, have = a.cols - col;
    const int64_t from = part * a.per, to = min(a.rows, from + a.per);
    const T *x = (const T *)a.x + col;
    float s[V];
#pragma unroll
    for (int k = 0; k < V; ++k) s[k] = 0.0f;
    auto add = [&](const piece_t<T, V> &in) __attribute__((always_inline)) {
        float f[V];
        to_floats<T, V>(in, f);
#pragma unroll
        for (int k = 0; k < V; ++k) s[k] += f[k];
    };
    int64_t r = from + group;
    for (; r + 16 * (U - 1) < to; r += 16 * U) {
        piece_t<T, V> in[U];
#pragma unroll
        for (int u = 0; u < U; ++u) in[u] = load_piece<T, V>(x + (r + 16 * u) * a.ldx, have);
#pragma unroll
        for (int u = 0; u < U; ++u) add(in[u]);
    }
    for (; r < to; r += 16) add(load_piece<T, V>(x + r * a.ldx, have));
#pragma unroll
    for (int k = 0; k < V; ++k) sums[group][l16 * V + k] = s[k];
    __syncthreads();
    const int c = threadIdx.x, at = strip * 16 * V + c;
    if (c >= 16 * V || at >= a.cols) return;
    float all = sums[0][c];
#pragma unroll
    for (int g = 1; g < 16; ++g) all += sums[g][c];
    a.out[(int64_t)part * a.cols + at] = all;
}

static int sum_strips(int64_t cols, int dtype) { return (int)((cols + (dtype == IMUNPACK_F32 ? 63 : 127)) / (dtype == IMUNPACK_F32 ? 64 : 128)); }
static int64_t sum_rows(int64_t rows, int64_t cols, int dtype) {  // of a part
    const int64_t parts = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(kSumParts, rows / kSumRows), kSumGroups / sum_strips(cols, dtype)));
    return std::max<int64_t>(1, (rows + parts - 1) / parts);
}
}  // namespace imu

using namespace imu;

extern "C" int imunpack_column_sums_workspace(int64_t rows, int64_t cols, int dtype, size_t *bytes) {
    if (rows < 0 || rows > (1ll << 31) || cols < 1 || cols > (1 << 24) || (dtype != IMUNPACK_F32 && dtype != IMUNPACK_BF16) || !bytes) return IMUNPACK_EINVAL;
    const int64_t per = sum_rows(rows, cols, dtype), parts = (rows + per - 1) / per;
    *bytes = parts > 1 ? (size_t)parts * (size_t)cols * sizeof(float) : 0;
    return IMUNPACK_OK;
}

extern "C" int imunpack_column_sums(const void *x, int64_t ldx, int64_t rows, int64_t cols, int dtype, float *out, void *workspace, size_t workspace_bytes, imunpack_stream_t stream) {
    size_t need = 0;
    IMU_TRY(imunpack_column_sums_workspace(rows, cols, dtype, &need));
    if (ldx < cols || (rows && !x) || !out || (need && (!workspace || ((uintptr_t)workspace & 15)))) return IMUNPACK_EINVAL;
    if (workspace_bytes < need) return IMUNPACK_ESMALL;
    const int64_t per = sum_rows(rows, cols, dtype), parts = std::max<int64_t>(1, (rows + per - 1) / per);
    const hipStream_t st = (hipStream_t)stream;
    auto launch = [&](int type, const SumsArgs &a, int64_t groups) {
        if (type == IMUNPACK_F32) hipLaunchKernelGGL(column_sums_kernel<float>, dim3((unsigned)groups), dim3(256), 0, st, a);
        else hipLaunchKernelGGL(column_sums_kernel<__bf16>, dim3((unsigned)groups), dim3(256), 0, st, a);
        return launch_status();
    };
    const int strips = sum_strips(cols, dtype);
    IMU_TRY(launch(dtype, {x, need ? (float *)workspace : out, ldx, rows, per, (int)cols, strips}, parts * strips));
    if (!need) return IMUNPACK_OK;
    const int wide = sum_strips(cols, IMUNPACK_F32);
    return launch(IMUNPACK_F32, {workspace, out, cols, parts, parts, (int)cols, wide}, wide);
}
