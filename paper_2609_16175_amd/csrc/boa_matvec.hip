// Products of a few vectors with rows of 4-bit codes:
//   y[m][n] = sum_k x[m][k] w[n][k],  w = s q + o  or, without offsets, s (q - 8),
// one scale (and offset) per row and group of consecutive k.
#include <algorithm>

#include "boa_ops.h"

using namespace boa;

namespace {

struct VecArgs {
    const void *x;
    const uint8_t *codes;
    const void *scales, *offsets;
    void *y;
    int64_t rows, x_stride, codes_stride, scale_stride, y_stride;
    int32_t M, K, group, scale_dtype;
};

__device__ inline float load_any(const void *p, int64_t i, int32_t dtype)
{
    if (dtype == BOA_T_F32) return ((const float *)p)[i];
    if (dtype == BOA_T_BF16) return (float)((const bf16_t *)p)[i];
    return (float)((const f16_t *)p)[i];
}

// Any shape: a wave per row of codes, a byte (two values of k) per lane and
// step, MB vectors at a time.
template <class T, int MB>
__global__ __launch_bounds__(256) void rows4_any_kernel(VecArgs a)
{
    const int lane = threadIdx.x & 63;
    const int64_t n = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (n >= a.rows) return;
    const uint8_t *codes = a.codes + n * a.codes_stride;
    const int32_t bytes = (a.K + 1) / 2;
    for (int m0 = 0; m0 < a.M; m0 += MB) {
        float acc[MB];
#pragma unroll
        for (int m = 0; m < MB; ++m) acc[m] = 0.0f;
        for (int b = lane; b < bytes; b += 64) {
            const uint32_t c = codes[b];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int k = 2 * b + h;
                if (k >= a.K) continue;
                const int64_t at = n * a.scale_stride + k / a.group;
                const float s = load_any(a.scales, at, a.scale_dtype);
                const float q = (float)((c >> (4 * h)) & 15u);
                const float w = a.offsets ? fmaf(s, q, load_any(a.offsets, at, a.scale_dtype)) : s * (q - 8.0f);
#pragma unroll
                for (int m = 0; m < MB; ++m)
                    if (m0 + m < a.M) acc[m] = fmaf((float)((const T *)a.x)[(m0 + m) * a.x_stride + k], w, acc[m]);
            }
        }
#pragma unroll
        for (int m = 0; m < MB; ++m) {
            const float v = wave_sum(acc[m]);
            if (lane == 0 && m0 + m < a.M) ((T *)a.y)[(m0 + m) * a.y_stride + n] = (T)v;
        }
    }
}

template <class T>
int launch_rows4(const VecArgs &a, hipStream_t st)
{
    const dim3 grid((uint32_t)ceil_div(a.rows, 4));
    if (a.M == 1)
        rows4_any_kernel<T, 1><<<grid, 256, 0, st>>>(a);
    else
        rows4_any_kernel<T, 8><<<grid, 256, 0, st>>>(a);
    return launch_status("matvec_fourbit");
}

}  // namespace

extern "C" int boa_matvec_fourbit(const void *x, int64_t M, int64_t x_stride, int32_t dtype, const uint8_t *codes,
                                  int64_t rows, int32_t K, int64_t codes_stride, const void *scales,
                                  const void *offsets, int64_t scale_stride, int32_t scale_dtype, int32_t group,
                                  void *y, int64_t y_stride, void *stream)
{
    auto bad = [](const char *why) { return set_error(BOA_EINVAL, why); };
    if (!dtype_known(dtype) || !dtype_known(scale_dtype)) return bad("matvec_fourbit: unknown dtype");
    if (M < 0 || M > BOA_MAX_MATVEC_M) return bad("matvec_fourbit: M out of range [0, 65535]");
    if (rows < 0 || rows >= (int64_t)1 << 31) return bad("matvec_fourbit: rows out of range [0, 2^31)");
    if (K < 1 || K > BOA_MAX_MATVEC_K) return bad("matvec_fourbit: K out of range [1, 2^20]");
    if (group < 1) return bad("matvec_fourbit: group must be at least 1");
    if (codes_stride < (K + 1) / 2 && rows > 1) return bad("matvec_fourbit: stride of the codes smaller than a row");
    if (scale_stride < ceil_div(K, group) && rows > 1)
        return bad("matvec_fourbit: stride of the scales smaller than a row");
    if (M > 1 && (x_stride < K || y_stride < rows)) return bad("matvec_fourbit: row stride of x or y too small");
    if (M == 0 || rows == 0) return BOA_OK;
    if (!x || !codes || !scales || !y) return bad("matvec_fourbit: NULL input or output");
    VecArgs a{};
    a.x = x, a.codes = codes, a.scales = scales, a.offsets = offsets, a.y = y;
    a.rows = rows, a.x_stride = x_stride, a.codes_stride = codes_stride, a.scale_stride = scale_stride;
    a.y_stride = y_stride, a.M = (int32_t)M, a.K = K, a.group = group, a.scale_dtype = scale_dtype;
    hipStream_t st = (hipStream_t)stream;
    if (dtype == BOA_T_F32) return launch_rows4<float>(a, st);
    if (dtype == BOA_T_BF16) return launch_rows4<bf16_t>(a, st);
    return launch_rows4<f16_t>(a, st);
}
