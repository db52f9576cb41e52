// Layer norm of rows and its gradient.
//
// Forward, per row x of d values: mu = mean(x), v = mean((x - mu)^2),
// r = 1 / sqrt(v + eps), y = (x - mu) r w + b. Backward, with xh = (x - mu) r
// and g = dy w: dx = r (g - mean(g) - xh mean(g xh)); dw = sum over rows of
// dy xh, db = sum over rows of dy.
//
// Both are bound by memory (65,536 rows of 1,024 bfloat16 values: 48.5 us
// forward, 5.5 TB/s, some of it from the last-level cache; 84.2 us backward,
// 4.8 TB/s; a large copy reaches 5.2): a row is read once into registers (TPR threads, NV loads of 16 bytes each), its
// sums are taken in float32 over the values
// held (the variance from x - mu, so that a large mean costs no digits), and
// the result is written from the same registers. The backward pass keeps each
// thread's columns of dw and db in registers over all rows of its block and
// leaves one partial row per block, which a second kernel adds in block order:
// no atomics, so results do not depend on the schedule.
#include <algorithm>

#include "boa_ops.h"

using namespace boa;

namespace {

constexpr int THREADS = 256;
constexpr int64_t MAX_BLOCKS = 1024;   // of the backward pass: 4 per CU, each with one partial row of dw and db

struct NormArgs {
    const void *x, *dy, *w, *b;
    void *y;                     // forward: y; backward: dx
    float *mean, *rstd;
    float *partial;              // backward: blocks x 2 x d
    int64_t rows, x_stride, dy_stride;
    int32_t d;
    float eps;
};

// The arguments of the rows from `row` on that one launch takes.
template <class T>
NormArgs rows_from(NormArgs a, int64_t row)
{
    a.x = (const T *)a.x + row * a.x_stride;
    if (a.dy) a.dy = (const T *)a.dy + row * a.dy_stride;
    a.y = (T *)a.y + row * a.d;
    if (a.mean) a.mean += row;
    if (a.rstd) a.rstd += row;
    a.rows = std::min(LAUNCH_ROWS, a.rows - row);
    return a;
}

// A thread's columns of load i of a row: [c, c + VEC), moved back to end with
// the row where they would pass its end; the first `skip` of them are then
// another thread's too, or all (skip >= VEC). Every load is whole and within the
// row, with no branch around it. WHOLE: rows of whole loads, where skip is 0
// or at least VEC.
template <int VEC, int TPR>
struct Cols {
    int c, skip;
    __device__ Cols(int i, int lane, int32_t d)
    {
        const int c0 = (i * TPR + lane) * VEC;
        c = min(c0, d - VEC);
        skip = c0 - c;
    }
    __device__ bool any() const { return skip < VEC; }
    template <bool WHOLE>
    __device__ bool mine(int j) const { return WHOLE ? skip == 0 : j >= skip; }
};

// Sum of a value over the TPR threads of a row (a wave, or the block).
template <int TPR>
__device__ inline float row_sum(float v, float *red)
{
    v = wave_sum(v);
    if constexpr (TPR > 64) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[wave] = v;
        __syncthreads();
        v = 0.0f;
#pragma unroll
        for (int i = 0; i < TPR / 64; ++i) v += red[i];
    }
    return v;
}

// Two sums at once.
template <int TPR>
__device__ inline void row_sum2(float &a, float &b, float *red)
{
    a = wave_sum(a);
    b = wave_sum(b);
    if constexpr (TPR > 64) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) {
            red[wave] = a;
            red[4 + wave] = b;
        }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int i = 0; i < TPR / 64; ++i) {
            a += red[i];
            b += red[4 + i];
        }
    }
}

template <class T, class P, int NV, int TPR, bool WHOLE>
__global__ __launch_bounds__(THREADS) void norm_kernel(NormArgs a)
{
    constexpr int VEC = 16 / sizeof(T);
    __shared__ float red[8];
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (THREADS / TPR) + threadIdx.x / TPR;
    if (row >= a.rows) return;   // a whole wave (TPR 64) or block (TPR 256) leaves
    const int32_t d = a.d;
    const T *x = (const T *)a.x + row * a.x_stride;
    float v[NV][VEC];
    float s = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) load_loose<VEC, T>(v[i], x + Cols<VEC, TPR>(i, lane, d).c);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const Cols<VEC, TPR> at(i, lane, d);
#pragma unroll
        for (int j = 0; j < VEC; ++j) s += at.template mine<WHOLE>(j) ? v[i][j] : 0.0f;
    }
    const float mu = row_sum<TPR>(s, red) / (float)d;
    float q = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const Cols<VEC, TPR> at(i, lane, d);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            v[i][j] -= mu;
            const float t = at.template mine<WHOLE>(j) ? v[i][j] : 0.0f;
            q = fmaf(t, t, q);
        }
    }
    const float r = 1.0f / sqrtf(row_sum<TPR>(q, red) / (float)d + a.eps);
    if (lane == 0) {
        if (a.mean) a.mean[row] = mu;
        if (a.rstd) a.rstd[row] = r;
    }
    T *y = (T *)a.y + row * (int64_t)d;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const Cols<VEC, TPR> at(i, lane, d);
        float o[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j) o[j] = v[i][j] * r;
        if (a.w) {
            float w[VEC];
            load_loose<VEC, P>(w, (const P *)a.w + at.c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) o[j] *= w[j];
        }
        if (a.b) {
            float b[VEC];
            load_loose<VEC, P>(b, (const P *)a.b + at.c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) o[j] += b[j];
        }
        // two threads' common columns hold the same values
        if (at.any()) store_loose<VEC, T>(y + at.c, o);
    }
}

// Rows wider than the registers: a block per row, read three times (the
// second and third time from the caches).
template <class T, class P>
__global__ __launch_bounds__(THREADS) void norm_wide_kernel(NormArgs a)
{
    __shared__ float red[8];
    const int64_t row = blockIdx.x;
    const int32_t d = a.d;
    const T *x = (const T *)a.x + row * a.x_stride;
    T *y = (T *)a.y + row * (int64_t)d;
    float s = 0.0f;
    for (int c = threadIdx.x; c < d; c += THREADS) s += (float)x[c];
    const float mu = row_sum<THREADS>(s, red) / (float)d;
    float q = 0.0f;
    for (int c = threadIdx.x; c < d; c += THREADS) {
        const float t = (float)x[c] - mu;
        q = fmaf(t, t, q);
    }
    const float r = 1.0f / sqrtf(row_sum<THREADS>(q, red) / (float)d + a.eps);
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[row] = mu;
        if (a.rstd) a.rstd[row] = r;
    }
    for (int c = threadIdx.x; c < d; c += THREADS) {
        float o = ((float)x[c] - mu) * r;
        if (a.w) o *= (float)((const P *)a.w)[c];
        if (a.b) o += (float)((const P *)a.b)[c];
        y[c] = (T)o;
    }
}

// DP: dw and db are wanted.
template <class T, class P, int NV, int TPR, bool WHOLE, bool DP>
__global__ __launch_bounds__(THREADS) void norm_back_kernel(NormArgs a)
{
    constexpr int VEC = 16 / sizeof(T);
    __shared__ float red[8];
    extern __shared__ float cols[];   // 2 x d, where several rows share a block
    constexpr int GROUPS = THREADS / TPR;
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int32_t d = a.d;
    float w[NV][VEC], dw[NV][VEC], db[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const Cols<VEC, TPR> at(i, lane, d);
        if (a.w) load_loose<VEC, P>(w[i], (const P *)a.w + at.c);
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            // columns that are not this thread's count for nothing in the row's sums
            w[i][j] = !at.template mine<WHOLE>(j) ? 0.0f : a.w ? w[i][j] : 1.0f;
            dw[i][j] = db[i][j] = 0.0f;
        }
    }
    for (int64_t row = (int64_t)blockIdx.x * GROUPS + group; row < a.rows; row += (int64_t)gridDim.x * GROUPS) {
        const T *x = (const T *)a.x + row * a.x_stride;
        const T *dy = (const T *)a.dy + row * a.dy_stride;
        const float mu = a.mean[row], r = a.rstd[row];
        float xh[NV][VEC], g[NV][VEC];
        float c1 = 0.0f, c2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = Cols<VEC, TPR>(i, lane, d).c;
            load_loose<VEC, T>(xh[i], x + c);
            load_loose<VEC, T>(g[i], dy + c);
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                xh[i][j] = (xh[i][j] - mu) * r;
                if (DP) {
                    dw[i][j] = fmaf(g[i][j], xh[i][j], dw[i][j]);
                    db[i][j] += g[i][j];
                }
                g[i][j] *= w[i][j];
                c1 += g[i][j];
                c2 = fmaf(g[i][j], xh[i][j], c2);
            }
        }
        if (a.y) {
            row_sum2<TPR>(c1, c2, red);
            c1 /= (float)d;
            c2 /= (float)d;
            T *dx = (T *)a.y + row * (int64_t)d;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const Cols<VEC, TPR> at(i, lane, d);
                float o[VEC];
#pragma unroll
                for (int j = 0; j < VEC; ++j) o[j] = r * (g[i][j] - c1 - xh[i][j] * c2);
                if (WHOLE ? at.any() : at.skip == 0) {
                    store_loose<VEC, T>(dx + at.c, o);
                } else if (at.any()) {   // the first columns are the thread's before, whose g is here 0
#pragma unroll
                    for (int j = 0; j < VEC; ++j)
                        if (at.template mine<WHOLE>(j)) dx[at.c + j] = (T)o[j];
                }
            }
        }
    }
    if constexpr (DP) {
        float *out = a.partial + (int64_t)blockIdx.x * 2 * d;
        for (int k = 0; k < GROUPS; ++k) {   // the block's waves with a row each, added in order
            if (group == k) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const Cols<VEC, TPR> at(i, lane, d);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        if (!at.template mine<WHOLE>(j)) continue;
                        float *tw = (GROUPS == 1 ? out : cols) + at.c + j, *tb = tw + d;
                        *tw = k ? *tw + dw[i][j] : dw[i][j];
                        *tb = k ? *tb + db[i][j] : db[i][j];
                    }
                }
            }
            if (GROUPS > 1) __syncthreads();
        }
        if (GROUPS > 1)
            for (int c = threadIdx.x; c < 2 * d; c += THREADS) out[c] = cols[c];
    }
}

// Rows wider than the registers: dx by a block per row ...
template <class T, class P>
__global__ __launch_bounds__(THREADS) void norm_back_wide_kernel(NormArgs a)
{
    __shared__ float red[8];
    const int64_t row = blockIdx.x;
    const int32_t d = a.d;
    const T *x = (const T *)a.x + row * a.x_stride;
    const T *dy = (const T *)a.dy + row * a.dy_stride;
    const float mu = a.mean[row], r = a.rstd[row];
    float c1 = 0.0f, c2 = 0.0f;
    for (int c = threadIdx.x; c < d; c += THREADS) {
        const float g = (float)dy[c] * (a.w ? (float)((const P *)a.w)[c] : 1.0f);
        c1 += g;
        c2 = fmaf(g, ((float)x[c] - mu) * r, c2);
    }
    row_sum2<THREADS>(c1, c2, red);
    c1 /= (float)d;
    c2 /= (float)d;
    T *dx = (T *)a.y + row * (int64_t)d;
    for (int c = threadIdx.x; c < d; c += THREADS) {
        const float g = (float)dy[c] * (a.w ? (float)((const P *)a.w)[c] : 1.0f);
        dx[c] = (T)(r * (g - c1 - ((float)x[c] - mu) * r * c2));
    }
}

// ... and dw, db by a block per 256 columns and stripe of rows.
template <class T>
__global__ __launch_bounds__(THREADS) void norm_cols_kernel(NormArgs a)
{
    const int c = blockIdx.y * THREADS + threadIdx.x;
    const int32_t d = a.d;
    if (c >= d) return;
    float dw = 0.0f, db = 0.0f;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float g = (float)((const T *)a.dy)[row * a.dy_stride + c];
        const float xh = ((float)((const T *)a.x)[row * a.x_stride + c] - a.mean[row]) * a.rstd[row];
        dw = fmaf(g, xh, dw);
        db += g;
    }
    a.partial[(int64_t)blockIdx.x * 2 * d + c] = dw;
    a.partial[(int64_t)blockIdx.x * 2 * d + d + c] = db;
}

// Adds the blocks' partial rows: 16 columns of dw | db per block and 64 slices
// of the partial rows, so that even narrow rows spread over the GPU (20 us with
// 64 columns and 16 slices at 1,024 partial rows of 768, most of it waiting);
// then the slices in order.
constexpr int JOIN_COLS = 16, JOIN_SLICES = 64;

template <class P>
__global__ __launch_bounds__(JOIN_COLS * JOIN_SLICES) void norm_join_kernel(const float *partial, int32_t blocks, int32_t d,
                                                                          P *dw, P *db)
{
    __shared__ float part[JOIN_SLICES][JOIN_COLS + 1];
    const int col = threadIdx.x % JOIN_COLS, slice = threadIdx.x / JOIN_COLS;
    const int c = blockIdx.x * JOIN_COLS + col;
    float s = 0.0f;
    if (c < 2 * d)
#pragma unroll 4
        for (int i = slice; i < blocks; i += JOIN_SLICES) s += partial[(int64_t)i * 2 * d + c];
    part[slice][col] = s;
    __syncthreads();
    if (slice == 0 && c < 2 * d) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < JOIN_SLICES; ++i) s += part[i][col];
        if (c < d) {
            if (dw) dw[c] = (P)s;
        } else if (db) {
            db[c - d] = (P)s;
        }
    }
}

// Calls f(T{}, P{}) for an element type and a parameter type: the parameters
// have the rows' type or are float32.
template <class F>
int with_types(int32_t dtype, int32_t param, F f)
{
    if (dtype == BOA_T_F32) return f(0.0f, 0.0f);
    if (dtype == BOA_T_BF16) return param == BOA_T_F32 ? f(bf16_t{}, 0.0f) : f(bf16_t{}, bf16_t{});
    return param == BOA_T_F32 ? f(f16_t{}, 0.0f) : f(f16_t{}, f16_t{});
}

// The registers a row takes: f(NV, TPR, WHOLE) as compile-time constants. A
// wave per row up to 4 loads a lane, then a block per row; false where a row
// does not fit, or is shorter than a load.
template <int V>
struct Int {
    static constexpr int value = V;
};

template <int VEC, class F>
bool with_shape(int32_t d, F f)
{
    const int64_t n = ceil_div(d, VEC);
    if (d < VEC || n > 1024) return false;
    auto whole = [&](auto nv, auto tpr) { d % VEC ? f(nv, tpr, Int<0>{}) : f(nv, tpr, Int<1>{}); };
    if (n <= 64) whole(Int<1>{}, Int<64>{});
    else if (n <= 128) whole(Int<2>{}, Int<64>{});
    else if (n <= 192) whole(Int<3>{}, Int<64>{});
    else if (n <= 256) whole(Int<4>{}, Int<64>{});
    else if (n <= 512) whole(Int<2>{}, Int<256>{});
    else whole(Int<4>{}, Int<256>{});
    return true;
}

int check_norm(const char *what, const void *x, int64_t rows, int32_t d, int64_t x_stride, int32_t dtype, int32_t param,
               bool has_param)
{
    char msg[160];
    const char *why = nullptr;
    if (!dtype_known(dtype)) why = "unknown dtype";
    else if (has_param && param != dtype && param != BOA_T_F32) why = "parameters must have the rows' type or be float32";
    else if (rows < 0 || rows >= (int64_t)1 << 31) why = "rows out of range [0, 2^31)";
    else if (d < 1 || d > BOA_MAX_NORM_D) why = "d out of range [1, 2^20]";
    else if (rows > 1 && x_stride < d) why = "row stride smaller than d";
    else if (rows && !x) why = "NULL rows";
    if (!why) return BOA_OK;
    __builtin_snprintf(msg, sizeof(msg), "%s: %s", what, why);
    return set_error(BOA_EINVAL, msg);
}

int64_t back_blocks(int64_t rows, int32_t d)
{
    // As many partial rows as blocks: at most 4 per CU; fewer of few rows, so that
    // writing and adding them stays small beside reading the rows, and of rows
    // above 16,384 values, which fill the GPU with blocks of columns: 128 MB of
    // them at most.
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(MAX_BLOCKS, ((int64_t)1 << 24) / d));
    return std::max<int64_t>(1, std::min(most, ceil_div(rows, 8)));
}

}  // namespace

extern "C" {

int boa_layer_norm(const void *x, int64_t rows, int32_t d, int64_t x_stride, int32_t dtype, const void *weight,
                   const void *bias, int32_t param_dtype, float eps, void *y, float *mean, float *rstd, void *stream)
{
    if (int rc = check_norm("layer_norm", x, rows, d, x_stride, dtype, param_dtype, weight || bias)) return rc;
    if (!(eps >= 0.0f)) return set_error(BOA_EINVAL, "layer_norm: eps must not be negative");
    if (rows && !y) return set_error(BOA_EINVAL, "layer_norm: NULL output");
    if (rows == 0) return BOA_OK;
    NormArgs a{};
    a.x = x, a.w = weight, a.b = bias, a.y = y, a.mean = mean, a.rstd = rstd;
    a.rows = rows, a.x_stride = x_stride, a.d = d, a.eps = eps;
    hipStream_t st = (hipStream_t)stream;
    return with_types(dtype, (weight || bias) ? param_dtype : dtype, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        constexpr int VEC = 16 / sizeof(T);
        for (int64_t row = 0; row < rows; row += LAUNCH_ROWS) {
            const NormArgs n = rows_from<T>(a, row);
            const bool fits = with_shape<VEC>(d, [&](auto nv, auto tpr, auto whole) {
                constexpr int NV = decltype(nv)::value, TPR = decltype(tpr)::value;
                constexpr bool WHOLE = decltype(whole)::value;
                const int64_t blocks = ceil_div(n.rows, THREADS / TPR);
                norm_kernel<T, P, NV, TPR, WHOLE><<<dim3((uint32_t)blocks), THREADS, 0, st>>>(n);
            });
            if (!fits) norm_wide_kernel<T, P><<<dim3((uint32_t)n.rows), THREADS, 0, st>>>(n);
        }
        return launch_status("layer_norm");
    });
}

int64_t boa_layer_norm_backward_workspace(int64_t rows, int32_t d)
{
    if (rows < 0 || d < 1) return 0;
    return back_blocks(rows, d) * 2 * d * (int64_t)sizeof(float);
}

int boa_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int64_t x_stride, int64_t rows, int32_t d,
                            int32_t dtype, const void *weight, int32_t param_dtype, const float *mean,
                            const float *rstd, void *dx, void *dweight, void *dbias, void *workspace,
                            int64_t workspace_bytes, void *stream)
{
    const bool params = dweight || dbias;
    if (int rc = check_norm("layer_norm_backward", x, rows, d, x_stride, dtype, param_dtype, weight || params)) return rc;
    if (rows && (!dy || !mean || !rstd)) return set_error(BOA_EINVAL, "layer_norm_backward: NULL input");
    if (rows > 1 && dy_stride < d) return set_error(BOA_EINVAL, "layer_norm_backward: row stride smaller than d");
    if (params && (!workspace || !aligned(workspace, 16)
                   || workspace_bytes < boa_layer_norm_backward_workspace(rows, d)))
        return set_error(BOA_EINVAL, "layer_norm_backward: workspace missing, unaligned or too small");
    if (!params && (!dx || rows == 0)) return BOA_OK;
    NormArgs a{};
    a.x = x, a.dy = dy, a.w = weight, a.y = dx, a.mean = const_cast<float *>(mean), a.rstd = const_cast<float *>(rstd);
    a.rows = rows, a.x_stride = x_stride, a.dy_stride = dy_stride, a.d = d, a.partial = (float *)workspace;
    hipStream_t st = (hipStream_t)stream;
    return with_types(dtype, (weight || params) ? param_dtype : dtype, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        constexpr int VEC = 16 / sizeof(T);
        const int64_t blocks = back_blocks(rows, d);
        const bool fits = with_shape<VEC>(d, [&](auto nv, auto tpr, auto whole) {
            constexpr int NV = decltype(nv)::value, TPR = decltype(tpr)::value;
            constexpr bool WHOLE = decltype(whole)::value;
            const size_t lds = TPR < THREADS ? (size_t)2 * d * sizeof(float) : 0;
            if (params)
                norm_back_kernel<T, P, NV, TPR, WHOLE, true><<<dim3((uint32_t)blocks), THREADS, lds, st>>>(a);
            else
                norm_back_kernel<T, P, NV, TPR, WHOLE, false><<<dim3((uint32_t)blocks), THREADS, 0, st>>>(a);
        });
        if (!fits) {
            for (int64_t row = 0; dx && row < rows; row += LAUNCH_ROWS) {
                const NormArgs n = rows_from<T>(a, row);
                norm_back_wide_kernel<T, P><<<dim3((uint32_t)n.rows), THREADS, 0, st>>>(n);
            }
            if (params)
                norm_cols_kernel<T><<<dim3((uint32_t)blocks, (uint32_t)ceil_div(d, THREADS)), THREADS, 0, st>>>(a);
        }
        if (params)
            norm_join_kernel<P><<<dim3((uint32_t)ceil_div(2 * (int64_t)d, JOIN_COLS)), JOIN_COLS * JOIN_SLICES, 0, st>>>(
                (const float *)workspace, (int32_t)blocks, d, (P *)dweight, (P *)dbias);
        return launch_status("layer_norm_backward");
    });
}

}  // extern "C"
