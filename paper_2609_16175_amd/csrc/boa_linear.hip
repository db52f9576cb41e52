// Linear layers with bias, activation and residual in the product's epilogue,
// and their gradients.
//
//   z = x w^T + bias        y = act(z) + residual
//   dz = dy act'(z)         dx = dz w         dw = dz^T x         dbias = sum over rows of dz
//
// A few rows (serving) read the weights once and are bound by that; more are
// bound by the matrix instructions. 16-bit operands go there as they are, with
// float32 sums; z is kept for the backward pass in f16 (11 bits, infinite
// beyond its range, where every activation's slope is constant, and for relu never 0
// where z is above 0), and dz, an operand of two products, is rounded to the
// layer's type. Float32 operands become two f16
// parts of 11 bits each, scaled by a power of two per row (or per column, where
// the sum runs over rows) so that the largest value lies below 2^15: three
// products, each value exact to 2^-22 of itself or 2^-40 of its row's largest.
// That is 3 / 16 of the time of float32 instructions; z stays float32.
#include <algorithm>
#include <type_traits>

#include "boa_gemm.h"

using namespace boa;

namespace {

// ---------------------------------------------------------------------------
// activations

constexpr float LOG2E = 1.4426950408889634f;
constexpr float INV_SQRT_2PI = 0.39894228040143268f;
constexpr float SQRT_2_PI = 0.79788456080286536f;
constexpr float CUBE = 0.044715f;

// FINE: float32 layers, with the library's exponential. For 16 bits the hardware's
// exponential and reciprocal (2^-22 of their values), since in a product's
// epilogue every instruction counts.
template <bool FINE>
__device__ inline float sigmoid(float z)
{
    if constexpr (FINE) return 1.0f / (1.0f + expf(-z));
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-LOG2E * z));
}

// The share of the normal distribution above m = |z|, and e = e^(-z^2 / 2), for 16
// bits: t P(t) e with t = 1 / (1 + 0.292 m), P fitted over [0, 13.5] for the least maximum of
// the error against the smaller of 2e-7 and 2^-13 of the share. As float32 works it
// out it is good to 2^-20 of itself up to 1, 2^-19 up to 2 and 2^-14 beyond, below
// every 16-bit rounding of gelu. A fit to 1.5e-7 of 1 in place of the share, a term
// shorter, would pass float16's from z = -4 on, and takes as long.
__device__ inline float share_above(float m, float z, float &e)
{
    e = __builtin_amdgcn_exp2f(-0.5f * LOG2E * z * z);
    const float t = __builtin_amdgcn_rcpf(fmaf(0.292f, m, 1.0f));
    float s = fmaf(t, -0.086612165f, 0.27031502f);
    s = fmaf(t, s, -0.07571438f);
    s = fmaf(t, s, 0.17060435f);
    s = fmaf(t, s, 0.10396614f);
    s = fmaf(t, s, 0.117441036f);
    return s * t * e;
}

// The same for float32, each to a few roundings of itself wherever it is a normal
// number: t P(t) e with t = 1 / (1 + 0.26 m) and P the polynomial whose largest
// relative error over [0, 14.5] is least (2^-25, 2^-21 as float32 works it out), fitted to the
// distribution; e with what m^2 leaves out of a float32. (1 + erf(z / sqrt 2)) / 2
// would cancel below 0, to a tenth of the value at -5 and all of it from -5.5 on,
// and erfc(-z / sqrt 2) / 2 is off by z^2 2^-23. Forward, 10,000 x 768 x 1024: 88.3 us, with
// erfc 89.4, with erf 86.8.
__device__ inline float fine_share_above(float m, float &e)
{
    const float square = m * m;
    e = expf(-0.5f * square);
    e = fmaf(-0.5f * fmaf(m, m, -square), e, e);
    const float t = 1.0f / fmaf(0.26f, m, 1.0f);
    float s = fmaf(t, 0.030230144f, -0.15149373f);
    s = fmaf(t, s, 0.24873184f);
    s = fmaf(t, s, -0.14778788f);
    s = fmaf(t, s, 0.15875782f);
    s = fmaf(t, s, 0.05196519f);
    s = fmaf(t, s, 0.1027886f);
    s = fmaf(t, s, 0.103050984f);
    s = fmaf(t, s, 0.103757024f);
    return s * t * e;
}

// The normal distribution's function and density at z.
template <bool FINE>
__device__ inline void normal(float z, float &below, float &density)
{
    if constexpr (FINE) {
        const float above = fine_share_above(fminf(fabsf(z), 40.0f), density);   // beyond 14.5 nothing is left of e
        below = z > 0.0f ? 1.0f - above : above;
    } else {
        const float above = share_above(fabsf(z), z, density);
        below = z > 0.0f ? 1.0f - above : above;
    }
    density *= INV_SQRT_2PI;
}

// Activations and their slopes; an activation's limit at -inf is 0, a slope's far from 0 is 0 or 1.
template <bool FINE, int ACT>
__device__ inline float act_of(float z)
{
    float y;
    if constexpr (ACT == BOA_ACT_RELU) {
        return z > 0.0f ? z : z != z ? z : 0.0f;
    } else if constexpr (ACT == BOA_ACT_SILU) {
        y = z * sigmoid<FINE>(z);
    } else if constexpr (ACT == BOA_ACT_GELU && !FINE) {
        // max(z, 0) - |z| (1 - erf(|z| / sqrt 2)) / 2; beyond 40 the share is 0, and |z| could be infinite
        float e;
        const float m = fminf(fabsf(z), 40.0f);
        return fmaf(-m, share_above(m, z, e), fmaxf(z, 0.0f));
    } else if constexpr (ACT == BOA_ACT_GELU) {
        float below, density;
        normal<FINE>(z, below, density);
        y = z * below;
    } else if constexpr (ACT == BOA_ACT_GELU_TANH) {
        y = z * sigmoid<FINE>(2.0f * SQRT_2_PI * z * fmaf(CUBE * z, z, 1.0f));   // (1 + tanh u) / 2 = sigmoid(2 u)
    } else {
        return z;
    }
    return z == -INFINITY ? 0.0f : y;
}

template <bool FINE, int ACT>
__device__ inline float slope_of(float z)
{
    float s, far;
    if constexpr (ACT == BOA_ACT_RELU) {
        return z > 0.0f ? 1.0f : z != z ? z : 0.0f;
    } else if constexpr (ACT == BOA_ACT_SILU) {
        const float g = sigmoid<FINE>(z);
        s = fmaf(z * g, 1.0f - g, g), far = 100.0f;
    } else if constexpr (ACT == BOA_ACT_GELU) {
        float below, density;
        normal<FINE>(z, below, density);
        s = fmaf(z, density, below), far = 20.0f;
    } else if constexpr (ACT == BOA_ACT_GELU_TANH) {
        const float g = sigmoid<FINE>(2.0f * SQRT_2_PI * z * fmaf(CUBE * z, z, 1.0f));
        s = fmaf(z * g * (1.0f - g), 2.0f * SQRT_2_PI * fmaf(3.0f * CUBE * z, z, 1.0f), g), far = 20.0f;
    } else {
        return 1.0f;
    }
    return fabsf(z) > far ? (z > 0.0f ? 1.0f : 0.0f) : s;
}

// Calls f with the activation as a constant: one branch for many values.
template <int N>
struct Act {
    static constexpr int value = N;
};

template <class F>
__device__ inline void with_act(int32_t act, F f)
{
    switch (act) {
    case BOA_ACT_RELU: f(Act<BOA_ACT_RELU>{}); break;
    case BOA_ACT_SILU: f(Act<BOA_ACT_SILU>{}); break;
    case BOA_ACT_GELU: f(Act<BOA_ACT_GELU>{}); break;
    case BOA_ACT_GELU_TANH: f(Act<BOA_ACT_GELU_TANH>{}); break;
    default: f(Act<BOA_ACT_NONE>{});
    }
}

// ---------------------------------------------------------------------------
// epilogue

struct Epilogue {
    void *out;
    int64_t ld;
    const void *bias;
    int32_t bias_f32;
    const void *residual;
    int64_t residual_ld;
    void *pre;
    int32_t act;
    int32_t rows, cols;
    const float *max_a, *max_b;   // of scaled operands: the largest magnitudes
    float *partial;               // of splits: rows x pad8(cols) sums each, in place of all that
    int64_t partial_ld, partial_split;
};

// Power of two that brings magnitudes of up to m below 2^15.
__device__ inline int up(float m) { return 15 - __builtin_amdgcn_frexp_expf(m); }

template <class TO>
__device__ inline float bias_at(const Epilogue &e, int32_t q)
{
    return !e.bias ? 0.0f : e.bias_f32 ? ((const float *)e.bias)[q] : (float)((const TO *)e.bias)[q];
}

// What eight neighbouring columns keep over the rows that a lane finishes: their
// bias and scales (where the rows have all eight), and where the row's values are.
template <class TO>
struct Columns {
    typedef std::conditional_t<sizeof(TO) == 4, float, f16_t> Z;
    float bias[8];
    int shift[sizeof(TO) == 4 ? 8 : 1];
    TO *out;
    const TO *residual;
    Z *pre;
    int64_t out_step, residual_step, pre_step;
    __device__ void down() { out += out_step, residual += residual_step, pre += pre_step; }
};

template <class TO>
__device__ inline Columns<TO> columns_at(const Epilogue &e, int64_t p, int32_t q, int step)
{
    constexpr bool WIDE = sizeof(TO) == 4;
    Columns<TO> c;
    c.out = (TO *)e.out + p * e.ld + q, c.out_step = step * e.ld;
    c.residual = (const TO *)e.residual + p * e.residual_ld + q, c.residual_step = step * e.residual_ld;
    c.pre = (typename Columns<TO>::Z *)e.pre + p * e.cols + q, c.pre_step = (int64_t)step * e.cols;
    const bool whole = q + 8 <= e.cols;
    if (!e.bias) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c.bias[i] = 0.0f;
    } else if (whole && (e.bias_f32 || WIDE)) {
        load_loose<8, float>(c.bias, (const float *)e.bias + q);
    } else if (whole) {
        if constexpr (!WIDE) load_loose<8, TO>(c.bias, (const TO *)e.bias + q);
    }
    if constexpr (WIDE) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c.shift[i] = e.max_b && q + i < e.cols ? up(e.max_b[q + i]) : 0;
    }
    return c;
}

// z as it is kept. relu's slope is 1 above 0 however near, and a float16 that
// rounded to 0 would not say so: such z are kept as its smallest value. The other
// slopes are the same there and at 0 to 2^-24.
template <class Z, int ACT>
__device__ inline float to_keep(float z)
{
    if constexpr (sizeof(Z) == 2 && ACT == BOA_ACT_RELU) return z > 0.0f ? fmaxf(z, 0x1p-24f) : z;
    return z;
}

// One value, at row p and column q.
template <class TO, int ACT>
__device__ inline void finish_one(const Epilogue &e, int64_t p, int32_t q, float v, float bias)
{
    typedef std::conditional_t<sizeof(TO) == 4, float, f16_t> Z;
    v += bias;
    if (e.pre) ((Z *)e.pre)[p * e.cols + q] = (Z)to_keep<Z, ACT>(v);
    v = act_of<sizeof(TO) == 4, ACT>(v);
    if (e.residual) v += (float)((const TO *)e.residual)[p * e.residual_ld + q];
    ((TO *)e.out)[p * e.ld + q] = (TO)v;
}

template <class E>
__device__ inline void store8(E *to, const float (&v)[8])
{
    if constexpr (sizeof(E) == 4) {
        store_loose<4, E>(to, *(const float(*)[4])v);
        store_loose<4, E>(to + 4, *(const float(*)[4])(v + 4));
    } else {
        store_loose<8, E>(to, v);
    }
}

// Eight sums from column q on, of which the row may have fewer.
template <class TO, int ACT>
__device__ inline void finish_run(const Epilogue &e, int64_t p, int32_t q, const float *sums, const Columns<TO> &c)
{
    constexpr bool WIDE = sizeof(TO) == 4;
    const int s = WIDE && e.max_a ? up(e.max_a[p]) : 0;
    if (q + 8 > e.cols) {
#pragma unroll 1
        for (int i = 0; q + i < e.cols; ++i) {
            float v = sums[i];
            if constexpr (WIDE) v = ldexpf(v, e.max_a ? -(s + up(e.max_b[q + i])) : 0);
            finish_one<TO, ACT>(e, p, q + i, v, bias_at<TO>(e, q + i));
        }
        return;
    }
    words4 r[sizeof(TO) / 2];   // asked for before the sums are worked on
    if (e.residual) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(TO) / 2; ++i) r[i] = ((const loose4 *)c.residual)[i];
    }
    float v[8];
    load_f32<4, float>(*(float(*)[4])v, sums);
    load_f32<4, float>(*(float(*)[4])(v + 4), sums + 4);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (WIDE) v[i] = ldexpf(v[i], -(s + c.shift[i]));
        v[i] += c.bias[i];
    }
    if (e.pre) {
        float z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = to_keep<typename Columns<TO>::Z, ACT>(v[i]);
        store8(c.pre, z);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = act_of<WIDE, ACT>(v[i]);
    if (e.residual) {
        typedef Pack<8, TO> P8;
        struct Both {
            words4 w[sizeof(TO) / 2];
        } both;
#pragma unroll
        for (int i = 0; i < (int)sizeof(TO) / 2; ++i) both.w[i] = r[i];
        const P8 t = __builtin_bit_cast(P8, both);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] += (float)t.v[i];
    }
    store8(c.out, v);
}

// A forward product (both operands along k) has the whole epilogue, the
// gradients' none. 32,768 x 1024 x 4096 in bfloat16: forward 398 us, 230 of them
// products and the rest the writing of y and z at the memory's rate; dx 265, dw
// 263 (1,040 TFLOP/s). 10,000 x 768 x 1024 as parts: 76, 57, 63 (630 to 830).
template <class S, bool ACROSS_A, bool ACROSS_B, class TO>
__device__ inline void product_block(const Product &pr, const Epilogue &e, const Place &w, char *lds)
{
    f32x16 acc[S::TB][S::TA];
    clear<S>(acc);
    if (!tile_product<S, ACROSS_A, ACROSS_B, sizeof(TO) == 4>(pr, w, (typename S::T *)lds, acc)) return;
    if (e.partial) {
        float *out = e.partial + w.split * e.partial_split;
        each_run<S>(w, acc, lds, [](int32_t, int32_t, int) { return Nothing{}; }, [&](int32_t p, int32_t q, const float *v, const Nothing &) {
            if (p >= e.rows || q >= e.cols) return;
            float *to = out + p * e.partial_ld + q;
            *(f32x4 *)to = *(const f32x4 *)v;
            *(f32x4 *)(to + 4) = *(const f32x4 *)(v + 4);
        });
        return;
    }
    auto all = [&](auto act) {
        each_run<S>(w, acc, lds, [&](int32_t p, int32_t q, int step) { return columns_at<TO>(e, p, q, step); },
            [&](int32_t p, int32_t q, const float *v, const Columns<TO> &c) {
                if (p < e.rows && q < e.cols) finish_run<TO, decltype(act)::value>(e, p, q, v, c);
            });
    };
    if constexpr (ACROSS_A || ACROSS_B) all(Act<BOA_ACT_NONE>{});
    else with_act(e.act, all);
}

template <class S, bool ACROSS_A, bool ACROSS_B, class TO>
__global__ __launch_bounds__(S::THREADS, S::WAVES_PER_SIMD) void product_kernel(Product pr, Epilogue e)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    product_block<S, ACROSS_A, ACROSS_B, TO>(pr, e, place_of(pr, blockIdx.x, gridDim.x), lds);
}

// Both gradients' products in one launch, where their tiles fit on the GPU
// together and neither sum is so long that splits of it would be faster: the first
// `blocks` for dx, the others for dw. M x K x N in bfloat16, one launch and two: 200
// x 768 x 768 7.0 and 11.3 us, 1000 x 2048 x 768 15.6 and 18.8, 2000 x 768 x 768
// 18.3 and 20.1; beyond PAIR_STAGES 4000 x 512 x 512 32 and 19. float32, with its
// copies: 200 x 768 x 768 32 and 34, 1000 x 1024 x 1024 46 and 51, 4000 x 512 x 512
// 92 and 63.
constexpr int PAIR_STAGES = 32;

template <class S, class TO>
__global__ __launch_bounds__(S::THREADS, S::WAVES_PER_SIMD) void pair_kernel(Product dx, Epilogue ex, Product dw, Epilogue ew, uint32_t blocks)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    if (blockIdx.x < blocks) product_block<S, false, true, TO>(dx, ex, place_of(dx, blockIdx.x, blocks), lds);
    else product_block<S, true, true, TO>(dw, ew, place_of(dw, blockIdx.x - blocks, gridDim.x - blocks), lds);
}

// The sum of the splits' shares, in their order; bound by memory (4 splits of 4096
// x 1024: 13 us, 5.8 TB/s).
template <class TO>
__global__ __launch_bounds__(256) void product_join_kernel(Epilogue e, int32_t splits)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, runs = e.partial_ld / 8;
    const int64_t p = i / runs;
    const int32_t q = (int32_t)(i % runs) * 8;
    if (p >= e.rows) return;
    f32x4 v0 = {0.0f, 0.0f, 0.0f, 0.0f}, v1 = v0;
    const float *from = e.partial + p * e.partial_ld + q;
#pragma unroll 4
    for (int s = 0; s < splits; ++s) {
        v0 += *(const f32x4 *)(from + s * e.partial_split);
        v1 += *(const f32x4 *)(from + s * e.partial_split + 4);
    }
    __shared__ __attribute__((aligned(16))) float sums[256 * 8];
    float *mine = sums + threadIdx.x * 8;
    *(f32x4 *)mine = v0;
    *(f32x4 *)(mine + 4) = v1;
    with_act(e.act, [&](auto act) { finish_run<TO, decltype(act)::value>(e, p, q, mine, columns_at<TO>(e, p, q, 0)); });
}

// ---------------------------------------------------------------------------
// operands that cannot be read in place

// rows x cols, `ld` apart, to rows of pad8(cols) with zeros at the end
struct CopyArgs {
    const void *src;
    void *dst;
    int64_t ld, rows;
    int32_t cols, pad;
    int32_t across;   // of parts by column: log2 of the threads along a row
    float *most;   // of parts: the largest magnitude per row or column
};

// What one launch copies: a job for each blockIdx.z.
struct CopyJobs {
    CopyArgs job[3];
    int32_t n;
    uint32_t x, y;   // blocks that the largest of them takes
    void add(const CopyArgs &c, int64_t nx, int64_t ny)
    {
        job[n++] = c;
        x = std::max(x, (uint32_t)nx), y = std::max(y, (uint32_t)ny);
    }
    dim3 grid() const { return dim3(x, y, (uint32_t)n); }
};

// Bound by memory: x and w of 9,973 x 413 x 777 in float16 take 5.8 us.
template <class T>
__global__ __launch_bounds__(256) void pad_kernel(CopyJobs jobs)
{
    const CopyArgs &a = jobs.job[blockIdx.z];
    const int64_t chunks = a.pad / 8, n = a.rows * chunks;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / chunks;
        const int32_t c = (int32_t)(i % chunks) * 8;
        const T *from = (const T *)a.src + r * a.ld + c;
        words4 w;
        if (c + 8 <= a.cols) {
            w = *(const loose4 *)from;
        } else {
            Pack<8, T> t;
#pragma unroll
            for (int e = 0; e < 8; ++e) t.v[e] = c + e < a.cols ? from[e] : (T)0.0f;
            w = __builtin_bit_cast(words4, t);
        }
        *(words4 *)((T *)a.dst + r * a.pad + c) = w;
    }
}

__device__ inline float finite_abs(float v) { return fabsf(v) < INFINITY ? fabsf(v) : 0.0f; }

__device__ inline void read8(float (&v)[8], const float *from, int32_t c, int32_t cols)
{
    if (c + 8 <= cols) {
        load_loose<8, float>(v, from + c);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? from[c + e] : 0.0f;
    }
}

// eight values as two parts; s: their exponents' shifts
__device__ inline void write_parts(const float (&v)[8], const int (&s)[8], f16_t *to, int64_t part)
{
    f16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float t = ldexpf(v[e], s[e]);
        hi[e] = (f16_t)t;
        lo[e] = (f16_t)(fabsf(t) < INFINITY ? t - (float)hi[e] : 0.0f);
    }
    *(f16x8 *)to = hi;
    *(f16x8 *)(to + part) = lo;
}

// Parts scaled by row, whose 32 values of the first and of the second part
// alternate, up to `pad` of each: a wave per row, which it reads twice (the second
// time from the cache). Bound by memory: x, w and dz of 10,000 x 768 x 1024 take 34
// us, 4.4 TB/s.
__global__ __launch_bounds__(256) void row_parts_kernel(CopyJobs jobs)
{
    const CopyArgs &a = jobs.job[blockIdx.z];
    const int lane = threadIdx.x & 63;
    for (int64_t r = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); r < a.rows; r += (int64_t)gridDim.x * 4) {
        const float *from = (const float *)a.src + r * a.ld;
        float m = 0.0f;
        for (int32_t c = lane * 8; c < a.cols; c += 512) {
            float v[8];
            read8(v, from, c, a.cols);
#pragma unroll
            for (int e = 0; e < 8; ++e) m = fmaxf(m, finite_abs(v[e]));
        }
        m = wave_max(m);
        if (lane == 0) a.most[r] = m;
        const int u = up(m), s[8] = {u, u, u, u, u, u, u, u};
        for (int32_t c = lane * 8; c < a.pad; c += 512) {
            float v[8];
            read8(v, from, c, a.cols);
            write_parts(v, s, (f16_t *)a.dst + r * 2 * a.pad + c / 32 * 64 + c % 32, 32);
        }
    }
}

template <class T>
__global__ __launch_bounds__(256) void zero_kernel(T *p, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = (T)0.0f;
}

// Largest magnitudes per column: the maximum of bit patterns, whose order does not
// matter. x and w of 10,000 x 768 x 1024: 16 us, latency.
__global__ __launch_bounds__(256) void col_max_kernel(CopyJobs jobs)
{
    const CopyArgs &a = jobs.job[blockIdx.z];
    const int32_t c = blockIdx.x * 256 + threadIdx.x;
    if (c >= a.cols) return;
    float m = 0.0f;
#pragma unroll 8
    for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) m = fmaxf(m, finite_abs(((const float *)a.src)[r * a.ld + c]));
    if (m > 0.0f) atomicMax((uint32_t *)a.most + c, __float_as_uint(m));
}

// Parts scaled by column: 32 rows of the first part and of the second
// alternate, with rows of zeros at the end. A thread has 8 columns, whose scales
// it works out once, of every few rows: of a block's threads 2^across lie side by
// side. Bound by memory: x, w and dz of 10,000 x 768 x 1024 take 48 us in one launch,
// 43 in three that leave the GPU idle between them (62 with the scales worked out at
// every run).
__global__ __launch_bounds__(256) void col_parts_kernel(CopyJobs jobs)
{
    const CopyArgs &a = jobs.job[blockIdx.z];
    const int32_t c = ((int32_t)(blockIdx.x << a.across) + (threadIdx.x & ((1 << a.across) - 1))) * 8, step = 256 >> a.across;
    if (c >= a.pad) return;
    int s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = c + e < a.cols ? up(a.most[c + e]) : 0;
    const int64_t deep = (a.rows + 31) / 32 * 32;
#pragma unroll 4
    for (int64_t r = (int64_t)blockIdx.y * step + (threadIdx.x >> a.across); r < deep; r += (int64_t)gridDim.y * step) {
        float v[8];
        read8(v, (const float *)a.src + min(r, a.rows - 1) * a.ld, c, a.cols);
        if (r >= a.rows)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.0f;
        write_parts(v, s, (f16_t *)a.dst + (r / 32 * 64 + r % 32) * a.pad + c, 32 * (int64_t)a.pad);
    }
}

// ---------------------------------------------------------------------------
// gradient of z

struct SlopeArgs {
    const void *dy, *pre;
    void *dz;          // rows of `pad` values, or null
    float *partial;    // stripes x N sums over rows, or null
    float *most;       // N: the columns' largest magnitudes (zeros at first), or null
    int64_t M, ld;
    int32_t N, pad, act;
};

// dz = dy act'(z), its sums over the rows of a stripe and, of float32, the columns'
// largest magnitudes. A thread has VEC columns of every 8th row of its block's.
// Bound by memory: 32,768 x 4096 in bfloat16 168 us, 4.8 TB/s.
template <class T>
__global__ __launch_bounds__(256) void slope_kernel(SlopeArgs a)
{
    typedef std::conditional_t<sizeof(T) == 4, float, f16_t> Z;
    constexpr int VEC = 8;
    __shared__ float sums[8][32 * VEC];
    const int col = threadIdx.x & 31, part = threadIdx.x >> 5;
    const int32_t c = (blockIdx.x * 32 + col) * VEC;
    float s[VEC] = {}, m[VEC] = {};
    if (c < a.N) {
        const bool whole = c + VEC <= a.N;
        for (int64_t r = (int64_t)blockIdx.y * 8 + part; r < a.M; r += (int64_t)gridDim.y * 8) {
            const T *dy = (const T *)a.dy + r * a.ld + c;
            const Z *z = (const Z *)a.pre + r * a.N + c;
            float g[VEC], x[VEC];
            if (whole) {
                load_loose<VEC, T>(g, dy);
                if (a.act) load_loose<VEC, Z>(x, z);
            } else {
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    g[e] = c + e < a.N ? (float)dy[e] : 0.0f;
                    x[e] = a.act && c + e < a.N ? (float)z[e] : 0.0f;
                }
            }
            if (a.act)
                with_act(a.act, [&](auto act) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) g[e] *= slope_of<sizeof(T) == 4, decltype(act)::value>(x[e]);
                });
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                s[e] += g[e];
                if (sizeof(T) == 4) m[e] = fmaxf(m[e], finite_abs(g[e]));
            }
            if (a.dz) {   // rows have room for whole runs
                T *to = (T *)a.dz + r * a.pad + c;
                if constexpr (sizeof(T) == 4) {
                    store_f32<4, T>(to, *(float(*)[4])g);
                    store_f32<4, T>(to + 4, *(float(*)[4])(g + 4));
                } else {
                    store_f32<VEC, T>(to, g);
                }
            }
        }
    }
    const int32_t mine = blockIdx.x * 32 * VEC + threadIdx.x;
    const int at = (threadIdx.x % VEC) * 32 + threadIdx.x / VEC;
    if (a.partial) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) sums[part][e * 32 + col] = s[e];
        __syncthreads();
        if (mine < a.N) {
            float t = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) t += sums[k][at];
            a.partial[(int64_t)blockIdx.y * a.N + mine] = t;
        }
        __syncthreads();
    }
    if (sizeof(T) == 4 && a.most) {   // the maximum of bit patterns, whose order does not matter
#pragma unroll
        for (int e = 0; e < VEC; ++e) sums[part][e * 32 + col] = m[e];
        __syncthreads();
        if (mine < a.N) {
            float t = 0.0f;
#pragma unroll
            for (int k = 0; k < 8; ++k) t = fmaxf(t, sums[k][at]);
            atomicMax((uint32_t *)a.most + mine, __float_as_uint(t));
        }
    }
}

// Adds the stripes' sums: 16 columns a block and 16 slices of the stripes (128 of
// 4,096 columns: 4.9 us).
template <class P>
__global__ __launch_bounds__(256) void bias_join_kernel(const float *partial, int32_t stripes, int32_t N, P *db)
{
    __shared__ float part[16][17];
    const int col = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const int32_t c = blockIdx.x * 16 + col;
    float s = 0.0f;
    if (c < N)
#pragma unroll 4
        for (int i = slice; i < stripes; i += 16) s += partial[(int64_t)i * N + c];
    part[slice][col] = s;
    __syncthreads();
    if (slice == 0 && c < N) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += part[i][col];
        db[c] = (P)s;
    }
}

// ---------------------------------------------------------------------------
// a few rows

struct FewArgs {
    const void *x, *w;
    int64_t x_ld, w_ld;
    int32_t M, N, K;
    Epilogue e;
};

constexpr int FEW_WAVES = 16, FEW_MOST = 8;   // FEW_MOST x 16 rows of x at most

// What a lane gives to the matrix instructions at a time: 16 bytes of a row, 8
// values of 16 bits for one of them or 4 float32 values for four (whose k are
// then not in their order, which the sum does not mind).
template <class T>
struct Few {
    typedef typename Vec<T>::v8 V;
    static constexpr int PER = 8;
    static __device__ f32x4 times(V w, V x, f32x4 acc) { return mfma16(w, x, acc); }
};
template <>
struct Few<float> {
    typedef f32x4 V;
    static constexpr int PER = 4;
    static __device__ f32x4 times(V w, V x, f32x4 acc)
    {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], x[e], acc, 0, 0, 0);
        return acc;
    }
};

// 16 rows of weights and 16 MT of x a block; its 16 waves share k and their sums
// are added through LDS in order. Fragments come straight from memory: every weight
// is read once, every state by each block from the cache. Rows past the end are
// read as the last one, and what they give is dropped. Bound by memory where there
// are blocks enough (1 x 4096 x 4096: 7.2 us in bfloat16, 15.5 in float32, 4.3 to
// 4.7 TB/s), else by the latency of a block's k (1 x 768 x 768: 3.5 and 4.3 us; 1 x
// 4096 x 1024: 6.7 and 11.8). Blocks of 8 or 4 rows of weights, of which there are
// more, take as long or longer: a wave asks for as many lines.
template <class T, int MT>
__global__ __launch_bounds__(64 * FEW_WAVES) void few_kernel(FewArgs a)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    typedef typename Few<T>::V V;
    constexpr int PER = Few<T>::PER, STEP = 4 * PER;   // k of a step
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, part = lane >> 4;
    const int32_t n0 = blockIdx.x * 16;
    const T *w = (const T *)a.w + (int64_t)min(n0 + r, a.N - 1) * a.w_ld;
    const T *x[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) x[j] = (const T *)a.x + (int64_t)min(j * 16 + r, a.M - 1) * a.x_ld;
    const int32_t whole = a.K / STEP, each = (whole + FEW_WAVES - 1) / FEW_WAVES;
    const int32_t end = min(whole, (wave + 1) * each);
    auto get = [](const T *p) { return __builtin_bit_cast(V, (words4) * (const loose4 *)p); };
    f32x4 acc[MT];
#pragma unroll
    for (int j = 0; j < MT; ++j) acc[j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    constexpr int AHEAD = MT == 1 ? 8 : MT == 2 ? 4 : MT == 4 ? 2 : 1;   // steps whose loads are on their way together
    for (int32_t s = wave * each; s < end; s += AHEAD) {
        V fw[AHEAD], fx[AHEAD][MT];
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (s + u < end) {
                const int32_t k = (s + u) * STEP + part * PER;
                fw[u] = get(w + k);
#pragma unroll
                for (int j = 0; j < MT; ++j) fx[u][j] = get(x[j] + k);
            }
#pragma unroll
        for (int u = 0; u < AHEAD; ++u)
            if (s + u < end) {
#pragma unroll
                for (int j = 0; j < MT; ++j) acc[j] = Few<T>::times(fw[u], fx[u][j], acc[j]);
            }
    }
    if (a.K % STEP && wave == FEW_WAVES - 1) {   // the last values of k, zeros past them
        auto some = [&](const T *p) {
            V f;
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const int32_t k = whole * STEP + part * PER + e;
                f[e] = k < a.K ? p[k] : (T)0.0f;
            }
            return f;
        };
        const V fw = some(w);
#pragma unroll
        for (int j = 0; j < MT; ++j) acc[j] = Few<T>::times(fw, some(x[j]), acc[j]);
    }
    float *sums = (float *)lds;   // [wave][row of x][row of w]
#pragma unroll
    for (int j = 0; j < MT; ++j) *(f32x4 *)(sums + ((wave * MT + j) * 16 + r) * 16 + part * 4) = acc[j];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * 256; i += 64 * FEW_WAVES) {
        float v = 0.0f;
#pragma unroll
        for (int k = 0; k < FEW_WAVES; ++k) v += sums[k * MT * 256 + i];
        const int32_t m = i >> 4, n = n0 + (i & 15);
        if (m < a.M && n < a.N) {
            const float bias = bias_at<T>(a.e, n);
            with_act(a.e.act, [&](auto act) { finish_one<T, decltype(act)::value>(a.e, m, n, v, bias); });
        }
    }
}

// ---------------------------------------------------------------------------
// host

bool in_place(const void *p, int64_t ld, int64_t rows, int64_t cols)
{
    return aligned(p, 16) && cols % 8 == 0 && (rows <= 1 || (ld % 8 == 0 && ld < 1 << 21));
}

template <class S, bool ACROSS_A, bool ACROSS_B, class TO>
void launch(Product pr, const Epilogue &e, hipStream_t st)
{
    pr.tiles_a = (int32_t)ceil_div(pr.a.own, S::BA);
    pr.tiles_b = (int32_t)ceil_div(pr.b.own, S::BB);
    const auto kernel = product_kernel<S, ACROSS_A, ACROSS_B, TO>;
    if (S::LDS > 64 << 10)   // has to be asked for
        (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
    in_launches((int64_t)pr.tiles_a * pr.tiles_b * pr.splits, S::THREADS, [&](uint32_t first, uint32_t blocks) {
        pr.first = first;
        kernel<<<dim3(blocks), S::THREADS, S::LDS, st>>>(pr, e);
    });
}

// out = a b^T with its epilogue; T: the operands' type in the product, TO: the layer's.
template <class T, class TO, bool ACROSS_A, bool ACROSS_B>
void product(Operand a, Operand b, int32_t K, Epilogue e, Arena &mem, bool run, hipStream_t st, bool small = false)
{
    const Cut cut = small ? Cut{SMALL, 1, (int32_t)ceil_div(K, sizeof(TO) == 4 ? 32 : 64)} : choose(a.own, b.own, K, sizeof(TO) == 4, 1, false, true);
    Product pr{};
    pr.a = a, pr.b = b, pr.K = K, pr.batches = 1, pr.splits = cut.splits, pr.steps = cut.steps;
    e.rows = a.own, e.cols = b.own;
    if (cut.splits > 1) {
        e.partial_ld = pad8(b.own);
        e.partial_split = e.partial_ld * a.own;
        e.partial = (float *)mem.take(e.partial_split * cut.splits * 4);
    }
    if (!run) return;
    with_tile<T>(cut.shape, [&](auto tile) { launch<decltype(tile), ACROSS_A, ACROSS_B, TO>(pr, e, st); });
    if (cut.splits > 1)
        product_join_kernel<TO><<<dim3((uint32_t)ceil_div(e.partial_ld / 8 * a.own, 256)), 256, 0, st>>>(e, cut.splits);
}

// rows x cols at `src` as an operand, in place or copied.
template <class T>
Operand operand(const void *src, int64_t ld, int64_t rows, int32_t cols, bool across, Arena &mem, CopyJobs &pads)
{
    Operand o{};
    o.own = (int32_t)(across ? cols : rows);
    if (in_place(src, ld, rows, cols)) {
        o.p = src, o.ld = rows > 1 ? ld : pad8(cols);
        return o;
    }
    CopyArgs c{};
    c.src = src, c.ld = ld, c.rows = rows, c.cols = cols, c.pad = pad8(cols);
    c.dst = mem.take(rows * c.pad * 2);
    o.p = c.dst, o.ld = c.pad;
    pads.add(c, spread(rows * (c.pad / 8)), 1);
    return o;
}

// float32 rows x cols at `src` as two parts: along k scaled per row ...
Operand row_parts(const void *src, int64_t ld, int64_t rows, int32_t cols, const float **most, Arena &mem, CopyJobs &jobs)
{
    CopyArgs c{};
    c.src = src, c.ld = ld, c.rows = rows, c.cols = cols, c.pad = (int32_t)ceil_div(cols, 32) * 32;
    c.dst = mem.take(rows * 2 * (int64_t)c.pad * 2);
    c.most = (float *)mem.take(rows * 4);
    *most = c.most;
    Operand o{};
    o.own = (int32_t)rows, o.p = c.dst, o.ld = 2 * (int64_t)c.pad, o.part = 32, o.block = 64;
    jobs.add(c, std::min<int64_t>(ceil_div(rows, 4), 1 << 14), 1);
    return o;
}

// ... and across scaled per column. most: the magnitudes that the scales come
// from, zeros that a job of `maxima` raises unless they are known.
Operand col_parts(const void *src, int64_t ld, int64_t rows, int32_t cols, float *most, bool known, Arena &mem, CopyJobs &maxima, CopyJobs &jobs)
{
    CopyArgs c{};
    c.src = src, c.ld = ld, c.rows = rows, c.cols = cols, c.pad = pad8(cols), c.most = most;
    const int64_t deep = ceil_div(rows, 32) * 32;
    c.dst = mem.take(deep * 2 * c.pad * 2);
    Operand o{};
    o.own = cols, o.p = c.dst, o.ld = c.pad, o.part = 32 * (int64_t)c.pad, o.block = 64 * (int64_t)c.pad;
    if (!known) {
        const int64_t strips = ceil_div(cols, 256);
        maxima.add(c, strips, std::max<int64_t>(1, std::min<int64_t>(ceil_div(rows, 32), 2048 / strips)));
    }
    while (c.across < 5 && 8 << c.across < c.pad) ++c.across;
    const int64_t wide = ceil_div(c.pad, 8 << c.across);
    jobs.add(c, wide, std::max<int64_t>(1, std::min<int64_t>(ceil_div(deep, 256 >> c.across), 2048 / wide)));
    return o;
}

template <class F>
int with_type(int32_t dtype, F f)
{
    if (dtype == BOA_T_F32) return f(0.0f);
    return dtype == BOA_T_BF16 ? f(bf16_t{}) : f(f16_t{});
}

// Whether a forward product is done by few_kernel. It takes a time for every row
// of x and k, the tiles one for every weight in float32 (their parts) and nearly
// the same whatever M: 32 x 1024 x 4096 in bfloat16 5.4 us (tiles 6.8), 64 x 1024
// x 4096 7.4 (6.9), 32 x 4096 x 1024 13.0 (9.2); in float32 128 x 1024 x 4096 20
// (27), 64 x 4096 x 4096 45 (59), 128 x 4096 x 4096 68 (66), 64 x 4096 x 1024 44 (32).
bool is_few(int64_t M, int64_t N, int64_t K, int32_t dtype)
{
    if (M <= BOA_LINEAR_FEW) return true;
    if (dtype != BOA_T_F32) return M <= 64 && M * K <= 49152;
    return M <= 16 * FEW_MOST && ceil_div(M, 16) * 16 * K * ceil_div(N, 4096) <= 71000 + N * K / 64;
}

int check(const char *what, const boa_dense *d, bool grad)
{
    const char *why = nullptr;
    if (!d) return set_error(BOA_EINVAL, "linear: NULL arguments");
    const int32_t last = BOA_ACT_GELU_TANH;
    if (!dtype_known(d->dtype)) why = "unknown dtype";
    else if (d->activation < 0 || d->activation > last) why = "unknown activation";
    else if (d->M < 0 || d->M > BOA_MAX_LINEAR_ROWS) why = "M out of range [0, 2^31 - 256]";
    else if (d->N < 1 || d->N > BOA_MAX_LINEAR) why = "N out of range [1, 2^17]";
    else if (d->K < 1 || d->K > BOA_MAX_LINEAR) why = "K out of range [1, 2^17]";
    else if (d->M > 1 && d->x_stride < d->K) why = "x's row stride smaller than K";
    else if (d->N > 1 && d->w_stride < d->K) why = "w's row stride smaller than K";
    else if (d->param_dtype != d->dtype && d->param_dtype != BOA_T_F32) why = "the bias must have the layer's type or be float32";
    else if (d->M && !d->x) why = "NULL x";
    else if (!d->w) why = "NULL w";
    else if (!grad && d->residual && d->M > 1 && d->residual_stride < d->N) why = "the residual's row stride smaller than N";
    else if (!grad && d->M && !d->y) why = "NULL y";
    else if (grad && d->M && !d->dy) why = "NULL dy";
    else if (grad && d->M > 1 && d->dy_stride < d->N) why = "dy's row stride smaller than N";
    else if (grad && d->M && d->activation != BOA_ACT_NONE && !d->pre) why = "NULL pre";
    if (!why) return BOA_OK;
    char msg[160];
    __builtin_snprintf(msg, sizeof(msg), "%s: %s", what, why);
    return set_error(BOA_EINVAL, msg);
}

template <class TO>
void forward(const boa_dense &d, Arena &mem, bool run, hipStream_t st)
{
    constexpr bool WIDE = sizeof(TO) == 4;
    typedef std::conditional_t<WIDE, f16_t, TO> T;
    const int32_t M = (int32_t)d.M;
    Epilogue e{};
    e.out = d.y, e.ld = d.N, e.bias = d.bias, e.bias_f32 = d.param_dtype == BOA_T_F32;
    e.residual = d.residual, e.residual_ld = d.residual_stride, e.pre = d.pre, e.act = d.activation;
    e.rows = M, e.cols = d.N;
    if (is_few(M, d.N, d.K, d.dtype)) {
        if (!run) return;
        const FewArgs a{d.x, d.w, d.x_stride, d.w_stride, M, d.N, d.K, e};
        auto launch = [&](auto kernel, int mt) {
            const int lds = FEW_WAVES * mt * 1024;
            if (lds > 64 << 10)   // has to be asked for
                (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, lds);
            kernel<<<dim3((uint32_t)ceil_div(d.N, 16)), 64 * FEW_WAVES, lds, st>>>(a);
        };
        if (M <= 16) launch(few_kernel<TO, 1>, 1);
        else if (M <= 32) launch(few_kernel<TO, 2>, 2);
        else if (M <= 64) launch(few_kernel<TO, 4>, 4);
        else if constexpr (WIDE) launch(few_kernel<TO, FEW_MOST>, FEW_MOST);
        return;
    }
    CopyJobs jobs{};
    Operand x{}, w{};
    if constexpr (WIDE) {
        x = row_parts(d.x, d.x_stride, M, d.K, &e.max_a, mem, jobs);
        w = row_parts(d.w, d.w_stride, d.N, d.K, &e.max_b, mem, jobs);
        if (run) row_parts_kernel<<<jobs.grid(), 256, 0, st>>>(jobs);
    } else {
        x = operand<T>(d.x, d.x_stride, M, d.K, false, mem, jobs);
        w = operand<T>(d.w, d.w_stride, d.N, d.K, false, mem, jobs);
        if (run && jobs.n) pad_kernel<T><<<jobs.grid(), 256, 0, st>>>(jobs);
    }
    product<T, TO, false, false>(x, w, d.K, e, mem, run, st);
}

template <class TO>
void backward(const boa_dense &d, Arena &mem, bool run, hipStream_t st)
{
    constexpr bool WIDE = sizeof(TO) == 4;
    typedef std::conditional_t<WIDE, f16_t, TO> T;
    const int32_t M = (int32_t)d.M;
    const bool act = d.activation != BOA_ACT_NONE;
    // dz: dy itself where the activation has none and it can be read as it is
    SlopeArgs s{};
    s.dy = d.dy, s.ld = d.dy_stride, s.pre = d.pre, s.M = M, s.N = d.N, s.pad = pad8(d.N), s.act = d.activation;
    const void *dz = d.dy;
    int64_t dz_ld = d.dy_stride;
    if ((d.dx || d.dw) && (act || (!WIDE && !in_place(d.dy, d.dy_stride, M, d.N)))) {
        s.dz = mem.take((int64_t)M * s.pad * sizeof(TO));
        dz = s.dz, dz_ld = s.pad;
    }
    float *most_z = nullptr, *most_w = nullptr, *most_x = nullptr;
    if (WIDE && M && (d.dx || d.dw)) {   // magnitudes of dz's, w's and x's columns
        const int64_t n = d.N + 2 * (int64_t)d.K;
        most_z = (float *)mem.take(n * 4), most_w = most_z + d.N, most_x = most_w + d.K;
        if (run) zero_kernel<float><<<spread(n), 256, 0, st>>>(most_z, n);
        if (d.dw && (s.dz || d.dbias)) s.most = most_z;   // the kernel runs anyway
    }
    const int64_t strips = ceil_div(d.N, 256);
    const int32_t stripes = (int32_t)std::max<int64_t>(1, std::min<int64_t>(ceil_div(M, 16), std::max<int64_t>(1, 2048 / strips)));
    if (d.dbias) s.partial = (float *)mem.take((int64_t)stripes * d.N * 4);
    if (run && (s.dz || d.dbias)) slope_kernel<TO><<<dim3((uint32_t)strips, (uint32_t)stripes), 256, 0, st>>>(s);
    if (run && d.dbias) {
        const uint32_t grid = (uint32_t)ceil_div(d.N, 16);
        if (d.param_dtype == BOA_T_F32) bias_join_kernel<float><<<grid, 256, 0, st>>>(s.partial, stripes, d.N, (float *)d.dbias);
        else bias_join_kernel<TO><<<grid, 256, 0, st>>>(s.partial, stripes, d.N, (TO *)d.dbias);
    }
    // dz along k and w across give dx, both across give dw
    const bool dx = d.dx && M, dw = d.dw && M;
    const float *rows_z = nullptr;
    Operand z_dx{}, w_dx{}, z_dw{}, x_dw{};
    if constexpr (WIDE) {
        CopyJobs along{}, maxima{}, across{};
        if (dx) {
            z_dx = row_parts(dz, dz_ld, M, d.N, &rows_z, mem, along);
            w_dx = col_parts(d.w, d.w_stride, d.N, d.K, most_w, false, mem, maxima, across);
        }
        if (dw) {
            z_dw = col_parts(dz, dz_ld, M, d.N, most_z, s.most, mem, maxima, across);
            x_dw = col_parts(d.x, d.x_stride, M, d.K, most_x, false, mem, maxima, across);
        }
        if (run && along.n) row_parts_kernel<<<along.grid(), 256, 0, st>>>(along);
        if (run && maxima.n) col_max_kernel<<<maxima.grid(), 256, 0, st>>>(maxima);
        if (run && across.n) col_parts_kernel<<<across.grid(), 256, 0, st>>>(across);
    } else {
        CopyJobs pads{};
        z_dx.p = dz, z_dx.ld = M > 1 || s.dz ? dz_ld : s.pad;
        z_dw = z_dx, z_dx.own = M, z_dw.own = d.N;
        if (dx) w_dx = operand<T>(d.w, d.w_stride, d.N, d.K, true, mem, pads);
        if (dw) x_dw = operand<T>(d.x, d.x_stride, M, d.K, true, mem, pads);
        if (run && pads.n) pad_kernel<T><<<pads.grid(), 256, 0, st>>>(pads);
    }
    Epilogue e{};
    e.act = BOA_ACT_NONE;
    const int64_t kept = mem.used;   // the two products' sums take turns
    int64_t most = kept;
    using S = Small<T>;
    auto tiles = [](int64_t a, int64_t b) { return ceil_div(a, S::BA) * ceil_div(b, S::BB); };
    const int64_t blocks = tiles(M, d.K), others = tiles(d.N, d.K);
    const int32_t deep = WIDE ? 32 : 64;   // k of a stage
    // by sizes alone: a gradient is the same with the other one and without
    const bool pair = blocks + others <= 256 * S::PER_CU && std::max(M, d.N) <= PAIR_STAGES * deep;
    if (pair && dx && dw) {
        if (run) {
            Product px{}, pw{};
            px.a = z_dx, px.b = w_dx, px.K = d.N, pw.a = z_dw, pw.b = x_dw, pw.K = M;
            Epilogue ex = e, ew = e;
            ex.out = d.dx, ex.ld = d.K, ex.max_a = rows_z, ex.max_b = most_w, ex.rows = M, ex.cols = d.K;
            ew.out = d.dw, ew.ld = d.K, ew.max_a = most_z, ew.max_b = most_x, ew.rows = d.N, ew.cols = d.K;
            for (Product *p : {&px, &pw}) {
                p->batches = p->splits = 1, p->steps = (int32_t)ceil_div(p->K, deep);
                p->tiles_a = (int32_t)ceil_div(p->a.own, S::BA), p->tiles_b = (int32_t)ceil_div(p->b.own, S::BB);
            }
            const auto kernel = pair_kernel<S, TO>;
            kernel<<<dim3((uint32_t)(blocks + others)), S::THREADS, S::LDS, st>>>(px, ex, pw, ew, (uint32_t)blocks);
        }
        return;
    }
    if (dx) {
        e.out = d.dx, e.ld = d.K, e.max_a = rows_z, e.max_b = most_w;
        product<T, TO, false, true>(z_dx, w_dx, d.N, e, mem, run, st, pair);
        most = mem.used;
        mem.used = kept;
    }
    if (dw) {
        e.out = d.dw, e.ld = d.K, e.max_a = most_z, e.max_b = most_x;
        product<T, TO, true, true>(z_dw, x_dw, M, e, mem, run, st, pair);
        most = std::max(most, mem.used);
    } else if (d.dw) {
        const int64_t n = (int64_t)d.N * d.K;
        if (run) zero_kernel<TO><<<spread(n), 256, 0, st>>>((TO *)d.dw, n);
    }
    mem.used = most;
}

int64_t measure(const boa_dense &d, bool grad)
{
    Arena mem;
    with_type(d.dtype, [&](auto t) {
        using TO = decltype(t);
        if (grad) backward<TO>(d, mem, false, nullptr);
        else forward<TO>(d, mem, false, nullptr);
        return 0;
    });
    return mem.used;
}

int call(const char *what, const boa_dense *d, bool grad, void *workspace, int64_t bytes, void *stream)
{
    if (int rc = check(what, d, grad)) return rc;
    if (!grad && d->M == 0) return BOA_OK;
    if (grad && !d->dx && !d->dw && !d->dbias) return BOA_OK;
    const int64_t need = measure(*d, grad);
    if (need && (!workspace || !aligned(workspace, 16) || bytes < need)) {
        char msg[96];
        __builtin_snprintf(msg, sizeof(msg), "%s: workspace missing, unaligned or too small", what);
        return set_error(BOA_EINVAL, msg);
    }
    Arena mem;
    mem.base = (char *)workspace;
    return with_type(d->dtype, [&](auto t) {
        using TO = decltype(t);
        if (grad) backward<TO>(*d, mem, true, (hipStream_t)stream);
        else forward<TO>(*d, mem, true, (hipStream_t)stream);
        return launch_status(what);
    });
}

}  // namespace

extern "C" {

int64_t boa_linear_workspace(const boa_dense *d, int32_t grad)
{
    if (int rc = check("linear", d, grad != 0)) return rc;
    return measure(*d, grad != 0);
}

int boa_linear(const boa_dense *d, void *workspace, int64_t workspace_bytes, void *stream)
{
    return call("linear", d, false, workspace, workspace_bytes, stream);
}

int boa_linear_grad(const boa_dense *d, void *workspace, int64_t workspace_bytes, void *stream)
{
    return call("linear_backward", d, true, workspace, workspace_bytes, stream);
}

}  // extern "C"
