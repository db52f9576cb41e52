// What stands between two blocks of a residual tower, in one pass over the rows:
// the norm after a block, its gate, the residual sum, and the norm before the
// next block.
//
//   u = norm(f) pw + pb  (or f)     h = s x + g u     y = norm(h) w + b
//
// norm(v) = (v - mean(v)) r, r = 1 / sqrt(mean((v - mean(v))^2) + eps), or without
// the means (rms). Backward, from dh and dy:
//
//   dH = dh + r (dy w - mean(dy w) - hn mean(dy w hn))       dx = s dH
//   dg = dH u    du = dH g    df = the same step back through the first norm
//
// and sums over rows: dw = dy hn, db = dy, dpw = du fn, dpb = du, dg of a shared
// gate. With a shared gate the last three come of two: S = sum dH fn and
// s = sum dH give dpw = g S, dpb = g s, dg = pw S + pb s.
//
// Both are bound by memory. Forward reads x and f (and a gate per value) and
// writes h and y; backward reads x, f, dh and dy and writes dx and df: h is
// formed again from x and f in float32, which costs what reading it would and
// keeps the digits that its rounding loses. A row stays in registers, as in
// boa_norm.hip: backward a wave holds up to 512 values, two waves 1,024, four
// 4,096, eight 8,192, so that a thread has 8 columns in most cases and 16 at most
// and the column sums stay in registers too, over all rows of a block; they leave
// one partial row each per block, added in block order.
#include <algorithm>

#include "boa_rows.h"

using namespace boa;

namespace {

constexpr int THREADS = ROW_THREADS;
constexpr int SUMS = 4;   // over rows: dy hn, dy; t fn, t for t = dH, or du where every value has its gate
constexpr int64_t MAX_BLOCKS = 1024;

// Threads of a block whose rows take TPR of them each.
constexpr int threads_of(int tpr) { return tpr < 128 ? THREADS : tpr; }

struct BlockArgs {
    const void *x, *f, *gate, *pw, *pb, *w, *b, *dh, *dy;
    void *h, *y, *dx, *df, *dgate;   // dgate: of a gate per value
    float *stats;                    // mean and 1 / deviation of f's rows, then of h's: each `stats_rows` long
    float *back;                     // wide rows: the two means of the gradient through the second norm
    float *partial;
    int64_t rows, stats_rows, x_ld, f_ld, gate_ld, dh_ld, dy_ld;
    int32_t d, layer, post, pre, gate_rows;
    float scale, eps;
};

template <class T>
const T *plus(const void *p, int64_t n) { return p ? (const T *)p + n : nullptr; }
template <class T>
T *plus(void *p, int64_t n) { return p ? (T *)p + n : nullptr; }

// The arguments of the rows from `row` on, `most` at most.
template <class T>
BlockArgs rows_from(BlockArgs a, int64_t row, int64_t most)
{
    a.x = plus<T>(a.x, row * a.x_ld), a.f = plus<T>(a.f, row * a.f_ld);
    if (a.gate_rows) a.gate = plus<T>(a.gate, row * a.gate_ld);
    a.dh = plus<T>(a.dh, row * a.dh_ld), a.dy = plus<T>(a.dy, row * a.dy_ld);
    a.h = plus<T>(a.h, row * a.d), a.y = plus<T>(a.y, row * a.d), a.dx = plus<T>(a.dx, row * a.d);
    a.df = plus<T>(a.df, row * a.d), a.dgate = plus<T>(a.dgate, row * a.d);
    a.stats = plus<float>(a.stats, row), a.back = plus<float>(a.back, 2 * row);
    a.rows = std::min(most, a.rows - row);
    return a;
}

// f(arguments) for the rows of each launch of blocks of `threads` threads, which take `each` rows.
template <class T, class F>
void in_launches(const BlockArgs &a, int32_t threads, int32_t each, F f)
{
    const int64_t most = std::min(LAUNCH_ROWS, ((int64_t)1 << 31) / threads * each);   // 2^32 threads would be refused
    for (int64_t row = 0; row < a.rows; row += most) f(rows_from<T>(a, row, most));
}

// A vector of parameters at a thread's columns, `or_else` where there is none.
template <class P, int VEC>
__device__ inline void params(float (&to)[VEC], const void *p, int c, float or_else)
{
    if (p) {
        load_loose<VEC, P>(to, (const P *)p + c);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) to[j] = or_else;
    }
}

// Mean and 1 / deviation of a row held in registers, and the row without its mean.
template <int NV, int VEC, int TPR, bool WHOLE>
__device__ inline void row_stats(float (&v)[NV][VEC], int lane, int32_t d, bool layer, float eps, float *red, float &mu, float &r)
{
    mu = 0.0f;
    if (layer) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Cols<VEC, TPR> at(i, lane, d);
#pragma unroll
            for (int j = 0; j < VEC; ++j) s += at.template mine<WHOLE>(j) ? v[i][j] : 0.0f;
        }
        mu = row_sum<TPR>(s, red) / (float)d;
    }
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
    r = 1.0f / sqrtf(row_sum<TPR>(q, red) / (float)d + eps);
}

// Forward: 65,536 rows of 1,024 bfloat16 values 103 us, 5.2 TB/s; 9,973 of 413
// float32 with a gate per value 16 us, 5.1 TB/s.
template <class T, class P, int NV, int TPR, bool WHOLE>
__global__ __launch_bounds__(threads_of(TPR)) void block_kernel(BlockArgs a)
{
    constexpr int VEC = 16 / sizeof(T);
    __shared__ float red[16];
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (threads_of(TPR) / TPR) + threadIdx.x / TPR;
    if (row >= a.rows) return;   // a whole wave (TPR 64) or block leaves
    const int32_t d = a.d;
    const T *x = (const T *)a.x + row * a.x_ld, *f = (const T *)a.f + row * a.f_ld;
    float v[NV][VEC], h[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int c = Cols<VEC, TPR>(i, lane, d).c;
        load_loose<VEC, T>(v[i], f + c);
        load_loose<VEC, T>(h[i], x + c);
    }
    float mu, r;
    if (a.post) {
        row_stats<NV, VEC, TPR, WHOLE>(v, lane, d, a.layer, a.eps, red, mu, r);
        if (lane == 0 && a.stats) {
            a.stats[row] = mu;
            a.stats[a.stats_rows + row] = r;
        }
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const Cols<VEC, TPR> at(i, lane, d);
        if (a.post) {
            float pw[VEC], pb[VEC];
            params<P, VEC>(pw, a.pw, at.c, 1.0f);
            params<P, VEC>(pb, a.pb, at.c, 0.0f);
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i][j] = fmaf(v[i][j] * r, pw[j], pb[j]);
        }
        if (a.gate) {
            float g[VEC];
            if (a.gate_rows) load_loose<VEC, T>(g, (const T *)a.gate + row * a.gate_ld + at.c);
            else load_loose<VEC, P>(g, (const P *)a.gate + at.c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) v[i][j] *= g[j];
        }
#pragma unroll
        for (int j = 0; j < VEC; ++j) h[i][j] = fmaf(a.scale, h[i][j], v[i][j]);
        // two threads' common columns hold the same values
        if (at.any()) {
            store_loose<VEC, T>((T *)a.h + row * (int64_t)d + at.c, h[i]);
        }
    }
    if (!a.pre) return;
    row_stats<NV, VEC, TPR, WHOLE>(h, lane, d, a.layer, a.eps, red, mu, r);
    if (lane == 0 && a.stats) {
        a.stats[2 * a.stats_rows + row] = mu;
        a.stats[3 * a.stats_rows + row] = r;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const Cols<VEC, TPR> at(i, lane, d);
        float w[VEC], b[VEC];
        params<P, VEC>(w, a.w, at.c, 1.0f);
        params<P, VEC>(b, a.b, at.c, 0.0f);
#pragma unroll
        for (int j = 0; j < VEC; ++j) h[i][j] = fmaf(h[i][j] * r, w[j], b[j]);
        if (at.any()) store_loose<VEC, T>((T *)a.y + row * (int64_t)d + at.c, h[i]);
    }
}

// One thread's columns of a gradient: whole, or those that are its own.
template <class T, int VEC, int TPR, bool WHOLE>
__device__ inline void store_mine(T *row, const Cols<VEC, TPR> &at, const float (&v)[VEC])
{
    if (WHOLE ? at.any() : at.skip == 0) {
        store_loose<VEC, T>(row + at.c, v);
    } else if (at.any()) {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (at.template mine<WHOLE>(j)) row[at.c + j] = (T)v[j];
    }
}

// A row's values at a thread's columns, as they come from memory.
template <class T, int NV>
struct RawRow {
    words4 f[NV], x[NV], dh[NV], dy[NV], gate[NV];
    float stats[4];
};

template <class T, int VEC>
__device__ inline void unpack(float (&to)[VEC], words4 w)
{
    typedef Pack<VEC, T> PV;
    const PV p = __builtin_bit_cast(PV, w);
#pragma unroll
    for (int j = 0; j < VEC; ++j) to[j] = (float)p.v[j];
}

// Backward. DP: column sums are wanted. The next row is on its way while a row is
// worked on, and the parameters lie in LDS as float32: asked for from memory they
// would wait for that row. 65,536 rows of 1,024 bfloat16 values: 223 to 233 us, 3.5
// TB/s (419 with the row and the parameters loaded where they are needed, and
// registers for one wave a SIMD).
template <class T, int NV>
constexpr bool ROW_AHEAD = NV * 16 / sizeof(T) <= 8;   // with more columns a thread it would not fit the registers

// LDS that the four parameter vectors take, each thread's columns for itself.
template <class T, int NV, int TPR>
constexpr int PARAM_FLOATS = 4 * NV * 16 / (int)sizeof(T) * TPR;

template <class T, class P, int NV, int TPR, bool WHOLE, bool DP>
__global__ __launch_bounds__(threads_of(TPR), (ROW_AHEAD<T, NV> ? 2 : 1)) void block_back_kernel(BlockArgs a)
{
    constexpr int VEC = 16 / sizeof(T), BLOCK = threads_of(TPR), GROUPS = BLOCK / TPR;
    constexpr bool AHEAD = ROW_AHEAD<T, NV>;
    constexpr bool IN_LDS = PARAM_FLOATS<T, NV, TPR> <= 8192;
    __shared__ float red[16];
    extern __shared__ __attribute__((aligned(16))) float cols[];   // parameters; at the end, where rows share a block, SUMS x d sums
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int32_t d = a.d;
    if constexpr (IN_LDS) {
        if (group == 0) {
            const void *of[4] = {a.w, a.pw, a.pb, a.gate_rows ? nullptr : a.gate};
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    float v[VEC];
                    params<P, VEC>(v, of[k], Cols<VEC, TPR>(i, lane, d).c, k == 2 ? 0.0f : 1.0f);
#pragma unroll
                    for (int q = 0; q < VEC; q += 4)
                        store_f32<4, float>(cols + (((k * NV + i) * VEC + q) * TPR + lane * 4), *(float(*)[4])(v + q));
                }
        }
        __syncthreads();
    }
    enum { W, PW, PB, G };
    auto param = [&](float (&to)[VEC], int which, int i, int c) {
        if constexpr (IN_LDS) {   // a thread's own, 16 bytes a lane side by side
#pragma unroll
            for (int q = 0; q < VEC; q += 4)
                load_f32<4, float>(*(float(*)[4])(to + q), cols + (((which * NV + i) * VEC + q) * TPR + lane * 4));
        } else {
            params<P, VEC>(to, which == W ? a.w : which == PW ? a.pw : which == PB ? a.pb : a.gate, c, which == PB ? 0.0f : 1.0f);
        }
    };
    auto load = [&](RawRow<T, NV> &to, int64_t row) {
        auto raw = [](const void *p, int64_t at) { return (words4) * (const loose4 *)((const T *)p + at); };
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = Cols<VEC, TPR>(i, lane, d).c;
            to.f[i] = raw(a.f, row * a.f_ld + c);
            to.x[i] = raw(a.x, row * a.x_ld + c);
            to.dh[i] = a.dh ? raw(a.dh, row * a.dh_ld + c) : words4{0, 0, 0, 0};
            to.dy[i] = a.dy ? raw(a.dy, row * a.dy_ld + c) : words4{0, 0, 0, 0};
            if (a.gate_rows) to.gate[i] = raw(a.gate, row * a.gate_ld + c);
        }
        to.stats[0] = a.post ? a.stats[row] : 0.0f, to.stats[1] = a.post ? a.stats[a.stats_rows + row] : 1.0f;
        to.stats[2] = a.dy ? a.stats[2 * a.stats_rows + row] : 0.0f, to.stats[3] = a.dy ? a.stats[3 * a.stats_rows + row] : 0.0f;
    };
    float sums[SUMS][NV][VEC];
#pragma unroll
    for (int k = 0; k < SUMS; ++k)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) sums[k][i][j] = 0.0f;
    const int64_t stride = (int64_t)gridDim.x * GROUPS;
    int64_t row = (int64_t)blockIdx.x * GROUPS + group;
    RawRow<T, NV> next;
    if (AHEAD && row < a.rows) load(next, row);
    for (; row < a.rows; row += stride) {
        if (!AHEAD) load(next, row);
        // what is needed later stays as it came: float32 would take twice the registers
        words4 f[NV], dh[NV], dy[NV], gate[NV];
        float v[NV][VEC];   // x, then hn, then dH, then the gradient of norm(f)
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            f[i] = next.f[i], dh[i] = next.dh[i], dy[i] = next.dy[i];
            if (a.gate_rows) gate[i] = next.gate[i];
            unpack<T, VEC>(v[i], next.x[i]);
        }
        const float pm = next.stats[0], pr = next.stats[1], hm = next.stats[2], hr = next.stats[3];
        // Between the steps nothing is kept that can be read or formed again: parameters from LDS, values as float32.
        auto forget = [&] {
            if constexpr (AHEAD) {
#pragma unroll
                for (int i = 0; i < NV; ++i) asm volatile("" : "+v"(f[i]), "+v"(dy[i]) :: "memory");
            }
        };
        forget();
        if (AHEAD && row + stride < a.rows) load(next, row + stride);
        auto gate_at = [&](float (&g)[VEC], int i, int c) {
            if (a.gate_rows) unpack<T, VEC>(g, gate[i]);
            else param(g, G, i, c);
        };
        auto fn_at = [&](float (&fn)[VEC], int i) {
            unpack<T, VEC>(fn, f[i]);
#pragma unroll
            for (int j = 0; j < VEC; ++j) fn[j] = (fn[j] - pm) * pr;
        };
        // columns that are not this thread's count for nothing in the row's sums
        auto g1_at = [&](float (&g1)[VEC], const Cols<VEC, TPR> &at, int i) {
            float w[VEC];
            param(w, W, i, at.c);
            unpack<T, VEC>(g1, dy[i]);
#pragma unroll
            for (int j = 0; j < VEC; ++j) g1[j] = at.template mine<WHOLE>(j) ? g1[j] * w[j] : 0.0f;
        };
        // h again, its norm, and the gradient through it (without dy none of that is used)
        float c1 = 0.0f, c2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Cols<VEC, TPR> at(i, lane, d);
            float fn[VEC], pw[VEC], pb[VEC], g[VEC], g1[VEC], t[VEC];
            fn_at(fn, i);
            param(pw, PW, i, at.c);
            param(pb, PB, i, at.c);
            gate_at(g, i, at.c);
            g1_at(g1, at, i);
            unpack<T, VEC>(t, dy[i]);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[i][j] = (fmaf(a.scale, v[i][j], g[j] * fmaf(fn[j], pw[j], pb[j])) - hm) * hr;
                if (DP) {
                    sums[0][i][j] = fmaf(t[j], v[i][j], sums[0][i][j]);
                    sums[1][i][j] += t[j];
                }
                c1 += g1[j];
                c2 = fmaf(g1[j], v[i][j], c2);
            }
        }
        if (a.dy) {
            row_sum2<TPR>(c1, c2, red);
            c1 = a.layer ? c1 / (float)d : 0.0f;
            c2 /= (float)d;
        }
        forget();
        float p1 = 0.0f, p2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Cols<VEC, TPR> at(i, lane, d);
            float fn[VEC], pw[VEC], g[VEC], g1[VEC], o[VEC];
            fn_at(fn, i);
            param(pw, PW, i, at.c);
            gate_at(g, i, at.c);
            g1_at(g1, at, i);
            unpack<T, VEC>(o, dh[i]);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                v[i][j] = a.dy ? fmaf(hr, g1[j] - c1 - v[i][j] * c2, o[j]) : o[j];
                o[j] = a.scale * v[i][j];
            }
            if (a.dx) store_mine<T, VEC, TPR, WHOLE>((T *)a.dx + row * (int64_t)d, at, o);
            if (a.dgate) {
                float pb[VEC];
                param(pb, PB, i, at.c);
#pragma unroll
                for (int j = 0; j < VEC; ++j) o[j] = v[i][j] * fmaf(fn[j], pw[j], pb[j]);
                store_mine<T, VEC, TPR, WHOLE>((T *)a.dgate + row * (int64_t)d, at, o);
            }
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const float du = v[i][j] * g[j], t = a.gate_rows ? du : v[i][j];
                if (DP) {
                    sums[2][i][j] = fmaf(t, fn[j], sums[2][i][j]);
                    sums[3][i][j] += t;
                }
                v[i][j] = at.template mine<WHOLE>(j) ? du * pw[j] : 0.0f;
                p1 += v[i][j];
                p2 = fmaf(v[i][j], fn[j], p2);
            }
        }
        if (!a.df) continue;
        forget();
        if (a.post) {
            row_sum2<TPR>(p1, p2, red);
            p1 = a.layer ? p1 / (float)d : 0.0f;
            p2 /= (float)d;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Cols<VEC, TPR> at(i, lane, d);
            if (a.post) {
                float fn[VEC];
                fn_at(fn, i);
#pragma unroll
                for (int j = 0; j < VEC; ++j) v[i][j] = pr * (v[i][j] - p1 - fn[j] * p2);
            }
            store_mine<T, VEC, TPR, WHOLE>((T *)a.df + row * (int64_t)d, at, v[i]);
        }
    }
    if constexpr (DP) {
        float *out = a.partial + (int64_t)blockIdx.x * SUMS * d;
        if (GROUPS > 1) __syncthreads();   // the parameters have been read
        for (int k = 0; k < GROUPS; ++k) {   // the block's waves with a row each, added in order
            if (group == k) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const Cols<VEC, TPR> at(i, lane, d);
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        if (!at.template mine<WHOLE>(j)) continue;
#pragma unroll
                        for (int q = 0; q < SUMS; ++q) {
                            if (q == 0 && !a.dy) sums[q][i][j] = 0.0f;   // 0 times a row that is not finite
                            float *to = (GROUPS == 1 ? out : cols) + (int64_t)q * d + at.c + j;
                            *to = k ? *to + sums[q][i][j] : sums[q][i][j];
                        }
                    }
                }
            }
            if (GROUPS > 1) __syncthreads();
        }
        if (GROUPS > 1)
            for (int c = threadIdx.x; c < SUMS * d; c += BLOCK) out[c] = cols[c];
    }
}

// ---------------------------------------------------------------------------
// rows wider than the registers, or narrower than a load: a block per row, which
// reads it once for every sum (from the caches after the first time). 8,192 rows of
// 8,192 bfloat16 values would take 844 us forward and 1,899 backward; held in the
// registers of eight waves, as rows up to that width are, they take 112 and 369.

template <class T, class P>
struct Wide {
    const BlockArgs &a;
    int64_t row;
    float pm, pr, hm, hr;
    __device__ float param(const void *p, int32_t c, float or_else) const { return p ? (float)((const P *)p)[c] : or_else; }
    __device__ float gate(int32_t c) const
    {
        return !a.gate ? 1.0f : a.gate_rows ? (float)((const T *)a.gate)[row * a.gate_ld + c] : (float)((const P *)a.gate)[c];
    }
    __device__ float fn(int32_t c) const { return ((float)((const T *)a.f)[row * a.f_ld + c] - pm) * pr; }
    __device__ float u(int32_t c) const { return a.post ? fmaf(fn(c), param(a.pw, c, 1.0f), param(a.pb, c, 0.0f)) : fn(c); }
    __device__ float h(int32_t c) const { return fmaf(a.scale, (float)((const T *)a.x)[row * a.x_ld + c], gate(c) * u(c)); }
    __device__ float hn(int32_t c) const { return (h(c) - hm) * hr; }
    __device__ float dy(int32_t c) const { return a.dy ? (float)((const T *)a.dy)[row * a.dy_ld + c] : 0.0f; }
    __device__ float dH(int32_t c, float c1, float c2) const
    {
        const float dh = a.dh ? (float)((const T *)a.dh)[row * a.dh_ld + c] : 0.0f;
        return a.dy ? fmaf(hr, dy(c) * param(a.w, c, 1.0f) - c1 - hn(c) * c2, dh) : dh;
    }
    __device__ void read_stats()
    {
        pm = a.post ? a.stats[row] : 0.0f, pr = a.post ? a.stats[a.stats_rows + row] : 1.0f;
        hm = a.dy ? a.stats[2 * a.stats_rows + row] : 0.0f, hr = a.dy ? a.stats[3 * a.stats_rows + row] : 0.0f;
    }
};

template <class V>
__device__ inline void wide_stats(V value, int32_t d, bool layer, float eps, float *red, float &mu, float &r)
{
    mu = 0.0f;
    if (layer) {
        float s = 0.0f;
        for (int32_t c = threadIdx.x; c < d; c += THREADS) s += value(c);
        mu = row_sum<THREADS>(s, red) / (float)d;
    }
    float q = 0.0f;
    for (int32_t c = threadIdx.x; c < d; c += THREADS) {
        const float t = value(c) - mu;
        q = fmaf(t, t, q);
    }
    r = 1.0f / sqrtf(row_sum<THREADS>(q, red) / (float)d + eps);
}

template <class T, class P>
__global__ __launch_bounds__(THREADS) void block_wide_kernel(BlockArgs a)
{
    __shared__ float red[8];
    Wide<T, P> w{a, (int64_t)blockIdx.x, 0.0f, 1.0f, 0.0f, 1.0f};
    const int32_t d = a.d;
    if (a.post) {
        float mu, r;
        wide_stats([&](int32_t c) { return w.fn(c); }, d, a.layer, a.eps, red, mu, r);
        w.pm = mu, w.pr = r;
    }
    T *h = (T *)a.h + w.row * d, *y = (T *)a.y + w.row * d;
    for (int32_t c = threadIdx.x; c < d; c += THREADS) h[c] = (T)w.h(c);
    if (a.pre) {
        float mu, r;
        wide_stats([&](int32_t c) { return w.h(c); }, d, a.layer, a.eps, red, mu, r);
        w.hm = mu, w.hr = r;
        for (int32_t c = threadIdx.x; c < d; c += THREADS) y[c] = (T)fmaf(w.hn(c), w.param(a.w, c, 1.0f), w.param(a.b, c, 0.0f));
    }
    if (threadIdx.x == 0 && a.stats) {
        const float s[4] = {w.pm, w.pr, w.hm, w.hr};
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (k < 2 ? a.post : a.pre) a.stats[k * a.stats_rows + w.row] = s[k];
    }
}

template <class T, class P>
__global__ __launch_bounds__(THREADS) void block_back_wide_kernel(BlockArgs a)
{
    __shared__ float red[8];
    Wide<T, P> w{a, (int64_t)blockIdx.x, 0.0f, 0.0f, 0.0f, 0.0f};
    w.read_stats();
    const int32_t d = a.d;
    float c1 = 0.0f, c2 = 0.0f, p1 = 0.0f, p2 = 0.0f;
    if (a.dy) {
        for (int32_t c = threadIdx.x; c < d; c += THREADS) {
            const float g = w.dy(c) * w.param(a.w, c, 1.0f);
            c1 += g;
            c2 = fmaf(g, w.hn(c), c2);
        }
        row_sum2<THREADS>(c1, c2, red);
        c1 = a.layer ? c1 / (float)d : 0.0f;
        c2 /= (float)d;
    }
    if (threadIdx.x == 0 && a.back) {
        a.back[2 * w.row] = c1;
        a.back[2 * w.row + 1] = c2;
    }
    if (a.post) {
        for (int32_t c = threadIdx.x; c < d; c += THREADS) {
            const float g = w.dH(c, c1, c2) * w.gate(c) * w.param(a.pw, c, 1.0f);
            p1 += g;
            p2 = fmaf(g, w.fn(c), p2);
        }
        row_sum2<THREADS>(p1, p2, red);
        p1 = a.layer ? p1 / (float)d : 0.0f;
        p2 /= (float)d;
    }
    for (int32_t c = threadIdx.x; c < d; c += THREADS) {
        const float dH = w.dH(c, c1, c2);
        const int64_t at = w.row * d + c;
        if (a.dx) ((T *)a.dx)[at] = (T)(a.scale * dH);
        if (a.dgate) ((T *)a.dgate)[at] = (T)(dH * w.u(c));
        if (a.df) {
            const float g = dH * w.gate(c);
            ((T *)a.df)[at] = (T)(a.post ? w.pr * (g * w.param(a.pw, c, 1.0f) - p1 - w.fn(c) * p2) : g);
        }
    }
}

// The column sums of such rows: a block per 256 columns and stripe of rows.
template <class T, class P>
__global__ __launch_bounds__(THREADS) void block_cols_kernel(BlockArgs a)
{
    const int32_t c = blockIdx.y * THREADS + threadIdx.x, d = a.d;
    if (c >= d) return;
    float s[SUMS] = {};
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        Wide<T, P> w{a, row, 0.0f, 0.0f, 0.0f, 0.0f};
        w.read_stats();
        const float dH = w.dH(c, a.back[2 * row], a.back[2 * row + 1]), t = a.gate_rows ? dH * w.gate(c) : dH;
        if (a.dy) {
            const float dy = w.dy(c);
            s[0] = fmaf(dy, w.hn(c), s[0]);
            s[1] += dy;
        }
        s[2] = fmaf(t, w.fn(c), s[2]);
        s[3] += t;
    }
#pragma unroll
    for (int k = 0; k < SUMS; ++k) a.partial[((int64_t)blockIdx.x * SUMS + k) * d + c] = s[k];
}

// Adds the blocks' partial rows: 16 columns a block and 64 slices of the rows,
// then the slices in order; two of the four sums a block, and what comes of them
// (1,024 partial rows of 1,024 columns: 10 us).
constexpr int JOIN_COLS = 16, JOIN_SLICES = 64;

template <class P>
struct JoinArgs {
    const float *partial;
    const P *gate, *pw, *pb;    // of a shared gate; null: ones, ones, zeros
    P *dw, *db, *dpw, *dpb, *dgate;
    int32_t blocks, d;
};

template <class P>
__global__ __launch_bounds__(JOIN_COLS * JOIN_SLICES) void block_join_kernel(JoinArgs<P> a)
{
    __shared__ float part[2][JOIN_SLICES][JOIN_COLS + 1];
    const int col = threadIdx.x % JOIN_COLS, slice = threadIdx.x / JOIN_COLS;
    const bool first = blockIdx.y == 0;
    if (first ? !a.dw && !a.db : !a.dpw && !a.dpb && !a.dgate) return;
    const int32_t c = blockIdx.x * JOIN_COLS + col;
    const float *from = a.partial + (first ? 0 : 2) * (int64_t)a.d + c;
    float s0 = 0.0f, s1 = 0.0f;
    if (c < a.d)
#pragma unroll 4
        for (int i = slice; i < a.blocks; i += JOIN_SLICES) {
            s0 += from[(int64_t)i * SUMS * a.d];
            s1 += from[(int64_t)i * SUMS * a.d + a.d];
        }
    part[0][slice][col] = s0;
    part[1][slice][col] = s1;
    __syncthreads();
    if (slice == 0 && c < a.d) {
        s0 = s1 = 0.0f;
#pragma unroll
        for (int i = 0; i < JOIN_SLICES; ++i) {
            s0 += part[0][i][col];
            s1 += part[1][i][col];
        }
        if (first) {
            if (a.dw) a.dw[c] = (P)s0;
            if (a.db) a.db[c] = (P)s1;
        } else {
            const float g = a.gate ? (float)a.gate[c] : 1.0f;
            if (a.dpw) a.dpw[c] = (P)(g * s0);
            if (a.dpb) a.dpb[c] = (P)(g * s1);
            if (a.dgate) a.dgate[c] = (P)fmaf(a.pw ? (float)a.pw[c] : 1.0f, s0, (a.pb ? (float)a.pb[c] : 0.0f) * s1);
        }
    }
}

// The registers a row takes: f(NV, TPR, WHOLE) as compile-time constants; false
// where a row does not fit, or is shorter than a load. Forward, a wave per row up
// to 4 loads a lane (65,536 rows of 1,024 bfloat16 values: 98 us, two waves a row 117);
// backward, at most 8 columns a thread up to 2,048 values, 16 beyond (float32 rows
// of more than 4,096 keep some 50 registers in scratch).
template <int VEC, bool FORWARD, class F>
bool with_shape(int32_t d, F f)
{
    const int64_t n = ceil_div(d, VEC);
    if (d < VEC || n * VEC > 8192) return false;
    auto whole = [&](auto nv, auto tpr) { d % VEC ? f(nv, tpr, Int<0>{}) : f(nv, tpr, Int<1>{}); };
    constexpr int MOST = VEC == 4 ? 4 : 2;   // loads of 16 columns
    if constexpr (FORWARD) {
        if (n <= 64) whole(Int<1>{}, Int<64>{});
        else if (n <= 128) whole(Int<2>{}, Int<64>{});
        else if (n <= 256) whole(Int<4>{}, Int<64>{});
        else if (n <= 512) whole(Int<2>{}, Int<256>{});
        else if (n <= 1024 && VEC == 4) whole(Int<4>{}, Int<256>{});
        else whole(Int<MOST>{}, Int<512>{});
    } else if constexpr (VEC == 4) {
        if (n <= 64) whole(Int<1>{}, Int<64>{});
        else if (n <= 128) whole(Int<2>{}, Int<64>{});
        else if (n <= 256) whole(Int<2>{}, Int<128>{});
        else if (n <= 512) whole(Int<2>{}, Int<256>{});
        else if (n <= 1024) whole(Int<4>{}, Int<256>{});
        else whole(Int<MOST>{}, Int<512>{});
    } else {
        if (n <= 64) whole(Int<1>{}, Int<64>{});
        else if (n <= 128) whole(Int<1>{}, Int<128>{});
        else if (n <= 256) whole(Int<1>{}, Int<256>{});
        else if (n <= 512) whole(Int<2>{}, Int<256>{});
        else whole(Int<MOST>{}, Int<512>{});
    }
    return true;
}

int check(const char *what, const boa_block *d, bool grad)
{
    if (!d) return set_error(BOA_EINVAL, "block_norm: NULL arguments");
    const char *why = nullptr;
    const bool shared = d->gate && !d->gate_rows;
    const bool sums = grad && (d->dpost_weight || d->dpost_bias || d->dweight || d->dbias || (shared && d->dgate));
    const bool many = d->rows > 1;
    if (!dtype_known(d->dtype)) why = "unknown dtype";
    else if (d->param_dtype != d->dtype && d->param_dtype != BOA_T_F32) why = "parameters must have the rows' type or be float32";
    else if (d->norm != BOA_NORM_LAYER && d->norm != BOA_NORM_RMS) why = "unknown norm";
    else if (d->rows < 0 || d->rows >= (int64_t)1 << 31) why = "rows out of range [0, 2^31)";
    else if (d->d < 1 || d->d > BOA_MAX_NORM_D) why = "d out of range [1, 2^20]";
    else if (!(d->eps >= 0.0f)) why = "eps must not be negative";
    else if (!(d->scale - d->scale == 0.0f)) why = "scale must be finite";
    else if (many && (d->x_stride < d->d || d->f_stride < d->d)) why = "row stride smaller than d";
    else if (many && d->gate && d->gate_rows && d->gate_stride < d->d) why = "the gate's row stride smaller than d";
    else if (d->rows && (!d->x || !d->f)) why = "NULL rows";
    else if (!grad && d->rows && (!d->h || (d->pre && !d->y))) why = "NULL output";
    else if (grad && many && ((d->dh && d->dh_stride < d->d) || (d->dy && d->dy_stride < d->d))) why = "a gradient's row stride smaller than d";
    else if (grad && d->rows && !d->dh && !d->dy) why = "neither dh nor dy";
    else if (grad && d->dy && !d->pre) why = "dy without the second norm";
    else if (grad && d->rows && (d->post || d->dy) && !d->stats) why = "NULL stats";
    else if (grad && !d->gate && d->dgate) why = "a gradient of the gate without a gate";
    else if (grad && !d->post && (d->dpost_weight || d->dpost_bias)) why = "gradients of the first norm without it";
    else if (sums && (!d->workspace || !aligned(d->workspace, 16) || d->workspace_bytes < boa_block_norm_backward_workspace(d->rows, d->d)))
        why = "workspace missing, unaligned or too small";
    if (!why) return BOA_OK;
    char msg[160];
    __builtin_snprintf(msg, sizeof(msg), "%s: %s", what, why);
    return set_error(BOA_EINVAL, msg);
}

int64_t back_blocks(int64_t rows, int32_t d)
{
    // As many partial rows as blocks: at most 4 per CU, what the registers let
    // run at once; fewer of few rows, and of wide ones 128 MB of them at most.
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(MAX_BLOCKS, ((int64_t)1 << 25) / ((int64_t)SUMS * d)));
    return std::max<int64_t>(1, std::min(most, ceil_div(rows, d <= 512 ? 32 : 8)));   // 4 rows at a time, or one
}

BlockArgs args_of(const boa_block *b)
{
    BlockArgs a{};
    a.x = b->x, a.f = b->f, a.gate = b->gate, a.x_ld = b->x_stride, a.f_ld = b->f_stride, a.gate_ld = b->gate_stride;
    a.pw = b->post ? b->post_weight : nullptr, a.pb = b->post ? b->post_bias : nullptr, a.w = b->weight, a.b = b->bias;
    a.dh = b->dh, a.dh_ld = b->dh_stride, a.dy = b->dy, a.dy_ld = b->dy_stride;
    a.stats = b->stats, a.stats_rows = b->rows, a.rows = b->rows, a.d = b->d;
    a.layer = b->norm == BOA_NORM_LAYER, a.post = b->post != 0, a.pre = b->pre != 0, a.gate_rows = b->gate && b->gate_rows;
    a.scale = b->scale, a.eps = b->eps;
    return a;
}

}  // namespace

extern "C" {

int boa_block_norm(const boa_block *b, void *stream)
{
    if (int rc = check("block_norm", b, false)) return rc;
    if (b->rows == 0) return BOA_OK;
    BlockArgs a = args_of(b);
    a.dh = a.dy = nullptr;
    a.h = b->h, a.y = b->y;
    hipStream_t st = (hipStream_t)stream;
    return with_types(b->dtype, b->param_dtype, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        constexpr int VEC = 16 / sizeof(T);
        const bool fits = with_shape<VEC, true>(b->d, [&](auto nv, auto tpr, auto whole) {
            constexpr int NV = decltype(nv)::value, TPR = decltype(tpr)::value, BLOCK = threads_of(TPR), EACH = BLOCK / TPR;
            constexpr bool WHOLE = decltype(whole)::value;
            in_launches<T>(a, BLOCK, EACH, [&](const BlockArgs &n) {
                block_kernel<T, P, NV, TPR, WHOLE><<<dim3((uint32_t)ceil_div(n.rows, EACH)), BLOCK, 0, st>>>(n);
            });
        });
        if (!fits)
            in_launches<T>(a, THREADS, 1, [&](const BlockArgs &n) {
                block_wide_kernel<T, P><<<dim3((uint32_t)n.rows), THREADS, 0, st>>>(n);
            });
        return launch_status("block_norm");
    });
}

int64_t boa_block_norm_backward_workspace(int64_t rows, int32_t d)
{
    if (rows < 0 || d < 1) return 0;
    return (back_blocks(rows, d) * SUMS * d + 2 * rows) * (int64_t)sizeof(float);
}

int boa_block_norm_backward(const boa_block *b, void *stream)
{
    if (int rc = check("block_norm_backward", b, true)) return rc;
    BlockArgs a = args_of(b);
    a.dx = b->dx, a.df = b->df, a.dgate = a.gate_rows ? b->dgate : nullptr;
    const bool sums = b->dweight || b->dbias || b->dpost_weight || b->dpost_bias || (b->dgate && !a.gate_rows);
    if (!sums && (b->rows == 0 || (!a.dx && !a.df && !a.dgate))) return BOA_OK;
    const int64_t blocks = back_blocks(b->rows, b->d);
    if (sums) a.partial = (float *)b->workspace, a.back = a.partial + blocks * SUMS * b->d;
    hipStream_t st = (hipStream_t)stream;
    return with_types(b->dtype, b->param_dtype, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        constexpr int VEC = 16 / sizeof(T);
        const bool fits = with_shape<VEC, false>(b->d, [&](auto nv, auto tpr, auto whole) {
            constexpr int NV = decltype(nv)::value, TPR = decltype(tpr)::value;
            constexpr bool WHOLE = decltype(whole)::value;
            constexpr int own = PARAM_FLOATS<T, NV, TPR> <= 8192 ? PARAM_FLOATS<T, NV, TPR> : 0;
            const size_t lds = sizeof(float) * std::max<size_t>(own, TPR < 128 ? (size_t)SUMS * b->d : 0);
            const dim3 grid((uint32_t)blocks);
            if (sums) block_back_kernel<T, P, NV, TPR, WHOLE, true><<<grid, threads_of(TPR), lds, st>>>(a);
            else block_back_kernel<T, P, NV, TPR, WHOLE, false><<<grid, threads_of(TPR), lds, st>>>(a);
        });
        if (!fits) {
            in_launches<T>(a, THREADS, 1, [&](const BlockArgs &n) {
                block_back_wide_kernel<T, P><<<dim3((uint32_t)n.rows), THREADS, 0, st>>>(n);
            });
            if (sums) block_cols_kernel<T, P><<<dim3((uint32_t)blocks, (uint32_t)ceil_div(b->d, THREADS)), THREADS, 0, st>>>(a);
        }
        if (sums) {
            JoinArgs<P> j{};
            j.partial = a.partial, j.blocks = (int32_t)blocks, j.d = b->d;
            j.gate = a.gate_rows ? nullptr : (const P *)a.gate, j.pw = (const P *)a.pw, j.pb = (const P *)a.pb;
            j.dw = (P *)b->dweight, j.db = (P *)b->dbias, j.dpw = (P *)b->dpost_weight, j.dpb = (P *)b->dpost_bias;
            j.dgate = a.gate_rows ? nullptr : (P *)b->dgate;
            block_join_kernel<P><<<dim3((uint32_t)ceil_div(b->d, JOIN_COLS), 2), JOIN_COLS * JOIN_SLICES, 0, st>>>(j);
        }
        return launch_status("block_norm_backward");
    });
}

}  // extern "C"
