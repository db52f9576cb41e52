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
// gate.
//
// Both are bound by memory. Forward reads x and f (and a gate per value) and
// writes h and y; backward reads x, f, dh and dy and writes dx and df: h is
// formed again from x and f in float32, which costs what reading it would and
// keeps the digits that its rounding loses. A row stays in registers, as in boa_norm.hip: a
// wave holds up to 1,024 values, a block 4,096, and every thread at most 16
// columns, so that the five column sums stay in registers too, over all rows
// of a block; they leave one partial row each per block, added in block order.
#include <algorithm>

#include "boa_rows.h"

using namespace boa;

namespace {

constexpr int THREADS = ROW_THREADS;
constexpr int SUMS = 5;   // over rows: dw, db, dpw, dpb, dg
constexpr int64_t MAX_BLOCKS = 512;

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

// The arguments of the rows from `row` on that one launch takes.
template <class T>
BlockArgs rows_from(BlockArgs a, int64_t row)
{
    a.x = plus<T>(a.x, row * a.x_ld), a.f = plus<T>(a.f, row * a.f_ld);
    if (a.gate_rows) a.gate = plus<T>(a.gate, row * a.gate_ld);
    a.dh = plus<T>(a.dh, row * a.dh_ld), a.dy = plus<T>(a.dy, row * a.dy_ld);
    a.h = plus<T>(a.h, row * a.d), a.y = plus<T>(a.y, row * a.d), a.dx = plus<T>(a.dx, row * a.d);
    a.df = plus<T>(a.df, row * a.d), a.dgate = plus<T>(a.dgate, row * a.d);
    a.stats = plus<float>(a.stats, row), a.back = plus<float>(a.back, 2 * row);
    a.rows = std::min(LAUNCH_ROWS, a.rows - row);
    return a;
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

template <class T, class P, int NV, int TPR, bool WHOLE>
__global__ __launch_bounds__(THREADS) void block_kernel(BlockArgs a)
{
    constexpr int VEC = 16 / sizeof(T);
    __shared__ float red[8];
    const int lane = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (THREADS / TPR) + threadIdx.x / TPR;
    if (row >= a.rows) return;   // a whole wave (TPR 64) or block (TPR 256) leaves
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

// DP: column sums are wanted.
template <class T, class P, int NV, int TPR, bool WHOLE, bool DP>
__global__ __launch_bounds__(THREADS) void block_back_kernel(BlockArgs a)
{
    constexpr int VEC = 16 / sizeof(T), GROUPS = THREADS / TPR;
    __shared__ float red[8];
    extern __shared__ float cols[];   // SUMS x d, where several rows share a block
    const int lane = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const int32_t d = a.d;
    float sums[SUMS][NV][VEC];
#pragma unroll
    for (int k = 0; k < SUMS; ++k)
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) sums[k][i][j] = 0.0f;
    for (int64_t row = (int64_t)blockIdx.x * GROUPS + group; row < a.rows; row += (int64_t)gridDim.x * GROUPS) {
        float fn[NV][VEC], hn[NV][VEC], dH[NV][VEC], g1[NV][VEC];
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = Cols<VEC, TPR>(i, lane, d).c;
            load_loose<VEC, T>(fn[i], (const T *)a.f + row * a.f_ld + c);
            load_loose<VEC, T>(hn[i], (const T *)a.x + row * a.x_ld + c);
            if (a.dh) load_loose<VEC, T>(dH[i], (const T *)a.dh + row * a.dh_ld + c);
            if (a.dy) load_loose<VEC, T>(g1[i], (const T *)a.dy + row * a.dy_ld + c);
        }
        const float pm = a.post ? a.stats[row] : 0.0f, pr = a.post ? a.stats[a.stats_rows + row] : 1.0f;
        const float hm = a.dy ? a.stats[2 * a.stats_rows + row] : 0.0f, hr = a.dy ? a.stats[3 * a.stats_rows + row] : 0.0f;
        // h again, its norm, and the gradient through it
        float c1 = 0.0f, c2 = 0.0f;
        auto gate_at = [&](float (&g)[VEC], int c) {
            if (a.gate_rows) load_loose<VEC, T>(g, (const T *)a.gate + row * a.gate_ld + c);
            else params<P, VEC>(g, a.gate, c, 1.0f);
        };
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Cols<VEC, TPR> at(i, lane, d);
            float pw[VEC], pb[VEC], g[VEC], w[VEC];
            params<P, VEC>(pw, a.pw, at.c, 1.0f);
            params<P, VEC>(pb, a.pb, at.c, 0.0f);
            gate_at(g, at.c);
            params<P, VEC>(w, a.w, at.c, 1.0f);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                fn[i][j] = (fn[i][j] - pm) * pr;
                const float u = fmaf(fn[i][j], pw[j], pb[j]);
                hn[i][j] = (fmaf(a.scale, hn[i][j], g[j] * u) - hm) * hr;
                if (!a.dh) dH[i][j] = 0.0f;
                if (!a.dy) g1[i][j] = 0.0f;
                if (DP) {
                    sums[0][i][j] = fmaf(g1[i][j], hn[i][j], sums[0][i][j]);
                    sums[1][i][j] += g1[i][j];
                }
                // columns that are not this thread's count for nothing in the row's sums
                g1[i][j] = at.template mine<WHOLE>(j) ? g1[i][j] * w[j] : 0.0f;
                c1 += g1[i][j];
                c2 = fmaf(g1[i][j], hn[i][j], c2);
            }
        }
        if (a.dy) {
            row_sum2<TPR>(c1, c2, red);
            c1 = a.layer ? c1 / (float)d : 0.0f;
            c2 /= (float)d;
        }
        float p1 = 0.0f, p2 = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Cols<VEC, TPR> at(i, lane, d);
            float pw[VEC], pb[VEC], g[VEC], o[VEC];
            params<P, VEC>(pw, a.pw, at.c, 1.0f);
            params<P, VEC>(pb, a.pb, at.c, 0.0f);
            gate_at(g, at.c);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                dH[i][j] = fmaf(hr, g1[i][j] - c1 - hn[i][j] * c2, dH[i][j]);
                o[j] = a.scale * dH[i][j];
            }
            if (a.dx) store_mine<T, VEC, TPR, WHOLE>((T *)a.dx + row * (int64_t)d, at, o);
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                o[j] = dH[i][j] * fmaf(fn[i][j], pw[j], pb[j]);
                if (DP) sums[4][i][j] += o[j];
                dH[i][j] *= g[j];
                if (DP) {
                    sums[2][i][j] = fmaf(dH[i][j], fn[i][j], sums[2][i][j]);
                    sums[3][i][j] += dH[i][j];
                }
                dH[i][j] = at.template mine<WHOLE>(j) ? dH[i][j] * pw[j] : 0.0f;
                p1 += dH[i][j];
                p2 = fmaf(dH[i][j], fn[i][j], p2);
            }
            if (a.dgate) store_mine<T, VEC, TPR, WHOLE>((T *)a.dgate + row * (int64_t)d, at, o);
        }
        if (!a.df) continue;
        if (a.post) {
            row_sum2<TPR>(p1, p2, red);
            p1 = a.layer ? p1 / (float)d : 0.0f;
            p2 /= (float)d;
        } else {
            p1 = p2 = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Cols<VEC, TPR> at(i, lane, d);
            float o[VEC];
#pragma unroll
            for (int j = 0; j < VEC; ++j) o[j] = pr * (dH[i][j] - p1 - fn[i][j] * p2);
            store_mine<T, VEC, TPR, WHOLE>((T *)a.df + row * (int64_t)d, at, o);
        }
    }
    if constexpr (DP) {
        float *out = a.partial + (int64_t)blockIdx.x * SUMS * d;
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
                            float *to = (GROUPS == 1 ? out : cols) + (int64_t)q * d + at.c + j;
                            *to = k ? *to + sums[q][i][j] : sums[q][i][j];
                        }
                    }
                }
            }
            if (GROUPS > 1) __syncthreads();
        }
        if (GROUPS > 1)
            for (int c = threadIdx.x; c < SUMS * d; c += THREADS) out[c] = cols[c];
    }
}

// ---------------------------------------------------------------------------
// rows wider than the registers, or narrower than a load: a block per row, which
// reads it once for every sum (from the caches after the first time)

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
        const float dy = w.dy(c), dH = w.dH(c, a.back[2 * row], a.back[2 * row + 1]), du = dH * w.gate(c);
        s[0] = fmaf(dy, w.hn(c), s[0]);
        s[1] += dy;
        s[2] = fmaf(du, w.fn(c), s[2]);
        s[3] += du;
        s[4] = fmaf(dH, w.u(c), s[4]);
    }
#pragma unroll
    for (int k = 0; k < SUMS; ++k) a.partial[((int64_t)blockIdx.x * SUMS + k) * d + c] = s[k];
}

// Adds the blocks' partial rows: 16 columns a block and 64 slices of the rows, then the slices in order.
constexpr int JOIN_COLS = 16, JOIN_SLICES = 64;

template <class P>
struct JoinArgs {
    const float *partial;
    P *to[SUMS];
    int32_t blocks, d;
};

template <class P>
__global__ __launch_bounds__(JOIN_COLS * JOIN_SLICES) void block_join_kernel(JoinArgs<P> a)
{
    __shared__ float part[JOIN_SLICES][JOIN_COLS + 1];
    const int col = threadIdx.x % JOIN_COLS, slice = threadIdx.x / JOIN_COLS, which = blockIdx.y;
    P *to = a.to[which];
    if (!to) return;
    const int32_t c = blockIdx.x * JOIN_COLS + col;
    const float *from = a.partial + (int64_t)which * a.d + c;
    float s = 0.0f;
    if (c < a.d)
#pragma unroll 4
        for (int i = slice; i < a.blocks; i += JOIN_SLICES) s += from[(int64_t)i * SUMS * a.d];
    part[slice][col] = s;
    __syncthreads();
    if (slice == 0 && c < a.d) {
        s = 0.0f;
#pragma unroll
        for (int i = 0; i < JOIN_SLICES; ++i) s += part[i][col];
        to[c] = (P)s;
    }
}

// The registers a row takes: f(NV, TPR, WHOLE) as compile-time constants, at
// most 16 columns a thread; false where a row does not fit, or is shorter than a load.
template <int VEC, class F>
bool with_shape(int32_t d, F f)
{
    const int64_t n = ceil_div(d, VEC);
    if (d < VEC || n * VEC > 4096) return false;
    auto whole = [&](auto nv, auto tpr) { d % VEC ? f(nv, tpr, Int<0>{}) : f(nv, tpr, Int<1>{}); };
    if (n <= 64) whole(Int<1>{}, Int<64>{});
    else if (n <= 128) whole(Int<2>{}, Int<64>{});
    else if constexpr (VEC == 4) {
        if (n <= 192) whole(Int<3>{}, Int<64>{});
        else if (n <= 256) whole(Int<4>{}, Int<64>{});
        else if (n <= 512) whole(Int<2>{}, Int<256>{});
        else whole(Int<4>{}, Int<256>{});
    } else {
        if (n <= 256) whole(Int<1>{}, Int<256>{});
        else whole(Int<2>{}, Int<256>{});
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
    // As many partial rows as blocks: at most 2 per CU, what the registers let
    // run at once; fewer of few rows, and of wide ones 128 MB of them at most.
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(MAX_BLOCKS, ((int64_t)1 << 25) / ((int64_t)SUMS * d)));
    return std::max<int64_t>(1, std::min(most, ceil_div(rows, 8)));
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
        for (int64_t row = 0; row < b->rows; row += LAUNCH_ROWS) {
            const BlockArgs n = rows_from<T>(a, row);
            const bool fits = with_shape<VEC>(b->d, [&](auto nv, auto tpr, auto whole) {
                constexpr int NV = decltype(nv)::value, TPR = decltype(tpr)::value;
                constexpr bool WHOLE = decltype(whole)::value;
                block_kernel<T, P, NV, TPR, WHOLE><<<dim3((uint32_t)ceil_div(n.rows, THREADS / TPR)), THREADS, 0, st>>>(n);
            });
            if (!fits) block_wide_kernel<T, P><<<dim3((uint32_t)n.rows), THREADS, 0, st>>>(n);
        }
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
    void *to[SUMS] = {b->dweight, b->dbias, b->dpost_weight, b->dpost_bias, a.gate_rows ? nullptr : b->dgate};
    const bool sums = std::any_of(to, to + SUMS, [](void *p) { return p != nullptr; });
    if (!sums && (b->rows == 0 || (!a.dx && !a.df && !a.dgate))) return BOA_OK;
    const int64_t blocks = back_blocks(b->rows, b->d);
    if (sums) a.partial = (float *)b->workspace, a.back = a.partial + blocks * SUMS * b->d;
    hipStream_t st = (hipStream_t)stream;
    return with_types(b->dtype, b->param_dtype, [&](auto t, auto p) {
        using T = decltype(t);
        using P = decltype(p);
        constexpr int VEC = 16 / sizeof(T);
        const bool fits = with_shape<VEC>(b->d, [&](auto nv, auto tpr, auto whole) {
            constexpr int NV = decltype(nv)::value, TPR = decltype(tpr)::value;
            constexpr bool WHOLE = decltype(whole)::value;
            const size_t lds = sums && TPR < THREADS ? (size_t)SUMS * b->d * sizeof(float) : 0;
            if (sums) block_back_kernel<T, P, NV, TPR, WHOLE, true><<<dim3((uint32_t)blocks), THREADS, lds, st>>>(a);
            else block_back_kernel<T, P, NV, TPR, WHOLE, false><<<dim3((uint32_t)blocks), THREADS, 0, st>>>(a);
        });
        if (!fits) {
            for (int64_t row = 0; row < b->rows; row += LAUNCH_ROWS) {
                const BlockArgs n = rows_from<T>(a, row);
                block_back_wide_kernel<T, P><<<dim3((uint32_t)n.rows), THREADS, 0, st>>>(n);
            }
            if (sums) block_cols_kernel<T, P><<<dim3((uint32_t)blocks, (uint32_t)ceil_div(b->d, THREADS)), THREADS, 0, st>>>(a);
        }
        if (sums) {
            JoinArgs<P> j{};
            j.partial = a.partial, j.blocks = (int32_t)blocks, j.d = b->d;
            for (int k = 0; k < SUMS; ++k) j.to[k] = (P *)to[k];
            block_join_kernel<P><<<dim3((uint32_t)ceil_div(b->d, JOIN_COLS), SUMS), JOIN_COLS * JOIN_SLICES, 0, st>>>(j);
        }
        return launch_status("block_norm_backward");
    });
}

}  // extern "C"
