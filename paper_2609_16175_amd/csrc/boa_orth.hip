// Orthogonalisation of a weight's update by Newton-Schulz products.
//
//   X = G / (|G| + eps), |G| the root of the sum of squares; then some times
//   X <- a X + (b A + c A^2) X,   A = X X^T
//
// which takes every singular value s of X to a s + b s^3 + c s^5 and leaves the
// singular vectors: towards 1 with the right coefficients. X lies so that A is
// the smaller of the two Gram matrices (m x m, m <= n). A and A^2 are symmetric:
// half of their tiles are computed, and written twice. What is left is
// 3 m^2 n + m^3 multiply-adds a step, which bound it for all but small matrices.
//
// The products run on the f16 matrix instructions. X itself is kept in float32 beside
// its f16 copy: values that have shrunk towards 0 are multiplied by a at every
// step, and rounding X to 16 bits would put noise into directions that G does
// not have and let it grow (a relative error of 0.04 for updates of rank 8 in
// 512 x 512, 0.0004 so); rounding the products' operands only
// turns the directions that are there. For bfloat16 updates of at least 128
// rows and columns A, b A + c A^2 and X are rounded to f16 (11 bits) as operands,
// which puts results off by less than their rounding to bfloat16 does; for
// others every operand is two f16 parts (22 bits), and three products. G is
// scaled by a power of two, which rounds nothing; the rest of 1 / |G| goes into the
// first step's coefficients.
#include <cmath>

#include "boa_gemm.h"

using namespace boa;

namespace {

constexpr int SUM_BLOCKS = 256;   // per matrix, at most
// What f16 copies hold of X, A and b A + c A^2: values times 2^10, 2^10, 2^8, or
// less in steps whose singular values could take them out of float16's range.
constexpr float X_UP = 1024.0f, A_UP = 1024.0f, B_UP = 256.0f;

struct Scales {
    float x, a, b;
};

struct Step {
    float a, b, c;
};

struct PrepArgs {
    const void *g;
    int64_t ld, batch;          // of g
    int32_t rows, cols, turned; // turned: X is g transposed
    int32_t m, n, x_ld;         // of X
    int64_t x_size, parts;      // values of one X; the same for copies of two parts (0: one part)
    float *x;
    f16_t *x16;
    double *sums;               // SUM_BLOCKS per matrix
    int32_t sum_blocks;
    float eps;
    Step *first;                // per matrix: the first step's coefficients
    Step step0;
};

// Sums of squares of a stripe of rows, in float64: float32's smallest values square
// below its range, its largest above. 4096 x 2048 in bfloat16: 9 us.
template <class T>
__global__ __launch_bounds__(256) void square_kernel(PrepArgs a)
{
    __shared__ double part[4];
    const T *g = (const T *)a.g + blockIdx.y * a.batch;
    const int32_t runs = (a.cols + 7) / 8;
    double s = 0.0;
    // a group of threads per row, as wide as the row has runs of eight, up to the block
    int32_t wide = 256;
    while (wide > 8 && wide / 2 >= runs) wide /= 2;
    const int32_t mine = threadIdx.x % wide, group = threadIdx.x / wide, groups = 256 / wide;
    for (int64_t r = (int64_t)blockIdx.x * groups + group; r < a.rows; r += (int64_t)gridDim.x * groups)
        for (int32_t c = mine * 8; c < a.cols; c += wide * 8) {
            const T *from = g + r * a.ld + c;
            float v[8];
            if (c + 8 <= a.cols) {
                load_loose<8, T>(v, from);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = c + e < a.cols ? (float)from[e] : 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) s = fma((double)v[e], (double)v[e], s);
        }
#pragma unroll
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) a.sums[(int64_t)blockIdx.y * SUM_BLOCKS + blockIdx.x] = part[0] + part[1] + part[2] + part[3];
}

// eight values as an f16 copy, and what it leaves out as the second part
__device__ inline void write16(f16_t *to, int64_t parts, const float (&v)[8])
{
    f16x8 hi, lo;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        hi[e] = (f16_t)v[e];
        lo[e] = (f16_t)(v[e] - (float)hi[e]);
    }
    *(f16x8 *)to = hi;
    if (parts) *(f16x8 *)(to + parts) = lo;
}

// The power of two that brings |G| = total into [1, 2), and the first step's
// coefficients for G times it in place of G / (|G| + eps).
struct First {
    int up;
    Step step;
};

__device__ inline First first_step(double total, float eps, const Step &s)
{
    First f;
    f.up = total > 0.0 && total < INFINITY ? 1 - __builtin_amdgcn_frexp_exp(total) : 0;
    const double by = total < INFINITY ? 1.0 / ldexp(total + (double)eps, f.up) : NAN, b3 = by * by * by;
    // |G| = 0 and eps = 0: X is 0, not NaN
    f.step = total == 0.0 ? Step{0.0f, 0.0f, 0.0f} : Step{(float)(s.a * by), (float)(s.b * b3), (float)(s.c * b3 * by * by)};
    return f;
}

// X of the first step: G times the power of two that brings |G| into [1, 2), as
// float32 and f16, in tiles of 64 x 64; and that step's coefficients. 4096 x 2048 in
// bfloat16, which is turned: 19 us, 3.6 TB/s.
template <class T>
__global__ __launch_bounds__(256) void prep_kernel(PrepArgs a)
{
    __shared__ float tile[64][65];
    __shared__ double total;
    const int32_t z = blockIdx.z;
    if (threadIdx.x < 64) {
        double s = 0.0;
#pragma unroll
        for (int k = 0; k < SUM_BLOCKS / 64; ++k) {
            const int32_t i = k * 64 + (int32_t)threadIdx.x;
            s += i < a.sum_blocks ? a.sums[(int64_t)z * SUM_BLOCKS + i] : 0.0;
        }
#pragma unroll
        for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o);
        if (threadIdx.x == 0) total = sqrt(s);
    }
    const T *g = (const T *)a.g + z * a.batch;
    const int32_t r0 = (a.turned ? blockIdx.x : blockIdx.y) * 64, c0 = (a.turned ? blockIdx.y : blockIdx.x) * 64;
    for (int i = threadIdx.x; i < 64 * 64; i += 256) {
        const int r = i >> 6, c = i & 63;
        const float v = r0 + r < a.rows && c0 + c < a.cols ? (float)g[(int64_t)(r0 + r) * a.ld + c0 + c] : 0.0f;
        if (a.turned) tile[c][r] = v;
        else tile[r][c] = v;
    }
    __syncthreads();
    const First first = first_step(total, a.eps, a.step0);
    const int up = first.up;
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.first[z] = first.step;
    const int32_t p0 = blockIdx.y * 64, q0 = blockIdx.x * 64;
    for (int i = threadIdx.x; i < 64 * 8; i += 256) {
        const int p = i >> 3, q = (i & 7) * 8;
        if (p0 + p >= a.m || q0 + q >= a.x_ld) continue;
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = ldexpf(tile[p][q + e], up);
        const int64_t at = z * a.x_size + (int64_t)(p0 + p) * a.x_ld + q0 + q;
        store_f32<4, float>(a.x + at, *(float(*)[4])v);
        store_f32<4, float>(a.x + at + 4, *(float(*)[4])(v + 4));
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= X_UP;
        write16(a.x16 + at + z * a.parts, a.parts, v);   // the parts of a matrix follow each other
    }
}

enum Kind { GRAM, POLY, UPDATE, LAST };

struct StepArgs {
    Kind kind;
    f16_t *to;               // GRAM: A; POLY: b A + c A^2; UPDATE: X
    int64_t to_ld, to_size, to_parts;   // to_size: from matrix to matrix
    const f16_t *a;          // POLY: A, laid out as `to`
    float *x;                // UPDATE: X, in place; LAST: read only
    int64_t x_size;
    void *out;               // LAST
    int64_t out_ld, out_size;
    int32_t rows, cols;      // that are written (columns of `to` up to its padding)
    int32_t dtype, turned;
    Step step;
    const Step *first;       // per matrix, in place of `step`, or null
    Scales up;               // of this step's copies
    float x_next;            // UPDATE: X's in the next one
};

// tile_product and what becomes of it. B_ACROSS: X, whose rows are k. 4096 x 2048 in
// bfloat16: A and b A + c A^2 36 us each (half of the tiles of 34 and 17 GFLOP), X 52
// us (660 TFLOP/s); four of 768 x 768 as parts: 24 us each, latency of 24 stages.
template <class S, bool B_ACROSS, bool PARTS>
__global__ __launch_bounds__(S::THREADS, S::WAVES_PER_SIMD) void step_kernel(Product pr, StepArgs e)
{
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const Place w = place_of(pr, blockIdx.x, gridDim.x);
    if (!is_needed(pr, w)) return;
    f32x16 acc[S::TB][S::TA];
    clear<S>(acc);
    if (!tile_product<S, false, B_ACROSS, PARTS>(pr, w, (f16_t *)lds, acc)) return;
    const Step k = e.first ? e.first[w.batch] : e.step;
    const int64_t base = w.batch * e.to_size;
    if constexpr (!B_ACROSS) {
        // powers of two, all of them
        const float gram = e.up.a / (e.up.x * e.up.x), linear = e.up.b / e.up.a, quadratic = e.up.b / (e.up.a * e.up.a);
        auto value = [&](float v, int64_t at) {
            if (e.kind == GRAM) return v * gram;
            float was = (float)e.a[at];
            if (e.to_parts) was += (float)e.a[at + e.to_parts];
            return k.b * was * linear + k.c * (v * quadratic);
        };
        each_run<S>(w, acc, lds, [](int32_t, int32_t, int) { return Nothing{}; },
            [&](int32_t p, int32_t q, const float *v, const Nothing &) {
                if (p >= e.rows || q >= e.to_ld) return;
                const int64_t at = base + p * e.to_ld + q;
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = value(v[i], at + i);
                write16(e.to + at, e.to_parts, o);
            },
            w.ta != w.tb,
            [&](int32_t p, int32_t q, const float (&v)[8]) {   // the mirrored tile
                if (q >= e.rows || p >= e.to_ld) return;
                const int64_t at = base + q * e.to_ld + p;
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = value(v[i], at + i);
                write16(e.to + at, e.to_parts, o);
            });
    } else {
        float *x = e.x + w.batch * e.x_size;
        const float by = 1.0f / (e.up.b * e.up.x);
        auto put = [&](int64_t at, float v) {
            const int64_t i = w.batch * e.out_size + at;
            if (e.dtype == BOA_T_F32) ((float *)e.out)[i] = v;
            else if (e.dtype == BOA_T_BF16) ((bf16_t *)e.out)[i] = (bf16_t)v;
            else ((f16_t *)e.out)[i] = (f16_t)v;
        };
        each_run<S>(w, acc, lds, [](int32_t, int32_t, int) { return Nothing{}; },
            [&](int32_t p, int32_t q, const float *v, const Nothing &) {
                if (p >= e.rows || q >= e.to_ld) return;
                const int64_t at = p * e.to_ld + q;
                float was[8], o[8];
                load_f32<4, float>(*(float(*)[4])was, x + at);
                load_f32<4, float>(*(float(*)[4])(was + 4), x + at + 4);
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = fmaf(k.a, was[i], v[i] * by);
                if (e.kind == UPDATE) {
                    store_f32<4, float>(x + at, *(float(*)[4])o);
                    store_f32<4, float>(x + at + 4, *(float(*)[4])(o + 4));
#pragma unroll
                    for (int i = 0; i < 8; ++i) o[i] *= e.x_next;
                    write16(e.to + base + at, e.to_parts, o);
                } else if (!e.turned) {
                    if (q + 8 <= e.cols && e.dtype != BOA_T_F32) {
                        void *to = (char *)e.out + (w.batch * e.out_size + p * e.out_ld + q) * 2;
                        if (e.dtype == BOA_T_BF16) store_loose<8, bf16_t>((bf16_t *)to, o);
                        else store_loose<8, f16_t>((f16_t *)to, o);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (q + i < e.cols) put(p * e.out_ld + q + i, o[i]);
                    }
                }
            },
            e.kind == LAST && e.turned,
            [&](int32_t p, int32_t q, const float (&v)[8]) {   // rows p of X are columns of the output
                if (q >= e.cols) return;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (p + i < e.rows) put(q * e.out_ld + p + i, fmaf(k.a, x[(p + i) * e.to_ld + q], v[i] * by));
            });
    }
}

// ---------------------------------------------------------------------------
// small matrices: a block does all steps on one, in LDS and in float32

constexpr int SMALL_WAVES = 16, SMALL_TILES = 8;   // tiles of X a wave may have
constexpr int SMALL_LDS = 158 << 10;

struct SmallArgs {
    const void *g;
    int64_t ld, batch;
    void *out;
    int32_t rows, cols, turned, m, n, m_pad, n_pad, steps;   // pads: multiples of 16
    float eps;
    Step step[BOA_MAX_ORTH_STEPS];
};

// Waves that share the sum of a tile of X X': 16 or 4 where it has 1 or 4 tiles, if the sum is long enough to pay for
// the joining.
__host__ __device__ inline int small_slices(int32_t m_pad, int32_t n_pad)
{
    return n_pad < 192 || m_pad > 32 ? 1 : m_pad <= 16 ? SMALL_WAVES : SMALL_WAVES / 4;
}

// LDS rows are 4 values longer than their tiles, so that 16 rows x 16 values read together lie in all banks.
inline int64_t small_bytes(int32_t m_pad, int32_t n_pad)
{
    return ((int64_t)m_pad * (n_pad + 4) + 2 * (int64_t)m_pad * (m_pad + 4) + (small_slices(m_pad, n_pad) > 1 ? SMALL_WAVES * 256 : 0)) * 4;
}

// Products by float32 matrix instructions, a 16 x 16 tile a wave at a time.
// X (m x n), A and B = b A + c A^2 (m x m) stay in LDS; every wave holds its
// TILES tiles of the new X until all have read the old one. Bound by the
// latencies of four short phases a step: 32 x 96, 5 steps, 17 us (82 in the 17
// launches of the large kernels); 64 x 256 73 (109); 64 x 400 115 (123); 64 x
// 480, the longest that fits, 134 (122), but 256 of them together 155 (508).
// TILES = 8 for all would cost 32 x 96 3 us of instruction fetches; a sum of 16
// x 1,024 split over 16 waves saves 24 us.
template <class T, int TILES>
__global__ __launch_bounds__(64 * SMALL_WAVES) void small_kernel(SmallArgs s)
{
    extern __shared__ __attribute__((aligned(16))) float x[];
    __shared__ double part[SMALL_WAVES];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, r = lane & 15, q = lane >> 4;
    const int xl = s.n_pad + 4, al = s.m_pad + 4, mt = s.m_pad / 16, nt = s.n_pad / 16;
    float *a = x + s.m_pad * xl, *b = a + s.m_pad * al;
    const T *g = (const T *)s.g + blockIdx.x * s.batch;
    double sum = 0.0;
    for (int from = threadIdx.x; from < s.m_pad * s.n_pad; from += 4 * 64 * SMALL_WAVES) {   // four loads on their way
        float v[4];
        int at[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int i = from + e * 64 * SMALL_WAVES;
            const int row = s.turned ? i % s.m_pad : i / s.n_pad, col = s.turned ? i / s.m_pad : i % s.n_pad;
            const int64_t to = min(row, s.m - 1), along = min(col, s.n - 1);
            v[e] = (float)(s.turned ? g[along * s.ld + to] : g[to * s.ld + along]);
            if (row >= s.m || col >= s.n) v[e] = 0.0f;
            at[e] = i < s.m_pad * s.n_pad ? row * xl + col : -1;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (at[e] < 0) continue;
            x[at[e]] = v[e];
            sum = fma((double)v[e], (double)v[e], sum);
        }
    }
#pragma unroll
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int i = 0; i < SMALL_WAVES; ++i) sum += part[i];
    const First first = first_step(sqrt(sum), s.eps, s.step[0]);
    for (int i = threadIdx.x; i < s.m_pad * s.n_pad; i += 64 * SMALL_WAVES) {
        float *v = x + i / s.n_pad * xl + i % s.n_pad;
        *v = ldexpf(*v, first.up);
    }
    __syncthreads();
    // sum over k in [from, to) of a row of `u` times a row, or `down` a column, of `v`; a lane's four k are next to each other
    auto product = [&](const float *u, int ul, int ti, const float *v, int vl, int tj, int from, int to, auto down) {
        f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
        const float *pu = u + (ti * 16 + r) * ul + 4 * q, *pv = down ? v + 4 * q * vl + tj * 16 + r : v + (tj * 16 + r) * vl + 4 * q;
#pragma unroll 2
        for (int k = from; k < to; k += 16) {
            const f32x4 f = *(const f32x4 *)(pu + k);
            f32x4 g;
            if constexpr (down) {
#pragma unroll
                for (int e = 0; e < 4; ++e) g[e] = pv[(k + e) * vl];
            } else {
                g = *(const f32x4 *)(pv + k);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(f[e], g[e], acc, 0, 0, 0);
        }
        return acc;
    };
    // u u' for a symmetric result, its tiles to `to`; few tiles: each sum over several waves, joined in order
    const int tiles = mt * mt;
    f32x4 *joined = (f32x4 *)(b + s.m_pad * al);
    auto square = [&](const float *u, int ul, int K, int slices, auto to) {
        if (slices == 1) {
            for (int t = wave; t < tiles; t += SMALL_WAVES)
                to(t, product(u, ul, t / mt, u, ul, t % mt, 0, K, std::false_type{}));   // mirrored tiles: the same roundings
        } else {
            const int t = wave % tiles, at = wave / tiles, k = K / 16;
            joined[threadIdx.x] = product(u, ul, t / mt, u, ul, t % mt, k * at / slices * 16, k * (at + 1) / slices * 16, std::false_type{});
            __syncthreads();
            if (wave < tiles) {
                f32x4 v = joined[threadIdx.x];
                for (int i = 1; i < slices; ++i) v += joined[threadIdx.x + i * tiles * 64];
                to(wave, v);
            }
        }
        __syncthreads();
    };
    for (int it = 0; it < s.steps; ++it) {
        const Step k = it ? s.step[it] : first.step;
        square(x, xl, s.n_pad, small_slices(s.m_pad, s.n_pad), [&](int tile, const f32x4 &v) {
#pragma unroll
            for (int e = 0; e < 4; ++e) a[(tile / mt * 16 + 4 * q + e) * al + tile % mt * 16 + r] = v[e];
        });
        square(a, al, s.m_pad, 1, [&](int tile, const f32x4 &v) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int at = (tile / mt * 16 + 4 * q + e) * al + tile % mt * 16 + r;
                b[at] = fmaf(k.b, a[at], k.c * v[e]);
            }
        });
        f32x4 now[TILES];
#pragma unroll
        for (int u = 0; u < TILES; ++u) {
            const int t = wave + u * SMALL_WAVES;
            if (t < mt * nt) now[u] = product(b, al, t / nt, x, xl, t % nt, 0, s.m_pad, std::true_type{});
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < TILES; ++u) {
            const int t = wave + u * SMALL_WAVES;
            if (t < mt * nt)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float *v = x + (t / nt * 16 + 4 * q + e) * xl + t % nt * 16 + r;
                    *v = fmaf(k.a, *v, now[u][e]);
                }
        }
        __syncthreads();
    }
    T *out = (T *)s.out + (int64_t)blockIdx.x * s.rows * s.cols;
    for (int i = threadIdx.x; i < s.rows * s.cols; i += 64 * SMALL_WAVES) {
        const int row = i / s.cols, col = i % s.cols;
        out[i] = (T)(s.turned ? x[col * xl + row] : x[row * xl + col]);
    }
}

// ---------------------------------------------------------------------------
// host

template <class S, bool B_ACROSS, bool PARTS>
void launch(Product pr, const StepArgs &e, hipStream_t st)
{
    pr.tiles_a = (int32_t)ceil_div(pr.a.own, S::BA);
    pr.tiles_b = (int32_t)ceil_div(pr.b.own, S::BB);
    const int64_t tiles = tiles_of(pr);
    const auto kernel = step_kernel<S, B_ACROSS, PARTS>;
    if (S::LDS > 64 << 10)   // has to be asked for
        (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, S::LDS);
    kernel<<<dim3((uint32_t)(tiles * pr.batches)), S::THREADS, S::LDS, st>>>(pr, e);
}

template <bool B_ACROSS>
void step(const Operand &a, const Operand &b, int32_t K, bool parts, int64_t batches, const StepArgs &e, hipStream_t st)
{
    Product pr{};
    const Cut cut = choose(a.own, b.own, K, parts, batches, !B_ACROSS, false);
    pr.a = a, pr.b = b, pr.K = K, pr.splits = 1, pr.batches = (int32_t)batches;
    pr.steps = cut.steps, pr.symmetric = !B_ACROSS;
    with_tile<f16_t>(cut.shape, [&](auto tile) {
        if (parts) launch<decltype(tile), B_ACROSS, true>(pr, e, st);
        else launch<decltype(tile), B_ACROSS, false>(pr, e, st);
    });
}

// The power of two, `most` at most, that keeps values of up to m below 2^13: an eighth of float16's range, which leaves
// room for what the roundings of the copies add to singular values.
float scale_for(double m, double most)
{
    int e = 0;
    (void)std::frexp(m, &e);
    return (float)std::min(most, std::ldexp(1.0, std::max(13 - e, -100)));
}

// The scales of each step. No value of a matrix is above its largest singular
// value. That is below 2 for the first X (whose coefficients make a step of values
// up to 1 of it), then at most the largest that a step makes of all values up to
// the bound before it; beyond 2^30 it is not followed. Polynomials over [0, end]
// have their extremes at its end or where their slopes are 0 (places that do not
// exist are infinite or NaN, and not in there).
void scales_of(const Step *step, int32_t steps, Scales *to)
{
    double s = 1.0;
    for (int i = 0; i < steps; ++i) {
        const double x = i ? s : 2.0, a = step[i].a, b = step[i].b, c = step[i].c, end = s * s;   // u = s^2 from here
        auto largest = [&](auto f, std::initializer_list<double> flat) {
            double m = std::fabs(f(end));
            for (double u : flat)
                if (u > 0.0 && u < end) m = std::max(m, std::fabs(f(u)));
            return m;
        };
        const double poly = largest([&](double u) { return u * (b + u * c); }, {-b / (2 * c)});
        to[i] = Scales{scale_for(x, X_UP), scale_for(x * x, A_UP), scale_for(poly, B_UP)};
        const double root = std::sqrt(9 * b * b - 20 * a * c);
        s = std::min(0x1p30, largest([&](double u) { return std::sqrt(u) * (a + u * (b + u * c)); },
                                     {(-3 * b + root) / (10 * c), (-3 * b - root) / (10 * c), -a / (3 * b)}));   // the last where c is 0
    }
}

int check(const boa_orth *d)
{
    if (!d) return set_error(BOA_EINVAL, "orthogonalize: NULL arguments");
    const char *why = nullptr;
    if (!dtype_known(d->dtype)) why = "unknown dtype";
    else if (d->count < 0 || d->count > BOA_MAX_ORTH_COUNT) why = "count out of range [0, 2^16)";
    else if (d->rows < 1 || d->rows > BOA_MAX_ORTH || d->cols < 1 || d->cols > BOA_MAX_ORTH) why = "rows and cols out of range [1, 2^14]";
    else if (d->steps < 1 || d->steps > BOA_MAX_ORTH_STEPS) why = "steps out of range [1, 32]";
    else if (!d->coefficients) why = "NULL coefficients";
    else if (!(d->eps >= 0.0f)) why = "eps must not be negative";
    else if (d->rows > 1 && d->update_stride < d->cols) why = "row stride smaller than cols";
    else if (d->count && (!d->update || !d->out)) why = "NULL matrices";
    if (!why)
        for (int i = 0; i < 3 * d->steps; ++i)
            if (!(d->coefficients[i] - d->coefficients[i] == 0.0f)) why = "coefficients must be finite";
    if (!why) return BOA_OK;
    char msg[160];
    __builtin_snprintf(msg, sizeof(msg), "orthogonalize: %s", why);
    return set_error(BOA_EINVAL, msg);
}

void orthogonalize(const boa_orth &d, Arena &mem, bool run, hipStream_t st)
{
    const bool turned = d.rows > d.cols;
    const int32_t m = turned ? d.cols : d.rows, n = turned ? d.rows : d.cols;
    auto coefficients = [&](int i) { return Step{d.coefficients[3 * i], d.coefficients[3 * i + 1], d.coefficients[3 * i + 2]}; };
    const int32_t m_pad = (m + 15) / 16 * 16, n_pad = (n + 15) / 16 * 16;
    if (m_pad <= 64 && m_pad * n_pad <= 256 * SMALL_WAVES * SMALL_TILES && small_bytes(m_pad, n_pad) <= SMALL_LDS) {
        if (!run) return;
        SmallArgs s{};
        s.g = d.update, s.ld = d.rows > 1 ? d.update_stride : d.cols, s.batch = d.update_batch, s.out = d.out;
        s.rows = d.rows, s.cols = d.cols, s.turned = turned, s.m = m, s.n = n, s.m_pad = m_pad, s.n_pad = n_pad;
        s.steps = d.steps, s.eps = d.eps;
        for (int i = 0; i < d.steps; ++i) s.step[i] = coefficients(i);
        const size_t lds = (size_t)small_bytes(m_pad, n_pad);
        auto launch = [&](auto kernel) {
            if (lds > 60 << 10)   // has to be asked for
                (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, SMALL_LDS);
            kernel<<<dim3((uint32_t)d.count), 64 * SMALL_WAVES, lds, st>>>(s);
        };
        auto small = [&](auto t) {
            const int32_t each = (int32_t)ceil_div(m_pad / 16 * (n_pad / 16), SMALL_WAVES);
            if (each == 1) launch(small_kernel<decltype(t), 1>);
            else if (each <= 4) launch(small_kernel<decltype(t), 4>);
            else launch(small_kernel<decltype(t), SMALL_TILES>);
        };
        if (d.dtype == BOA_T_F32) small(0.0f);
        else if (d.dtype == BOA_T_BF16) small(bf16_t{});
        else small(f16_t{});
        return;
    }
    const bool parts = d.dtype != BOA_T_BF16 || m < 128;
    const int32_t x_ld = pad8(n), a_ld = pad8(m);
    const int64_t x_size = (int64_t)m * x_ld, a_size = (int64_t)m * a_ld, C = d.count, copies = parts ? 2 : 1;
    float *x = (float *)mem.take(C * x_size * 4);
    f16_t *x16[2];   // the update reads the one and writes the other
    for (auto &p : x16) p = (f16_t *)mem.take(C * x_size * copies * 2);
    f16_t *a16 = (f16_t *)mem.take(C * a_size * copies * 2), *b16 = (f16_t *)mem.take(C * a_size * copies * 2);
    double *sums = (double *)mem.take(C * SUM_BLOCKS * 8);
    Step *first = (Step *)mem.take(C * (int64_t)sizeof(Step));
    if (!run) return;
    PrepArgs p{};
    p.g = d.update, p.ld = d.rows > 1 ? d.update_stride : d.cols, p.batch = d.update_batch, p.rows = d.rows, p.cols = d.cols;
    p.turned = turned, p.m = m, p.n = n, p.x_ld = x_ld, p.x_size = x_size, p.parts = parts ? x_size : 0;
    p.x = x, p.x16 = x16[0], p.sums = sums, p.eps = d.eps, p.first = first, p.step0 = coefficients(0);
    p.sum_blocks = (int32_t)std::min<int64_t>(SUM_BLOCKS, ceil_div((int64_t)d.rows * d.cols, 8192));
    const dim3 squares((uint32_t)p.sum_blocks, (uint32_t)C), tiles((uint32_t)ceil_div(x_ld, 64), (uint32_t)ceil_div(m, 64), (uint32_t)C);
    auto prepare = [&](auto t) {
        using T = decltype(t);
        square_kernel<T><<<squares, 256, 0, st>>>(p);
        prep_kernel<T><<<tiles, 256, 0, st>>>(p);
    };
    if (d.dtype == BOA_T_F32) prepare(0.0f);
    else if (d.dtype == BOA_T_BF16) prepare(bf16_t{});
    else prepare(f16_t{});

    auto operand = [&](const f16_t *p, int64_t ld, int64_t size, int32_t own, bool across) {
        Operand o{};
        o.p = p, o.ld = ld, o.part = size, o.block = across ? 32 * ld : 32, o.batch = size * copies, o.own = own;
        return o;
    };
    const Operand A = operand(a16, a_ld, a_size, m, false), B = operand(b16, a_ld, a_size, m, false);
    Step each[BOA_MAX_ORTH_STEPS];
    Scales up[BOA_MAX_ORTH_STEPS];
    for (int i = 0; i < d.steps; ++i) each[i] = coefficients(i);
    scales_of(each, d.steps, up);
    for (int i = 0; i < d.steps; ++i) {
        const Operand X = operand(x16[i & 1], x_ld, x_size, m, false), Xk = operand(x16[i & 1], x_ld, x_size, x_ld, true);
        StepArgs e{};
        e.step = each[i], e.first = i == 0 ? first : nullptr, e.up = up[i];
        e.rows = m, e.to_ld = a_ld, e.to_size = a_size * copies, e.to_parts = parts ? a_size : 0;
        e.kind = GRAM, e.to = a16;
        step<false>(X, X, n, parts, C, e, st);
        e.kind = POLY, e.to = b16, e.a = a16;
        step<false>(A, A, m, parts, C, e, st);
        e.kind = i + 1 < d.steps ? UPDATE : LAST;
        e.to = x16[(i + 1) & 1], e.to_ld = x_ld, e.to_size = x_size * copies, e.to_parts = parts ? x_size : 0;
        e.x = x, e.x_size = x_size, e.x_next = i + 1 < d.steps ? up[i + 1].x : 0.0f;
        e.out = d.out, e.out_ld = d.cols, e.out_size = (int64_t)d.rows * d.cols, e.cols = n, e.dtype = d.dtype, e.turned = turned;
        step<true>(B, Xk, m, parts, C, e, st);
    }
}

}  // namespace

extern "C" {

int64_t boa_orthogonalize_workspace(const boa_orth *d)
{
    if (int rc = check(d)) return rc;
    Arena mem;
    orthogonalize(*d, mem, false, nullptr);
    return mem.used;
}

int boa_orthogonalize(const boa_orth *d, void *workspace, int64_t workspace_bytes, void *stream)
{
    if (int rc = check(d)) return rc;
    if (d->count == 0) return BOA_OK;
    const int64_t need = boa_orthogonalize_workspace(d);
    if (need && (!workspace || !aligned(workspace, 16) || workspace_bytes < need))
        return set_error(BOA_EINVAL, "orthogonalize: workspace missing, unaligned or too small");
    Arena mem;
    mem.base = (char *)workspace;
    orthogonalize(*d, mem, true, (hipStream_t)stream);
    return launch_status("orthogonalize");
}

}  // extern "C"
