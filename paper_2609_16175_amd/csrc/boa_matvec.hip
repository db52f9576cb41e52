// Products of a few vectors with rows of 4-bit codes:
//   y[m][n] = sum_k x[m][k] w[n][k],  w = s q + o  or, without offsets, s (q - 8),
// one scale (and offset) per row and group of consecutive k.
#include <algorithm>
#include <type_traits>

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

// ---------------------------------------------------------------------------
// Rows of whole 16-byte chunks (32 codes), groups of whole chunks.
//
// Bound by reading the codes: at half a byte per weight even the few steps
// that turn a code into a number count, so the products run on the 16x16x32
// bf16 matrix instruction and a code becomes a bf16 number in two steps: its
// four bits under an exponent are 16 + q times a power of two, DOWN. x is held
// exactly as bf16 parts (1 of bfloat16, 2 of float16, 3 of float32), each a
// column of its own, and sum (16 + q) x has 24 (or 16) times sum x taken off by
// starting there, which leaves sum (q - 8) x (or sum q x). All of them are DOWN
// times what they stand for until the result is written: so sums over a chunk's
// 32 values, up to 31 times as large as them each, stay finite for any finite x.
//
// A lane holds one row's chunk: lane l has row l & 15 and chunk l >> 4 of four
// in a step of 128 k, so a wave reads 64 bytes of 16 rows at once. Lanes of
// different chunks may need different scales, so their sums must stay apart:
// columns are laid out as 4 chunks x 4 slots, x being zero except in the slots
// of the lane's own chunk. Result row 4 c + s of the matrix instruction is
// then chunk c's sum for slot s, and it lies in the lanes that hold chunk c
// and its scale. The zeros cost matrix time only, which is idle here.
//
// One bfloat16 vector against 1,000,000 rows of 768 codes: 90 us, 4.6 TB/s
// (a read alone 5.8); vector instructions are busy two thirds of that. Five
// float32 vectors against 999,983 rows of 128: 35 us, 3.3 TB/s.

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int FAST_WAVES = 8;               // per block
constexpr int AHEAD = 2;                    // units of loads a wave keeps in flight
constexpr int ROWS_W = 32;                  // rows of a wave: two tiles of 16
constexpr size_t FAST_LDS = 64 << 10;       // x of one stretch of k, at most
constexpr float DOWN = 1.0f / 2048.0f;      // a power of two, 32 x (31 + 24) of which stay below 1

template <class T>
constexpr int parts_v = sizeof(T) == 4 ? 3 : std::is_same<T, bf16_t>::value ? 1 : 2;

// bytes of x in LDS per step of 128 k: 4 chunks x (4 pieces of 8 k x 4 slots x 16 bytes, and 4 sums) per column set
constexpr int step_bytes(int nc) { return nc * (1024 + 64); }

struct FastArgs {
    VecArgs v;
    int32_t m0, vectors;       // the vectors of this launch
    int32_t split_k;           // waves of a block that share rows, each taking every split_k-th step
    int32_t steps, stretch;    // steps of 128 k in a row; of them held in LDS at a time
    uint32_t group_inv;        // 2^32 / (chunks per group), rounded up; 0: one chunk per group
};

// value[0..VALS) of both tiles, summed over the four chunks' lanes; afterwards
// quarter q of the wave holds values 2u + (q & 1) of tile q >> 1 in out[u].
template <int VALS>
__device__ inline void join_chunks(const float (&a)[2][VALS], float (&out)[(VALS + 1) / 2])
{
    float half[VALS + 1];
#pragma unroll
    for (int i = 0; i < VALS; ++i) {
        const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(a[0][i]), __float_as_uint(a[1][i]), false, false);
        half[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    half[VALS] = 0.0f;
#pragma unroll
    for (int u = 0; u < (VALS + 1) / 2; ++u) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(half[2 * u]), __float_as_uint(half[2 * u + 1]), false, false);
        out[u] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
}

// NC column sets of 4 slots; a vector takes parts_v<T> slots in a row.
template <class T, class SC, int NC, bool OFFSETS>
__global__ __launch_bounds__(64 * FAST_WAVES) void rows4_kernel(FastArgs f)
{
    constexpr int PARTS = parts_v<T>, VALS = NC * 4 / PARTS;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    const VecArgs &a = f.v;
    // x: [step][piece j of 4][set][chunk][slot][8 k] bf16; sums: [step][set][chunk][slot]; then a step of zeros
    bf16x8 *xs = (bf16x8 *)lds;
    f32x4 *sums = (f32x4 *)(lds + (size_t)f.stretch * NC * 1024);
    const int zero_at = f.stretch * NC * 68;   // in units of 16 bytes: past x and the sums, NC * 64 of them
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, chunk = lane >> 4, r = lane & 15;
    const int split = wave % f.split_k, per_block = FAST_WAVES / f.split_k;
    const int64_t tiles = (a.rows + ROWS_W - 1) / ROWS_W;

    // x of steps [step0, step0 + stretch): the parts, then their sums
    auto fill = [&](int step0) {
        for (int i = threadIdx.x; i < f.stretch * NC * 64; i += 64 * FAST_WAVES) {
            const int slot = i & 3, c = (i >> 2) & 3, j = (i >> 4) & 3, set = (i >> 6) % NC, step = i / (64 * NC);
            const int col = set * 4 + slot, m = col / PARTS, part = col % PARTS;
            const int k0 = (step0 + step) * 128 + c * 32 + j * 8;
            const bool live = col < VALS * PARTS && m < f.vectors && k0 < a.K;
            const T *x = (const T *)a.x + (int64_t)(f.m0 + m) * a.x_stride + k0;
            bf16x8 to;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                // codes k and k + 4 of a word share a register
                float rest = live ? (float)x[(k >> 1) + (k & 1) * 4] : 0.0f, top = rest;
                if constexpr (PARTS > 1) {
#pragma unroll
                    for (int p = 0; p < PARTS; ++p) {
                        const float cut = __uint_as_float(__float_as_uint(rest) & 0xFFFF0000u);
                        if (p == part) top = cut;
                        rest = fabsf(rest) < INFINITY ? rest - cut : 0.0f;
                    }
                }
                to[k] = (bf16_t)top;
            }
            xs[((step * 4 + j) * NC + set) * 16 + c * 4 + slot] = to;
        }
        for (int i = threadIdx.x; i < NC * 64; i += 64 * FAST_WAVES) ((u32x4 *)lds)[zero_at + i] = u32x4{0, 0, 0, 0};
        __syncthreads();
        for (int i = threadIdx.x; i < f.stretch * NC * 16; i += 64 * FAST_WAVES) {
            const int at = i & 15, set = (i >> 4) % NC, step = i / (16 * NC);
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const bf16x8 v = xs[((step * 4 + j) * NC + set) * 16 + at];
#pragma unroll
                for (int k = 0; k < 8; ++k) sum += DOWN * (float)v[k];
            }
            ((float *)sums)[(step * NC + set) * 16 + at] = sum;
        }
        __syncthreads();
    };

    // this lane's rows of a tile
    struct Rows {
        const uint8_t *codes[2];
        int64_t sc[2];
    };
    auto rows_of = [&](Rows &to, int64_t tile) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const int64_t row = min(tile * ROWS_W + t * 16 + r, a.rows - 1);
            to.codes[t] = a.codes + row * a.codes_stride;
            to.sc[t] = row * a.scale_stride;
        }
    };
    // one step of a tile's codes and scales, for this lane's rows and chunk
    struct Loaded {
        u32x4 w[2];
        SC s[2], o[2];
    };
    auto load = [&](Loaded &to, const Rows &rows, int step) {
        const int c = step * 4 + chunk;
        const int cc = c * 32 < a.K ? c : 0;   // the last step may have fewer than four chunks; x is 0 there
        const int g = f.group_inv ? (int)__umulhi((uint32_t)cc, f.group_inv) : cc;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            to.w[t] = *(const u32x4 *)(rows.codes[t] + cc * 16);
            to.s[t] = ((const SC *)a.scales)[rows.sc[t] + g];
            if (OFFSETS) to.o[t] = ((const SC *)a.offsets)[rows.sc[t] + g];
        }
    };
    // where this lane's x lies in a step: in its own chunk's slots, else among the zeros, which all steps share
    const bool mine = (r >> 2) == chunk;
    const int x_at = mine ? chunk * 4 + (r & 3) : zero_at, x_step = mine ? NC * 64 : 0;
    // in registers, so that masking and setting the exponent are one instruction
    uint32_t four_bits = 0x00780078u, sixteen = 0x3C003C00u;   // 16 DOWN, twice
    asm volatile("" : "+v"(four_bits));
    asm volatile("" : "+s"(sixteen));
    float y[2][NC * 4];
    auto multiply = [&](const Loaded &from, int at) {   // at: the step's place in LDS
        f32x4 acc[2][NC], xsum[NC];
#pragma unroll
        for (int n = 0; n < NC; ++n) {
            xsum[n] = sums[(at * NC + n) * 4 + chunk];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[t][n][i] = (OFFSETS ? -16.0f : -24.0f) * xsum[n][i];
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            bf16x8 b[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const uint32_t q = from.w[t][j];
                u32x4 e;
                e[0] = ((q << 3) & four_bits) | sixteen;
                e[1] = ((q >> 1) & four_bits) | sixteen;
                e[2] = ((q >> 5) & four_bits) | sixteen;
                e[3] = ((q >> 9) & four_bits) | sixteen;
                b[t] = __builtin_bit_cast(bf16x8, e);
            }
#pragma unroll
            for (int n = 0; n < NC; ++n) {
                const bf16x8 x = xs[x_at + at * x_step + (j * NC + n) * 16];
#pragma unroll
                for (int t = 0; t < 2; ++t)
                    acc[t][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, b[t], acc[t][n], 0, 0, 0);
            }
        }
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int n = 0; n < NC; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    y[t][n * 4 + i] = fmaf((float)from.s[t], acc[t][n][i], y[t][n * 4 + i]);
                    if (OFFSETS) y[t][n * 4 + i] = fmaf((float)from.o[t], xsum[n][i], y[t][n * 4 + i]);
                }
    };
    auto clear = [&] {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < NC * 4; ++i) y[t][i] = 0.0f;
    };
    constexpr int OUT = (VALS + 1) / 2;
    auto totals = [&](float (&out)[OUT]) {   // the parts of a value, then the chunks
        float v[2][VALS];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < VALS; ++i) {
                v[t][i] = y[t][i * PARTS];
#pragma unroll
                for (int p = 1; p < PARTS; ++p) v[t][i] += y[t][i * PARTS + p];
            }
        join_chunks<VALS>(v, out);
    };
    auto write = [&](const float (&out)[OUT], int64_t tile) {
        const int64_t row = tile * ROWS_W + (chunk >> 1) * 16 + r;
        if (row >= a.rows) return;
#pragma unroll
        for (int u = 0; u < OUT; ++u) {
            const int m = 2 * u + (chunk & 1);
            if (m < VALS && m < f.vectors) ((T *)a.y)[(int64_t)(f.m0 + m) * a.y_stride + row] = (T)(out[u] / DOWN);
        }
    };

    if (f.split_k == 1 && f.steps <= f.stretch) {
        // A wave walks through its tiles' steps as one sequence with AHEAD units
        // of loads in flight. A unit is two steps, so that the two halves of a
        // row's 128-byte lines are asked for together.
        const int64_t stride = (int64_t)gridDim.x * FAST_WAVES;
        int64_t tile = (int64_t)blockIdx.x * FAST_WAVES + wave, next = tile;
        int step = 0, next_step = 0;
        Loaded buf[AHEAD][2];
        Rows rows;
        auto fetch = [&](Loaded (&to)[2]) {
            if (next < tiles) {
                if (next_step == 0) rows_of(rows, next);
                load(to[0], rows, next_step);
                if (next_step + 1 < f.steps) load(to[1], rows, next_step + 1);
            }
            next_step += 2;
            if (next_step >= f.steps) {
                next_step = 0;
                next += stride;
            }
        };
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) fetch(buf[i]);
        fill(0);
        clear();
        while (tile < tiles) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (tile < tiles) {
                    multiply(buf[i][0], step);
                    if (step + 1 < f.steps) multiply(buf[i][1], step + 1);
                    fetch(buf[i]);
                    step += 2;
                    if (step >= f.steps) {
                        float out[OUT];
                        totals(out);
                        write(out, tile);
                        clear();
                        step = 0;
                        tile += stride;
                    }
                }
            }
        }
        return;
    }
    // Few tiles, or rows longer than LDS holds of x: the waves of a tile take
    // its steps in turn and add their sums in order.
    for (int64_t t0 = (int64_t)blockIdx.x * per_block; t0 < tiles; t0 += (int64_t)gridDim.x * per_block) {
        const int64_t tile = t0 + wave / f.split_k;
        clear();
        Rows rows;
        rows_of(rows, tile);
        for (int step0 = 0; step0 < f.steps; step0 += f.stretch) {
            const int end = min(f.steps, step0 + f.stretch);
            int step = step0 + split;
            Loaded cur;
            if (step < end) load(cur, rows, step);
            if (t0 != (int64_t)blockIdx.x * per_block || step0) __syncthreads();
            fill(step0);
            for (; step < end; step += f.split_k) {
                Loaded nxt;
                if (step + f.split_k < end) load(nxt, rows, step + f.split_k);
                multiply(cur, step - step0);
                cur = nxt;
            }
        }
        float out[OUT];
        totals(out);
        if (f.split_k > 1) {
            __syncthreads();   // x has been read
            float *red = (float *)lds;
#pragma unroll
            for (int u = 0; u < OUT; ++u) red[(wave * OUT + u) * 64 + lane] = out[u];
            __syncthreads();
            if (split == 0)
                for (int k = 1; k < f.split_k; ++k)
#pragma unroll
                    for (int u = 0; u < OUT; ++u) out[u] += red[((wave + k) * OUT + u) * 64 + lane];
        }
        if (split == 0) write(out, tile);
    }
}

template <class T, class SC, int NC>
void launch_fast(FastArgs f, hipStream_t st)
{
    const VecArgs &a = f.v;
    f.steps = (int32_t)ceil_div(a.K, 128);
    f.stretch = (int32_t)std::min<int64_t>(f.steps, (FAST_LDS - NC * 1024) / step_bytes(NC));
    // exact for the at most 2^15 chunks of a row
    const int32_t per_group = a.group / 32;
    f.group_inv = per_group == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + per_group - 1) / per_group);
    const int64_t tiles = ceil_div(a.rows, ROWS_W);
    // waves share a tile's steps while there are too few tiles to give every
    // CU two blocks of them
    f.split_k = 1;
    while (f.split_k < FAST_WAVES && f.split_k * 2 <= f.steps && tiles * f.split_k < 512 * FAST_WAVES) f.split_k *= 2;
    const int64_t blocks = std::min<int64_t>(ceil_div(tiles, FAST_WAVES / f.split_k), f.split_k > 1 ? 4096 : 512);
    size_t lds = (size_t)f.stretch * step_bytes(NC) + NC * 1024;
    if (f.split_k > 1) lds = std::max(lds, (size_t)FAST_WAVES * NC * 2 * 64 * sizeof(float));
    if (a.offsets) rows4_kernel<T, SC, NC, true><<<dim3((uint32_t)blocks), 64 * FAST_WAVES, lds, st>>>(f);
    else rows4_kernel<T, SC, NC, false><<<dim3((uint32_t)blocks), 64 * FAST_WAVES, lds, st>>>(f);
}

template <class T, class SC>
void launch_sets(const VecArgs &a, hipStream_t st)
{
    constexpr int PARTS = parts_v<T>, MOST = 16 / PARTS;
    for (int32_t m0 = 0; m0 < a.M; m0 += MOST) {
        FastArgs f{};
        f.v = a, f.m0 = m0, f.vectors = std::min(MOST, a.M - m0);
        const int cols = f.vectors * PARTS;
        if (cols <= 4) launch_fast<T, SC, 1>(f, st);
        else if (cols <= 8) launch_fast<T, SC, 2>(f, st);
        else launch_fast<T, SC, 4>(f, st);
    }
}

template <class T>
int launch_rows4(const VecArgs &a, hipStream_t st)
{
    const bool chunks = a.K % 32 == 0 && a.group % 32 == 0 && aligned(a.codes, 16) && a.codes_stride % 16 == 0;
    if (chunks) {
        if (a.scale_dtype == BOA_T_F32) launch_sets<T, float>(a, st);
        else if (a.scale_dtype == BOA_T_BF16) launch_sets<T, bf16_t>(a, st);
        else launch_sets<T, f16_t>(a, st);
        return launch_status("matvec_fourbit");
    }
    for (int64_t row = 0; row < a.rows; row += LAUNCH_ROWS) {
        VecArgs n = a;
        const int64_t scale = row * a.scale_stride * dtype_bytes(a.scale_dtype);
        n.codes += row * a.codes_stride;
        n.scales = (const uint8_t *)a.scales + scale;
        if (a.offsets) n.offsets = (const uint8_t *)a.offsets + scale;
        n.y = (T *)a.y + row;
        n.rows = std::min(LAUNCH_ROWS, a.rows - row);
        const dim3 grid((uint32_t)ceil_div(n.rows, 4));
        if (a.M == 1)
            rows4_any_kernel<T, 1><<<grid, 256, 0, st>>>(n);
        else
            rows4_any_kernel<T, 8><<<grid, 256, 0, st>>>(n);
    }
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
