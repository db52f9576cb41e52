// Softmax cross entropy of B queries over V points as classes, with its
// gradients, in pieces of the points and without keeping the logits.
//
//   l_bv = scale h_b . c_v + bias_v     lse_b = log sum_v exp l_bv
//   loss_b = lse_b - l_b,y(b)           q_bv  = g_b (exp(l_bv - lse_b) - [v = y_b])
//   dh_b = scale sum_v q_bv c_v         dc_v  = scale sum_b q_bv h_b      dbias_v = sum_b q_bv
//
// Every product runs on the bf16 matrix instructions with float32 sums, one
// tile routine for all of them (tile_product). float32 inputs are split into
// three bf16 parts whose sum is the value (8 + 8 + 8 bits), and the six
// products of parts above 2^-24 of the result are added: float32's precision
// for six bf16 products, which the matrix instructions do in two thirds of the
// time of a float32 one (large products reach 1,387 and 154 TFLOP/s).
//
// The losses take one pass over the points: a block keeps, per query, the
// running maximum and sum of exponentials of its share of the points; the
// shares are joined afterwards. The gradients take a second pass over pieces
// of the points: probabilities of a piece from the logits formed again,
// rounded to the products' type, then the two products. The label's
// own entry is left out of the rounded probabilities, and out of the sums of
// exponentials until the shares are joined: with r the others' sum and e the
// label's term, its entry is -g r / (r + e), added in float32, and the loss of a
// query whose point has most of the probability log(1 + r / e). Neither is the
// small difference of larger numbers, whatever 1 - p is.
#include <algorithm>
#include <cmath>

#include "boa_ops.h"

using namespace boa;

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) bf16x8 LdsRow;
typedef __attribute__((address_space(3))) short4v LdsFour;

__device__ inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
// running maximum of nothing: exp2(-inf - NO_MAX) is 0 and not NaN, and logits at the type's lowest value still count
constexpr float NO_MAX = -__FLT_MAX__;

// One operand of a product: bf16 rows `ld` values apart, which run along k or,
// `across`, along the operand's own dimension (a row is then one k). Rows past
// the end are read as the last one, 16-byte chunks past `cols` as the row's
// first; what they give is dropped, or meets zeros on the other side.
struct Operand {
    const bf16_t *p;
    int64_t ld;
    int32_t rows, cols;
    const float *f;   // float32 rows in place of p, split into parts on the way to LDS: `cols` values
    int32_t vec;      // and whether 16 bytes of them may be read at a time
};

// A product of K values (a multiple of 16). With parts, the operands' parts
// are part_a and part_b values apart.
struct Product {
    Operand a, b;
    int32_t K;
    int64_t part_a, part_b;
};

// A block's tile: WM x WN waves of TM x TN tiles of 32 x 32. A stage of k in
// LDS is 32 values of k, or 16 of each of three parts. Blocks of four waves or
// fewer leave room for a second one on the CU.
template <int WM_, int WN_, int TM_, int TN_, int PARTS_>
struct Shape {
    static constexpr int WM = WM_, WN = WN_, TM = TM_, TN = TN_, PARTS = PARTS_;
    static constexpr int BM = WM * TM * 32, BN = WN * TN * 32, THREADS = 64 * WM * WN;
    static constexpr int BK = PARTS == 1 ? 32 : 16;
    static constexpr int STAGE = (BM + BN) * BK * PARTS;   // bf16 values
    static constexpr int ROOM = (THREADS == 512 ? 150 : 75) * 1024 / (STAGE * 2);
    static constexpr bool EVEN = BM * (BK / 8) % THREADS == 0 && BN * (BK / 8) % THREADS == 0;   // every wave loads the same
    static constexpr int STAGES = !EVEN ? 2 : ROOM > 4 ? 4 : ROOM;
    static_assert(ROOM >= 2, "two stages at least");
    // Up to 32 queries, float32 points are split into parts on the way to LDS:
    // reading them is the work. With more, the splitting would be done over for
    // every tile of queries, and a copy in parts serves them all (777 queries,
    // 100,003 x 768: 4.00 ms in place of 3.55).
    static constexpr bool SPLIT = PARTS == 3 && (BM == 32 || BN == 32);
};

// Waits until at most `left` of this wave's loads are on their way and its LDS
// reads are done, then for the other waves.
template <int LEFT>
__device__ inline void wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// One operand's side of tile_product: where this thread's loads come from and
// where its fragments lie. ROWS of the operand's own dimension.
//
// Along k, a stage holds ROWS rows of BK values whose 16-byte chunks are
// stored in the order chunk ^ (row / 4 & 3), or of two chunks chunk ^ (row / 8
// & 1); across, BK rows of ROWS values in the order chunk ^ (row & 3) * 4, and
// fragments are read transposed, 64 bytes of four rows by half a wave. Either
// way what lanes read together spreads over the banks. The permutation is
// applied to the addresses loaded from, since a load to LDS writes its lanes
// in order.
template <class S, int ROWS, bool ACROSS, bool F32>
struct Side {
    static constexpr int CHUNKS = ACROSS ? ROWS / 8 : S::BK / 8;      // of an LDS row
    static constexpr int N = (ROWS * (S::BK / 8) + S::THREADS - 1) / S::THREADS;   // loads of a part
    static constexpr int PER = S::THREADS / CHUNKS;                   // LDS rows of one load of all threads
    static constexpr int PART = ROWS * S::BK;                         // values of a part's stage
    // float32: four values a load
    static constexpr int QUADS = (ACROSS ? ROWS : S::BK) / 4, NF = ROWS * S::BK / 4 / S::THREADS, PERF = S::THREADS / QUADS;
    static_assert(!F32 || (S::PARTS == 3 && NF * S::THREADS * 4 == ROWS * S::BK), "float32 has parts");
    float held[F32 ? NF : 1][4];
    const float *f;
    int32_t vec, k_from;
    const bf16_t *p;
    int64_t ld, part;
    int32_t row, last, at;   // this thread's first row, the last there is, value within a row (across: of the tile's first)
    int32_t cols;
    static_assert(!ACROSS || ROWS >= 128, "the permutation takes 16 chunks");

    __device__ static int swap(int row) { return ACROSS ? (row & 3) * 4 : CHUNKS == 4 ? (row >> 2) & 3 : (row >> 3) & 1; }

    __device__ Side(const Operand &o, int64_t part_, int32_t row0, int32_t from_k)
    {
        const int t = threadIdx.x;
        ld = o.ld, part = part_, last = o.rows - 1, cols = o.cols;
        f = o.f, vec = o.vec, k_from = from_k;
        if constexpr (F32) {
            row = row0;
            at = 0;
            p = nullptr;
        } else if constexpr (ACROSS) {
            row = from_k + t / CHUNKS;
            at = row0;
            p = o.p;
        } else {
            static_assert(PER % 16 == 0 || N == 1, "one permutation for all of a thread's loads");
            row = row0 + t / CHUNKS;
            at = (t % CHUNKS ^ swap(t / CHUNKS)) * 8;
            p = o.p + from_k;
        }
    }
    // loads k [k0, k0 + BK); K: end of k
    __device__ void load(bf16_t *to, int32_t k0, int32_t K) const
    {
        const int t = threadIdx.x, wave = t >> 6;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (!S::EVEN && i * S::THREADS + wave * 64 >= ROWS * (S::BK / 8)) continue;
            const bf16_t *from;
            if constexpr (ACROSS) {
                const int c = at + (t % CHUNKS ^ swap(t / CHUNKS + i * PER)) * 8;
                from = p + (int64_t)min(row + k0 + i * PER, last) * ld + (c < cols ? c : 0);
            } else {
                from = p + (int64_t)min(row + i * PER, last) * ld + (k0 + at < K ? k0 + at : 0);
            }
#pragma unroll
            for (int q = 0; q < S::PARTS; ++q)
                __builtin_amdgcn_global_load_lds(
                    (const __attribute__((address_space(1))) void *)(from + q * part),
                    (__attribute__((address_space(3))) void *)(to + q * PART + (i * S::THREADS + wave * 64) * 8), 16, 0, 0);
        }
    }
    // float32: k [k0, k0 + BK) into registers, and from there as parts to LDS
    __device__ void fetch(int32_t k0)
    {
        const int t = threadIdx.x;
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            const int r = t / QUADS + i * PERF, q = t % QUADS * 4;
            const int32_t c = ACROSS ? row + q : k_from + k0 + q;   // value within a row
            const float *from = f + (int64_t)min((ACROSS ? k_from + k0 : row) + r, last) * ld + c;
            if (vec && c < cols) {
                load_f32<4, float>(held[i], from);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) held[i][e] = c + e < cols ? from[e] : 0.0f;
            }
        }
    }
    __device__ void put(bf16_t *to)
    {
        const int t = threadIdx.x;
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            const int r = t / QUADS + i * PERF, q = t % QUADS;
            bf16_t *at_row = to + r * CHUNKS * 8 + ((q >> 1) ^ swap(r)) * 8 + (q & 1) * 4;
#pragma unroll
            for (int part_i = 0; part_i < S::PARTS; ++part_i) {
                bf16x4 four;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float top = __uint_as_float(__float_as_uint(held[i][e]) & 0xFFFF0000u);
                    four[e] = (bf16_t)top;
                    held[i][e] = fabsf(top) < INFINITY ? held[i][e] - top : 0.0f;
                }
                *(bf16x4 *)(at_row + part_i * PART) = four;
            }
        }
    }
    // where this lane's fragments begin in a stage, in bytes; row0: the wave's first row of the tile
    __device__ static uint32_t lane_at(int row0)
    {
        const int lane = threadIdx.x & 63, half = lane >> 5, r = lane & 31;
        if constexpr (ACROSS) {
            const int row = 8 * half + ((lane & 15) >> 2), chunk = row0 / 8 + ((lane >> 4) & 1) * 2 + ((lane >> 1) & 1);
            return row * ROWS * 2 + (chunk ^ swap(row)) * 16 + (lane & 1) * 8;
        } else {
            return (row0 + r) * S::BK * 2 + (half ^ swap(r)) * 16;
        }
    }
    // The fragment of the wave's tile i, k step s and part q. `at`: lane_at plus
    // the stage; tiles and steps are exclusive ors on bits that nothing carries
    // into, so one address serves them all.
    __device__ static bf16x8 fragment(uint32_t at, int i, int s, int q)
    {
        if constexpr (ACROSS) {
            bf16x8 f;
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
                const uint32_t a = (at ^ (i * 64)) + q * PART * 2 + (16 * s + 4 * jj) * ROWS * 2;
                const bf16x4 v = __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsFour *)(uintptr_t)a));
#pragma unroll
                for (int e = 0; e < 4; ++e) f[4 * jj + e] = v[e];
            }
            return f;
        } else {
            return *(const LdsRow *)(uintptr_t)((at ^ (s * 32)) + q * PART * 2 + i * 32 * S::BK * 2);
        }
    }
};

// acc += A[row0a ..][k] * B[row0b ..][k], k in [from_k, from_k + K). Loads run
// STAGES - 1 stages ahead of the matrix instructions (a stage of 256 x 256 is
// 1000 cycles of them, 3000 with parts), which bound it: the losses of 777
// queries x 100,003 points x 768 float32 values take 0.80 ms, 1,030 TFLOP/s for
// the 896 rows that are multiplied (890 for the 777), the gradients' products,
// whose tiles are shorter, 0.90 to 0.95 ms each, 870 to 920 (755 to 800). Of
// parts, the six products above 2^-24 of the result are added, smallest first.
// ACROSS_A, ACROSS_B: the operand's rows are k; F32_A, F32_B: it is float32 in memory.
template <class S, bool ACROSS_A, bool ACROSS_B, bool F32_A = false, bool F32_B = false>
__device__ inline void tile_product(const Product &pr, int32_t row0a, int32_t row0b, bf16_t *lds,
                                    f32x16 (&acc)[S::TM][S::TN], int32_t from_k, int32_t K)
{
    constexpr int STAGES = S::STAGES, BK = S::BK;
    const int wave = threadIdx.x >> 6, wm = wave % S::WM, wn = wave / S::WM;
    using A = Side<S, S::BM, ACROSS_A, F32_A>;
    using B = Side<S, S::BN, ACROSS_B, F32_B>;
    A a(pr.a, pr.part_a, row0a, from_k);
    B b(pr.b, pr.part_b, row0b, from_k);
    // loads to LDS that may be on their way when a stage is waited for
    constexpr int COUNTED = (STAGES - 2) * S::PARTS * ((F32_A ? 0 : A::N) + (F32_B ? 0 : B::N));
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) bf16_t *)lds;
    const uint32_t lane_a = A::lane_at(wm * S::TM * 32), lane_b = B::lane_at(wn * S::TN * 32);
    const int total = (K + BK - 1) / BK;
    auto load = [&](int it) {   // past the end, the last stage again: it is not used
        bf16_t *to = lds + it % STAGES * S::STAGE;
        const int k0 = min(it, total - 1) * BK;
        if constexpr (F32_A) a.fetch(k0);
        if constexpr (F32_B) b.fetch(k0);
        if constexpr (!F32_A) a.load(to, k0, K);
        if constexpr (!F32_B) b.load(to + S::BM * BK * S::PARTS, k0, K);
    };
    auto put = [&](int it) {
        bf16_t *to = lds + it % STAGES * S::STAGE;
        if constexpr (F32_A) a.put(to);
        if constexpr (F32_B) b.put(to + S::BM * BK * S::PARTS);
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) {
        load(i);
        put(i);
    }
    auto step = [&](int it, auto steps) {
        wait_and_meet<COUNTED>();
        load(it + STAGES - 1);
        const uint32_t stage = base + it % STAGES * S::STAGE * 2;
        const uint32_t at_a = stage + lane_a, at_b = stage + S::BM * BK * S::PARTS * 2 + lane_b;
#pragma unroll
        for (int s = 0; s < decltype(steps)::value; ++s) {
            constexpr int PAIRS = S::PARTS == 1 ? 1 : 6, QA = S::PARTS - 1;
            constexpr int qa[6] = {QA, QA / 2, 0, QA / 2, 0, 0}, qb[6] = {0, 1, 2, 0, 1, 0};
            // with parts, a row of tiles at a time: all fragments at once do not fit the registers
            constexpr int ROW = S::PARTS == 1 ? S::TM : S::TM > 2 ? 2 : 1;
            bf16x8 fb[S::PARTS][S::TN];
#pragma unroll
            for (int q = 0; q < S::PARTS; ++q)
#pragma unroll
                for (int j = 0; j < S::TN; ++j) fb[q][j] = B::fragment(at_b, j, s, q);
#pragma unroll
            for (int i0 = 0; i0 < S::TM; i0 += ROW) {
                bf16x8 fa[S::PARTS][ROW];
#pragma unroll
                for (int q = 0; q < S::PARTS; ++q)
#pragma unroll
                    for (int i = 0; i < ROW; ++i)
                        fa[q][i] = A::fragment(at_a, i0 + i, s, q);
#pragma unroll
                for (int q = 0; q < PAIRS; ++q)
#pragma unroll
                    for (int i = 0; i < ROW; ++i)
#pragma unroll
                        for (int j = 0; j < S::TN; ++j)
                            acc[i0 + i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fa[qa[q]][i], fb[qb[q]][j],
                                                                                     acc[i0 + i][j], 0, 0, 0);
                if (S::PARTS > 1) __builtin_amdgcn_sched_barrier(0);
            }
        }
        put(it + STAGES - 1);
    };
    for (int it = 0; it < K / BK; ++it) step(it, std::integral_constant<int, BK / 16>{});
    if (K % BK) step(total - 1, std::integral_constant<int, 1>{});
    wait_and_meet<0>();
}

// Row of a 32 x 32 tile that a lane's value i stands for (the column is lane & 31).
__device__ inline int tile_row(int i, int half) { return (i >> 2) * 8 + half * 4 + (i & 3); }

// Work item of a block: `minor` blocks that share operand rows run on one XCD
// (blocks go to the 8 XCDs in turn). False: nothing to do.
__device__ inline bool split_block(int32_t majors, int32_t minors, int32_t *major, int32_t *minor)
{
    const int32_t id = (int32_t)blockIdx.x, local = id >> 3;
    *major = (id & 7) + 8 * (local / minors);
    *minor = local % minors;
    return *major < majors;
}
inline uint32_t split_grid(int64_t majors, int64_t minors) { return (uint32_t)(ceil_div(majors, 8) * 8 * minors); }

template <class S>
__device__ inline void clear(f32x16 (&acc)[S::TM][S::TN])
{
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
}

// ---------------------------------------------------------------------------
// operands

// Copies rows (R x C) as bf16 parts, zeros past the end: `plain`
// [part][rows_pad][plain_ld], and `kept` the same without the rows that are left
// out (whatever they hold, zeros take their place). Either may be null. Of
// queries it also gives the labels: -1 where a query has none, past the last
// one too.
struct PartsArgs {
    const void *src;
    int64_t stride, plain_ld, plain_part;
    int32_t R, C, rows_pad;
    bf16_t *plain, *kept;
    const int64_t *labels;   // of queries, or null
    int32_t V;
    int32_t *label;          // rows_pad
};

// A thread makes 8 values of a row (plain_ld is a multiple of 16).
template <class T>
__device__ inline void make_parts(const PartsArgs &a, int64_t i)
{
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    const int64_t chunks = a.plain_ld / 8;
    const int64_t r = i / chunks;
    const int32_t c = (int32_t)(i % chunks) * 8;
    if (r >= a.rows_pad) return;
    bool live = true;
    if (a.labels) {
        const int64_t y = r < a.R ? a.labels[r] : -1;
        live = y >= 0 && y < a.V;
        if (c == 0) a.label[r] = live ? (int32_t)y : -1;
    }
    float v[8];
    const T *from = (const T *)a.src + r * a.stride + c;
    if (r < a.R && c + 8 <= a.C && aligned16(from)) {
        constexpr int N = 16 / sizeof(T);
#pragma unroll
        for (int e = 0; e < 8; e += N) load_f32<N, T>(*(float(*)[N])(v + e), from + e);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = r < a.R && c + e < a.C ? (float)from[e] : 0.0f;
    }
    float first[8] = {};
#pragma unroll
    for (int p = 0; p < PARTS; ++p) {
        bf16x8 part, nil;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            nil[e] = (bf16_t)0.0f;
            if constexpr (PARTS == 1) {
                part[e] = (bf16_t)v[e];
            } else {
                const float top = __uint_as_float(__float_as_uint(v[e]) & 0xFFFF0000u);
                // A point's infinity times a query's part of 0 would be NaN: the part is the smallest normal number,
                // which alters no sum of products that is not itself next to that.
                part[e] = (bf16_t)(p && a.labels && top == 0.0f && fabsf(first[e]) >= 0x1p-100f
                                       ? copysignf(0x1p-126f, first[e]) : top);
                if (p == 0) first[e] = top;
                v[e] = fabsf(top) < INFINITY ? v[e] - top : 0.0f;   // an infinity or NaN is its first part alone
            }
        }
        const int64_t at = p * a.plain_part + r * a.plain_ld + c;
        if (a.plain) *(bf16x8 *)(a.plain + at) = part;
        if (a.kept) *(bf16x8 *)(a.kept + at) = live ? part : nil;
    }
}

template <class T>
__global__ __launch_bounds__(256) void parts_kernel(PartsArgs a)
{
    make_parts<T>(a, (int64_t)blockIdx.x * 256 + threadIdx.x);
}

inline int64_t parts_blocks(const PartsArgs &a) { return ceil_div((int64_t)a.rows_pad * (a.plain_ld / 8), 256); }

// A point's bias in base 2. Finite ones stay finite, masks of the type's lowest
// value among them.
__device__ inline float base2(float bias)
{
    return fabsf(bias) < INFINITY ? fmaxf(-__FLT_MAX__, fminf(__FLT_MAX__, bias * LOG2E)) : bias;
}

// What a call begins with, in one launch: the queries as parts; the points'
// biases in base 2, -inf past the last point (`to`, or null); the points' first
// queries (or null) and the blocks that are done cleared.
struct PrepArgs {
    PartsArgs queries;
    int32_t query_blocks, point_blocks;
    const float *bias;
    float *to;
    int32_t V, padded;
    int32_t *first;
    uint32_t *done;
};

template <class T>
__global__ __launch_bounds__(256) void prep_kernel(PrepArgs a)
{
    if (blockIdx.x < (uint32_t)a.query_blocks) {
        if (blockIdx.x == 0 && threadIdx.x == 0) *a.done = 0;
        make_parts<T>(a.queries, (int64_t)blockIdx.x * 256 + threadIdx.x);
        return;
    }
    const int64_t step = (int64_t)a.point_blocks * 256;
    for (int64_t i = (int64_t)(blockIdx.x - a.query_blocks) * 256 + threadIdx.x; i < a.padded; i += step) {
        if (a.to) a.to[i] = i >= a.V ? -INFINITY : a.bias ? base2(a.bias[i]) : 0.0f;
        if (a.first && i < a.V) a.first[i] = -1;
    }
}

// ---------------------------------------------------------------------------
// losses

struct RowState {
    float m, s;   // running maximum (base 2) and sum of exponentials, the label's own left out
};

// sum += x with what rounding loses kept in `lost` and brought in by the next
// addition: thousands of small exponentials would vanish one by one beside a
// large sum.
__device__ inline void add_kept(float &sum, float &lost, float x)
{
    const float y = x - lost, t = sum + y;
    lost = (t - sum) - y;
    sum = t;
}

struct StatsArgs {
    Product pr;              // a: points, b: queries
    const float *bias;
    RowState *part;          // splits x B
    const int32_t *label;    // of the queries, padded
    float *pick;             // B: the label's logit, base 2
    float scale2;            // scale * log2(e)
    int32_t B, V, v0, tiles_v, tiles_b, splits;   // v0: the first point among all
};

__device__ inline void join(RowState &a, float m, float s)
{
    const float top = fmaxf(a.m, m);
    a.s = a.s * __builtin_amdgcn_exp2f(a.m - top) + s * __builtin_amdgcn_exp2f(m - top);
    a.m = top;
}

// A block takes every splits-th tile of points for one tile of queries. A
// lane's values belong to TN queries (the columns of its tiles), so the
// running states stay in its registers until the end.
template <class S>
__global__ __launch_bounds__(S::THREADS, 2) void stats_kernel(StatsArgs a)
{
    extern __shared__ __attribute__((aligned(256))) bf16_t lds[];
    int32_t split, tb;
    if (!split_block(a.splits, a.tiles_b, &split, &tb)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5;
    const int wm = wave % S::WM, wn = wave / S::WM;
    RowState st[S::TN];
    float lost[S::TN];
    int32_t lab[S::TN];
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
        st[j] = RowState{NO_MAX, 0.0f};
        lost[j] = 0.0f;
        lab[j] = a.label[tb * S::BN + (wn * S::TN + j) * 32 + (lane & 31)] - a.v0;
    }
    for (int32_t tv = split; tv < a.tiles_v; tv += a.splits) {
        f32x16 acc[S::TM][S::TN];
        clear<S>(acc);
        tile_product<S, false, false, S::SPLIT, false>(a.pr, tv * S::BM, tb * S::BN, lds, acc, 0, a.pr.K);
#pragma unroll
        for (int i = 0; i < S::TM; ++i) {
            const int32_t v0 = tv * S::BM + (wm * S::TM + i) * 32;
            float off[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int32_t v = v0 + tile_row(e, half);
                off[e] = v >= a.V ? -INFINITY : a.bias ? base2(a.bias[v]) : 0.0f;
            }
#pragma unroll
            for (int j = 0; j < S::TN; ++j) {
                float top = st[j].m;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    acc[i][j][e] = fmaf(acc[i][j][e], a.scale2, off[e]);
                    top = fmaxf(top, acc[i][j][e]);
                }
                const int32_t rel = lab[j] - v0;
                const float by = __builtin_amdgcn_exp2f(st[j].m - top);
                float s = 0.0f;
                if (__any((uint32_t)rel < 32u)) {   // a query's own point is among these: it is joined later
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const bool here = rel == tile_row(e, half);
                        if (here) a.pick[tb * S::BN + (wn * S::TN + j) * 32 + (lane & 31)] = acc[i][j][e];
                        s += here ? 0.0f : __builtin_amdgcn_exp2f(acc[i][j][e] - top);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) s += __builtin_amdgcn_exp2f(acc[i][j][e] - top);
                }
                st[j].m = top;
                st[j].s *= by;
                lost[j] *= by;
                add_kept(st[j].s, lost[j], s);
            }
        }
    }
    RowState *red = (RowState *)lds;   // WM x BN; the product has passed its last barrier
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
        const float m = __shfl_xor(st[j].m, 32), s = __shfl_xor(st[j].s, 32);
        join(st[j], m, s);
        if (half == 0) red[wm * S::BN + (wn * S::TN + j) * 32 + lane] = st[j];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < S::BN; c += S::THREADS) {
        const int32_t b = tb * S::BN + c;
        if (b >= a.B) continue;
        RowState one = red[c];
        for (int w = 1; w < S::WM; ++w) join(one, red[w * S::BN + c].m, red[w * S::BN + c].s);
        a.part[(int64_t)split * a.B + b] = one;
    }
}

struct RowArgs {
    const int64_t *labels;
    const float *dloss, *pick;
    const RowState *part;
    float *loss;             // per query (the caller's, or scratch where the loss is reduced)
    float *lse;              // the caller's, or null
    float *top;              // rows_pad: what the sum is relative to, base 2
    float *rowf;             // rows_pad: g / sum of 2^(l - top) over all points, 0 for a query without gradient
    float *coef;             // B: g * (p_label - 1), by way of the others' sum
    int32_t *label;          // rows_pad: the label, or -1 where it has no entry
    int32_t B, V, shares, reduction, rows_pad;
    uint32_t *done;          // blocks that are done, 0 at the start
    float *total, *factor;   // the reduced loss and the factor every gradient gets, or null
};

// A wave per query: joins the shares of its statistics. The last block to end
// adds the losses, in order whichever it is.
__global__ __launch_bounds__(256) void row_kernel(RowArgs a)
{
    const int lane = threadIdx.x & 63;
    const int32_t b = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (b >= a.B) {
        if (lane == 0 && b < a.rows_pad) {
            a.top[b] = INFINITY;   // probabilities of 0 whatever the bias
            a.rowf[b] = 0.0f;
        }
    } else {
        RowState st{NO_MAX, 0.0f};
        for (int i = lane; i < a.shares; i += 64) {
            const RowState o = a.part[(int64_t)i * a.B + b];
            join(st, o.m, o.s);
        }
#pragma unroll
        for (int o = 32; o; o >>= 1) {
            const float m = __shfl_xor(st.m, o), s = __shfl_xor(st.s, o);
            join(st, m, s);
        }
        if (lane == 0) {
            const int64_t y = a.labels[b];
            const bool in = y >= 0 && y < a.V;
            const float l2 = in ? a.pick[b] : 0.0f;
            const float mine = in ? __builtin_amdgcn_exp2f(l2 - st.m) : 0.0f, all = st.s + mine;
            const bool none = all == 0.0f;   // every point left out
            const float log_s = __builtin_amdgcn_logf(all);
            float loss = 0.0f;
            if (y >= a.V) loss = NAN;
            else if (in) loss = none ? INFINITY : mine > st.s ? log1pf(st.s / mine) : ((st.m - l2) + log_s) * LN2;
            a.loss[b] = loss;
            if (a.lse) a.lse[b] = none ? -INFINITY : (st.m + log_s) * LN2;
            const float g = !in || none ? 0.0f : a.reduction == BOA_REDUCE_NONE && a.dloss ? a.dloss[b] : 1.0f;
            a.top[b] = none || !in ? INFINITY : st.m;
            a.rowf[b] = g == 0.0f ? 0.0f : g / all;
            if (none || !in) a.label[b] = -1;
            if (a.coef) a.coef[b] = in && !none ? -g * (st.s / all) : 0.0f;
        }
    }
    if (!a.total && !a.factor) return;
    __shared__ bool last;
    __shared__ float ls[4], ns[4];
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        last = atomicAdd(a.done, 1u) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    float s = 0.0f, n = 0.0f;
    for (int32_t i = threadIdx.x; i < a.B; i += 256) {
        s += __builtin_nontemporal_load(a.loss + i);
        n += a.labels[i] >= 0 ? 1.0f : 0.0f;
    }
    s = wave_sum(s);
    n = wave_sum(n);
    if (lane == 0) {
        ls[threadIdx.x >> 6] = s;
        ns[threadIdx.x >> 6] = n;
    }
    __syncthreads();
    if (threadIdx.x) return;
    s = ls[0] + ls[1] + ls[2] + ls[3];
    n = ns[0] + ns[1] + ns[2] + ns[3];
    const float by = a.reduction == BOA_REDUCE_MEAN ? fmaxf(n, 1.0f) : 1.0f;
    if (a.total) *a.total = s / by;
    if (a.factor) *a.factor = (a.dloss && a.reduction != BOA_REDUCE_NONE ? *a.dloss : 1.0f) / by;
}

// ---------------------------------------------------------------------------
// gradients

struct ProbArgs {
    Product pr;              // a: queries, b: points of the piece
    const float *bias;       // of the piece
    const float *top, *rowf;
    const int32_t *label;
    bf16_t *p;               // [part][rows_pad][cols_pad], or null
    float *col;              // tiles_b x cols_pad: sums over the tile's queries, or null
    float scale2;
    int32_t B, V, v0;        // v0: the piece's first point
    int32_t n, cols_pad, rows_pad, tiles_b, tiles_v;
};

// bf16 part `part` of PARTS of a value (see parts_kernel); one part rounds.
template <int PARTS>
__device__ inline bf16_t part_of(float v, int part)
{
    if constexpr (PARTS == 1) return (bf16_t)v;
    float top = __uint_as_float(__float_as_uint(v) & 0xFFFF0000u);
#pragma unroll
    for (int i = 0; i < PARTS - 1; ++i)
        if (i < part) {
            v -= top;
            top = __uint_as_float(__float_as_uint(v) & 0xFFFF0000u);
        }
    return (bf16_t)top;
}

// Probabilities of a tile of queries and points of the piece, without the
// labels' own entries, written through LDS as rows of queries.
template <class S>
__global__ __launch_bounds__(S::THREADS, 2) void prob_kernel(ProbArgs a)
{
    constexpr int PARTS = S::PARTS;
    extern __shared__ __attribute__((aligned(256))) bf16_t lds[];
    int32_t tv, tb;
    if (!split_block(a.tiles_v, a.tiles_b, &tv, &tb)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, r = lane & 31;
    const int wm = wave % S::WM, wn = wave / S::WM;
    f32x16 acc[S::TM][S::TN];
    clear<S>(acc);
    tile_product<S, false, false, false, S::SPLIT>(a.pr, tb * S::BM, tv * S::BN, lds, acc, 0, a.pr.K);
    float off[S::TN];
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
        const int32_t v = tv * S::BN + (wn * S::TN + j) * 32 + r;
        off[j] = v >= a.n ? -INFINITY : a.bias ? base2(a.bias[v]) : 0.0f;
    }
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
        const int32_t b0 = tb * S::BM + (wm * S::TM + i) * 32;
        const int32_t mine = a.label[b0 + r] - a.v0;
#pragma unroll
        for (int e = 0; e < 16; ++e) {
            const int32_t b = b0 + tile_row(e, half);
            const float top = a.top[b], f = a.rowf[b];
#pragma unroll
            for (int j = 0; j < S::TN; ++j) {
                const float l = fmaf(acc[i][j][e], a.scale2, off[j]);
                acc[i][j][e] = f == 0.0f ? 0.0f : f * __builtin_amdgcn_exp2f(l - top);
            }
        }
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
            const int32_t c0 = tv * S::BN + (wn * S::TN + j) * 32;
            if (__any(mine >= c0 && mine < c0 + 32)) {
#pragma unroll
                for (int e = 0; e < 16; ++e)
                    if (__shfl(mine, tile_row(e, half)) == c0 + r) acc[i][j][e] = 0.0f;
            }
        }
    }
    if (a.col) {
        float *red = (float *)lds;   // WM x BN
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
            float s = 0.0f;
#pragma unroll
            for (int i = 0; i < S::TM; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) s += acc[i][j][e];
            s += __shfl_xor(s, 32);
            if (half == 0) red[wm * S::BN + (wn * S::TN + j) * 32 + r] = s;
        }
        __syncthreads();
        for (int c = threadIdx.x; c < S::BN; c += S::THREADS) {
            float s = 0.0f;
            for (int w = 0; w < S::WM; ++w) s += red[w * S::BN + c];
            a.col[(int64_t)tb * a.cols_pad + tv * S::BN + c] = s;
        }
        __syncthreads();
    }
    if (!a.p) return;
    constexpr int LD = S::BN + 8;
#pragma unroll 1
    for (int part = 0; part < PARTS; ++part) {
#pragma unroll
        for (int i = 0; i < S::TM; ++i)
#pragma unroll
            for (int j = 0; j < S::TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    bf16_t one;
                    if constexpr (PARTS == 1) {
                        one = (bf16_t)acc[i][j][e];
                    } else {   // the parts one after the other: what is left stays in acc
                        const float top = __uint_as_float(__float_as_uint(acc[i][j][e]) & 0xFFFF0000u);
                        one = (bf16_t)top;
                        acc[i][j][e] -= top;
                    }
                    lds[((wm * S::TM + i) * 32 + tile_row(e, half)) * LD + (wn * S::TN + j) * 32 + r] = one;
                }
        __syncthreads();
        bf16_t *to = a.p + ((int64_t)part * a.rows_pad + tb * S::BM) * a.cols_pad + tv * S::BN;
        for (int c = threadIdx.x; c < S::BM * (S::BN / 8); c += S::THREADS) {
            const int row = c / (S::BN / 8), col = c % (S::BN / 8) * 8;
            *(bf16x8 *)(to + (int64_t)row * a.cols_pad + col) = *(const bf16x8 *)(lds + row * LD + col);
        }
        __syncthreads();
    }
}

struct DhArgs {
    Product pr;              // a: probabilities, b: the piece's points, across
    float *part;             // splits x rows_pad x ld
    int32_t d, ld, rows_pad, tiles_b, tiles_d, splits, k_split, first;
};

// A split's share of sum_v p_bv c_v over the piece, added to what earlier
// pieces left.
template <class S>
__global__ __launch_bounds__(S::THREADS, 2) void dh_kernel(DhArgs a)
{
    extern __shared__ __attribute__((aligned(256))) bf16_t lds[];
    int32_t split, tile;
    if (!split_block(a.splits, a.tiles_b * a.tiles_d, &split, &tile)) return;
    const int32_t tb = tile / a.tiles_d, td = tile % a.tiles_d;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, r = lane & 31;
    const int wm = wave % S::WM, wn = wave / S::WM;
    const int32_t k0 = split * a.k_split, K = min(a.k_split, a.pr.K - k0);
    f32x16 acc[S::TM][S::TN];
    clear<S>(acc);
    if (K > 0) tile_product<S, false, true, false, S::SPLIT>(a.pr, tb * S::BM, td * S::BN, lds, acc, k0, K);
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
        for (int j = 0; j < S::TN; ++j) {
            const int32_t c = td * S::BN + (wn * S::TN + j) * 32 + r;
            if (c >= a.d) continue;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const int32_t b = tb * S::BM + (wm * S::TM + i) * 32 + tile_row(e, half);
                float *to = a.part + ((int64_t)split * a.rows_pad + b) * a.ld + c;
                *to = a.first ? acc[i][j][e] : *to + acc[i][j][e];
            }
        }
}

struct DcArgs {
    Product pr;              // a: probabilities, b: the queries, both across
    void *out;               // of the piece
    const int32_t *first;    // V: the first query of a point, or -1
    const float *own;        // B x d: the labels' own terms, by first query
    const float *factor;
    float scale;
    int32_t n, d, v0, tiles_v, tiles_d;
};

template <class S, class T>
__global__ __launch_bounds__(S::THREADS, 2) void dc_kernel(DcArgs a)
{
    extern __shared__ __attribute__((aligned(256))) bf16_t lds[];
    int32_t tv, td;
    if (!split_block(a.tiles_v, a.tiles_d, &tv, &td)) return;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, half = lane >> 5, r = lane & 31;
    const int wm = wave % S::WM, wn = wave / S::WM;
    f32x16 acc[S::TM][S::TN];
    clear<S>(acc);
    tile_product<S, true, true>(a.pr, tv * S::BM, td * S::BN, lds, acc, 0, a.pr.K);
    // out by way of LDS, a row of the waves' tiles at a time, so that rows are
    // written 16 bytes a lane (with single values the launch took twice as long
    // at 384 queries)
    const float by = a.scale * *a.factor;
    constexpr int LD = S::BN + 4, ROWS = S::WM * 32, V = 16 / sizeof(T);
    float *rows = (float *)lds;   // ROWS x LD
    const bool whole = a.d % V == 0 && aligned16(a.out);
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
        if (i) __syncthreads();
#pragma unroll
        for (int j = 0; j < S::TN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) rows[(wm * 32 + tile_row(e, half)) * LD + (wn * S::TN + j) * 32 + r] = acc[i][j][e];
        __syncthreads();
        for (int at = threadIdx.x; at < ROWS * (S::BN / V); at += S::THREADS) {
            const int row = at / (S::BN / V), col = at % (S::BN / V) * V;
            const int32_t v = tv * S::BM + (row / 32 * S::TM + i) * 32 + row % 32, c = td * S::BN + col;
            if (v >= a.n || c >= a.d) continue;
            float x[V];
#pragma unroll
            for (int k = 0; k < V; k += 4) load_f32<4, float>(*(float(*)[4])(x + k), rows + row * LD + col + k);
            const int32_t first = a.first[a.v0 + v];
#pragma unroll
            for (int k = 0; k < V; ++k) {
                if (first >= 0 && c + k < a.d) x[k] += a.own[(int64_t)first * a.d + c + k];
                x[k] *= by;
            }
            T *to = (T *)a.out + (int64_t)v * a.d + c;
            if (whole) {
                store_f32<V, T>(to, x);
            } else {
#pragma unroll
                for (int k = 0; k < V; ++k)
                    if (c + k < a.d) to[k] = (T)x[k];
            }
        }
    }
}

constexpr int OWN_AHEAD = 8;   // rows of queries on their way at a time

struct OwnArgs {
    const void *h;
    int64_t h_stride;
    int32_t B, d;
    const int32_t *label;
    const float *coef;
    int32_t *first;
    float *own, *own_bias;   // own may be null
};

// The labels' own terms, sum of coef_b h_b over the queries of one point, kept
// by the first of them. A block per query, which leaves unless its query is the
// first: every block reads all labels, so this is for few queries (up to
// SORT_FROM), where it shares a launch with other work; more are sorted. Of the
// columns a block takes TH from c0.
template <class T, int TH>
__device__ inline void own_terms(const OwnArgs &a, int32_t b, int32_t c0)
{
    const T *h = (const T *)a.h;
    const int64_t h_stride = a.h_stride;
    const int32_t B = a.B, d = a.d, *label = a.label;
    const float *coef = a.coef;
    int32_t *first = a.first;
    float *own = a.own, *own_bias = a.own_bias;
    __shared__ int earlier;
    __shared__ int32_t list[TH];
    __shared__ float by[TH];
    __shared__ int count;
    const int32_t y = label[b];
    if (y < 0) return;
    if (threadIdx.x == 0) earlier = 0;
    __syncthreads();
    for (int32_t i = threadIdx.x; i < b; i += TH)
        if (label[i] == y) earlier = 1;
    __syncthreads();
    if (earlier) return;
    const int32_t c = c0 + (int32_t)threadIdx.x;
    float sb = 0.0f, acc = 0.0f;
    for (int32_t i0 = b; i0 < B; i0 += TH) {
        // the queries of this stretch that share the label, in order
        __syncthreads();
        if (threadIdx.x == 0) count = 0;
        __syncthreads();
        const int32_t i = i0 + threadIdx.x;
        const bool hit = i < B && label[i] == y;
        const uint64_t in_wave = __ballot(hit);
        for (int w = 0; w < TH / 64; ++w) {
            if ((threadIdx.x >> 6) == w && in_wave) {
                const int at = count + __popcll(in_wave & ((1ull << (threadIdx.x & 63)) - 1));
                if (hit) {
                    list[at] = i;
                    by[at] = coef[i];
                }
                __builtin_amdgcn_wave_barrier();
                if ((threadIdx.x & 63) == 0) count += __popcll(in_wave);
            }
            __syncthreads();
        }
        for (int j = 0; j < count; ++j) sb += by[j];
        if (!own || c >= d) continue;
        for (int j0 = 0; j0 < count; j0 += OWN_AHEAD) {
            float v[OWN_AHEAD];
#pragma unroll
            for (int u = 0; u < OWN_AHEAD; ++u) v[u] = (float)h[(int64_t)list[min(j0 + u, count - 1)] * h_stride + c];
#pragma unroll
            for (int u = 0; u < OWN_AHEAD; ++u)
                if (j0 + u < count) acc = fmaf(by[j0 + u], v[u], acc);
        }
    }
    if (own && c < d) own[(int64_t)b * d + c] = acc;
    if (threadIdx.x == 0 && c0 == 0) {
        first[y] = b;
        own_bias[b] = sb;
    }
}

template <class T>
__global__ __launch_bounds__(256) void own_kernel(OwnArgs a)
{
    own_terms<T, 256>(a, blockIdx.x, blockIdx.y * 256);
}

// ---------------------------------------------------------------------------
// Many queries: the same terms in time that grows with them. The queries are
// sorted by their label, stably, 8 bits a pass; a wave then adds up a stretch of
// the sorted order (8 positions, or 64 of many queries), and what a point's
// queries leave in later stretches than their first is joined to it. Every
// order is fixed by the labels alone, so results do not depend on the schedule.
constexpr int SORT_TILE = 2048, SORT_DIGITS = 256;   // queries a block sorts, 256 at a time
// More queries than SORT_FROM are sorted (the whole call at 2,048 x 10,000 x 32
// bfloat16: sorted 87 us whatever the labels; unsorted 81 with labels drawn at
// random, 277 with equal ones), up to SORT_BLOCK by one block in LDS, which is
// one launch in place of three a pass (8,192: 186 us in place of 217).
constexpr int64_t SORT_FROM = 1024, SORT_BLOCK = 8192;

struct SortArgs {
    const int32_t *label;             // the first pass' keys: a label of -1 comes last, as key V
    const uint32_t *key_in, *id_in;   // the later ones'
    uint32_t *key_out, *id_out;
    uint32_t *counts;                 // digits x tiles, then where each begins
    int32_t B, V, tiles, shift;

    __device__ uint32_t key(int32_t i) const
    {
        if (key_in) return key_in[i];
        return (uint32_t)(label[i] < 0 ? V : label[i]);
    }
};

__global__ __launch_bounds__(256) void sort_count_kernel(SortArgs a)
{
    __shared__ uint32_t count[SORT_DIGITS];
    const int t = threadIdx.x;
    count[t] = 0;
    __syncthreads();
    for (int r = 0; r < SORT_TILE; r += 256) {
        const int32_t i = blockIdx.x * SORT_TILE + r + t;
        if (i < a.B) atomicAdd(&count[a.key(i) >> a.shift & 255], 1u);
    }
    __syncthreads();
    a.counts[(int64_t)t * a.tiles + blockIdx.x] = count[t];
}

// counts[i] = sum of counts before i, by one block: a stretch per thread
__global__ __launch_bounds__(1024) void sort_scan_kernel(uint32_t *counts, int32_t n)
{
    __shared__ uint32_t waves[16];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int32_t per = (n + 1023) / 1024, from = min(n, t * per), to = min(n, from + per);
    uint32_t sum = 0;
    for (int32_t i = from; i < to; ++i) sum += counts[i];
    uint32_t upto = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = __shfl_up(upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == 63) waves[wave] = upto;
    __syncthreads();
    uint32_t at = upto - sum;
    for (int w = 0; w < wave; ++w) at += waves[w];
    for (int32_t i = from; i < to; ++i) {
        const uint32_t c = counts[i];
        counts[i] = at;
        at += c;
    }
}

// The wave's queries of a lane's digit: how many, and how many before it.
struct SameDigit {
    uint32_t count, rank;
    __device__ SameDigit(bool live, uint32_t digit)
    {
        uint64_t same = __ballot(live);
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const uint64_t set = __ballot(digit >> b & 1);
            same &= digit >> b & 1 ? set : ~set;
        }
        count = __popcll(same);
        rank = __popcll(same & ((1ull << (threadIdx.x & 63)) - 1));
    }
};

__global__ __launch_bounds__(256) void sort_place_kernel(SortArgs a)
{
    __shared__ uint32_t base[SORT_DIGITS], mine[4][SORT_DIGITS];
    const int t = threadIdx.x, wave = t >> 6;
    base[t] = a.counts[(int64_t)t * a.tiles + blockIdx.x];
    for (int r = 0; r < SORT_TILE; r += 256) {
#pragma unroll
        for (int w = 0; w < 4; ++w) mine[w][t] = 0;
        __syncthreads();
        const int32_t i = blockIdx.x * SORT_TILE + r + t;
        const bool live = i < a.B;
        const uint32_t key = live ? a.key(i) : 0, digit = key >> a.shift & 255;
        const SameDigit same(live, digit);
        if (live && same.rank == 0) mine[wave][digit] = same.count;
        __syncthreads();
        if (live) {
            uint32_t at = base[digit] + same.rank;
            for (int w = 0; w < wave; ++w) at += mine[w][digit];
            a.key_out[at] = key;
            a.id_out[at] = a.key_in ? a.id_in[i] : (uint32_t)i;
        }
        __syncthreads();
        base[t] += mine[0][t] + mine[1][t] + mine[2][t] + mine[3][t];
    }
}

// Up to SORT_BLOCK queries, all passes in LDS: keys and queries of before and
// after a pass, 1024 queries at a time.
__global__ __launch_bounds__(1024) void sort_block_kernel(SortArgs a)
{
    extern __shared__ uint32_t sort_lds[];   // 2 x B keys, the digits' counters, 2 x B ids of 16 bits
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int32_t B = a.B;
    uint32_t *base = sort_lds + 2 * B, (*mine)[SORT_DIGITS] = (uint32_t(*)[SORT_DIGITS])(base + SORT_DIGITS);
    uint16_t *ids = (uint16_t *)(base + 17 * SORT_DIGITS);
    for (int32_t i = t; i < B; i += 1024) {
        sort_lds[i] = a.key(i);
        ids[i] = (uint16_t)i;
    }
    int from = 0;
    for (int shift = 0; shift < 32 && ((uint32_t)a.V >> shift); shift += 8, from ^= 1) {
        const uint32_t *key_in = sort_lds + from * B;
        const uint16_t *id_in = ids + from * B;
        uint32_t *key_out = sort_lds + (from ^ 1) * B;
        uint16_t *id_out = ids + (from ^ 1) * B;
        if (t < SORT_DIGITS) base[t] = 0;
        __syncthreads();
        for (int32_t i = t; i < B; i += 1024) atomicAdd(&base[key_in[i] >> shift & 255], 1u);
        __syncthreads();
        if (t < 64) {   // the first wave: where each digit begins, four digits a lane
            uint32_t c[4], sum = 0;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                c[k] = base[t * 4 + k];
                sum += c[k];
            }
            uint32_t upto = sum;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const uint32_t v = __shfl_up(upto, o);
                if (lane >= o) upto += v;
            }
            uint32_t at = upto - sum;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                base[t * 4 + k] = at;
                at += c[k];
            }
        }
        for (int32_t r = 0; r < B; r += 1024) {
#pragma unroll
            for (int w = 0; w < 4; ++w) mine[wave][w * 64 + lane] = 0;
            __syncthreads();
            const int32_t i = r + t;
            const bool live = i < B;
            const uint32_t key = live ? key_in[i] : 0, digit = key >> shift & 255;
            const SameDigit same(live, digit);
            if (live && same.rank == 0) mine[wave][digit] = same.count;
            __syncthreads();
            if (live) {
                uint32_t at = base[digit] + same.rank;
                for (int w = 0; w < wave; ++w) at += mine[w][digit];
                key_out[at] = key;
                id_out[at] = id_in[i];
            }
            __syncthreads();
            if (t < SORT_DIGITS)
#pragma unroll
                for (int w = 0; w < 16; ++w) base[t] += mine[w][t];
            __syncthreads();
        }
    }
    for (int32_t i = t; i < B; i += 1024) {
        a.key_out[i] = sort_lds[from * B + i];
        a.id_out[i] = ids[from * B + i];
    }
}

struct SegArgs {
    OwnArgs o;
    const uint32_t *key, *id;   // sorted
    int32_t V, seg, segs;       // positions of a stretch, stretches
    float *head, *head_bias;    // segs x d, segs: what continues from the stretch before
};

// 256 columns of a stretch a wave, four columns a lane
template <class T>
__device__ inline void seg_terms(const SegArgs &a, int32_t seg, int32_t col)
{
    const int lane = threadIdx.x & 63;
    if (seg >= a.segs) return;
    const int32_t d = a.o.d, pos = seg * a.seg + lane, c0 = col + lane;
    const bool in = lane < a.seg && pos < a.o.B;
    const uint32_t key = in ? a.key[pos] : (uint32_t)a.V;
    const int n = __popcll(__ballot(key < (uint32_t)a.V));   // sorted: the live ones come first
    if (n == 0) return;
    const int32_t q = in ? (int32_t)a.id[pos] : 0;
    const float coef = lane < n ? a.o.coef[q] : 0.0f;
    uint32_t before = __shfl_up(key, 1);
    if (lane == 0) before = pos ? a.key[pos - 1] : ~0u;
    const uint64_t begins = __ballot(key != before);
    const T *h = (const T *)a.o.h;
    const bool rows = a.o.own != nullptr, first_cols = col == 0;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f}, sb = 0.0f;
    int32_t owner = -1;   // the query that keeps the sum, -1: it continues
    auto flush = [&] {
        if (rows) {
            float *to = owner < 0 ? a.head + (int64_t)seg * d : a.o.own + (int64_t)owner * d;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c0 + 64 * j < d) to[c0 + 64 * j] = acc[j];
        }
        if (first_cols && lane == 0) {
            if (owner < 0) a.head_bias[seg] = sb;
            else a.o.own_bias[owner] = sb;
        }
    };
    for (int i0 = 0; i0 < n; i0 += OWN_AHEAD) {
        float v[OWN_AHEAD][4];
        if (rows)
#pragma unroll
            for (int u = 0; u < OWN_AHEAD; ++u) {
                const T *from = h + (int64_t)__builtin_amdgcn_readlane(q, min(i0 + u, n - 1)) * a.o.h_stride;
#pragma unroll
                for (int j = 0; j < 4; ++j) v[u][j] = c0 + 64 * j < d ? (float)from[c0 + 64 * j] : 0.0f;
            }
#pragma unroll
        for (int u = 0; u < OWN_AHEAD; ++u) {
            const int i = i0 + u;
            if (i >= n) break;
            if (begins >> i & 1) {
                if (i) flush();
                owner = __builtin_amdgcn_readlane(q, i);
                if (first_cols && lane == i) a.o.first[key] = q;
                acc[0] = acc[1] = acc[2] = acc[3] = sb = 0.0f;
            }
            const float c = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(coef), i));
            sb += c;
            if (rows)
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[j] = fmaf(c, v[u][j], acc[j]);
        }
    }
    flush();
}

template <class T>
__global__ __launch_bounds__(256) void seg_kernel(SegArgs a)
{
    seg_terms<T>(a, blockIdx.x * 4 + (threadIdx.x >> 6), blockIdx.y * 256);
}

// What a point's queries left in the stretches after their first, by the block
// of the first of these: 16 waves take equal shares of them, added in order.
__global__ __launch_bounds__(1024) void seg_join_kernel(SegArgs a)
{
    __shared__ float part[16][256], part_bias[16];
    const int32_t seg = blockIdx.x + 1;
    const uint32_t key = a.key[(int64_t)seg * a.seg];
    if (key >= (uint32_t)a.V || a.key[(int64_t)seg * a.seg - 1] != key) return;        // nothing continues
    if (seg > 1 && a.key[(int64_t)(seg - 1) * a.seg - 1] == key) return;               // an earlier block's
    int32_t last = seg, end = a.segs;   // the last stretch that begins with the key: last <= it < end
    while (end - last > 1) {
        const int32_t mid = last + (end - last) / 2;
        if (a.key[(int64_t)mid * a.seg] == key) last = mid;
        else end = mid;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int32_t d = a.o.d, c0 = blockIdx.y * 256, per = (end - seg + 15) / 16;
    const int32_t from = min(end, seg + wave * per), to = min(end, from + per);
    const bool rows = a.o.own != nullptr;
    float acc[4] = {0.0f, 0.0f, 0.0f, 0.0f}, sb = 0.0f;
    if (rows)
#pragma unroll 4
        for (int32_t k = from; k < to; ++k)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (c0 + lane + 64 * j < d) acc[j] += a.head[(int64_t)k * d + c0 + lane + 64 * j];
    if (lane == 0 && blockIdx.y == 0)
#pragma unroll 4
        for (int32_t k = from; k < to; ++k) sb += a.head_bias[k];
#pragma unroll
    for (int j = 0; j < 4; ++j) part[wave][lane + 64 * j] = acc[j];
    if (lane == 0) part_bias[wave] = sb;
    __syncthreads();
    const int32_t owner = a.o.first[key], c = c0 + threadIdx.x;
    if (rows && threadIdx.x < 256 && c < d) {
        float s = a.o.own[(int64_t)owner * d + c];
#pragma unroll
        for (int w = 0; w < 16; ++w) s += part[w][threadIdx.x];
        a.o.own[(int64_t)owner * d + c] = s;
    }
    if (threadIdx.x == 0 && blockIdx.y == 0) {
        float s = a.o.own_bias[owner];
#pragma unroll
        for (int w = 0; w < 16; ++w) s += part_bias[w];
        a.o.own_bias[owner] = s;
    }
}

__global__ __launch_bounds__(256) void dbias_kernel(const float *col, int32_t tiles_b, int32_t cols_pad, int32_t n,
                                                    int32_t v0, const int32_t *first, const float *own_bias,
                                                    const float *factor, float *out)
{
    const int32_t v = blockIdx.x * 256 + threadIdx.x;
    if (v >= n) return;
    float s = 0.0f;
    for (int32_t t = 0; t < tiles_b; ++t) s += col[(int64_t)t * cols_pad + v];
    const int32_t f = first[v0 + v];
    if (f >= 0) s += own_bias[f];
    out[v] = s * *factor;
}

// dh = scale factor (sum of the splits + coef c_label), four values a thread
// (ld, a multiple of 4, is the splits' row)
template <class T>
__global__ __launch_bounds__(256) void dh_join_kernel(const float *part, int32_t splits, int32_t rows_pad, int32_t B,
                                                      int32_t d, int32_t ld, const T *points, int64_t points_stride,
                                                      const int32_t *label, const float *coef, const float *factor,
                                                      float scale, T *dh)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= (int64_t)B * (ld / 4)) return;
    const int32_t b = (int32_t)(i / (ld / 4)), c = (int32_t)(i % (ld / 4)) * 4;
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int32_t k = 0; k < splits; ++k) {
        float v[4];
        load_f32<4, float>(v, part + ((int64_t)k * rows_pad + b) * ld + c);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] += v[e];
    }
    const int32_t y = label[b];
    const float by = scale * *factor;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        if (c + e >= d) break;
        if (y >= 0) s[e] = fmaf(coef[b], (float)points[(int64_t)y * points_stride + c + e], s[e]);
        dh[(int64_t)b * d + c + e] = (T)(by * s[e]);
    }
}

// ---------------------------------------------------------------------------
// Rows of at most 128 values: one kernel for each pass, which forms a tile of
// logits, turns it into probabilities in registers and multiplies them on at
// once, so that they never leave the wave.
//
// A wave keeps TN tiles of 32 rows of one side (N) in registers and streams
// the other side (M) through LDS, 32 rows at a time. The logits are formed as
// M x N tiles: a lane then has 16 M values of one N row, its softmax
// statistics are its own, and the probabilities, rounded, are in place as the
// operand of the second product
//   out^T (values x N) += stream^T (values x M) * p (M x N),
// whose other operand is the same LDS tile read transposed. A lane's 16 values
// are rows 8 (i / 4) + 4 half + i % 4 of the tile; the second product takes
// its 32 k in that order on both sides, which is what two transposed reads of
// four rows give.
//   SWEEP_LOSS: N = queries, M = points: running maximum and sum
//   SWEEP_H:    the same and sum_v p c_v, relative to the running maximum
//   SWEEP_C:    N = points, M = queries: sum_b p h_b and sum_b p, p from the
//               first pass's statistics
// The maximum a column is taken relative to moves only when a logit exceeds it
// by 2^8: the sums have room for that, and the output is scaled rarely.
//
// A tile of 32 x 32 logits is 512 cycles of matrix instructions at 128 values
// and some 750 of vector instructions (about 120 of them at 4 cycles, 16
// exponentials at 16). 2,048 queries x 1,000,000 points x 128 values take
// 1.11 ms in SWEEP_H and 1.09 ms in SWEEP_C (940 and 960 TFLOP/s; a large library
// product reaches 1,387), which is some 1,300 cycles a tile: nearly the sum. Both
// tiles of a wave pass each phase together, with scheduling barriers between the
// phases, and the two waves of a SIMD hardly overlap. Forming the logits again in
// SWEEP_C costs 2 d operations a logit; storing and reading them back would be
// 6 bytes, more than twice the time at d = 128.
enum { SWEEP_LOSS = 0, SWEEP_H = 1, SWEEP_C = 2 };
constexpr float SLACK = 8.0f;
constexpr int SWEEP_THREADS = 256;

template <int DT_, int PARTS_, int MODE_, int TN_, int WN_>
struct Sweep {
    static constexpr int DT = DT_, PARTS = PARTS_, MODE = MODE_, TN = TN_, WN = WN_;
    static constexpr int WS = 4 / WN;                        // waves that share N rows and take M rows in turn
    static constexpr int NB = WN * TN * 32;                  // N rows of a block
    static constexpr int SR = WS > 1 ? 32 * WS : PARTS == 1 ? 64 : 32;   // M rows of a stage
    static constexpr int SUBS = SR / 32 / WS;                // tiles of a stage per wave
    static constexpr int CH = DT == 1 ? 4 : DT == 2 ? 8 : 16;            // 16-byte chunks of an LDS row
    static constexpr int ROWB = CH * 16, PLANE = SR * ROWB;
    static constexpr int SIDES = MODE == SWEEP_C ? 3 : 1;    // float arrays along M: bias, or top, factor and label
    static constexpr int STAGE = (PARTS * PLANE + SIDES * SR * 4 + 255) / 256 * 256;
    static constexpr bool STAGED = PARTS == 3 && MODE != SWEEP_C;        // float32 points: split on the way to LDS
    static constexpr int OUT_LD = DT * 32 + 4;               // floats of a row of the output in LDS
    // The kept rows' last k steps lie in LDS where the registers do not hold
    // them all: a spilled one would be waited for together with the loads on
    // their way to the next stage. SWEEP_H of 64 rows and 128 values a wave still
    // spills 11 registers, addresses that are read back once a stage before its
    // loads; with 32 rows shared by four waves 23, outside the loop.
    static constexpr int KS = 2 * DT, SHED = MODE != SWEEP_LOSS && PARTS * TN * DT >= 8 ? (MODE == SWEEP_H ? 2 : 1) : 0;
    static constexpr size_t lds()
    {
        return std::max<size_t>(2 * STAGE + SHED * TN * PARTS * SWEEP_THREADS * 16,
                                MODE == SWEEP_C ? 4 * 32 * OUT_LD * 4 : WS > 1 ? WS * 32 * (OUT_LD + 2) * 4 : 0);
    }
};

struct SweepArgs {
    const bf16_t *n, *m;      // bf16 rows of each side (parts n_part, m_part values apart)
    const float *nf, *mf;     // float32 points in their place
    int64_t n_ld, m_ld, n_part, m_part;
    int32_t N, M;             // rows of each side
    int32_t d, Kp;            // values of a row, and of it present in the bf16 rows (a multiple of 16)
    int32_t vec;              // float32 rows may be read 16 bytes at a time
    int32_t tiles_n, stages, splits, per_split;
    float scale2;
    const float *bias;        // padded: base 2, -inf past the last point
    const float *top, *rowf;  // padded (SWEEP_C)
    const int32_t *label;     // of the queries, padded
    float *pick;              // the label's logit, base 2
    RowState *part;           // splits x N
    float *out;               // splits x N x DT * 32 partial outputs
    float *col;               // splits x N partial sums of p, or null
    // SWEEP_C in one split: the results themselves
    void *dc;
    float *dbias;
    const int32_t *first;
    const float *own, *own_bias, *factor;
    float scale;
};

// The order of a row's chunks in LDS is chunk ^ sweep_swap(row): eight rows at
// one chunk (the first product) and four chunks of four rows (the second's
// transposed reads) both spread over all banks.
template <int CH>
__device__ constexpr int sweep_swap(int row)
{
    return CH == 16 ? ((row & 3) << 2) | ((row >> 2) & 3) : CH == 8 ? (row >> 1 & 1) << 2 | ((row >> 2) & 3) : (row >> 2) & 3;
}

template <class S>
__global__ __launch_bounds__(SWEEP_THREADS, 2) void sweep_kernel(SweepArgs a)
{
    constexpr int DT = S::DT, PARTS = S::PARTS, TN = S::TN, KS = S::KS, KEEP = KS - S::SHED;
    extern __shared__ __attribute__((aligned(256))) uint8_t smem[];
    int32_t split, tn0;
    if (S::MODE == SWEEP_C ? !split_block(a.tiles_n, a.splits, &tn0, &split)
                           : !split_block(a.splits, a.tiles_n, &split, &tn0))
        return;
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6, half = lane >> 5, r = lane & 31;
    const int wn = wave % S::WN, ws = wave / S::WN;
    const int32_t n0 = tn0 * S::NB + wn * TN * 32;
    const int32_t s_begin = split * a.per_split, s_end = min(a.stages, s_begin + a.per_split);

    // the kept side
    bf16x8 fn[PARTS][KEEP][TN], *shed = (bf16x8 *)(smem + 2 * S::STAGE) + t;
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        const int64_t row = min(n0 + j * 32 + r, a.N - 1);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            const int at = k * 16 + half * 8;
            bf16x8 f[PARTS];
            if constexpr (PARTS == 3 && S::MODE == SWEEP_C) {
                float v[8];
                const float *from = a.nf + row * a.n_ld + at;
                if (a.vec && at + 8 <= a.d) {
                    load_f32<4, float>(*(float(*)[4])v, from);
                    load_f32<4, float>(*(float(*)[4])(v + 4), from + 4);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = at + e < a.d ? from[e] : 0.0f;
                }
#pragma unroll
                for (int p = 0; p < PARTS; ++p)
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float top = __uint_as_float(__float_as_uint(v[e]) & 0xFFFF0000u);
                        f[p][e] = (bf16_t)top;
                        v[e] = fabsf(top) < INFINITY ? v[e] - top : 0.0f;
                    }
            } else {
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    if (at < a.Kp) {
                        f[p] = *(const bf16x8 *)(a.n + p * a.n_part + row * a.n_ld + at);
                    } else {
#pragma unroll
                        for (int e = 0; e < 8; ++e) f[p][e] = (bf16_t)0.0f;
                    }
                }
            }
#pragma unroll
            for (int p = 0; p < PARTS; ++p) {
                if (k < KEEP) fn[p][k < KEEP ? k : 0][j] = f[p];
                else shed[(((k - KEEP) * TN + j) * PARTS + p) * SWEEP_THREADS] = f[p];
            }
        }
    }

    // streamed rows: thread t's slots are rows t / CH + i * (256 / CH), stored chunk t % CH
    constexpr int PER = SWEEP_THREADS / S::CH, ITS = (S::SR + PER - 1) / PER;
    const int slot_row = t / S::CH, slot_chunk = (t % S::CH) ^ sweep_swap<S::CH>(slot_row);
    // Chunks past the values present are zeros: the other side has zeros there, and
    // whatever else the row holds, an infinity among it, would not do.
    const int slot_at = slot_chunk * 8;
    const bool present = slot_at < a.Kp;
    if (!S::STAGED && !present)
#pragma unroll
        for (int i = 0; i < 2 * PARTS * ITS; ++i) {
            if (S::SR % PER && wave * 64 >= S::SR * S::CH) continue;
            bf16x8 nil;
#pragma unroll
            for (int e = 0; e < 8; ++e) nil[e] = (bf16_t)0.0f;
            *(bf16x8 *)(smem + i / (PARTS * ITS) * S::STAGE + i / ITS % PARTS * S::PLANE
                        + (i % ITS * SWEEP_THREADS + t) * 16) = nil;
        }
    auto dma = [&](int buf, int32_t stage) {
        uint8_t *to = smem + buf * S::STAGE;
        uint32_t side_at = t * 4;
        asm volatile("" : "+v"(side_at));
#pragma unroll
        for (int k = 0; k < S::SIDES; ++k) {
            const void *side = S::MODE != SWEEP_C ? (const void *)a.bias
                             : k == 0 ? (const void *)a.top : k == 1 ? (const void *)a.rowf : (const void *)a.label;
            if (wave * 64 < S::SR && t < S::SR)
                __builtin_amdgcn_global_load_lds(
                    (const __attribute__((address_space(1))) void *)((const uint8_t *)side + (int64_t)stage * S::SR * 4 + side_at),
                    (__attribute__((address_space(3))) void *)(to + PARTS * S::PLANE + k * S::SR * 4 + wave * 256), 4, 0, 0);
        }
        if constexpr (!S::STAGED) {
            // a stage's rows lie within 32 bits of its first one (a.m_ld is below 2^24):
            // one address for the wave and an offset per lane, made anew each time to save registers
            const uint8_t *first = (const uint8_t *)(a.m + (int64_t)stage * S::SR * a.m_ld);
            int32_t row0 = slot_row;
            asm volatile("" : "+v"(row0));
            const int32_t last = a.M - 1 - stage * S::SR;
#pragma unroll
            for (int p = 0; p < PARTS; ++p)
#pragma unroll
                for (int i = 0; i < ITS; ++i) {
                    if (S::SR % PER && wave * 64 >= S::SR * S::CH) continue;
                    const uint32_t at = ((uint32_t)min(i * PER + row0, last) * (uint32_t)a.m_ld + slot_at) * 2;
                    if (present) __builtin_amdgcn_global_load_lds(
                        (const __attribute__((address_space(1))) void *)(first + p * a.m_part * 2 + at),
                        (__attribute__((address_space(3))) void *)(to + p * S::PLANE + (i * SWEEP_THREADS + wave * 64) * 16),
                        16, 0, 0);
                }
        }
    };
    // float32 points: 8 threads a row, DT * 4 values each, split into parts on the way
    float held[S::STAGED ? DT : 1][4];
    auto fetch = [&](int32_t stage) {
        if constexpr (S::STAGED) {
            const float *from = a.mf + (int64_t)min(stage * S::SR + (t >> 3), a.M - 1) * a.m_ld;
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                const int at = ((t & 7) + 8 * i) * 4;
                if (a.vec && at < a.d) {
                    load_f32<4, float>(held[i], from + at);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) held[i][e] = at + e < a.d ? from[at + e] : 0.0f;
                }
            }
        }
    };
    auto put = [&](int buf) {
        if constexpr (S::STAGED) {
            const int row = t >> 3;
#pragma unroll
            for (int i = 0; i < DT; ++i) {
                const int q = (t & 7) + 8 * i;
                uint8_t *to = smem + buf * S::STAGE + row * S::ROWB + (((q >> 1) ^ sweep_swap<S::CH>(row)) * 16) + (q & 1) * 8;
#pragma unroll
                for (int p = 0; p < PARTS; ++p) {
                    bf16x4 four;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float top = __uint_as_float(__float_as_uint(held[i][e]) & 0xFFFF0000u);
                        four[e] = (bf16_t)top;
                        held[i][e] = fabsf(top) < INFINITY ? held[i][e] - top : 0.0f;
                    }
                    *(bf16x4 *)(to + p * S::PLANE) = four;
                }
            }
        }
    };

    f32x16 out[S::MODE == SWEEP_LOSS ? 1 : DT][TN];
    float mx[TN], sum[TN], lost[TN], off[TN];
    int32_t lab[TN];
#pragma unroll
    for (int j = 0; j < TN; ++j) {
#pragma unroll
        for (int i = 0; i < (S::MODE == SWEEP_LOSS ? 1 : DT); ++i)
#pragma unroll
            for (int e = 0; e < 16; ++e) out[i][j][e] = 0.0f;
        mx[j] = NO_MAX;
        sum[j] = lost[j] = 0.0f;
        const int32_t n = n0 + j * 32 + r;
        off[j] = S::MODE == SWEEP_C ? a.bias[min(n, a.N - 1)] : 0.0f;
        lab[j] = S::MODE != SWEEP_C && n < a.N ? a.label[n] : -1;
    }

    // lane's place in transposed reads: group g of 16 lanes takes values 16 (g & 1).. of rows 4 half..
    const int tr_row = ((lane & 15) >> 2) + 4 * half, tr_chunk = ((lane >> 4) & 1) * 2 + ((lane >> 1) & 1);
    const uint32_t base = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) uint8_t *)smem;
    const uint32_t s_lane = r * S::ROWB + ((half ^ sweep_swap<S::CH>(r)) * 16);
    const uint32_t t_lane = tr_row * S::ROWB + ((tr_chunk ^ sweep_swap<S::CH>(tr_row)) * 16) + (lane & 1) * 8;

    if (s_begin < s_end) {
        dma(0, s_begin);
        fetch(s_begin);
        put(0);
    }
    wait_and_meet<0>();   // a barrier alone does not wait for loads to LDS
    for (int32_t stage = s_begin; stage < s_end; ++stage) {
        const int buf = (stage - s_begin) & 1;
        if (stage + 1 < s_end) {
            dma(buf ^ 1, stage + 1);
            fetch(stage + 1);
        }
        const uint8_t *from = smem + buf * S::STAGE;
        const float *side = (const float *)(from + PARTS * S::PLANE);
#pragma unroll 1
        for (int sub = 0; sub < S::SUBS; ++sub) {   // not unrolled: the registers are full
            const int row0 = (sub * S::WS + ws) * 32;   // of the stage
            // Both reads' addresses: the chunk's permutation is an exclusive or on
            // bits that rows and stages leave alone.
            const uint32_t s_at = base + buf * S::STAGE + row0 * S::ROWB + s_lane;
            const uint32_t t_at = base + buf * S::STAGE + row0 * S::ROWB + t_lane;
            f32x16 acc[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int e = 0; e < 16; ++e) acc[j][e] = 0.0f;
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                if (S::TN * S::DT >= 8 && k && k % 2 == 0) __builtin_amdgcn_sched_barrier(0);
                bf16x8 fm[PARTS];
#pragma unroll
                for (int p = 0; p < PARTS; ++p) fm[p] = *(const LdsRow *)(uintptr_t)((s_at ^ (k * 32)) + p * S::PLANE);
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    bf16x8 f[PARTS];   // a thread reads back what it put there itself
#pragma unroll
                    for (int p = 0; p < PARTS; ++p)
                        f[p] = k < KEEP ? fn[p][k < KEEP ? k : 0][j] : shed[(((k - KEEP) * TN + j) * PARTS + p) * SWEEP_THREADS];
                    if constexpr (PARTS == 3) {
                        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fm[2], f[0], acc[j], 0, 0, 0);
                        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fm[1], f[1], acc[j], 0, 0, 0);
                        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fm[0], f[2], acc[j], 0, 0, 0);
                        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fm[1], f[0], acc[j], 0, 0, 0);
                        acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fm[0], f[1], acc[j], 0, 0, 0);
                    }
                    acc[j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fm[0], f[0], acc[j], 0, 0, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);   // the registers are full: the phases stay apart
            // logits to probabilities
            if constexpr (S::MODE != SWEEP_C) {
                float top[TN];
#pragma unroll
                for (int j = 0; j < TN; ++j) top[j] = NO_MAX;
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float bias[4];
                    load_f32<4, float>(bias, side + row0 + 8 * q + 4 * half);
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            acc[j][4 * q + e] = fmaf(acc[j][4 * q + e], a.scale2, bias[e]);
                            top[j] = fmaxf(top[j], acc[j][4 * q + e]);
                        }
                }
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    if (__any(top[j] > mx[j] + SLACK)) {
                        const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(top[j]), __float_as_uint(top[j]), false, false);
                        const float now = fmaxf(fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])), mx[j]);
                        const float by = __builtin_amdgcn_exp2f(mx[j] - now);
                        sum[j] *= by;
                        lost[j] *= by;
                        if constexpr (S::MODE == SWEEP_H)
#pragma unroll
                            for (int i = 0; i < DT; ++i)
#pragma unroll
                                for (int e = 0; e < 16; ++e) out[i][j][e] *= by;
                        mx[j] = now;
                    }
                    const int32_t rel = lab[j] - (stage * S::SR + row0);
                    const bool mine = (uint32_t)rel < 32u;
                    if (__any(mine)) {   // a column's own point is among these rows: it is joined later
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const bool here = rel == tile_row(e, half);
                            if (here) a.pick[n0 + j * 32 + r] = acc[j][e];
                            acc[j][e] = here ? -INFINITY : acc[j][e];
                        }
                    }
                    float s = 0.0f;
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        acc[j][e] = __builtin_amdgcn_exp2f(acc[j][e] - mx[j]);
                        s += acc[j][e];
                    }
                    add_kept(sum[j], lost[j], s);
                }
            } else {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    float top[4], f[4];
                    load_f32<4, float>(top, side + row0 + 8 * q + 4 * half);
                    load_f32<4, float>(f, side + S::SR + row0 + 8 * q + 4 * half);
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            acc[j][4 * q + e] = f[e] * __builtin_amdgcn_exp2f(fmaf(acc[j][4 * q + e], a.scale2, off[j]) - top[e]);
                }
                const int32_t own = ((const int32_t *)side)[2 * S::SR + row0 + r];
                if (__any((uint32_t)(own - n0) < (uint32_t)(32 * TN))) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const int32_t y = __shfl(own, tile_row(e, half));
#pragma unroll
                        for (int j = 0; j < TN; ++j)
                            if (y == n0 + j * 32 + r) acc[j][e] = 0.0f;
                    }
                }
                if (a.col || a.dbias)
#pragma unroll
                    for (int j = 0; j < TN; ++j) {
                        float s = 0.0f;
#pragma unroll
                        for (int e = 0; e < 16; ++e) s += acc[j][e];
                        add_kept(sum[j], lost[j], s);
                    }
            }
            // the second product
            if constexpr (S::MODE != SWEEP_LOSS) {
                bf16x8 fp[2][PARTS][TN];
#pragma unroll
                for (int j = 0; j < TN; ++j)
#pragma unroll
                    for (int e = 0; e < 16; ++e)
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) fp[e >> 3][p][j][e & 7] = part_of<PARTS>(acc[j][e], p);
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int kb = 0; kb < 2; ++kb) {
#pragma unroll
                    for (int i = 0; i < DT; ++i) {
                        bf16x8 fm[PARTS];
#pragma unroll
                        for (int p = 0; p < PARTS; ++p)
#pragma unroll
                            for (int jj = 0; jj < 2; ++jj) {
                                // of chunk i * 4 + tr_chunk of row 16 kb + 8 jj + tr_row
                                const uint32_t at = (t_at ^ ((i * 64) ^ (jj * 32)))
                                                    + p * S::PLANE + (16 * kb + 8 * jj) * S::ROWB;
                                const short4v four = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsFour *)(uintptr_t)at);
                                const bf16x4 v = __builtin_bit_cast(bf16x4, four);
#pragma unroll
                                for (int e = 0; e < 4; ++e) fm[p][4 * jj + e] = v[e];
                            }
#pragma unroll
                        for (int j = 0; j < TN; ++j) {
                            if constexpr (PARTS == 3) {
                                out[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fm[2], fp[kb][0][j], out[i][j], 0, 0, 0);
                                out[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fm[1], fp[kb][1][j], out[i][j], 0, 0, 0);
                                out[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fm[0], fp[kb][2][j], out[i][j], 0, 0, 0);
                                out[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fm[1], fp[kb][0][j], out[i][j], 0, 0, 0);
                                out[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fm[0], fp[kb][1][j], out[i][j], 0, 0, 0);
                            }
                            out[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fm[0], fp[kb][0][j], out[i][j], 0, 0, 0);
                        }
                    }
                }
            }
        }
        if (stage + 1 < s_end) put(buf ^ 1);
        wait_and_meet<0>();
    }

#pragma unroll
    for (int j = 0; j < TN; ++j) sum[j] += __shfl_xor(sum[j], 32);
    if constexpr (S::WS > 1) {   // the waves that share these rows: brought to one maximum and added, in order
        constexpr int ROW = DT * 32 + 4;
        float *mine = (float *)smem + ws * 32 * (ROW + 2) + r * (ROW + 2);   // out, then maximum and sum; TN is 1
        if constexpr (S::MODE == SWEEP_H)
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) mine[i * 32 + tile_row(e, half)] = out[i][0][e];
        if (half == 0) {
            mine[ROW] = mx[0];
            mine[ROW + 1] = sum[0];
        }
        __syncthreads();
        if (ws) return;
        float by[S::WS], top = mx[0];
#pragma unroll
        for (int w = 1; w < S::WS; ++w) top = fmaxf(top, mine[w * 32 * (ROW + 2) + ROW]);
#pragma unroll
        for (int w = 0; w < S::WS; ++w) by[w] = __builtin_amdgcn_exp2f(mine[w * 32 * (ROW + 2) + ROW] - top);
        mx[0] = top;
        sum[0] *= by[0];
#pragma unroll
        for (int w = 1; w < S::WS; ++w) sum[0] = fmaf(by[w], mine[w * 32 * (ROW + 2) + ROW + 1], sum[0]);
        if constexpr (S::MODE == SWEEP_H)
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    out[i][0][e] *= by[0];
#pragma unroll
                    for (int w = 1; w < S::WS; ++w)
                        out[i][0][e] = fmaf(by[w], mine[w * 32 * (ROW + 2) + i * 32 + tile_row(e, half)], out[i][0][e]);
                }
    }
    const int64_t share = split;
    if constexpr (S::MODE != SWEEP_C) {
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int32_t n = n0 + j * 32 + r;
            if (n >= a.N) continue;
            // the halves move their maximum together, except where one never saw a logit above the start
            const float other = __shfl_xor(mx[j], 32);
            if (half == 0) a.part[share * a.N + n] = RowState{fmaxf(mx[j], other), sum[j]};
            if constexpr (S::MODE == SWEEP_H)
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int q = 0; q < 4; ++q) {
                        const float four[4] = {out[i][j][4 * q], out[i][j][4 * q + 1], out[i][j][4 * q + 2], out[i][j][4 * q + 3]};
                        store_f32<4, float>(a.out + (share * a.N + n) * (DT * 32) + i * 32 + 8 * q + 4 * half, four);
                    }
        }
    } else {
        float *mine = (float *)smem + wave * 32 * S::OUT_LD;
        const bool whole = a.splits == 1;
        const float factor = whole ? *a.factor : 1.0f;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int32_t base = n0 + j * 32;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float four[4] = {out[i][j][4 * q], out[i][j][4 * q + 1], out[i][j][4 * q + 2], out[i][j][4 * q + 3]};
                    store_f32<4, float>(mine + r * S::OUT_LD + i * 32 + 8 * q + 4 * half, four);
                }
            __syncthreads();
            if (half == 0 && base + r < a.N) {
                if (!whole && a.col) a.col[(int64_t)split * a.N + base + r] = sum[j];
                if (whole && a.dbias) {
                    const int32_t f = a.first[base + r];
                    a.dbias[base + r] = factor * (f >= 0 ? sum[j] + a.own_bias[f] : sum[j]);
                }
            }
            if (whole && !a.dc) continue;   // the biases' gradient alone
            constexpr int CHUNKS = DT * 4, ROWS = 64 / CHUNKS > 0 ? 64 / CHUNKS : 1;   // chunks of 8 values, rows at once
            for (int row = lane / CHUNKS; row < 32; row += ROWS) {
                const int32_t n = base + row;
                const int at = (lane % CHUNKS) * 8;
                if (n >= a.N || lane >= ROWS * CHUNKS || at >= a.d) continue;
                float v[8];
                load_f32<4, float>(*(float(*)[4])v, mine + row * S::OUT_LD + at);
                load_f32<4, float>(*(float(*)[4])(v + 4), mine + row * S::OUT_LD + at + 4);
                if (!whole) {
                    float *to = a.out + ((int64_t)split * a.N + n) * (DT * 32) + at;
                    store_f32<4, float>(to, *(float(*)[4])v);
                    store_f32<4, float>(to + 4, *(float(*)[4])(v + 4));
                    continue;
                }
                const int32_t f = a.first[n];
                const float by = a.scale * factor;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (f >= 0 && at + e < a.d) v[e] += a.own[(int64_t)f * a.d + at + e];
                    v[e] *= by;
                }
                using T = typename std::conditional<PARTS == 3, float, bf16_t>::type;
                T *to = (T *)a.dc + (int64_t)n * a.d + at;
                if (a.d % 8 == 0 && aligned16(a.dc)) {
                    constexpr int V = 16 / sizeof(T);
#pragma unroll
                    for (int e = 0; e < 8; e += V) store_f32<V, T>(to + e, *(float(*)[V])(v + e));
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (at + e < a.d) to[e] = (T)v[e];
                }
            }
        }
    }
}

// The splits of SWEEP_C added in order, and what a single split writes itself.
template <class T>
__global__ __launch_bounds__(256) void dc_join_kernel(const float *out, const float *col, int32_t splits, int32_t N, int32_t d,
                                                      int32_t ld, const int32_t *first, const float *own,
                                                      const float *own_bias, const float *factor, float scale, T *dc,
                                                      float *dbias)
{
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (dc && i < (int64_t)N * d) {
        const int64_t n = i / d;
        const int c = (int)(i % d);
        float s = 0.0f;
        for (int k = 0; k < splits; ++k) s += out[((int64_t)k * N + n) * ld + c];
        const int32_t f = first[n];
        if (f >= 0) s += own[(int64_t)f * d + c];
        dc[i] = (T)(scale * *factor * s);
    }
    if (dbias && i < N) {
        float s = 0.0f;
        for (int k = 0; k < splits; ++k) s += col[(int64_t)k * N + i];
        const int32_t f = first[i];
        if (f >= 0) s += own_bias[f];
        dbias[i] = *factor * s;
    }
}

// The shares of SWEEP_H, brought to the common maximum:
// dh = scale factor (g / sum  sum_shares 2^(m - top) out + coef c_label)
struct DhShares {
    const float *out;        // shares x B x ld
    const RowState *part;
    int32_t shares, ld;
    const float *top, *rowf, *factor;
    const void *points;
    int64_t points_stride;
    float scale;
    void *dh;
};

// A block per query: ld / 4 threads take four values each, and as many times as
// they fit the block they part the shares, whose sums are then added in order.
template <class T, int TH>
__device__ inline void dh_of_shares(const DhShares &a, const OwnArgs &o, int32_t b)
{
    __shared__ float part[TH * 4];
    const int cols = a.ld / 4, slices = TH / cols, col = threadIdx.x % cols, slice = threadIdx.x / cols;
    const float f = a.rowf[b], m = a.top[b];
    float s[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (f != 0.0f && slice < slices)
#pragma unroll 4
        for (int32_t k = slice; k < a.shares; k += slices) {
            const int64_t at = (int64_t)k * o.B + b;
            float v[4];
            load_f32<4, float>(v, a.out + at * a.ld + col * 4);
            const float by = __builtin_amdgcn_exp2f(a.part[at].m - m);
#pragma unroll
            for (int e = 0; e < 4; ++e) s[e] = fmaf(by, v[e], s[e]);
        }
    store_f32<4, float>(part + threadIdx.x * 4, s);
    __syncthreads();
    const int c = threadIdx.x;
    if (c >= o.d) return;
    float sum = 0.0f;
    for (int k = 0; k < slices; ++k) sum += part[(k * cols) * 4 + c];
    sum *= f;
    const int32_t y = o.label[b];
    if (y >= 0) sum = fmaf(o.coef[b], (float)((const T *)a.points)[(int64_t)y * a.points_stride + c], sum);
    ((T *)a.dh)[(int64_t)b * o.d + c] = (T)(a.scale * *a.factor * sum);
}

// Between the sweeps: the queries' gradients, a block each, and beside them the
// labels' own terms. TH: 1024 threads where there are many shares to add, which
// are many where there are few queries.
template <class T, int TH>
__global__ __launch_bounds__(TH) void between_kernel(OwnArgs o, DhShares s, SegArgs g)
{
    const int32_t dh = s.dh ? o.B : 0, b = (int32_t)blockIdx.x - dh;   // d is at most 128
    if (b < 0) dh_of_shares<T, TH>(s, o, blockIdx.x);
    else if (g.key) seg_terms<T>(g, b * (TH / 64) + (threadIdx.x >> 6), 0);
    else own_terms<T, TH>(o, b, 0);
}

// ---------------------------------------------------------------------------
// host side

int64_t round_up(int64_t a, int64_t to) { return ceil_div(a, to) * to; }

// Where everything lies in the workspace, for one call's sizes.
struct Plan {
    int32_t parts, Kp, tile_b, rows_pad, tiles_b;
    bool direct;               // the points are read where they are
    bool sweep;                // rows of at most 128 values: sweep_kernel
    int32_t ld;                // sweep: values of a padded row
    int32_t splits, shares, per_split;               // of the statistics
    int32_t c_splits, c_per_split, c_tiles;          // sweep: of the points' gradient
    int64_t Vc, cols_pad;      // points per piece, and its padded size
    int64_t copied;            // points that are held as a copy at a time
    int32_t dh_splits, dh_k, tile_d, tiles_d;
    int64_t off_h, off_c, off_part, off_loss, off_top, off_rowf, off_coef, off_label, off_pick, off_factor, off_done;
    bool sorted;               // the queries are sorted by label for the labels' own terms
    int32_t sort_tiles, seg, segs;
    int64_t off_p, off_col, off_dh, off_first, off_own, off_ownb, off_bias, off_hz, off_dc, total;
    int64_t off_keys, off_counts, off_head, off_headb;   // sorted only
};

// Whether the tiles can be read where the points are: bfloat16 rows of whole
// 16-byte chunks, an even number of them.
bool points_direct(const boa_xent *x)
{
    return x->dtype == BOA_T_BF16 && x->d % 16 == 0 && aligned(x->points, 16) && x->points_stride % 8 == 0
           && x->points_stride < (1 << 24);
}

Plan make_plan(const boa_xent *x, bool grad)
{
    Plan p{};
    p.parts = x->dtype == BOA_T_F32 ? 3 : 1;
    p.direct = points_direct(x);
    p.sweep = x->d <= 128;
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t o = at;
        at += round_up(std::max<int64_t>(bytes, 16), 256);
        return o;
    };
    const bool dh = grad && x->dh, dc = grad && x->dpoints, db = grad && x->dbias;
    if (p.sweep) {
        p.ld = (int32_t)round_up(x->d, 32);
        // up to 32 queries the waves of a block share them and part the points
        p.tile_b = p.parts == 1 ? (x->B <= 32 ? 32 : x->B <= 128 ? 128 : 256) : 128;
        const int32_t rows = p.tile_b == 32 ? 128 : p.parts == 1 ? 64 : 32;
        p.tiles_b = (int32_t)ceil_div(x->B, p.tile_b);
        p.rows_pad = (int32_t)round_up(x->B, 256);
        const int64_t stages = ceil_div(x->V, rows);
        // two blocks per CU; whole multiples of the 8 XCDs, so that none gets a block more
        int64_t splits = std::max<int64_t>(1, 512 / p.tiles_b);
        if (splits > 8) splits = splits / 8 * 8;
        splits = std::min(splits, stages);
        p.per_split = (int32_t)ceil_div(stages, splits);
        p.splits = (int32_t)ceil_div(stages, p.per_split);
        p.shares = p.splits;
        p.off_bias = take(round_up(x->V, 128) * 4);
        p.off_h = take((int64_t)p.parts * p.rows_pad * p.ld * 2);
        if (x->dtype == BOA_T_BF16 && !p.direct) p.off_c = take(x->V * (int64_t)p.ld * 2);
        if (dh) p.off_dh = take((int64_t)p.shares * x->B * p.ld * 4);
        if (dc || db) {
            p.off_hz = take((int64_t)p.parts * p.rows_pad * p.ld * 2);
            const int64_t c_stages = ceil_div(x->B, p.parts == 1 ? 64 : 32);
            p.c_tiles = (int32_t)ceil_div(x->V, p.parts == 1 ? 256 : 128);
            // few points: the queries are parted, and the parts joined
            const int64_t c_splits = std::min(c_stages, std::max<int64_t>(1, p.c_tiles < 256 ? 512 / p.c_tiles : 1));
            p.c_per_split = (int32_t)ceil_div(c_stages, c_splits);
            p.c_splits = (int32_t)ceil_div(c_stages, p.c_per_split);
            if (p.c_splits > 1) {
                p.off_dc = take((int64_t)p.c_splits * x->V * p.ld * 4);
                p.off_col = take((int64_t)p.c_splits * x->V * 4);
            }
        }
    } else {
        p.Kp = (int32_t)round_up(x->d, 16);
        // rows of queries in a tile: 256, or 128 where that leaves 10% less past the end
        p.tile_b = x->B <= 32 ? 32 : round_up(x->B, 256) * 10 > round_up(x->B, 128) * 11 ? 128 : 256;
        p.tiles_b = (int32_t)ceil_div(x->B, p.tile_b);
        p.rows_pad = p.tiles_b * p.tile_b;
        const int64_t tiles_v = ceil_div(x->V, 256);
        // the losses' splits: a block per CU (its stages fill LDS), and no more than there are tiles
        const int64_t resident = p.tile_b == 256 ? 256 : 512;   // blocks
        int64_t splits = std::max<int64_t>(1, resident / p.tiles_b);
        if (splits > 8) splits = splits / 8 * 8;   // none of the 8 XCDs with a block more
        p.splits = (int32_t)std::min(tiles_v, splits);
        // columns of dh's product: 256, or 128 where that leaves 15% less past the end
        p.tile_d = round_up(x->d, 256) * 100 > round_up(x->d, 128) * 115 ? 128 : 256;
        p.tiles_d = (int32_t)ceil_div(x->d, p.tile_d);
        // A piece's probabilities take up to 256 MB, or four tiles of points where
        // there are more than 131,072 queries (43,690 with parts). Of the numbers
        // of pieces that do, the one whose launches fill the GPU best: each launch takes
        // whole rounds of resident blocks.
        // Points that cannot be read where they are get a copy: of all of them up
        // to 2 GB, so that it serves both passes, else a piece at a time, which
        // then is no larger than that either.
        if (p.parts == 3) p.direct = p.tile_b == 32;   // Shape::SPLIT
        const int64_t per = (int64_t)p.rows_pad * 2 * p.parts;
        const int64_t point = (int64_t)p.Kp * 2 * p.parts, copy = (int64_t)2 << 30;
        const bool by_pieces = !p.direct && x->V * point > copy;
        int64_t most = std::max<int64_t>(4, ((int64_t)256 << 20) / per / 256);   // tiles of points
        if (by_pieces) most = std::min(most, copy / point / 256);   // at least 341 tiles
        const int64_t least = ceil_div(tiles_v, most);
        int64_t best = -1, best_cost = 0;
        for (int64_t n = least; n < least + 6; ++n) {
            const int64_t tv = ceil_div(tiles_v, n), c_tiles = ceil_div(x->d, 128);
            // rounds, each worth the work of its blocks
            const int64_t cost = n * (ceil_div(tv * p.tiles_b, resident) * resident * p.tile_b * x->d
                                      + ceil_div(tv * c_tiles, 512) * 512 * 128 * p.rows_pad);
            if (best < 0 || cost < best_cost) best = tv, best_cost = cost;
        }
        p.Vc = best * 256;
        p.cols_pad = p.Vc;
        p.copied = p.direct ? 0 : by_pieces ? p.Vc : x->V;
        const int64_t pieces = by_pieces ? ceil_div(x->V, p.Vc) : 1;
        p.shares = p.splits * (int32_t)pieces;   // a piece's tiles are split like all of them
        p.off_h = take((int64_t)p.parts * p.rows_pad * p.Kp * 2);
        p.off_c = take(p.copied * point);
        if (dh) {
            // The points are split where the tiles alone do not fill the GPU. All
            // tiles of a split run on one XCD, so splits come in eights; a block
            // pays for reading and adding to its share of the sums as for `over`
            // values of k (26 us and 32 cycles each, six times less with parts).
            const int64_t tiles = (int64_t)p.tiles_b * p.tiles_d, over = (p.parts == 1 ? 2000 : 330) * p.tile_b / 256;
            const int64_t room = p.tile_b == 256 && p.tile_d == 256 ? 32 : 64;   // blocks an XCD holds
            int64_t splits = 1, split_cost = 0;
            for (int64_t n = 1; n <= 512 && n * 256 <= p.cols_pad; n += n < 8 ? n : 8) {
                const int64_t cost = ceil_div(ceil_div(n, 8) * tiles, room) * (ceil_div(p.cols_pad, n) + over);
                if (n == 1 || cost < split_cost) splits = n, split_cost = cost;
            }
            p.dh_k = (int32_t)round_up(ceil_div(p.cols_pad, splits), 64);
            p.dh_splits = (int32_t)ceil_div(p.cols_pad, p.dh_k);
            p.off_dh = take((int64_t)p.dh_splits * p.rows_pad * p.Kp * 4);
        }
        if (dh || dc) p.off_p = take(per * p.cols_pad);
        if (dc || db) p.off_hz = take((int64_t)p.parts * p.rows_pad * p.Kp * 2);
        if (db) p.off_col = take((int64_t)p.tiles_b * p.cols_pad * 4);
    }
    p.off_part = take((int64_t)p.shares * x->B * sizeof(RowState));
    p.off_loss = take(x->B * 4);
    p.off_pick = take(x->B * 4);
    p.off_top = take((int64_t)p.rows_pad * 4);
    p.off_rowf = take((int64_t)p.rows_pad * 4);
    p.off_label = take((int64_t)p.rows_pad * 4);
    p.off_factor = take(16);
    p.off_done = take(16);
    if (grad) p.off_coef = take(x->B * 4);
    if (dc || db) {
        p.off_first = take(x->V * 4);
        p.off_ownb = take(x->B * 4);
        if (dc) p.off_own = take(x->B * (int64_t)x->d * 4);
        p.sorted = x->B > SORT_FROM;
        if (p.sorted) {
            p.sort_tiles = (int32_t)ceil_div(x->B, SORT_TILE);
            p.seg = x->B <= SORT_BLOCK ? 8 : 64;   // 64 lanes know a stretch; few queries give more waves something to do
            p.segs = (int32_t)ceil_div(x->B, p.seg);
            p.off_keys = take(4 * x->B * 4);   // keys and queries, before and after a pass
            p.off_counts = take((int64_t)SORT_DIGITS * p.sort_tiles * 4);
            if (dc) p.off_head = take((int64_t)p.segs * x->d * 4);
            p.off_headb = take((int64_t)p.segs * 4);
        }
    }
    p.total = at;
    return p;
}

template <class S>
constexpr size_t stage_bytes()
{
    return S::STAGES * S::STAGE * sizeof(bf16_t);
}

template <class K, class A>
void run(K kernel, uint32_t grid, uint32_t threads, size_t lds, hipStream_t st, const A &args)
{
    if (lds > 64 << 10)   // has to be asked for
        (void)hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    kernel<<<dim3(grid), threads, lds, st>>>(args);
}

template <class F>
void with_tile(int32_t n, F f)   // 32, 128 or 256 rows of the smaller side
{
    if (n <= 32) f(std::integral_constant<int, 32>{});
    else if (n <= 128) f(std::integral_constant<int, 128>{});
    else f(std::integral_constant<int, 256>{});
}

// Waves of 128 x 64 (or 64 x 128) where a tile has room: 6 fragments for 8
// matrix instructions, which LDS delivers in half their time.
template <int BM, int BN, int PARTS>
struct Pick;
template <int P> struct Pick<256, 256, P> { using S = Shape<2, 4, 4, 2, P>; };
template <int P> struct Pick<256, 128, P> { using S = Shape<2, 2, 4, 2, P>; };
template <int P> struct Pick<128, 256, P> { using S = Shape<2, 2, 2, 4, P>; };
template <int P> struct Pick<128, 128, P> { using S = Shape<2, 2, 2, 2, P>; };
template <> struct Pick<256, 32, 1> { using S = Shape<2, 1, 4, 1, 1>; };
template <> struct Pick<32, 256, 1> { using S = Shape<1, 2, 1, 4, 1>; };
template <> struct Pick<32, 128, 1> { using S = Shape<1, 2, 1, 2, 1>; };
template <> struct Pick<256, 32, 3> { using S = Shape<4, 1, 2, 1, 3>; };
template <> struct Pick<32, 256, 3> { using S = Shape<1, 4, 1, 2, 3>; };
template <> struct Pick<32, 128, 3> { using S = Shape<1, 4, 1, 1, 3>; };

int check(const boa_xent *x, bool grad)
{
    auto bad = [](const char *why) { return set_error(BOA_EINVAL, why); };
    if (!x) return bad("softmax_xent: NULL arguments");
    if (x->dtype == BOA_T_F16)
        return set_error(BOA_EUNSUPPORTED, "softmax_xent: float16 does not hold the probabilities of many points; use bfloat16 or float32");
    if (x->dtype != BOA_T_F32 && x->dtype != BOA_T_BF16) return bad("softmax_xent: unknown dtype");
    if (x->d < 1 || x->d > BOA_MAX_XENT_D) return bad("softmax_xent: d out of range [1, 4096]");
    // two blocks per query, or a thread per four values of them, stay below a launch's 2^32 threads
    if (x->B < 0 || x->B > BOA_MAX_XENT_B) return bad("softmax_xent: B out of range [0, 2^21]");
    if (x->V < 1 || x->V > ((int64_t)1 << 31) - (1 << 16)) return bad("softmax_xent: V out of range");
    if (x->reduction < BOA_REDUCE_NONE || x->reduction > BOA_REDUCE_MEAN) return bad("softmax_xent: unknown reduction");
    if ((x->B > 1 && x->h_stride < x->d) || (x->V > 1 && x->points_stride < x->d))
        return bad("softmax_xent: row stride smaller than d");
    if (!std::isfinite(x->scale)) return bad("softmax_xent: scale must be finite");
    if (grad && x->dbias && !x->bias) return bad("softmax_xent: a gradient of bias without a bias");
    return BOA_OK;
}

// What one call's steps share.
template <class T>
struct Work {
    const boa_xent *x;
    bool grad;
    Plan p;
    uint8_t *ws;
    hipStream_t st;

    template <class P>
    P *at(int64_t off) const { return (P *)(ws + off); }
    float *row_loss() const { return x->reduction == BOA_REDUCE_NONE ? x->loss : at<float>(p.off_loss); }
    bool want_c() const { return grad && (x->dpoints || x->dbias); }

    // queries as parts and their labels, and the points' side of it
    void prep(int32_t ld, bf16_t *kept, float *bias, int32_t padded) const
    {
        PrepArgs a{};
        PartsArgs &q = a.queries;
        q.src = x->h, q.stride = x->h_stride, q.R = (int32_t)x->B, q.C = x->d, q.rows_pad = p.rows_pad;
        q.plain = at<bf16_t>(p.off_h), q.plain_ld = ld, q.plain_part = (int64_t)p.rows_pad * ld, q.kept = kept;
        q.labels = x->labels, q.V = (int32_t)x->V, q.label = at<int32_t>(p.off_label);
        a.query_blocks = (int32_t)parts_blocks(q);
        a.bias = x->bias, a.to = bias, a.V = (int32_t)x->V, a.padded = padded;
        a.first = want_c() ? at<int32_t>(p.off_first) : nullptr;
        a.point_blocks = a.to || a.first ? (int32_t)std::min<int64_t>(1024, ceil_div(padded, 256)) : 0;
        a.done = at<uint32_t>(p.off_done);
        prep_kernel<T><<<dim3((uint32_t)(a.query_blocks + a.point_blocks)), 256, 0, st>>>(a);
    }

    // after the statistics: losses, and what the gradients need of each query
    void rows(int32_t shares) const
    {
        RowArgs r{};
        r.labels = x->labels, r.dloss = grad ? x->dloss : nullptr, r.pick = at<float>(p.off_pick);
        r.part = at<RowState>(p.off_part), r.loss = row_loss(), r.lse = x->lse;
        r.top = at<float>(p.off_top), r.rowf = at<float>(p.off_rowf), r.label = at<int32_t>(p.off_label);
        r.coef = grad ? at<float>(p.off_coef) : nullptr;
        r.B = (int32_t)x->B, r.V = (int32_t)x->V, r.shares = shares, r.reduction = x->reduction, r.rows_pad = p.rows_pad;
        r.done = at<uint32_t>(p.off_done);
        r.total = x->reduction != BOA_REDUCE_NONE ? x->loss : nullptr, r.factor = grad ? at<float>(p.off_factor) : nullptr;
        row_kernel<<<dim3((uint32_t)ceil_div(p.rows_pad, 4)), 256, 0, st>>>(r);
    }

    OwnArgs own() const
    {
        OwnArgs o{};
        o.h = x->h, o.h_stride = x->h_stride, o.B = (int32_t)x->B, o.d = x->d;
        o.label = at<int32_t>(p.off_label), o.coef = at<float>(p.off_coef);
        if (want_c()) {
            o.first = at<int32_t>(p.off_first), o.own_bias = at<float>(p.off_ownb);
            o.own = x->dpoints ? at<float>(p.off_own) : nullptr;
        }
        return o;
    }

    // the queries sorted by label: what seg_kernel takes
    SegArgs sort(const OwnArgs &o) const
    {
        const int32_t B = (int32_t)x->B;
        uint32_t *keys[2] = {at<uint32_t>(p.off_keys), at<uint32_t>(p.off_keys) + 2 * x->B};
        SortArgs s{};
        s.label = o.label, s.counts = at<uint32_t>(p.off_counts);
        s.B = B, s.V = (int32_t)x->V, s.tiles = p.sort_tiles;
        s.key_out = keys[0], s.id_out = keys[0] + x->B;
        if (B <= SORT_BLOCK) {
            run(sort_block_kernel, 1, 1024, (size_t)B * 12 + 17 * SORT_DIGITS * 4, st, s);
        } else {
            const dim3 tiles((uint32_t)p.sort_tiles);
            int to = 0;
            for (s.shift = 0; s.shift < 32 && (x->V >> s.shift); s.shift += 8) {   // keys up to V
                s.key_out = keys[to], s.id_out = keys[to] + x->B;
                sort_count_kernel<<<tiles, 256, 0, st>>>(s);
                sort_scan_kernel<<<dim3(1), 1024, 0, st>>>(s.counts, SORT_DIGITS * p.sort_tiles);
                sort_place_kernel<<<tiles, 256, 0, st>>>(s);
                s.key_in = s.key_out, s.id_in = s.id_out;
                to ^= 1;
            }
        }
        SegArgs a{};
        a.o = o, a.key = s.key_out, a.id = s.id_out, a.V = s.V, a.seg = p.seg, a.segs = p.segs;
        a.head = x->dpoints ? at<float>(p.off_head) : nullptr, a.head_bias = at<float>(p.off_headb);
        return a;
    }

    void join_segs(const SegArgs &a) const
    {
        const uint32_t cols = a.o.own ? (uint32_t)ceil_div(x->d, 256) : 1;
        if (p.segs > 1) seg_join_kernel<<<dim3((uint32_t)p.segs - 1, cols), 1024, 0, st>>>(a);
    }

    // the labels' own terms, in launches of their own
    void own_terms(const OwnArgs &o) const
    {
        const uint32_t cols = o.own ? (uint32_t)ceil_div(x->d, 256) : 1;
        if (!p.sorted) {
            own_kernel<T><<<dim3((uint32_t)x->B, cols), 256, 0, st>>>(o);
            return;
        }
        const SegArgs a = sort(o);
        seg_kernel<T><<<dim3((uint32_t)ceil_div(p.segs, 4), cols), 256, 0, st>>>(a);
        join_segs(a);
    }
};

template <class S>
void launch_sweep(const SweepArgs &a, hipStream_t st)
{
    const uint32_t grid = S::MODE == SWEEP_C ? split_grid(a.tiles_n, a.splits) : split_grid(a.splits, a.tiles_n);
    run(sweep_kernel<S>, grid, SWEEP_THREADS, S::lds(), st, a);
}

template <int DT, int MODE, class T>
void sweep(const SweepArgs &a, int32_t tile, hipStream_t st)
{
    if constexpr (sizeof(T) == 4) {
        launch_sweep<Sweep<DT, 3, MODE, 1, 4>>(a, st);
    } else if constexpr (MODE == SWEEP_C) {
        launch_sweep<Sweep<DT, 1, MODE, 2, 4>>(a, st);
    } else {
        if (tile == 32) launch_sweep<Sweep<DT, 1, MODE, 1, 1>>(a, st);
        else if (tile == 128) launch_sweep<Sweep<DT, 1, MODE, 1, 4>>(a, st);
        else launch_sweep<Sweep<DT, 1, MODE, 2, 4>>(a, st);
    }
}

template <int MODE, class T>
void sweep(const SweepArgs &a, int32_t tile, int32_t ld, hipStream_t st)
{
    if (ld == 32) sweep<1, MODE, T>(a, tile, st);
    else if (ld == 64) sweep<2, MODE, T>(a, tile, st);
    else if (ld == 96) sweep<3, MODE, T>(a, tile, st);
    else sweep<4, MODE, T>(a, tile, st);
}

template <class T>
int run_sweeps(const Work<T> &w)
{
    const boa_xent *x = w.x;
    const Plan &p = w.p;
    const int32_t B = (int32_t)x->B, V = (int32_t)x->V, d = x->d;
    hipStream_t st = w.st;
    bf16_t *h = w.template at<bf16_t>(p.off_h), *hz = w.want_c() ? w.template at<bf16_t>(p.off_hz) : nullptr;
    int32_t *first = w.want_c() ? w.template at<int32_t>(p.off_first) : nullptr;
    float *bias = w.template at<float>(p.off_bias);
    const int32_t v_pad = (int32_t)round_up(V, 128);

    w.prep(p.ld, hz, bias, v_pad);
    SweepArgs c{};   // the points' side of the arguments
    if constexpr (sizeof(T) == 4) {
        c.mf = (const float *)x->points, c.m_ld = x->points_stride;
        c.vec = d % 4 == 0 && x->points_stride % 4 == 0 && aligned(x->points, 16);
        c.Kp = p.ld;
    } else if (p.direct) {
        c.m = (const bf16_t *)x->points, c.m_ld = x->points_stride, c.Kp = d;
    } else {
        bf16_t *copy = w.template at<bf16_t>(p.off_c);
        for (int64_t v0 = 0; v0 < V; v0 += LAUNCH_ROWS) {
            PartsArgs a{};
            a.src = (const T *)x->points + v0 * x->points_stride, a.stride = x->points_stride;
            a.R = a.rows_pad = (int32_t)std::min<int64_t>(LAUNCH_ROWS, V - v0), a.C = d;
            a.plain = copy + v0 * p.ld, a.plain_ld = p.ld;
            parts_kernel<T><<<dim3((uint32_t)parts_blocks(a)), 256, 0, st>>>(a);
        }
        c.m = copy, c.m_ld = p.ld, c.Kp = p.ld;
    }
    SweepArgs a = c;
    a.n = h, a.n_ld = p.ld, a.n_part = (int64_t)p.rows_pad * p.ld, a.N = B, a.M = V, a.d = d;
    a.Kp = p.ld;
    if (p.direct) a.Kp = d;   // h has zeros there, the points other values
    a.tiles_n = p.tiles_b, a.splits = p.splits, a.per_split = p.per_split;
    a.stages = (int32_t)ceil_div(V, p.tile_b == 32 ? 128 : p.parts == 1 ? 64 : 32);
    a.scale2 = x->scale * LOG2E, a.bias = bias, a.label = w.template at<int32_t>(p.off_label);
    a.pick = w.template at<float>(p.off_pick), a.part = w.template at<RowState>(p.off_part);
    const bool dh = w.grad && x->dh;
    if (dh) {
        a.out = w.template at<float>(p.off_dh);
        sweep<SWEEP_H, T>(a, p.tile_b, p.ld, st);
    } else {
        sweep<SWEEP_LOSS, T>(a, p.tile_b, p.ld, st);
    }
    w.rows(p.shares);
    if (!w.grad) return launch_status("softmax_xent");
    const float *factor = w.template at<float>(p.off_factor);
    const OwnArgs own = w.own();
    DhShares shares{};
    if (dh) {
        shares.out = a.out, shares.part = a.part, shares.shares = p.shares, shares.ld = p.ld;
        shares.top = w.template at<float>(p.off_top), shares.rowf = w.template at<float>(p.off_rowf);
        shares.factor = factor, shares.points = x->points, shares.points_stride = x->points_stride;
        shares.scale = x->scale, shares.dh = x->dh;
    }
    if (dh || w.want_c()) {
        SegArgs g{};
        if (w.want_c() && p.sorted) g = w.sort(own);
        const int threads = p.shares > 64 ? 1024 : 256;
        const int64_t terms = !w.want_c() ? 0 : p.sorted ? ceil_div(p.segs, threads / 64) : B;
        const dim3 grid((uint32_t)((dh ? B : 0) + terms));
        if (threads == 1024) between_kernel<T, 1024><<<grid, 1024, 0, st>>>(own, shares, g);
        else between_kernel<T, 256><<<grid, 256, 0, st>>>(own, shares, g);
        if (g.key) w.join_segs(g);
    }
    if (w.want_c()) {
        SweepArgs g = c;
        g.n = c.m, g.nf = c.mf, g.n_ld = c.m_ld, g.N = V, g.M = B, g.d = d;
        g.m = hz, g.mf = nullptr, g.m_ld = p.ld, g.m_part = (int64_t)p.rows_pad * p.ld;
        g.tiles_n = p.c_tiles, g.splits = p.c_splits, g.per_split = p.c_per_split;
        g.stages = (int32_t)ceil_div(B, p.parts == 1 ? 64 : 32);
        g.scale2 = a.scale2, g.bias = bias, g.label = a.label;
        g.top = w.template at<float>(p.off_top), g.rowf = w.template at<float>(p.off_rowf);
        g.first = first, g.factor = factor, g.scale = x->scale;
        g.own = own.own, g.own_bias = own.own_bias;
        g.dc = x->dpoints, g.dbias = x->dbias;
        if (p.c_splits > 1) {
            g.out = w.template at<float>(p.off_dc);
            g.col = x->dbias ? w.template at<float>(p.off_col) : nullptr;
        }
        sweep<SWEEP_C, T>(g, 0, p.ld, st);
        if (p.c_splits > 1)
            dc_join_kernel<T><<<dim3((uint32_t)ceil_div((int64_t)V * (x->dpoints ? d : 1), 256)), 256, 0, st>>>(
                g.out, g.col, p.c_splits, V, d, p.ld, first, g.own, g.own_bias, factor, x->scale, (T *)x->dpoints, x->dbias);
    }
    return launch_status("softmax_xent_grad");
}

template <class T>
int run_tiles(const Work<T> &w)
{
    constexpr int PARTS = sizeof(T) == 4 ? 3 : 1;
    const boa_xent *x = w.x;
    const Plan &p = w.p;
    const bool grad = w.grad;
    uint8_t *ws = w.ws;
    hipStream_t st = w.st;
    const int32_t B = (int32_t)x->B, V = (int32_t)x->V, d = x->d;
    bf16_t *hp = (bf16_t *)(ws + p.off_h), *hz = w.want_c() ? (bf16_t *)(ws + p.off_hz) : nullptr;
    float *factor = (float *)(ws + p.off_factor);
    const int64_t h_part = (int64_t)p.rows_pad * p.Kp, c_part = p.copied * p.Kp;
    w.prep(p.Kp, hz, nullptr, V);

    const int32_t pieces = (int32_t)ceil_div(V, p.Vc);
    const bool whole = p.copied >= V;   // the points' copy serves both passes
    auto points_of = [&](int64_t v0, int32_t n, bool again) {
        Operand o{};
        o.rows = n, o.ld = x->points_stride;
        if (p.direct) {
            if constexpr (PARTS == 3) {
                o.f = (const float *)x->points + v0 * x->points_stride, o.cols = d;
                o.vec = d % 4 == 0 && x->points_stride % 4 == 0 && aligned(x->points, 16);
            } else {
                o.p = (const bf16_t *)x->points + v0 * x->points_stride, o.cols = p.Kp;
            }
            return o;
        }
        bf16_t *copy = (bf16_t *)(ws + p.off_c) + (whole ? v0 * p.Kp : 0);
        o.p = copy, o.ld = o.cols = p.Kp;
        if (!(whole && again)) {
            PartsArgs a{};
            a.src = (const T *)x->points + v0 * x->points_stride, a.stride = x->points_stride;
            a.R = a.rows_pad = n, a.C = d, a.plain_ld = p.Kp, a.plain_part = c_part, a.plain = copy;
            parts_kernel<T><<<dim3((uint32_t)parts_blocks(a)), 256, 0, st>>>(a);
        }
        return o;
    };

    // losses: all points at once where they are read in place, else by pieces
    {
        const int32_t step = p.direct || whole ? V : (int32_t)p.Vc;
        int32_t used = 0;
        for (int64_t v0 = 0; v0 < V; v0 += step) {
            const int32_t n = (int32_t)std::min<int64_t>(step, V - v0);
            StatsArgs a{};
            a.pr.a = points_of(v0, n, false);
            a.pr.b = Operand{hp, p.Kp, p.rows_pad, p.Kp};
            a.pr.K = p.Kp;
            a.pr.part_a = c_part, a.pr.part_b = h_part;
            a.bias = x->bias ? x->bias + v0 : nullptr;
            a.scale2 = x->scale * LOG2E;
            a.label = (const int32_t *)(ws + p.off_label), a.pick = (float *)(ws + p.off_pick);
            a.B = B, a.V = n, a.v0 = (int32_t)v0, a.tiles_b = p.tiles_b;
            a.tiles_v = (int32_t)ceil_div(n, 256);
            a.splits = std::min(p.splits, a.tiles_v);
            a.part = (RowState *)(ws + p.off_part) + (int64_t)used * B;
            used += a.splits;
            with_tile(p.tile_b, [&](auto bn) {
                using S = typename Pick<256, decltype(bn)::value, PARTS>::S;
                run(stats_kernel<S>, split_grid(a.splits, a.tiles_b), S::THREADS, stage_bytes<S>(), st, a);
            });
        }
        w.rows(used);
    }
    if (!grad || !(x->dh || x->dpoints || x->dbias)) return launch_status("softmax_xent");

    const int32_t *label = (const int32_t *)(ws + p.off_label);
    const float *coef = (const float *)(ws + p.off_coef);
    const OwnArgs oa = w.own();
    const int32_t *first = oa.first;
    const float *own = oa.own, *own_bias = oa.own_bias;
    if (w.want_c()) w.own_terms(oa);
    const int64_t p_part = (int64_t)p.rows_pad * p.cols_pad;
    for (int32_t i = 0; i < pieces; ++i) {
        const int32_t v0 = (int32_t)(i * p.Vc), n = (int32_t)std::min<int64_t>(p.Vc, V - v0);
        const int32_t tiles_v = (int32_t)ceil_div(n, 256);
        ProbArgs a{};
        a.pr.a = Operand{hp, p.Kp, p.rows_pad, p.Kp};
        a.pr.b = points_of(v0, n, true);
        a.pr.K = p.Kp;
        a.pr.part_a = h_part, a.pr.part_b = c_part;
        a.bias = x->bias ? x->bias + v0 : nullptr;
        a.top = (const float *)(ws + p.off_top), a.rowf = (const float *)(ws + p.off_rowf), a.label = label;
        a.p = x->dh || x->dpoints ? (bf16_t *)(ws + p.off_p) : nullptr;
        a.col = x->dbias ? (float *)(ws + p.off_col) : nullptr;
        a.scale2 = x->scale * LOG2E;
        a.B = B, a.V = V, a.v0 = v0, a.n = n, a.cols_pad = (int32_t)p.cols_pad, a.rows_pad = p.rows_pad;
        a.tiles_b = p.tiles_b, a.tiles_v = tiles_v;
        with_tile(p.tile_b, [&](auto bm) {
            using S = typename Pick<decltype(bm)::value, 256, PARTS>::S;
            const size_t lds = std::max(stage_bytes<S>(), sizeof(bf16_t) * (size_t)S::BM * (S::BN + 8));
            run(prob_kernel<S>, split_grid(tiles_v, p.tiles_b), S::THREADS, lds, st, a);
        });
        if (x->dbias)
            dbias_kernel<<<dim3((uint32_t)ceil_div(n, 256)), 256, 0, st>>>(a.col, p.tiles_b, (int32_t)p.cols_pad, n, v0, first,
                                                                          own_bias, factor, x->dbias + v0);
        if (x->dh) {
            DhArgs g{};
            g.pr.a = Operand{a.p, p.cols_pad, p.rows_pad, (int32_t)p.cols_pad};
            g.pr.b = a.pr.b;
            g.pr.K = tiles_v * 256;
            g.pr.part_a = p_part, g.pr.part_b = c_part;
            g.part = (float *)(ws + p.off_dh);
            g.d = d, g.ld = p.Kp, g.rows_pad = p.rows_pad, g.tiles_b = p.tiles_b, g.splits = p.dh_splits, g.k_split = p.dh_k, g.first = i == 0;
            g.tiles_d = p.tiles_d;
            with_tile(p.tile_b, [&](auto bm) {
                constexpr int BM = decltype(bm)::value;
                const uint32_t grid = split_grid(g.splits, g.tiles_b * g.tiles_d);
                if (p.tile_d == 128) {
                    using S = typename Pick<BM, 128, PARTS>::S;
                    run(dh_kernel<S>, grid, S::THREADS, stage_bytes<S>(), st, g);
                } else {
                    using S = typename Pick<BM, 256, PARTS>::S;
                    run(dh_kernel<S>, grid, S::THREADS, stage_bytes<S>(), st, g);
                }
            });
        }
        if (x->dpoints) {
            DcArgs g{};
            g.pr.a = Operand{a.p, p.cols_pad, p.rows_pad, (int32_t)p.cols_pad};
            g.pr.b = Operand{hz, p.Kp, p.rows_pad, p.Kp};
            g.pr.K = p.rows_pad;
            g.pr.part_a = p_part, g.pr.part_b = h_part;
            g.out = (T *)x->dpoints + (int64_t)v0 * d;
            g.first = first, g.own = own, g.factor = factor, g.scale = x->scale;
            // tiles of 256 x 128, two blocks a CU: one writes its rows while the
            // other multiplies (256 x 256: 285 us in place of 267 at 2,000 queries)
            g.n = n, g.d = d, g.v0 = v0, g.tiles_v = tiles_v, g.tiles_d = (int32_t)ceil_div(d, 128);
            using S = typename Pick<256, 128, PARTS>::S;
            run(dc_kernel<S, T>, split_grid(tiles_v, g.tiles_d), S::THREADS, stage_bytes<S>(), st, g);
        }
    }
    if (x->dh)
        dh_join_kernel<T><<<dim3((uint32_t)ceil_div((int64_t)B * (p.Kp / 4), 256)), 256, 0, st>>>(
            (const float *)(ws + p.off_dh), p.dh_splits, p.rows_pad, B, d, p.Kp, (const T *)x->points, x->points_stride, label,
            coef, factor, x->scale, (T *)x->dh);
    return launch_status("softmax_xent_grad");
}

template <class T>
__global__ __launch_bounds__(256) void zero_kernel(T *p, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = (T)0.0f;
}

template <class T>
void zero(T *p, int64_t n, hipStream_t st)
{
    if (p && n) zero_kernel<<<dim3((uint32_t)std::min<int64_t>(4096, ceil_div(n, 256))), 256, 0, st>>>(p, n);
}

int xent(const boa_xent *x, bool grad, void *ws, int64_t ws_bytes, void *stream)
{
    if (int rc = check(x, grad)) return rc;
    auto bad = [](const char *why) { return set_error(BOA_EINVAL, why); };
    if (!x->points || (x->B && (!x->h || !x->labels))) return bad("softmax_xent: NULL input");
    if (!x->loss && (x->B || x->reduction != BOA_REDUCE_NONE)) return bad("softmax_xent: NULL loss");
    hipStream_t st = (hipStream_t)stream;
    if (x->B == 0) {   // nothing to learn from: a loss of 0, gradients of 0
        if (x->reduction != BOA_REDUCE_NONE) zero(x->loss, 1, st);
        if (grad) {
            if (x->dtype == BOA_T_F32) zero((float *)x->dpoints, x->V * x->d, st);
            else zero((bf16_t *)x->dpoints, x->V * x->d, st);
            zero(x->dbias, x->V, st);
        }
        return launch_status("softmax_xent");
    }
    if (!ws || !aligned(ws, 16) || ws_bytes < make_plan(x, grad).total)
        return bad("softmax_xent: workspace missing, unaligned or too small");
    if (x->dtype == BOA_T_F32) {
        const Work<float> w{x, grad, make_plan(x, grad), (uint8_t *)ws, st};
        return w.p.sweep ? run_sweeps(w) : run_tiles(w);
    }
    const Work<bf16_t> w{x, grad, make_plan(x, grad), (uint8_t *)ws, st};
    return w.p.sweep ? run_sweeps(w) : run_tiles(w);
}

}  // namespace

extern "C" {

int64_t boa_softmax_xent_workspace(const boa_xent *x, int32_t grad)
{
    if (int rc = check(x, grad != 0)) return rc;
    return x->B ? make_plan(x, grad != 0).total : 0;
}

int boa_softmax_xent(const boa_xent *x, void *workspace, int64_t workspace_bytes, void *stream)
{
    return xent(x, false, workspace, workspace_bytes, stream);
}

int boa_softmax_xent_grad(const boa_xent *x, void *workspace, int64_t workspace_bytes, void *stream)
{
    return xent(x, true, workspace, workspace_bytes, stream);
}

}  // extern "C"
