// Matrix products of the query tower's layers on the 16-bit matrix
// instructions: out[p][q] = sum_k a(p, k) b(q, k), float32 sums.
//
// An operand's rows run along k, or "across": a row is then one k and runs
// along the operand's own dimension. A linear layer's forward product has both
// along k, its input's gradient the weights across, its weights' gradient both.
// Float32 operands come as two f16 parts, a = a0 + a1, and the products of parts
// above 2^-22 of the result are added: a1 b0 + a0 b1 + a0 b0.
#pragma once

#include <algorithm>

#include "boa_ops.h"

namespace boa {

typedef bf16_t bf16x8 __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x4 __attribute__((ext_vector_type(4)));
typedef f16_t f16x8 __attribute__((ext_vector_type(8)));
typedef f16_t f16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));

template <class T>
struct Vec;
template <>
struct Vec<bf16_t> {
    typedef bf16x8 v8;
    typedef bf16x4 v4;
};
template <>
struct Vec<f16_t> {
    typedef f16x8 v8;
    typedef f16x4 v4;
};

__device__ inline f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x16 mfma32(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ inline f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// One operand: rows `ld` values apart from a 16-byte aligned address, ld a
// multiple of 8 and below 2^21, whole 16-byte chunks in every row. Of parts, the
// second lies `part` values behind the first, and 32 values of k lie `block`
// values from the next 32 (along k: 32 where the parts are two matrices, 64 where
// they alternate). own: the operand's extent in the output. batch: from one
// product of a batch to the next.
struct Operand {
    const void *p;
    int64_t ld, part, block, batch;
    int32_t own;
};

struct Product {
    Operand a, b;
    int32_t K;
    int32_t tiles_a, tiles_b, splits, batches;
    int32_t steps;     // stages of k a split takes
    int32_t symmetric; // the output is: tiles with ta <= tb only
    uint32_t first;    // work item of this launch's first block
};

// A block's tile: WA x WB waves of TA x TB tiles of 32 x 32, 64 values of k a
// stage; GROUPS such sets of waves, which share k and add their sums at the end;
// PER_CU blocks of it at once on a CU.
template <class T_, int WA_, int WB_, int TA_, int TB_, int GROUPS_, int STAGES_, int PER_CU_>
struct Tile {
    typedef T_ T;
    static constexpr int WA = WA_, WB = WB_, TA = TA_, TB = TB_, BK = 64, GROUPS = GROUPS_, STAGES = STAGES_, PER_CU = PER_CU_;
    static constexpr int BA = WA * TA * 32, BB = WB * TB * 32, SET = 64 * WA * WB, THREADS = SET * GROUPS;
    static constexpr int WAVES_PER_SIMD = PER_CU * THREADS / 256;
    static_assert(STAGES >= 2, "a stage is read while the next one arrives");
    static constexpr int STAGE = (BA + BB) * BK;   // values
    // columns that a wave turns over at a time at the end, and what that takes
    static constexpr int TURN_COLS = TB % 2 ? 32 : 64, TURN_BYTES = TA * 32 * (TURN_COLS + 4) * 4;
    static constexpr int ROOM = GROUPS * STAGES * STAGE * 2;
    static constexpr int LDS = ROOM > WA * WB * TURN_BYTES ? ROOM : WA * WB * TURN_BYTES;
    static_assert((GROUPS - 1) * BA * BB * 4 <= LDS && LDS * PER_CU <= 160 << 10, "LDS");
};

constexpr uint32_t NOWHERE = 0x80000000u;   // an offset past every buffer: such loads give zeros

// A buffer of 2^31 - 1 bytes from an address that all lanes share.
__device__ inline words4 buffer_at(const void *p)
{
    const uint64_t a = (uint64_t)p;
    words4 r;
    r[0] = __builtin_amdgcn_readfirstlane((uint32_t)a);
    r[1] = __builtin_amdgcn_readfirstlane((uint32_t)(a >> 32));
    r[2] = 0x7FFFFFFFu;
    r[3] = 0x00027000u;
    return r;
}

template <class T>
__device__ inline uint32_t lds_address(const T *p)
{
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const T *)p;
}

// 16 bytes a lane from the buffer to LDS, lane after lane from `to`; an offset
// past the buffer's end gives zeros. Written out because the compiler waits for
// all such loads that it knows of before any transposed read; here the kernel's
// own waits count them.
__device__ inline void load_to_lds(words4 buffer, uint32_t offset, uint32_t to)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(buffer)
                 : "memory");
}

// One operand's side of a stage: where this thread's loads come from, and where
// its fragments lie. A stage is 64 values of k, or 32 of the first part and the
// same 32 of the second behind them.
//
// Along k, a stage holds ROWS rows of 64 values whose 16-byte chunks are stored
// in the order chunk ^ (row / 2 & 7): the same chunk of any 16 rows that follow
// each other lies in all banks; across, 64 rows of ROWS values in the order
// chunk ^ (row & 3) * 4, and fragments are read transposed, 64 bytes of four
// rows by half a wave. Either way what lanes read together spreads over the
// banks. The permutation is applied to the addresses loaded from, since a load
// to LDS writes its lanes in order. Rows past the operand's end and k past K are
// loaded as zeros (an offset that the buffer's bounds check refuses).
template <class S, int ROWS, bool ACROSS, bool PARTS>
struct Side {
    typedef typename S::T T;
    static constexpr int CHUNKS = ACROSS ? ROWS / 8 : S::BK / 8;   // of an LDS row
    static constexpr int N = ROWS * (S::BK / 8) / S::SET;         // loads of a stage
    static constexpr int PER = S::SET / CHUNKS;                   // LDS rows of one load of a set of waves
    static_assert(N * S::SET == ROWS * (S::BK / 8) && PER * CHUNKS == S::SET, "whole loads");
    static_assert(ACROSS ? PER % 4 == 0 || N == 1 : PER % 8 == 0, "across, one permutation for all of a thread's loads");
    uint32_t at[N];   // byte offsets from the stage's base
    int32_t k;        // place of load 0

    __device__ static int swap(int row) { return ACROSS ? (ROWS >= 128 ? (row & 3) * 4 : (row & 1) * 4) : (row >> 1) & 7; }

    __device__ Side(const Operand &o, int32_t own0)
    {
        const int t = threadIdx.x % S::SET, row = t / CHUNKS, chunk = t % CHUNKS ^ swap(t / CHUNKS);
        if constexpr (ACROSS) {
            k = row;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t from = (uint32_t)k_of(i) * (uint32_t)o.ld * 2 + (second(i) ? (uint32_t)o.part * 2 : 0);
                at[i] = own0 + chunk * 8 < o.own ? from + chunk * 16 : NOWHERE;
            }
        } else {
            k = chunk * 8;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const uint32_t from = (uint32_t)(row + i * PER) * (uint32_t)o.ld * 2 + (second(i) ? (uint32_t)o.part * 2 : 0);
                at[i] = own0 + row + i * PER < o.own ? from + k_of(i) * 2 : NOWHERE;
            }
        }
    }
    // the place of load i among a stage's 64 rows or values, its k, and whether it is of the second part
    __device__ int place(int i) const { return ACROSS ? k + i * PER : k ^ (i * PER / 2 & 7) * 8; }
    __device__ int k_of(int i) const { return PARTS ? place(i) & 31 : place(i); }
    __device__ bool second(int i) const { return PARTS && place(i) >= 32; }
    // loads a stage from `base`, of which the first k_left values of k count
    __device__ void load(T *to, const T *base, int32_t k_left) const
    {
        const words4 rsrc = buffer_at(base);
        const uint32_t lds = lds_address(to) + (threadIdx.x % S::SET >> 6) * 1024;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t off = k_of(i) < k_left ? at[i] : NOWHERE;
            load_to_lds(rsrc, off, __builtin_amdgcn_readfirstlane(lds + i * S::SET * 16));
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
    // The fragment of the wave's tile i and k step s. `at`: lane_at plus the
    // stage; tiles and steps are exclusive ors on bits that nothing carries into.
    __device__ static typename Vec<T>::v8 fragment(uint32_t at, int i, int s)
    {
        typedef typename Vec<T>::v8 v8;
        typedef typename Vec<T>::v4 v4;
        if constexpr (ACROSS) {
            typedef __attribute__((address_space(3))) short4v Four;
            v8 f;
#pragma unroll
            for (int jj = 0; jj < 2; ++jj) {
                const uint32_t a = (at ^ (i * 64)) + (16 * s + 4 * jj) * ROWS * 2;
                const v4 v = __builtin_bit_cast(v4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((Four *)(uintptr_t)a));
#pragma unroll
                for (int e = 0; e < 4; ++e) f[4 * jj + e] = v[e];
            }
            return f;
        } else {
            typedef __attribute__((address_space(3))) v8 Row;
            return *(const Row *)(uintptr_t)((at ^ (s * 32)) + i * 32 * S::BK * 2);
        }
    }
};

// Waits until at most LEFT of this wave's loads are on their way and its LDS
// reads are done, then for the other waves.
template <int LEFT>
__device__ inline void wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// What a block works on.
struct Place {
    int32_t ta, tb, split, batch;
};

// Tiles a side of a symmetric output's squares.
constexpr uint32_t SQUARE = 4;

// Work items of an output.
__host__ __device__ inline uint32_t tiles_of(const Product &pr)
{
    const uint32_t squares = (pr.tiles_b + SQUARE - 1) / SQUARE;
    return pr.symmetric ? squares * (squares + 1) / 2 * SQUARE * SQUARE : (uint32_t)pr.tiles_a * pr.tiles_b;
}

// Whether a symmetric output's work item is a tile on or above the diagonal.
__device__ inline bool is_needed(const Product &pr, const Place &w) { return !pr.symmetric || (w.ta <= w.tb && w.tb < pr.tiles_b); }

// Work item of block id of n. Blocks go to the 8 XCDs in turn; each XCD takes a run of
// tiles that share operand rows in its L2: bands of 8 tiles of a, one tile of b
// after the other.
__device__ inline Place place_of(const Product &pr, uint32_t id, uint32_t n)
{
    const uint32_t x = id & 7, per = n >> 3, extra = n & 7;
    uint32_t t = pr.first + x * per + min(x, extra) + (id >> 3);
    const uint32_t tiles = tiles_of(pr);
    Place w;
    const uint32_t layer = t / tiles;
    t -= layer * tiles;
    w.batch = layer / pr.splits;
    w.split = layer - w.batch * pr.splits;
    if (pr.symmetric) {   // squares of tiles, which share rows; a square's own diagonal has some that are not needed
        const uint32_t square = t / (SQUARE * SQUARE), within = t - square * (SQUARE * SQUARE);
        uint32_t c = (uint32_t)((sqrtf(8.0f * (float)square + 1.0f) - 1.0f) * 0.5f);
        while (c * (c + 1) / 2 > square) --c;
        while ((c + 1) * (c + 2) / 2 <= square) ++c;
        w.tb = c * SQUARE + within / SQUARE;
        w.ta = (square - c * (c + 1) / 2) * SQUARE + within % SQUARE;
        return w;
    }
    const uint32_t band = t / (8 * pr.tiles_b), first = band * 8, rows = min(8u, pr.tiles_a - first);
    t -= band * 8 * pr.tiles_b;
    w.tb = t / rows;
    w.ta = first + t - w.tb * rows;
    return w;
}

// acc[i][j] += tile i of b times tile j of a: lane (l & 31) holds row j * 32 +
// (l & 31) of a's side, its values e columns i * 32 + 8 (e / 4) + 4 (l / 32) +
// e % 4 of b's side. Fragments are read one step of 16 ahead of the matrix
// instructions. Before the last step of a stage the next one is waited for and
// the waves meet: all fragments of the stage are in registers then, its place
// takes the loads of the stage STAGES further on, and that step's instructions
// cover the meeting and the next stage's first reads. True for the waves that
// have the sums.
template <class S, bool ACROSS_A, bool ACROSS_B, bool PARTS>
__device__ inline bool tile_product(const Product &pr, const Place &w, typename S::T *lds, f32x16 (&acc)[S::TB][S::TA])
{
    typedef typename S::T T;
    constexpr int STAGES = S::STAGES, BK = S::BK;
    using A = Side<S, S::BA, ACROSS_A, PARTS>;
    using B = Side<S, S::BB, ACROSS_B, PARTS>;
    constexpr int DEEP = PARTS ? 32 : BK;   // k of a stage
    const int set = S::GROUPS == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / S::SET);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x % S::SET >> 6), wa = wave % S::WA, wb = wave / S::WA;
    const int32_t a0 = w.ta * S::BA, b0 = w.tb * S::BB;
    const A a(pr.a, a0);
    const B b(pr.b, b0);
    const int32_t all = (pr.K + DEEP - 1) / DEEP;
    const int32_t from = w.split * pr.steps, steps = min(pr.steps, all - from);
    const int32_t each = (steps + S::GROUPS - 1) / S::GROUPS;   // stages of a set of waves
    const int32_t last = from + min(steps, (set + 1) * each);
    const T *pa = (const T *)pr.a.p + w.batch * pr.a.batch + (ACROSS_A ? (int64_t)a0 : a0 * pr.a.ld);
    const T *pb = (const T *)pr.b.p + w.batch * pr.b.batch + (ACROSS_B ? (int64_t)b0 : b0 * pr.b.ld);
    const int64_t next_a = PARTS ? pr.a.block : ACROSS_A ? BK * pr.a.ld : BK, next_b = PARTS ? pr.b.block : ACROSS_B ? BK * pr.b.ld : BK;
    lds += set * STAGES * S::STAGE;
    int32_t at = from + set * each, stage = 0;   // of the next load
    auto load = [&]() {
        const int32_t left = at < last ? pr.K - at * DEEP : 0;   // past the end zeros
        T *to = lds + stage * S::STAGE;
        a.load(to, pa + at * next_a, left);
        b.load(to + S::BA * BK, pb + at * next_b, left);
        if (++stage == STAGES) stage = 0;
        ++at;
    };
    const uint32_t base = lds_address(lds);
    const uint32_t lane_a = A::lane_at(wa * S::TA * 32), lane_b = B::lane_at(wb * S::TB * 32) + S::BA * BK * 2;
    // A step's fragments: of 16 values of k, or of 16 of both parts. Two steps'
    // at a time, but for parts in a tile that has no registers left for that.
    constexpr int P = PARTS ? 2 : 1, STEPS = BK / 16 / P, BUFFERS = PARTS && S::TA * S::TB > 4 ? 1 : 2;
    typename Vec<T>::v8 fa[BUFFERS][P][S::TA], fb[BUFFERS][P][S::TB];
    auto read = [&](int to, int32_t slot, int s) {
        const uint32_t at_a = base + slot * S::STAGE * 2 + lane_a, at_b = base + slot * S::STAGE * 2 + lane_b;
#pragma unroll
        for (int q = 0; q < P; ++q) {
#pragma unroll
            for (int j = 0; j < S::TA; ++j) fa[to][q][j] = A::fragment(at_a, j, s + q * STEPS);
#pragma unroll
            for (int i = 0; i < S::TB; ++i) fb[to][q][i] = B::fragment(at_b, i, s + q * STEPS);
        }
    };
    auto multiply = [&](int from_buffer) {
        const auto &u = fa[from_buffer];
        const auto &v = fb[from_buffer];
#pragma unroll
        for (int q = P == 2 ? 0 : 2; q < 3; ++q)
#pragma unroll
            for (int i = 0; i < S::TB; ++i)
#pragma unroll
                for (int j = 0; j < S::TA; ++j) acc[i][j] = mfma32(v[q == 1 ? P - 1 : 0][i], u[q == 0 ? P - 1 : 0][j], acc[i][j]);
    };
    constexpr int LOADS = A::N + B::N;
    for (int i = 0; i < STAGES; ++i) load();
    wait_and_meet<(STAGES - 1) * LOADS>();
    int32_t cur = 0;
    if (BUFFERS == 2) read(0, 0, 0);
    for (int32_t it = 0; it < each; ++it) {
        const int32_t next = cur + 1 == STAGES ? 0 : cur + 1;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            if (BUFFERS == 1) read(0, cur, s);
            if (s + 1 < STEPS) {
                if (BUFFERS == 2) read((s + 1) & 1, cur, s + 1);
            } else {
                wait_and_meet<(STAGES - 2) * LOADS>();
                load();
                if (BUFFERS == 2) read(0, next, 0);
            }
            // else the reads would be gathered before the instructions that use them (4096^3: 1,010 in place of 1,170 TFLOP/s);
            // transposed ones are as well off without (1,220 and 1,170)
            if constexpr (!ACROSS_A && !ACROSS_B) __builtin_amdgcn_sched_barrier(0);
            multiply(s & (BUFFERS - 1));
        }
        cur = next;
    }
    wait_and_meet<0>();
    if constexpr (S::GROUPS > 1) {   // the first set adds the others' sums, in their order
        f32x4 *sums = (f32x4 *)(lds - set * STAGES * S::STAGE);
        constexpr int PIECES = S::TA * S::TB * 4;
        const int t = threadIdx.x % S::SET;
        if (set) {
#pragma unroll
            for (int i = 0; i < S::TB; ++i)
#pragma unroll
                for (int j = 0; j < S::TA; ++j)
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x16 &v = acc[i][j];
                        sums[((set - 1) * PIECES + (i * S::TA + j) * 4 + g) * S::SET + t] =
                            f32x4{v[4 * g], v[4 * g + 1], v[4 * g + 2], v[4 * g + 3]};
                    }
        }
        __syncthreads();
        if (!set)
            for (int s = 0; s < S::GROUPS - 1; ++s)
#pragma unroll
                for (int i = 0; i < S::TB; ++i)
#pragma unroll
                    for (int j = 0; j < S::TA; ++j)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const f32x4 v = sums[(s * PIECES + (i * S::TA + j) * 4 + g) * S::SET + t];
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][j][4 * g + e] += v[e];
                        }
        __syncthreads();
    }
    return set == 0;
}

template <class S>
__device__ inline void clear(f32x16 (&acc)[S::TB][S::TA])
{
#pragma unroll
    for (int i = 0; i < S::TB; ++i)
#pragma unroll
        for (int j = 0; j < S::TA; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
}

// Nothing to keep.
struct Nothing {
    __device__ void down() {}
};

// Hands the sums out in runs of eight neighbouring columns: f(row of a's side,
// first column of b's side, the eight sums in LDS, kept). A lane keeps its columns
// over every `step`th row: kept is what(first row, column, step), asked for once
// (addresses, the columns' bias), and kept.down() takes it a step on. Each wave turns its tiles over in its own piece of LDS, two columns of tiles at
// a time, so that what follows is written once, and stores fill whole lines.
// `turned`: g(first row, column, eight sums down that column) for all of them
// too, for a transposed output. The stages must no longer be in use.
template <class S, class W, class F, class G>
__device__ inline void each_run(const Place &w, const f32x16 (&acc)[S::TB][S::TA], char *lds, W what, F f, bool turned, G g)
{
    constexpr int WIDE = S::TURN_COLS / 32, RUNS = S::TURN_COLS / 8, LD = S::TURN_COLS + 4;   // + 4: rows begin in other banks
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wa = wave % S::WA, wb = wave / S::WA;
    const int lane = threadIdx.x & 63, half = lane >> 5, r = lane & 31;
    float *mine = (float *)lds + wave * (S::TURN_BYTES / 4);
    const int32_t p0 = w.ta * S::BA + wa * S::TA * 32, q0 = w.tb * S::BB + wb * S::TB * 32;
#pragma unroll
    for (int i0 = 0; i0 < S::TB; i0 += WIDE) {
        constexpr int STEP = 64 / RUNS;
        const int32_t col = lane % RUNS * 8, q = q0 + i0 * 32 + col;
        auto kept = what(p0 + lane / RUNS, q, STEP);
#pragma unroll
        for (int i = 0; i < WIDE; ++i)
#pragma unroll
            for (int j = 0; j < S::TA; ++j)
#pragma unroll
                for (int g4 = 0; g4 < 4; ++g4) {
                    const f32x16 &v = acc[i0 + i][j];
                    *(f32x4 *)(mine + (j * 32 + r) * LD + i * 32 + g4 * 8 + half * 4) =
                        f32x4{v[4 * g4], v[4 * g4 + 1], v[4 * g4 + 2], v[4 * g4 + 3]};
                }
        __builtin_amdgcn_wave_barrier();
#pragma unroll 2
        for (int row = lane / RUNS; row < S::TA * 32; row += STEP) {
            f(p0 + row, q, (const float *)(mine + row * LD + col), kept);
            kept.down();
        }
        if (turned)
#pragma unroll 1
            for (int k = lane; k < S::TURN_COLS * S::TA * 4; k += 64) {
                const int run = k % (S::TA * 4), c = k / (S::TA * 4);
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = mine[(run * 8 + e) * LD + c];
                g(p0 + run * 8, q0 + i0 * 32 + c, v);
            }
        __builtin_amdgcn_wave_barrier();
    }
}

template <class S, class W, class F>
__device__ inline void each_run(const Place &w, const f32x16 (&acc)[S::TB][S::TA], char *lds, W what, F f)
{
    each_run<S>(w, acc, lds, what, f, false, [](int32_t, int32_t, const float (&)[8]) {});
}

// ---------------------------------------------------------------------------
// host

// Work memory handed out piece by piece; without a base it only counts.
struct Arena {
    char *base = nullptr;
    int64_t used = 0;
    void *take(int64_t bytes)
    {
        void *p = base ? base + used : nullptr;
        used += ceil_div(bytes, 256) * 256;
        return p;
    }
};

inline int32_t pad8(int64_t n) { return (int32_t)(ceil_div(n, 8) * 8); }

inline uint32_t spread(int64_t items) { return (uint32_t)std::max<int64_t>(1, std::min<int64_t>(ceil_div(items, 256), 1 << 14)); }

// The tiles there are: 256 x 256 for large outputs; 128 x 128, two at once on a
// CU, or one with its loads four stages ahead where a CU gets no second; 64 x 64,
// four at once, or two with two sets of waves, or one of those with its loads
// four stages ahead. A smaller tile reads more of LDS for the same products:
// 1,170, 980 and 630 TFLOP/s where there are tiles enough (k = 4,096); it is taken
// where the larger would leave CUs without one.
template <class T>
using Large = Tile<T, 4, 2, 2, 4, 1, 2, 1>;
template <class T>
using Middle = Tile<T, 2, 2, 2, 2, 1, 2, 2>;
template <class T>
using MiddleAlone = Tile<T, 2, 2, 2, 2, 1, 4, 1>;
template <class T>
using Small = Tile<T, 2, 2, 1, 1, 1, 2, 4>;
template <class T>
using SmallPair = Tile<T, 2, 2, 1, 1, 2, 2, 2>;
template <class T>
using SmallAlone = Tile<T, 2, 2, 1, 1, 2, 4, 1>;

// How a product is cut into blocks.
struct Cut {
    int shape, splits;
    int32_t steps;   // stages of k a split takes
};
constexpr int SMALL = 3;   // Small's shape

// f(first block, blocks) for the launches that a number of blocks takes: one may not have 2^32 threads.
template <class F>
void in_launches(int64_t blocks, int32_t threads, F f)
{
    const int64_t most = ((int64_t)1 << 31) / threads;
    for (int64_t at = 0; at < blocks; at += most) f((uint32_t)at, (uint32_t)std::min(most, blocks - at));
}

// f with the tile of a shape
template <class T, class F>
void with_tile(int shape, F f)
{
    if (shape == 0) f(Large<T>{});
    else if (shape == 1) f(Middle<T>{});
    else if (shape == 2) f(MiddleAlone<T>{});
    else if (shape == SMALL) f(Small<T>{});
    else if (shape == 4) f(SmallPair<T>{});
    else f(SmallAlone<T>{});
}

// The cheapest of the tiles and some numbers of splits by a model of the
// time: rounds of blocks over the GPU's 256 CUs, each as long as its stages
// and a beginning and end; splits also write and read their sums. symmetric:
// only the tiles on one side of the diagonal.
inline Cut choose(int64_t A, int64_t B, int64_t K, bool parts, int64_t batches, bool symmetric, bool may_split)
{
    struct Cost {
        int side, at_once, sets;
        double stage, alone, ends;   // us a stage in a full CU and in a CU of its own, us of beginning and end
    };
    // measured on outputs of 0.5 to 8 tiles a CU and k of 512 to 4,096
    static const Cost costs[6] = {{256, 1, 1, 1.75, 1.40, 9.0}, {128, 2, 1, 0.98, 0.62, 6.5}, {128, 1, 1, 0.68, 0.60, 6.0},
                                  {64, 4, 1, 0.72, 0.36, 4.5}, {64, 2, 2, 0.80, 0.62, 5.0}, {64, 1, 2, 0.55, 0.50, 4.5}};
    static const int counts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
    const int64_t steps = ceil_div(K, parts ? 32 : 64);
    const double longer = parts ? 1.25 : 1.0;   // a stage's time: three products of half its values
    Cut best{0, 1, (int32_t)steps};
    double least = 1e30;
    for (int s = 0; s < 6; ++s)
        for (int n : counts) {
            if (n > 1 && (!may_split || n > steps || (double)n * A * B * 4 > 256e6)) break;
            const Cost &c = costs[s];
            const int64_t each = ceil_div(steps, n), splits = ceil_div(steps, each), turns = ceil_div(each, c.sets);
            const double tiles_a = (double)ceil_div(A, c.side), tiles_b = (double)ceil_div(B, c.side);
            const double blocks = (symmetric ? tiles_a * (tiles_a + 1) / 2 : tiles_a * tiles_b) * splits * batches;
            const double room = 256.0 * c.at_once;
            const double full = (double)(int64_t)(blocks / room), rest = blocks - full * room;
            double t = full * (turns * c.stage * longer + c.ends);
            if (rest > 0)
                t += turns * longer * std::max(c.alone, c.stage * std::min(1.0, (double)ceil_div((int64_t)rest, 256) / c.at_once)) + c.ends;
            if (splits > 1) t += 4.0 + (double)splits * A * B * 8 / 4e6;
            if (t < least) least = t, best = {s, (int)splits, (int32_t)each};
        }
    return best;
}

}  // namespace boa
