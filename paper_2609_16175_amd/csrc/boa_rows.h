// Shared by the kernels that hold a row in registers (boa_norm.hip,
// boa_block.hip): which thread has which columns, sums over a row, the choice of
// a row's registers.
#pragma once

#include "boa_ops.h"

namespace boa {

constexpr int ROW_THREADS = 256;

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

// Two sums at once; red: two values a wave.
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
            red[TPR / 64 + wave] = b;
        }
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int i = 0; i < TPR / 64; ++i) {
            a += red[i];
            b += red[TPR / 64 + i];
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

template <int V>
struct Int {
    static constexpr int value = V;
};

}  // namespace boa
