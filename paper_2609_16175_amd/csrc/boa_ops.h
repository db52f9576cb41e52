// Shared by the query-tower operators (boa_norm.hip, boa_xent.hip,
// boa_matvec.hip): element types, wave reductions, error reporting.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "boa.h"

namespace boa {

// Records the thread's error message for boa_last_error() and returns the code (boa_api.hip).
int set_error(int code, const char *msg);

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

inline int64_t dtype_bytes(int32_t t) { return t == BOA_T_F32 ? 4 : 2; }
// Rows that one launch takes at up to 256 threads a row: a launch may not have
// 2^32 threads. More rows take several launches.
constexpr int64_t LAUNCH_ROWS = (int64_t)1 << 23;

inline bool dtype_known(int32_t t) { return t == BOA_T_F32 || t == BOA_T_BF16 || t == BOA_T_F16; }
inline bool aligned(const void *p, uintptr_t to) { return reinterpret_cast<uintptr_t>(p) % to == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// the error a launch left, as a return code of the C interface
inline int launch_status(const char *what)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return BOA_OK;
    char msg[256];
    __builtin_snprintf(msg, sizeof(msg), "%s: %s", what, hipGetErrorString(e));
    return set_error(BOA_EHIP, msg);
}

template <int N, class T>
struct alignas(N * sizeof(T)) Pack {
    T v[N];
};

template <int N, class T>
__device__ inline void load_f32(float (&to)[N], const T *p)
{
    const Pack<N, T> a = *reinterpret_cast<const Pack<N, T> *>(p);
#pragma unroll
    for (int i = 0; i < N; ++i) to[i] = (float)a.v[i];
}

template <int N, class T>
__device__ inline void store_f32(T *p, const float (&from)[N])
{
    Pack<N, T> a;
#pragma unroll
    for (int i = 0; i < N; ++i) a.v[i] = (T)from[i];
    *reinterpret_cast<Pack<N, T> *>(p) = a;
}

// The same at any element's address: 16-byte loads and stores need no alignment
// above two bytes.
typedef uint32_t words4 __attribute__((ext_vector_type(4)));
typedef words4 loose4 __attribute__((aligned(2)));

template <int N, class T>
__device__ inline void load_loose(float (&to)[N], const T *p)
{
    constexpr int V = 16 / sizeof(T);
    static_assert(N % V == 0, "whole 16-byte loads");
#pragma unroll
    for (int k = 0; k < N; k += V) {
        const words4 w = *reinterpret_cast<const loose4 *>(p + k);
        const Pack<V, T> a = __builtin_bit_cast(Pack<V, T>, w);
#pragma unroll
        for (int i = 0; i < V; ++i) to[k + i] = (float)a.v[i];
    }
}

template <int N, class T>
__device__ inline void store_loose(T *p, const float (&from)[N])
{
    static_assert(N * sizeof(T) == 16, "one 16-byte store");
    Pack<N, T> a;
#pragma unroll
    for (int i = 0; i < N; ++i) a.v[i] = (T)from[i];
    *reinterpret_cast<loose4 *>(p) = __builtin_bit_cast(words4, a);
}

__device__ inline float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

__device__ inline float wave_max(float v)
{
#pragma unroll
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

}  // namespace boa
