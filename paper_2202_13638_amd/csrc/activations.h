// What the operators of a policy with memory share: activations in three types, their checks on the host, and small device functions.
// Nothing here is part of the public ABI (see include/bagel.h).
#pragma once

#include <math.h>

#include "bagel_internal.h"

// Sets the message of bagel_last_error(NULL) on this thread and returns `code` (bagel_api.hip).
int bagel_refuse(int code, const char *format, ...) __attribute__((format(printf, 2, 3)));

inline int bagel_type_bytes(int dtype) { return dtype == BAGEL_FLOAT32 ? 4 : 2; }
inline bool bagel_type_ok(int dtype) { return dtype == BAGEL_FLOAT32 || dtype == BAGEL_BFLOAT16 || dtype == BAGEL_FLOAT16; }

// Whether a matrix that is there can be addressed: its start at a multiple of its type, and rows that do not overlap.
inline bool bagel_matrix_ok(const bagel_matrix &m, int64_t rows, int64_t width, int dtype)
{
    return !m.data || (((uintptr_t)m.data & (bagel_type_bytes(dtype) - 1)) == 0 && (rows <= 1 || (m.stride >= width && m.stride < (1ll << 40))));
}

// Launches f<type>() for the type that `dtype` says.
template <typename T> struct bagel_type { using type = T; };
template <typename F> hipError_t bagel_by_type(int dtype, F &&f)
{
    if (dtype == BAGEL_FLOAT32) return f(bagel_type<float>());
    if (dtype == BAGEL_BFLOAT16) return f(bagel_type<__bf16>());
    return f(bagel_type<_Float16>());
}

template <typename T> struct bagel_rows {
    T *data;
    int64_t stride;
    __device__ __forceinline__ T *row(int64_t r) const { return data + r * stride; }
};
template <typename T> inline bagel_rows<T> bagel_rows_of(const bagel_matrix &m) { return {(T *)m.data, m.stride}; }

// V entries of a row, one load or store of up to 16 bytes.
template <typename T, int V> using bagel_pack = T __attribute__((ext_vector_type(V)));

// one at any place of its type (the loads and stores of the hardware need no more)
template <typename T, int V> struct __attribute__((packed, aligned(sizeof(T)))) bagel_loose_pack {
    bagel_pack<T, V> x;
};

template <typename T, int V> __device__ __forceinline__ void bagel_load(const T *p, float (&v)[V])
{
    const bagel_pack<T, V> x = reinterpret_cast<const bagel_loose_pack<T, V> *>(p)->x;
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (float)x[i];
}

template <typename T, int V> __device__ __forceinline__ void bagel_store(T *p, const float (&v)[V])
{
    bagel_pack<T, V> x;
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (T)v[i];
    reinterpret_cast<bagel_loose_pack<T, V> *>(p)->x = x;
}

// Data-parallel moves within 16 lanes: 0xB1 swaps neighbours, 0x4E pairs, 0x141 mirrors 8 lanes, 0x140 all 16.
template <int MOVE> __device__ __forceinline__ float bagel_moved(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), MOVE, 0xF, 0xF, false));
}

// The sum over 8 lanes, the same in all of them.
__device__ __forceinline__ float bagel_sum_of_8(float v)
{
    v += bagel_moved<0xB1>(v);
    v += bagel_moved<0x4E>(v);
    return v + bagel_moved<0x141>(v);
}

// The sum over 16 lanes, the same in all of them.
__device__ __forceinline__ float bagel_sum_of_16(float v)
{
    v += bagel_moved<0xB1>(v);
    v += bagel_moved<0x4E>(v);
    v += bagel_moved<0x141>(v);
    v += bagel_moved<0x140>(v);
    return v;
}

// and over the 64 lanes of a wave.
__device__ __forceinline__ float bagel_wave_sum(float v)
{
    const int i = __float_as_int(bagel_sum_of_16(v));
    return (__int_as_float(__builtin_amdgcn_readlane(i, 0)) + __int_as_float(__builtin_amdgcn_readlane(i, 16))) +
           (__int_as_float(__builtin_amdgcn_readlane(i, 32)) + __int_as_float(__builtin_amdgcn_readlane(i, 48)));
}
