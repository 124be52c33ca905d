// Rows of activations that are held in registers while something is summed over them (block_join.hip, layer_norm.hip).
// Nothing here is part of the public ABI (see include/bagel.h).
#pragma once

#include "activations.h"

namespace {

// Sums of N values over the WAVES waves that share a row, in a fixed order.  Two buffers take turns (`turn`), so that one barrier is enough: a
// wave that is ahead writes the other one, and cannot come back to this one before all have read it.
template <int WAVES, int N, int LANES = 64> __device__ __forceinline__ void row_sum(float (&v)[N], float (*shared)[WAVES][4], int &turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = LANES == 8 ? bagel_sum_of_8(v[i]) : LANES == 16 ? bagel_sum_of_16(v[i]) : bagel_wave_sum(v[i]);
    if constexpr (WAVES > 1) {
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < N; ++i) shared[turn][wave][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = 0.0f;
#pragma unroll
            for (int k = 0; k < WAVES; ++k) v[i] += shared[turn][k][i];
        }
        turn ^= 1;
    }
}

// A row is held in registers by WAVES waves, K packs of V entries a lane: entry V (64 WAVES k + lane) + i, or (LANES = 16, 8) by a quarter or an eighth of a wave.  One
// wave or less to a row leaves several rows to a workgroup, which need nothing of each other.  Packs need not be aligned.  One that would reach over the end
// of the row is moved back to end there: its first entries are another pack's, and count as zero here.
template <int V, int K, int WAVES, int LANES = 64> struct tile {
    static_assert(LANES == 64 || ((LANES == 16 || LANES == 8) && WAVES == 1), "a row has whole waves, or 16 lanes or 8 of one");
    static constexpr int threads = WAVES == 1 ? 256 : 64 * WAVES, lanes = LANES * WAVES, rows = WAVES == 1 ? 256 / LANES : 1;
    __device__ static __forceinline__ int place(int k) { return V * (lanes * k + (int)threadIdx.x % lanes); }
    __device__ static __forceinline__ bool here(int k, int width) { return place(k) < width; }
    __device__ static __forceinline__ int column(int k, int width) { return min(place(k), width - V); }
    __device__ static __forceinline__ int twice(int k, int width) { return max(place(k) + V - width, 0); }    // entries that are another pack's
    __device__ static __forceinline__ int64_t first_row() { return WAVES == 1 ? (int64_t)blockIdx.x * rows + threadIdx.x / LANES : blockIdx.x; }
    __device__ static __forceinline__ int64_t next_row() { return (int64_t)gridDim.x * rows; }
    // vectors of the row's width, ones where there is none
    __device__ static __forceinline__ void vector(const float *p, int width, float (&v)[K][V])
    {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = p && here(k, width) ? p[column(k, width) + i] : 1.0f;
    }
    __device__ static __forceinline__ void product(const float *p, const float *q, int width, float (&v)[K][V])
    {
        float w[K][V];
        vector(p, width, v);
        vector(q, width, w);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] *= w[k][i];
    }
    // a row on its way, and what it is
    template <typename T> struct packed {
        bagel_pack<T, V> x[K];
        __device__ __forceinline__ void load(const bagel_rows<T> &m, int64_t r, int width)
        {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (m.data && here(k, width)) x[k] = reinterpret_cast<const bagel_loose_pack<T, V> *>(m.row(r) + column(k, width))->x;
                else x[k] = (bagel_pack<T, V>)(T)0.0f;
            }
        }
        __device__ __forceinline__ void arrived(int width)
        {
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (V > 1 && here(k, width) && twice(k, width))
#pragma unroll
                    for (int i = 0; i < V - 1; ++i) x[k][i] = i < twice(k, width) ? (T)0.0f : x[k][i];
        }
        __device__ __forceinline__ float operator()(int k, int i) const { return (float)x[k][i]; }
        // From here on the packs are what they are and not what they were converted to, which would be twice the registers.
        __device__ __forceinline__ void keep()
        {
            if constexpr (sizeof(T) == 2 && V > 1) {
                using words = uint32_t __attribute__((ext_vector_type(V / 2)));
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    words w = __builtin_bit_cast(words, x[k]);
                    asm volatile("" : "+v"(w));
                    x[k] = __builtin_bit_cast(bagel_pack<T, V>, w);
                }
            }
        }
    };
    template <typename T> __device__ static __forceinline__ void store(T *row, int width, int k, const float (&v)[V])
    {
        if (!here(k, width)) return;
        T *to = row + column(k, width);
        bagel_pack<T, V> x;
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (T)v[i];
        if (V == 1 || !twice(k, width)) reinterpret_cast<bagel_loose_pack<T, V> *>(to)->x = x;
        else
#pragma unroll
            for (int i = 1; i < V; ++i)
                if (i >= twice(k, width)) to[i] = x[i];
    }
    template <typename T> __device__ static __forceinline__ void store(T *row, int width, const float (&v)[K][V])
    {
#pragma unroll
        for (int k = 0; k < K; ++k) store(row, width, k, v[k]);
    }
};

}  // namespace
