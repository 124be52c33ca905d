// What the translation units of linear attention share (linear_attention.hip: the calls; linear_attention_pass.h: the pass over the rows, compiled for
// each type on its own).  Nothing here is part of the public ABI (see include/bagel.h).
#pragma once

#include "activations.h"

template <typename T> struct bagel_heads_of {
    T *data;
    int64_t stride, head;
    __device__ __forceinline__ T *at(int64_t row, int h) const { return data + row * stride + h * head; }
};
template <typename T> inline bagel_heads_of<T> bagel_heads_from(const bagel_heads &h) { return {(T *)h.data, h.stride, h.head}; }

constexpr int BAGEL_ATTENTION_CHUNK = 64;            // rows that are gone through at a time

// One linear attention: memory = decay memory + scale_b b c^T, out = scale memory^T a.  a and out have `qs` heads to a memory, b and c `ks`, of which
// one or both are 1.  `back`: from a sequence's last row to its first, and the memory is multiplied by its decay behind a row, not before.
// A sequence is gone through in segments of `segment` rows (of the last fewer), each by another workgroup.  Segment s of sequence i is number
// offsets[i] / segment + i + s: that leaves room for all segments of the sequences before, whatever their lengths.
template <typename T> struct bagel_attention_pass {
    int64_t rows;
    int sequences, each, states, qs, ks, wb, wc;     // each: rows of a sequence where there are no offsets; wb: width of a and b, wc: of c and out
    bool back;
    float scale, scale_b;
    const int32_t *offsets;
    const float *log_decay;
    bagel_heads_of<T> a, b, c, out;
    const float *first;                              // memories before the first row (gone through), null: zero
    float *last;                                     // and behind the last, null: not wanted
    int64_t step_b, step_c;                          // of their entries: [sequences][states] times wb, wc in either order
    int64_t segment;                                 // a multiple of the chunk
    int64_t slots;                                   // numbers of segments; 1 for each sequence where `segment` holds any of them
    float *memories;                                 // [slots][states][wb][wc]: behind every segment; null: one segment to a sequence
};

// Zeros in the results' rows behind the last sequence, by workgroup number `group` of `groups`.
template <typename T> __device__ __forceinline__ void bagel_clear_behind(const bagel_attention_pass<T> &p, int64_t group, int64_t groups)
{
    const int64_t end = min(max((int64_t)p.offsets[p.sequences], (int64_t)0), p.rows), each = (int64_t)p.states * p.qs * p.wc, n = (p.rows - end) * each;
    for (int64_t i = group * blockDim.x + threadIdx.x; i < n; i += groups * blockDim.x) {
        const int64_t r = i / each;
        const int j = (int)(i - r * each);
        p.out.at(end + r, j / p.wc)[j % p.wc] = (T)0.0f;
    }
}

// (wb and wc are 16 bytes at least)
template <typename T> hipError_t bagel_launch_attention_pass(const bagel_attention_pass<T> &p, hipStream_t stream);
