// What the translation units of linear attention share (linear_attention.hip: the calls; linear_attention_pass.h: the pass over the rows, compiled for
// each type on its own).  Nothing here is part of the public ABI (see include/bagel.h).
#pragma once

#include <algorithm>

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
//
// A sequence is gone through in segments of `segment` rows (of the last fewer), each by another workgroup, which begins with the memory behind the segment
// before.  The first segments of all sequences have the numbers 0 to sequences - 1.  Segment s >= 1 of sequence i is number
// sequences + offsets[i] / segment + s - 1: that leaves room for those of the sequences before, whatever their lengths.
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
    int64_t step_b, step_c;                          // of a memory's entries, wb times wc in either order; [sequences][states] of them
    int64_t segment;                                 // a multiple of the chunk
    int64_t further;                                 // numbers of segments that are not the first of their sequence
    bool join;                                       // whether a segment joins what those before it have added, which then no launch has done
    float *memories;                                 // [sequences + further][states][..]: behind every segment but the last; null: one segment to a sequence
    int64_t groups, launched;                        // workgroups of all launches, and of those before this one
};

// A grid has fewer than 2^32 threads, and a workgroup up to 512: more workgroups than these go by several launches, each `kernel(workgroups, those before)`.
constexpr int64_t BAGEL_ATTENTION_GROUPS = 1 << 22;
template <typename F> hipError_t bagel_attention_launches(int64_t groups, F &&kernel)
{
    hipError_t e = hipSuccess;
    for (int64_t from = 0; from < groups && e == hipSuccess; from += BAGEL_ATTENTION_GROUPS) {
        kernel((unsigned)std::min(groups - from, BAGEL_ATTENTION_GROUPS), from);
        e = hipGetLastError();
    }
    return e;
}

// The memories behind all segments but the last of their sequences, of one pass or two (with as many sequences, rows, states and segments).
template <typename T> hipError_t bagel_launch_attention_memories(const bagel_attention_pass<T> *p, int n, hipStream_t stream);

// The gradients of keys and values in one pass: `p` is that of the values (memory R, a = key, b = query, c = gradient of the results), `q` that of the
// keys (R transposed, a = value, b = gradient of the results, c = query).  Only where bagel_attention_keys_fit.
template <typename T> hipError_t bagel_launch_attention_keys(const bagel_attention_pass<T> &p, const bagel_attention_pass<T> &q, hipStream_t stream);
// (Two memories of wide heads and the sums over several heads of queries are more than a lane's registers hold, and no other place for the sums has been built; in 32 bits the
// tiles of 64 leave room for one workgroup only, those of 128 for none.)
template <typename T> inline bool bagel_attention_keys_fit(int key_width, int value_width, int heads_to_a_memory)
{
    return sizeof(T) == 2 && (key_width <= 64) == (value_width <= 64) && (key_width <= 64 || heads_to_a_memory == 1);
}

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
