// The pass of linear attention over the rows (bagel_attention_pass in linear_attention.h), with the matrix instructions of one type.
//
// A chunk of 64 rows, with l the decay, S the memory before it and m, n rows of it in the order they are gone through:
//   out_m = scale (l^(m+1) S^T a_m + sum_{n<=m} P_mn c_n),   P_mn = scale_b l^(m-n) a_m.b_n
//   S <- l^64 S + sum_n scale_b l^(63-n) b_n c_n^T                     (back: l^m S^T a_m, and l^(64-n))
// No power of l is negative, so nothing grows that the definition does not let grow.
#pragma once

#include "linear_attention.h"

namespace {

constexpr int CHUNK = BAGEL_ATTENTION_CHUNK;
constexpr int WAVES = 4, THREADS = 64 * WAVES;

using floats = float __attribute__((ext_vector_type(4)));

// Operands of a product over 32: index lane % 16 of the result, and of the 32, with g = lane / 16, 4 g + j in entries 0 to 3 and 16 + 4 g + j in 4 to 7.
// A result has index lane % 16 of its second operand and 4 g + j of its first one: two results are an operand as they are.
template <typename T> using operand = T __attribute__((ext_vector_type(8)));

__device__ __forceinline__ floats product(operand<__bf16> x, operand<__bf16> y, floats z) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ floats product(operand<_Float16> x, operand<_Float16> y, floats z) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ floats product(operand<float> x, operand<float> y, floats z)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) z = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], z, 0, 0, 0);
    return z;
}

// 64 rows in shared memory.  The 16 bytes between them bring the same column of neighbouring rows to other banks.
template <typename T, int W> struct tile {
    static constexpr int pitch = W + 16 / sizeof(T);
    T x[CHUNK * pitch];
    // operand with a row's entries 32 t on
    __device__ __forceinline__ operand<T> along(int row, int t) const
    {
        using half = T __attribute__((ext_vector_type(4)));
        const T *p = x + row * pitch + 32 * t + 4 * ((threadIdx.x & 63) >> 4);
        const half lo = *reinterpret_cast<const half *>(p), hi = *reinterpret_cast<const half *>(p + 16);
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    // operand with the rows 32 t on of columns `column` to `column` + 15
    __device__ __forceinline__ operand<T> across(int t, int column) const
    {
        const int g = (threadIdx.x & 63) >> 4, j = threadIdx.x & 15;
        if constexpr (sizeof(T) == 2) {
            // a group of 16 lanes reads 4 rows of 16 columns, and each lane gets one of them
            using half = short __attribute__((ext_vector_type(4)));
            using shared_half = __attribute__((address_space(3))) half;
            const T *p = x + (32 * t + 4 * g + j / 4) * pitch + column + 4 * (j % 4);
            const half lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared_half *)p);
            const half hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared_half *)(p + 16 * pitch));
            return __builtin_bit_cast(operand<T>, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            operand<T> r;
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = x[(32 * t + 4 * g + (i & 3) + 4 * (i & 4)) * pitch + column + j];
            return r;
        }
    }
};

// A tile on its way from memory: rows m < n are base + step m, what is not there is zero.
template <typename T, int W> struct incoming {
    static constexpr int V = 16 / sizeof(T), packs = CHUNK * W / V / THREADS;
    bagel_pack<T, V> x[packs];
    __device__ __forceinline__ void load(const bagel_heads_of<T> &h, int head, int64_t base, int step, int n, int width)
    {
#pragma unroll
        for (int k = 0; k < packs; ++k) {
            const int i = threadIdx.x + THREADS * k, m = i / (W / V), column = i % (W / V) * V;
            x[k] = (bagel_pack<T, V>)(T)0.0f;
            if (m >= n || column >= width) continue;
            const T *p = h.at(base + step * m, head) + column;
            if (column + V <= width) x[k] = reinterpret_cast<const bagel_loose_pack<T, V> *>(p)->x;
            else
#pragma unroll
                for (int j = 0; j < V - 1; ++j)
                    if (column + j < width) x[k][j] = p[j];
        }
    }
    __device__ __forceinline__ void put(tile<T, W> &to) const
    {
#pragma unroll
        for (int k = 0; k < packs; ++k) {
            const int i = threadIdx.x + THREADS * k;
            *reinterpret_cast<bagel_pack<T, V> *>(to.x + i / (W / V) * to.pitch + i % (W / V) * V) = x[k];
        }
    }
};

// l^e for whole e >= 0; l2 = log2(l), finite
__device__ __forceinline__ float power(float l2, int e) { return __builtin_amdgcn_exp2f(l2 * (float)e); }

// The largest magnitude in a wave (NaN does not count).
__device__ __forceinline__ float wave_largest(float v)
{
    v = fmaxf(v, bagel_moved<0xB1>(v));
    v = fmaxf(v, bagel_moved<0x4E>(v));
    v = fmaxf(v, bagel_moved<0x141>(v));
    v = fmaxf(v, bagel_moved<0x140>(v));
    const int i = __float_as_int(v);
    return fmaxf(fmaxf(__int_as_float(__builtin_amdgcn_readlane(i, 0)), __int_as_float(__builtin_amdgcn_readlane(i, 16))),
                 fmaxf(__int_as_float(__builtin_amdgcn_readlane(i, 32)), __int_as_float(__builtin_amdgcn_readlane(i, 48))));
}

// float16 holds 5 bits of exponent: what is rounded to it is brought below 2^15 first by a power of two, and back behind the product.  The others
// hold what float32 holds.
template <typename T> constexpr bool NARROW = sizeof(T) == 2 && __is_same(T, _Float16);
// The exponent e for which largest / 2^e is in [2^14, 2^15) (as far as e stays in what may be multiplied by; of zero and what is not finite, 0).
__device__ __forceinline__ int exponent_for(float largest)
{
    const int e = (int)(__float_as_uint(largest) >> 23) - 127 - 14;
    return largest > 0.0f && largest < INFINITY ? max(e, -100) : 0;
}

// Where a segment is.
struct place {
    int sequence;
    int64_t base;                // its first row, in the order they are gone through
    int64_t rows;
    bool first, last;            // of its sequence
    bool there;
};

// Which sequence a number of a segment belongs to: the last that does not begin behind it.  All lanes look, at one in 64 of the sequences each time.
template <typename T> __device__ __forceinline__ place place_of(const bagel_attention_pass<T> &p, int64_t slot)
{
    place r;
    int64_t begin, end, s;
    if (!p.offsets) {
        const int64_t each = max((p.each + p.segment - 1) / p.segment, (int64_t)1);
        r.sequence = (int)(slot / each);
        s = slot - r.sequence * each;
        begin = (int64_t)r.sequence * p.each;
        end = begin + p.each;
    } else {
        const int lane = threadIdx.x & 63;
        const auto number = [&](int i) { return (int64_t)p.offsets[i] / p.segment + i; };
        int lo = 0, count = p.sequences;
        while (count > 1) {
            const int step = (count + 63) / 64;
            const uint64_t ok = __ballot(lane * step < count && number(lo + min(lane * step, count - 1)) <= slot);
            const int k = max(__popcll(ok) - 1, 0);
            lo += k * step;
            count = min(step, count - k * step);
        }
        r.sequence = __builtin_amdgcn_readfirstlane(lo);
        // (offsets that break the rules lead nowhere outside of the rows)
        begin = min(max((int64_t)p.offsets[r.sequence], (int64_t)0), p.rows);
        end = min(max((int64_t)p.offsets[r.sequence + 1], begin), p.rows);
        s = slot - (begin / p.segment + r.sequence);
    }
    const int64_t length = end - begin, from = s * p.segment;
    r.first = s == 0;
    r.there = s == 0 || (s > 0 && from < length);
    r.rows = min(length - from, p.segment);
    r.last = from + p.segment >= length;
    r.base = p.back ? end - 1 - from : begin + from;
    return r;
}

// Four waves to a segment of a memory.  Every wave has a quarter of the memory's columns, in float32 in its registers, and the same columns of c and out; the rows'
// products with each other, P, are shared out by rows of P and meet in shared memory.
// SUMS: only the memory behind the segment, from zero where it is not the first of its sequence.
template <typename T, int WB, int WC, bool SUMS> __global__ __launch_bounds__(THREADS) void chunks_kernel(bagel_attention_pass<T> p)
{
    constexpr int NB = WB / 16, NC = WC / 64, KB = WB / 32;
    __shared__ tile<T, WB> sb;
    __shared__ tile<T, WC> sc;
    __shared__ tile<T, SUMS ? 16 : WB> sa;
    __shared__ tile<T, SUMS ? 16 : CHUNK> sp;
    __shared__ int sp_exponent[4];
    const int64_t segments = p.slots * p.states;
    if ((int64_t)blockIdx.x >= segments) {           // rows behind the last sequence
        const int64_t end = min(max((int64_t)p.offsets[p.sequences], (int64_t)0), p.rows), each = (int64_t)p.states * p.qs * p.wc, n = (p.rows - end) * each;
        for (int64_t i = ((int64_t)blockIdx.x - segments) * THREADS + threadIdx.x; i < n; i += ((int64_t)gridDim.x - segments) * THREADS) {
            const int64_t r = i / each;
            const int j = (int)(i - r * each);
            p.out.at(end + r, j / p.wc)[j % p.wc] = (T)0.0f;
        }
        return;
    }
    const int64_t slot = blockIdx.x / p.states;
    const int state = blockIdx.x % p.states;
    const place at = place_of(p, slot);
    if (!at.there || (SUMS && at.last)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, j16 = lane & 15;
    const int column = wave * (WC / 4);
    const float l2 = fmaxf(p.log_decay[state], -1e30f) * 1.44269504f;
    const int step = p.back ? -1 : 1, behind = p.back ? 1 : 0;       // of powers of l

    // entry (16 bt + 4 g + j, column + 16 nc + j16) of the memory
    floats S[NB][NC];
    const int64_t size = (int64_t)p.wb * p.wc, memory = ((int64_t)at.sequence * p.states + state) * size;
    {
        const float *from = at.first ? p.first : SUMS ? nullptr : p.memories + ((slot - 1) * p.states + state) * size;
        const int64_t start = at.first ? memory : 0, step_b = at.first ? p.step_b : p.wc, step_c = at.first ? p.step_c : 1;
#pragma unroll
        for (int bt = 0; bt < NB; ++bt)
#pragma unroll
            for (int nc = 0; nc < NC; ++nc)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int b = 16 * bt + 4 * g + j, c = column + 16 * nc + j16;
                    S[bt][nc][j] = from && b < p.wb && c < p.wc ? from[start + b * step_b + c * step_c] : 0.0f;
                }
    }
    // powers of l that are the same for all chunks: of P's rows of this wave, of the rows' distance to the memory before, and to the one behind
    float weight_p[4][4], weight_in[4], weight_out[2][8];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int d = 16 * (wave - t) + j16 - 4 * g - j;
            weight_p[t][j] = d >= 0 ? power(l2, d) * p.scale_b : 0.0f;
        }
        weight_in[t] = power(l2, 16 * t + j16 + 1 - behind);
    }
    const auto weigh_out = [&](int n) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int i = 0; i < 8; ++i) weight_out[t][i] = power(l2, max(n - 1 - (32 * t + 4 * g + (i & 3) + 4 * (i & 4)), 0) + behind) * p.scale_b;
    };
    weigh_out(CHUNK);

    const int heads = max(p.qs, p.ks);
    const int64_t steps = (at.rows + CHUNK - 1) / CHUNK * heads;
    incoming<T, SUMS ? 16 : WB> na;
    incoming<T, WB> nb;
    incoming<T, WC> nc_;
    const auto ask = [&](int64_t k) {
        const int64_t chunk = heads == 1 ? k : k / heads;
        const int h = heads == 1 ? 0 : (int)(k - chunk * heads), n = (int)min(at.rows - chunk * CHUNK, (int64_t)CHUNK);
        const int64_t base = at.base + step * chunk * CHUNK;
        if constexpr (!SUMS)
            if (h == 0 || p.qs > 1) na.load(p.a, state * p.qs + (p.qs > 1 ? h : 0), base, step, n, p.wb);
        if (h == 0 || p.ks > 1) {
            nb.load(p.b, state * p.ks + (p.ks > 1 ? h : 0), base, step, n, p.wb);
            nc_.load(p.c, state * p.ks + (p.ks > 1 ? h : 0), base, step, n, p.wc);
        }
    };
    if (steps > 0) ask(0);
    floats O[4][NC];
    for (int64_t k = 0; k < steps; ++k) {
        const int64_t chunk = heads == 1 ? k : k / heads;
        const int h = heads == 1 ? 0 : (int)(k - chunk * heads), n = (int)min(at.rows - chunk * CHUNK, (int64_t)CHUNK);
        __syncthreads();
        if constexpr (!SUMS)
            if (h == 0 || p.qs > 1) na.put(sa);
        if (h == 0 || p.ks > 1) {
            nb.put(sb);
            nc_.put(sc);
        }
        __syncthreads();
        if (k + 1 < steps) ask(k + 1);

        operand<T> c[2][NC];
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
            for (int nc = 0; nc < NC; ++nc) c[t][nc] = sc.across(t, column + 16 * nc);
        if constexpr (!SUMS) {
            // the wave's 16 rows of P, transposed: a lane has four entries of a row
            floats P[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) P[t] = (floats)0.0f;
            operand<T> a[KB];
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) a[kb] = sa.along(16 * wave + j16, kb);
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (t <= wave) {
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) P[t] = product(sb.along(16 * t + j16, kb), a[kb], P[t]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) P[t][j] = t < wave || 4 * g + j <= j16 ? P[t][j] * weight_p[t][j] : 0.0f;
                }
            float down = 1.0f;
            if constexpr (NARROW<T>) {
                float top = 0.0f;
#pragma unroll
                for (int t = 0; t < 4; ++t)
#pragma unroll
                    for (int j = 0; j < 4; ++j) top = fmaxf(top, fabsf(P[t][j]));
                const int e = exponent_for(wave_largest(top));
                down = ldexpf(1.0f, -e);
                if (lane == 0) sp_exponent[wave] = e;
            }
#pragma unroll
            for (int t = 0; t < 4; ++t)
                if (t <= (wave | 1)) {               // (products over 32 rows: their second half may be beyond the wave's rows, and zero)
                    bagel_pack<T, 4> x;
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = (T)(NARROW<T> ? P[t][j] * down : P[t][j]);
                    *reinterpret_cast<bagel_pack<T, 4> *>(sp.x + (16 * wave + j16) * sp.pitch + 16 * t + 4 * g) = x;
                }
            __syncthreads();
            if (p.out.data) {
                if (h == 0 || p.qs > 1) {
                    int e = 0;
                    float down = 1.0f;
                    if constexpr (NARROW<T>) {
                        float top = 0.0f;
#pragma unroll
                        for (int bt = 0; bt < NB; ++bt)
#pragma unroll
                            for (int nc = 0; nc < NC; ++nc)
#pragma unroll
                                for (int j = 0; j < 4; ++j) top = fmaxf(top, fabsf(S[bt][nc][j]));
                        e = exponent_for(wave_largest(top));
                        down = ldexpf(1.0f, -e);
                    }
#pragma unroll
                    for (int nc = 0; nc < NC; ++nc) {
                        operand<T> s[KB];
#pragma unroll
                        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                            for (int i = 0; i < 8; ++i) s[kb][i] = (T)(NARROW<T> ? S[2 * kb + i / 4][nc][i % 4] * down : S[2 * kb + i / 4][nc][i % 4]);
#pragma unroll
                        for (int it = 0; it < 4; ++it) {
                            floats o = (floats)0.0f;
#pragma unroll
                            for (int kb = 0; kb < KB; ++kb) o = product(s[kb], sa.along(16 * it + j16, kb), o);
                            const float w = NARROW<T> ? ldexpf(weight_in[it], e) : weight_in[it];
#pragma unroll
                            for (int j = 0; j < 4; ++j) O[it][nc][j] = o[j] * w;
                        }
                    }
                }
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    operand<T> row[2];
                    row[0] = sp.along(16 * it + j16, 0);
                    if (it >= 2) row[1] = sp.along(16 * it + j16, 1);
#pragma unroll
                    for (int nc = 0; nc < NC; ++nc) {
                        floats o = NARROW<T> ? (floats)0.0f : O[it][nc];
                        o = product(c[0][nc], row[0], o);
                        if (it >= 2) o = product(c[1][nc], row[1], o);
                        if constexpr (NARROW<T>) {
                            const float up = ldexpf(1.0f, sp_exponent[it]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) O[it][nc][j] = fmaf(o[j], up, O[it][nc][j]);
                        } else {
                            O[it][nc] = o;
                        }
                    }
                }
                if (h == heads - 1 || p.qs > 1) {
                    const int head = state * p.qs + (p.qs > 1 ? h : 0);
#pragma unroll
                    for (int it = 0; it < 4; ++it) {
                        const int m = 16 * it + j16;
                        if (m >= n) continue;
                        T *to = p.out.at(at.base + step * (chunk * CHUNK + m), head);
#pragma unroll
                        for (int nc = 0; nc < NC; ++nc) {
                            const int first = column + 16 * nc + 4 * g;
                            bagel_pack<T, 4> x;
#pragma unroll
                            for (int j = 0; j < 4; ++j) x[j] = (T)(O[it][nc][j] * p.scale);
                            if (first + 4 <= p.wc) reinterpret_cast<bagel_loose_pack<T, 4> *>(to + first)->x = x;
                            else
#pragma unroll
                                for (int j = 0; j < 3; ++j)
                                    if (first + j < p.wc) to[first + j] = x[j];
                        }
                    }
                }
            }
        }
        // The memory behind the chunk.  c is weighed, and what that makes is held to 24 bits as a sum of operands (22 in float16): the memory is kept in
        // float32, and one rounding to 8 or 11 bits of every row would be left in it.
        if (p.ks > 1 || h == heads - 1) {
            if (n != CHUNK) weigh_out(n);
            const float keep = p.ks == 1 || h == 0 ? power(l2, n) : 1.0f;
#pragma unroll
            for (int nc = 0; nc < NC; ++nc) {
                int e = 0;
                float w[2][8];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[t][i] = (float)c[t][nc][i] * weight_out[t][i];
                if constexpr (NARROW<T>) {
                    float top = 0.0f;
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(w[t][i]));
                    e = exponent_for(wave_largest(top));
                    const float down = ldexpf(1.0f, -e);
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int i = 0; i < 8; ++i) w[t][i] *= down;
                }
                constexpr int PARTS = sizeof(T) == 4 ? 1 : NARROW<T> ? 2 : 3;
                operand<T> part[PARTS][2];
#pragma unroll
                for (int t = 0; t < 2; ++t)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
#pragma unroll
                        for (int q = 0; q < PARTS; ++q) {
                            part[q][t][i] = (T)w[t][i];
                            w[t][i] -= (float)part[q][t][i];
                        }
#pragma unroll
                for (int bt = 0; bt < NB; ++bt) {
                    const operand<T> b0 = sb.across(0, 16 * bt), b1 = sb.across(1, 16 * bt);
                    floats s = NARROW<T> ? (floats)0.0f : S[bt][nc];
                    if constexpr (!NARROW<T>)
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[j] *= keep;
#pragma unroll
                    for (int q = PARTS - 1; q >= 0; --q) {
                        s = product(b0, part[q][0], s);
                        s = product(b1, part[q][1], s);
                    }
                    if constexpr (NARROW<T>) {
                        const float up = ldexpf(1.0f, e);
#pragma unroll
                        for (int j = 0; j < 4; ++j) s[j] = fmaf(S[bt][nc][j], keep, s[j] * up);
                    }
                    S[bt][nc] = s;
                }
            }
        }
    }
    float *to = SUMS ? p.memories + (slot * p.states + state) * size : at.last && p.last ? p.last + memory : nullptr;
    if (!to) return;
    const int64_t step_b = SUMS ? p.wc : p.step_b, step_c = SUMS ? 1 : p.step_c;
#pragma unroll
    for (int bt = 0; bt < NB; ++bt)
#pragma unroll
        for (int nc = 0; nc < NC; ++nc)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int b = 16 * bt + 4 * g + j, c = column + 16 * nc + j16;
                if (b < p.wb && c < p.wc) to[b * step_b + c * step_c] = S[bt][nc][j];
            }
}

// What segments have added to the memory, into the memory behind each: a thread to an entry, along its sequence's segments but the last.
template <typename T> __global__ __launch_bounds__(256) void memories_kernel(bagel_attention_pass<T> p, int blocks)
{
    const int size = p.wb * p.wc;
    for (int64_t work = blockIdx.x; work < (int64_t)p.sequences * p.states * blocks; work += gridDim.x) {
        const int i = (int)(work % blocks) * 256 + threadIdx.x, state = (int)(work / blocks % p.states), sequence = (int)(work / blocks / p.states);
        int64_t length = p.each, slot;
        if (!p.offsets) {
            slot = (int64_t)sequence * max((length + p.segment - 1) / p.segment, (int64_t)1);
        } else {
            const int64_t begin = min(max((int64_t)p.offsets[sequence], (int64_t)0), p.rows);
            length = min(max((int64_t)p.offsets[sequence + 1], begin), p.rows) - begin;
            slot = begin / p.segment + sequence;
        }
        const int64_t segments = (length + p.segment - 1) / p.segment, each = (int64_t)p.states * size;
        if (i >= size || segments < 3) continue;     // (of two, the first one's is whole)
        const float keep = __builtin_amdgcn_exp2f(fmaxf(p.log_decay[state], -1e30f) * 1.44269504f * (float)p.segment);
        float *m = p.memories + (slot * p.states + state) * size + i;
        float s = m[0];
        constexpr int AHEAD = 8;
        for (int64_t k = 1; k < segments - 1; k += AHEAD) {
            float add[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) add[j] = k + j < segments - 1 ? m[(k + j) * each] : 0.0f;
#pragma unroll
            for (int j = 0; j < AHEAD; ++j)
                if (k + j < segments - 1) m[(k + j) * each] = s = fmaf(keep, s, add[j]);
        }
    }
}

template <typename T, int WB, int WC> hipError_t launch_pass(const bagel_attention_pass<T> &p, hipStream_t stream)
{
    const int64_t work = p.slots * p.states;
    if (p.memories && work > 0) {
        chunks_kernel<T, WB, WC, true><<<(unsigned)work, THREADS, 0, stream>>>(p);
        const int blocks = (p.wb * p.wc + 255) / 256;
        const int64_t all = (int64_t)p.sequences * p.states * blocks;
        memories_kernel<T><<<(unsigned)(all < 1 << 20 ? all : 1 << 20), 256, 0, stream>>>(p, blocks);
    }
    const int64_t clear = p.offsets && p.out.data && p.rows > 0 ? 32 : 0;
    if (work + clear > 0) chunks_kernel<T, WB, WC, false><<<(unsigned)(work + clear), THREADS, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

template <typename T> hipError_t bagel_launch_attention_pass(const bagel_attention_pass<T> &p, hipStream_t stream)
{
    if (p.wb <= 64) return p.wc <= 64 ? launch_pass<T, 64, 64>(p, stream) : launch_pass<T, 64, 128>(p, stream);
    return p.wc <= 64 ? launch_pass<T, 128, 64>(p, stream) : launch_pass<T, 128, 128>(p, stream);
}
