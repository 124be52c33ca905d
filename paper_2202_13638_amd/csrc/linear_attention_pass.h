// The pass of linear attention over the rows (bagel_attention_pass in linear_attention.h), with the matrix instructions of one type.
//
// A chunk of 64 rows, with l the decay, S the memory before it and m, n rows of it in the order they are gone through:
//   out_m = scale (l^(m+1) S^T a_m + sum_{n<=m} P_mn c_n),   P_mn = scale_b l^(m-n) a_m.b_n
//   S <- l^64 S + sum_n scale_b l^(63-n) b_n c_n^T                     (back: l^m S^T a_m, and l^(64-n))
// No power of l is negative, so nothing grows that the definition does not let grow.
//   By the definition, row after row, the work is 3 to 5 operations for every entry of a memory and row, none of which a matrix instruction can do, and each row waits for the one
// before it.  By chunks it is matrix products throughout, and a chunk waits for a memory instead.  64 rows: with more of them P, which grows by their square, takes
// longer than the memory's update, with fewer the update, made once a chunk, takes longer than P.
#pragma once

#include <type_traits>

#include "linear_attention.h"

namespace {

constexpr int CHUNK = BAGEL_ATTENTION_CHUNK;

using floats = float __attribute__((ext_vector_type(4)));

// Operands of a product over 32: index lane % 16 of the result, and entries 8 g to 8 g + 7 of the 32, with g = lane / 16.  A result has index lane % 16 of its second
// operand and 4 g to 4 g + 3 of its first one.  With the first one's index r of two results taken as 8 (r / 4) + r % 4 and 4 more, a lane
// holds eight in a row of the two: they are an operand of the next product as they are.
template <typename T> using operand = T __attribute__((ext_vector_type(8)));

__device__ __forceinline__ floats product(operand<__bf16> x, operand<__bf16> y, floats z) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ floats product(operand<_Float16> x, operand<_Float16> y, floats z) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, z, 0, 0, 0); }
__device__ __forceinline__ floats product(operand<float> x, operand<float> y, floats z)
{
#pragma unroll
    for (int j = 0; j < 8; ++j) z = __builtin_amdgcn_mfma_f32_16x16x4f32(x[j], y[j], z, 0, 0, 0);
    return z;
}

// 64 rows in shared memory, read by rows and by columns.  A lane's part of an address is the same for all tiles of a width and made once; what differs is known to
// the compiler.
//   In 16 bits the slots of 16 bytes of a row are permuted by a number that the row's place among 16 gives.  Shared memory serves 256 bytes at a time: of reads of
// 16 bytes, lanes 0 to 3, 12 to 15 and 20 to 27 together, and 4 to 11, 16 to 19 and 28 to 31; of those of 8 bytes, lanes 0 to 31.  The numbers bring into different banks
// what is served together in 16 rows of one slot, of which those of odd lane groups are of the next (along, spread), and in two times four rows of two slots (across).
// Four rows of half of four slots (across_spread) meet in pairs whatever the numbers.  In 32 bits 16 bytes stand between the rows.
template <typename T, int W> struct tile {
    static constexpr bool PERMUTED = sizeof(T) == 2;
    static constexpr int pitch = PERMUTED ? W : W + 4, row_bytes = pitch * sizeof(T);
    alignas(32) T x[CHUNK * pitch];
    __host__ __device__ static constexpr int number(int row)
    {
        return W == 64 ? (row & 2) ^ (row >> 2 & 1) ^ (row & 4) ^ (row >> 1 & 4) : (row << 1 & 6) ^ (row >> 2 & 1) ^ (row << 1 & 8) ^ (row & 8);
    }
    static constexpr int four_on = PERMUTED ? number(4) * 16 : 0;        // what four rows further, of a row whose place has no four in it, change in the slot
    __device__ static __forceinline__ int place(int row, int column)     // of an entry
    {
        return row * pitch + (PERMUTED ? ((column >> 3 ^ number(row)) << 3) + (column & 7) : column);
    }
    __device__ static __forceinline__ int bytes(int row, int column) { return place(row, column) * (int)sizeof(T); }
    // `lane_part` (bytes) with `c` columns on, a multiple of 8 that the lane's own column does not carry into
    __device__ static __forceinline__ int on(int lane_part, int c) { return PERMUTED ? lane_part ^ c * 2 : lane_part + c * (int)sizeof(T); }
    template <typename P> __device__ __forceinline__ P &in_bytes(int offset) { return *reinterpret_cast<P *>(reinterpret_cast<char *>(x) + offset); }
    template <typename P> __device__ __forceinline__ const P &in_bytes(int offset) const { return *reinterpret_cast<const P *>(reinterpret_cast<const char *>(x) + offset); }

    // Operand with entries 32 t on of rows 16 r + lane % 16
    __device__ static __forceinline__ int lane_along() { return bytes(threadIdx.x & 15, 8 * ((threadIdx.x & 63) >> 4)); }
    __device__ __forceinline__ operand<T> &along(int lane_part, int r, int t) { return in_bytes<operand<T>>(on(lane_part, 32 * t) + r * 16 * row_bytes); }
    // Operand with entries 32 t on of rows 32 r + 8 (i / 4) + i % 4 + 4 half, i = lane % 16
    __device__ static __forceinline__ int lane_spread()
    {
        const int i = threadIdx.x & 15;
        return bytes(8 * (i / 4) + i % 4, 8 * ((threadIdx.x & 63) >> 4));
    }
    __device__ __forceinline__ operand<T> spread(int lane_part, int r, int half, int t) const
    {
        return in_bytes<operand<T>>((on(lane_part, 32 * t) ^ half * four_on) + (r * 32 + half * 4) * row_bytes);
    }
    // Four entries 16 c + 4 g on of row 16 r + lane % 16
    __device__ static __forceinline__ int lane_entries() { return bytes(threadIdx.x & 15, 4 * ((threadIdx.x & 63) >> 4)); }
    __device__ __forceinline__ bagel_pack<T, 4> &entries(int lane_part, int r, int c) { return in_bytes<bagel_pack<T, 4>>(on(lane_part, 16 * c) + r * 16 * row_bytes); }
    // Operands with rows 32 t + 8 g to 32 t + 8 g + 7 of a column to each of 16 lanes: 16 c + lane % 16, or (spread) 32 c + 8 (i / 4) + i % 4 + 4 half, i = lane % 16.
    // In 16 bits a group of 16 lanes reads 4 rows of four columns for each of its lanes, and each lane gets one of the 16.
    __device__ static __forceinline__ int lane_across(bool spread)
    {
        const int g = (threadIdx.x & 63) >> 4, i = threadIdx.x & 15;
        if (PERMUTED) return bytes(8 * g + i / 4, (spread ? 8 : 4) * (i % 4));
        return bytes(8 * g, spread ? 8 * (i / 4) + i % 4 : i);
    }
    __device__ __forceinline__ operand<T> column(int from) const
    {
        if constexpr (PERMUTED) {
            using half = short __attribute__((ext_vector_type(4)));
            using shared_half = __attribute__((address_space(3))) half;
            const half lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared_half *)&in_bytes<half>(from));
            const half hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared_half *)&in_bytes<half>((from ^ four_on) + 4 * row_bytes));
            return __builtin_bit_cast(operand<T>, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            operand<T> r;
#pragma unroll
            for (int i = 0; i < 8; ++i) r[i] = in_bytes<T>(from + i * row_bytes);
            return r;
        }
    }
    __device__ __forceinline__ operand<T> across(int lane_part, int t, int c) const { return column(on(lane_part, 16 * c) + 32 * t * row_bytes); }
    __device__ __forceinline__ operand<T> across_spread(int lane_part, int t, int c, int half) const
    {
        return column(on(lane_part, 32 * c) + half * 4 * (int)sizeof(T) + 32 * t * row_bytes);
    }
};

// A number that the compiler takes to be another one every time.  The addresses of the rarer ways are made of it, so that they are not all kept in registers
// through the loop over the chunks.
__device__ __forceinline__ int afresh(int x)
{
    asm volatile("" : "+v"(x));
    return x;
}

// A thread's packs of 16 bytes of a tile.
template <typename T, int W, int THREADS> struct packs_of {
    static constexpr int V = 16 / sizeof(T), in_row = W / V, count = CHUNK * in_row / THREADS, apart = THREADS / in_row;    // rows between a thread's packs
    static_assert(!tile<T, W>::PERMUTED || apart % 16 == 0, "a thread's rows have the same place among 16");
    using pack = bagel_pack<T, V>;
    __device__ static __forceinline__ int row(int k) { return threadIdx.x / in_row + k * apart; }
    __device__ static __forceinline__ int column() { return threadIdx.x % in_row * V; }
    __device__ static __forceinline__ int lane_part() { return tile<T, W>::bytes(row(0), column()); }
    template <typename Tile> __device__ static __forceinline__ auto &in(Tile &t, int lane_part, int k) { return t.template in_bytes<pack>(lane_part + k * apart * t.row_bytes); }
};

// A tile on its way from memory, the 64 rows up to its last one: those before the first are there too, but of the segment's first rows, where it is copied in
// their place.  Every thread loads from a place that is there, so that no branch and no wait stands between the loads and the products that go on
// meanwhile; a pack that would reach over the end of a row is the one that ends there (a row is a pack at least).  In shared memory the n rows that
// are there come first, the others are zero, and columns that are not there stay as they were.
template <typename T, int W, int THREADS> struct incoming {
    using in = packs_of<T, W, THREADS>;
    static constexpr int V = in::V;
    typename in::pack x[in::count];
    __device__ __forceinline__ void load(const T *from, int64_t stride, int width)
    {
        from += in::row(0) * stride + min(in::column(), width - V);
#pragma unroll
        for (int k = 0; k < in::count; ++k) x[k] = reinterpret_cast<const bagel_loose_pack<T, V> *>(from + k * (in::apart * stride))->x;
    }
    __device__ __forceinline__ void load_few(const T *from, int n, int64_t stride, int width)
    {
        from += min(in::column(), width - V);
#pragma unroll
        for (int k = 0; k < in::count; ++k) x[k] = reinterpret_cast<const bagel_loose_pack<T, V> *>(from + max(in::row(k) - (CHUNK - n), 0) * stride)->x;
    }
    __device__ __forceinline__ void put(tile<T, W> &to, int lane_part, int n, int width) const
    {
        if (n == CHUNK && width == W) {
#pragma unroll
            for (int k = 0; k < in::count; ++k) in::in(to, lane_part, k) = x[k];
            return;
        }
        const int column = afresh(in::column()), row = afresh(in::row(0));
        if (column >= width) return;
        const int back = width == W ? 0 : max(column + V - width, 0);
#pragma unroll
        for (int k = 0; k < in::count; ++k) {
            const int m = row + k * in::apart - (CHUNK - n), r = m < 0 ? m + CHUNK : m;
            const typename in::pack y = m < 0 ? (typename in::pack)(T)0.0f : x[k];
            if (back == 0) to.template in_bytes<typename in::pack>(to.bytes(r, column)) = y;
            else
#pragma unroll
                for (int j = 0; j < V; ++j) to.x[to.place(r, column - back + j)] = y[j];
        }
    }
};

// A tile of results to memory, in the same way: packs that end where their row ends write some entries twice.
template <typename T, int W, int THREADS> __device__ __forceinline__ void write_rows(tile<T, W> &from, int lane_part, T *to, int64_t stride, int n, int width)
{
    using in = packs_of<T, W, THREADS>;
    if (n == CHUNK && width == W) {
        T *at = to + in::row(0) * stride + in::column();
#pragma unroll
        for (int k = 0; k < in::count; ++k) reinterpret_cast<bagel_loose_pack<T, in::V> *>(at + k * (in::apart * stride))->x = in::in(from, lane_part, k);
        return;
    }
    const int column = afresh(in::column()), first = min(column, width - in::V), row = afresh(in::row(0));
    if (column >= width) return;
#pragma unroll
    for (int k = 0; k < in::count; ++k) {
        const int m = row + k * in::apart;
        if (m >= n) continue;
        typename in::pack y;
        if (width == W) y = in::in(from, lane_part, k);
        else
#pragma unroll
            for (int j = 0; j < in::V; ++j) y[j] = from.x[from.place(m, first + j)];
        reinterpret_cast<bagel_loose_pack<T, in::V> *>(to + m * stride + first)->x = y;
    }
}

template <typename T, int W> __device__ __forceinline__ void clear(tile<T, W> &t, int width)
{
    if (width < W)
        for (int i = threadIdx.x; i < CHUNK * t.pitch; i += blockDim.x) t.x[i] = (T)0.0f;
}

// The wait states between products and whatever uses their results, ahead of a branch: the compiler may count them along the longer way only.
__device__ __forceinline__ void settle(floats &x) { asm volatile("s_nop 9" : "+v"(x)); }
template <int N> __device__ __forceinline__ void settle(floats (&x)[N])
{
    static_assert(N == 2 || N == 4 || N == 8, "a memory's tiles, or a piece of P");
    if constexpr (N == 2) asm volatile("s_nop 9" : "+v"(x[0]), "+v"(x[1]));
    else if constexpr (N == 4) asm volatile("s_nop 9" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]));
    else asm volatile("s_nop 9" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]), "+v"(x[7]));
}

// Reads of shared memory and products stay on their side of it: left to itself the compiler puts each read right before its product, which then waits for it
// (131072 rows, 8 heads of 128 on 2 memories, bf16: 272 us without and 248 with what is read ahead; 64000 rows, 8 heads of 64: 64.0 and 62.8).  In 32 bits the products'
// own time is longer than a read, and 128 x 64 has no registers for what is read ahead (bf16, 64000 rows, 8 heads: 107 us without, 130 with).
template <typename T, int WB, int WC> constexpr bool AHEAD = sizeof(T) == 2 && !(WB == 128 && WC == 64);
template <bool WANTED> __device__ __forceinline__ void reads_before_products()
{
    if constexpr (WANTED) __builtin_amdgcn_sched_barrier(0x216);
}

// log2(l) of a memory, no less than what e times it can be said of; NaN stays NaN.
template <typename T> __device__ __forceinline__ float log2_decay(const bagel_attention_pass<T> &p, int state)
{
    const float d = p.log_decay[state];
    return (d < -1e30f ? -1e30f : d) * 1.44269504f;
}

// l^e for whole e >= 0; l2 = log2(l), not infinite
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
    int64_t before;              // the number of the segment before, -1: it is the first
    int64_t further;             // of its sequence's segments before, those that are not the first
    bool last, there;
};

// A sequence's rows; offsets that break the rules lead nowhere outside.
template <typename T> __device__ __forceinline__ void sequence_rows(const bagel_attention_pass<T> &p, int i, int64_t &begin, int64_t &end)
{
    if (!p.offsets) {
        begin = (int64_t)i * p.each;
        end = begin + p.each;
    } else {
        begin = min(max((int64_t)p.offsets[i], (int64_t)0), p.rows);
        end = min(max((int64_t)p.offsets[i + 1], begin), p.rows);
    }
}
template <typename T> __device__ __forceinline__ int64_t further_of_each(const bagel_attention_pass<T> &p) { return p.each > 0 ? (p.each - 1) / p.segment : 0; }

template <typename T> __device__ __forceinline__ place place_of(const bagel_attention_pass<T> &p, int64_t number)
{
    place r;
    int64_t s = 0;
    if (number < p.sequences) {
        r.sequence = (int)number;
        r.before = -1;
        r.further = 0;
    } else {
        const int64_t further = number - p.sequences;
        if (!p.offsets) {
            const int64_t each = max(further_of_each(p), (int64_t)1);
            r.sequence = (int)(further / each);
            s = further - r.sequence * each + 1;
        } else {
            // The last sequence whose further segments do not begin behind it.  All lanes look, at one in 64 of the sequences each time.
            const int lane = threadIdx.x & 63;
            int lo = 0, count = p.sequences;
            while (count > 1) {
                const int step = (count + 63) / 64;
                const uint64_t ok = __ballot(lane * step < count && (int64_t)p.offsets[lo + min(lane * step, count - 1)] / p.segment <= further);
                const int k = max(__popcll(ok) - 1, 0);
                lo += k * step;
                count = min(step, count - k * step);
            }
            r.sequence = __builtin_amdgcn_readfirstlane(lo);
            s = further - min(max((int64_t)p.offsets[r.sequence], (int64_t)0), p.rows) / p.segment + 1;
        }
        r.before = s == 1 ? r.sequence : number - 1;
        r.further = s - 1;
    }
    int64_t begin, end;
    sequence_rows(p, r.sequence, begin, end);
    const int64_t length = end - begin, from = s * p.segment;
    r.there = number < p.sequences || (s > 0 && from < length);
    r.rows = min(length - from, p.segment);
    r.last = from + p.segment >= length;
    r.base = p.back ? end - 1 - from : begin + from;
    return r;
}

// Workgroups go to the eight dies in turn.  Each die takes work that follows each other, so that the heads of the same rows, which lie side by side in memory,
// are read by one: the first segments, and then the further ones, which may not be there.
__device__ __forceinline__ int64_t by_dies(int64_t group, int64_t first, int64_t all)
{
    const int64_t begin = group < first ? 0 : first, n = group < first ? first : all - first, i = group - begin, die = i % 8;
    return begin + die * (n / 8) + min(die, n % 8) + i / 8;
}

// A lane's parts of addresses in shared memory.
template <typename T, int WB, int WC, int THREADS> struct lane_parts {
    const int along_a = tile<T, WB>::lane_along(), spread_b = tile<T, WB>::lane_spread();
    const int across_b = tile<T, WB>::lane_across(true), across_c = tile<T, WC>::lane_across(false), entries_o = tile<T, WC>::lane_entries();
    const int pack_b = packs_of<T, WB, THREADS>::lane_part(), pack_c = packs_of<T, WC, THREADS>::lane_part();
};

// Powers of l that are the same for all chunks, in shared memory.
struct powers {
    floats out[CHUNK / 4];       // from the rows to the memory behind the chunk, times scale_b
    floats p[3][2][64];          // between rows of a piece of P (a lane's eight entries) that begins 0, 16 and 32 rows before, times scale_b
    int exponent[2][4][2];       // of the pieces (float16)
    __device__ __forceinline__ void weigh_out(float l2, int behind, float scale_b, int n)
    {
        if ((int)threadIdx.x < CHUNK) reinterpret_cast<float *>(out)[threadIdx.x] = power(l2, max(n - 1 - (int)threadIdx.x, 0) + behind) * scale_b;
    }
    __device__ __forceinline__ void weigh_p(float l2, float scale_b)
    {
        const int lane = threadIdx.x & 63;
        for (int i = threadIdx.x >> 6; i < 6; i += blockDim.x >> 6) {
            floats x;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int d = 16 * (i / 2) + lane % 16 - (lane / 16 * 8 + i % 2 * 4 + j);
                x[j] = d >= 0 ? power(l2, d) * scale_b : 0.0f;
            }
            p[i / 2][i % 2][lane] = x;
        }
    }
};

// A wave's 16 columns of a memory in float32, a lane one of them: S[2 kb + half][j] is entry 32 kb + 8 g + 4 half + j of it.
template <int NB> __device__ __forceinline__ int memory_row(int bt, int j) { return bt / 2 * 32 + (threadIdx.x & 63) / 16 * 8 + bt % 2 * 4 + j; }
template <int NB> __device__ __forceinline__ void read_memory(floats (&S)[NB], const float *from, int64_t step_b, int64_t step_c, int column, int wb, int wc)
{
#pragma unroll
    for (int bt = 0; bt < NB; ++bt)
#pragma unroll
        for (int j = 0; j < 4; ++j) S[bt][j] = from && memory_row<NB>(bt, j) < wb && column < wc ? from[memory_row<NB>(bt, j) * step_b + column * step_c] : 0.0f;
#pragma unroll
    for (int bt = 0; bt < NB; ++bt) asm volatile("" : "+v"(S[bt]));      // it is there before anything else is asked for, so that no later wait is one for it
}
template <int NB> __device__ __forceinline__ void write_memory(const floats (&S)[NB], float *to, int64_t step_b, int64_t step_c, int column, int wb, int wc)
{
    asm volatile("" : "+v"(step_b));                 // its multiples are not kept from the beginning: they would take all scalar registers
    if (!to || column >= wc) return;
#pragma unroll
    for (int bt = 0; bt < NB; ++bt)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (memory_row<NB>(bt, j) < wb) to[memory_row<NB>(bt, j) * step_b + column * step_c] = S[bt][j];
}

// What is in float32 and becomes an operand, the memory before a chunk and P, is a sum of so many of them.  In 16 bits one alone would round it to 8 or 11 bits, which would be
// seen in the results (64000 rows, 8 heads of 64, bf16: 0.0023 from 64 bits, where the rounding of the results alone makes 0.0017).  Two hold 16 or 22 bits, of whose
// rounding nothing is left in results of 8 or 11.  They take up to 12 % of the time (that case 57 us with one, 63 with two; its gradient 181 and 193).
template <typename T> constexpr int PARTS = sizeof(T) == 4 ? 1 : 2;
// All parts but the last are cut off: what is left is exact, as it would be behind a rounding, which the compiler makes once for the operand and once more for what is left
// (844 instead of 612 vector instructions in two steps; 716 so).
template <typename T, int N> __device__ __forceinline__ void in_parts(float (&x)[8], operand<T> (&part)[N])
{
    using words = uint32_t __attribute__((ext_vector_type(4)));
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int q = 0; q < N - 1; ++q) {
            words w;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
                if constexpr (NARROW<T>) {
                    const auto both = __builtin_amdgcn_cvt_pkrtz(x[i], x[i + 1]);
                    w[i / 2] = __builtin_bit_cast(uint32_t, both);
                    x[i] = fmaf((float)both[0], -1.0f, x[i]);
                    x[i + 1] = fmaf((float)both[1], -1.0f, x[i + 1]);
                } else {
                    w[i / 2] = __builtin_amdgcn_perm(__float_as_uint(x[i + 1]), __float_as_uint(x[i]), 0x07060302);     // their upper halves
                    x[i] -= __uint_as_float(__float_as_uint(x[i]) & 0xFFFF0000u);
                    x[i + 1] -= __uint_as_float(__float_as_uint(x[i + 1]) & 0xFFFF0000u);
                }
            }
            part[q] = __builtin_bit_cast(operand<T>, w);
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) part[N - 1][i] = (T)x[i];
}

// The exponent that is taken off a memory that becomes operands (float16; otherwise none is), and its operands 32 kb.
template <typename T, int NB> __device__ __forceinline__ int exponent_of(const floats (&S)[NB])
{
    if (!NARROW<T>) return 0;
    float top = 0.0f;
#pragma unroll
    for (int bt = 0; bt < NB; ++bt)
#pragma unroll
        for (int j = 0; j < 4; ++j) top = fmaxf(top, fabsf(S[bt][j]));
    return exponent_for(wave_largest(top));
}
template <typename T, int NB> __device__ __forceinline__ void as_operands(const floats (&S)[NB], int kb, float down, operand<T> (&to)[PARTS<T>])
{
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = NARROW<T> ? S[2 * kb + i / 4][i % 4] * down : S[2 * kb + i / 4][i % 4];
    in_parts<T>(x, to);
}

// The pieces of P that are not zero, rows 16 it by rows 32 kb of b with kb <= it / 2, in shared memory as the operands that their lanes hold: slots of 16 bytes, one
// lane's next to another's.
template <typename T> struct pieces_of {
    using slot = uint32_t __attribute__((ext_vector_type(4)));
    static constexpr int SLOTS = sizeof(operand<T>) / 16;
    struct parts {
        slot x[SLOTS];
    };
    slot x[6][PARTS<T>][SLOTS][64];
    __device__ static constexpr int number(int it, int kb) { return it + it / 3 + kb; }
    __device__ __forceinline__ void put(int it, int kb, int q, operand<T> o)
    {
        const parts p = __builtin_bit_cast(parts, o);
#pragma unroll
        for (int i = 0; i < SLOTS; ++i) x[number(it, kb)][q][i][threadIdx.x & 63] = p.x[i];
    }
    // those of rows 16 it
    __device__ __forceinline__ void get(operand<T> (&to)[2][PARTS<T>], int it) const
    {
#pragma unroll
        for (int kb = 0; kb <= it / 2; ++kb)
#pragma unroll
            for (int q = 0; q < PARTS<T>; ++q) {
                parts p;
#pragma unroll
                for (int i = 0; i < SLOTS; ++i) p.x[i] = x[number(it, kb)][q][i][threadIdx.x & 63];
                to[kb][q] = __builtin_bit_cast(operand<T>, p);
            }
    }
};

// A piece of P, transposed: a lane has eight entries of a row.
template <bool EARLY, typename T, int W>
__device__ __forceinline__ void make_piece(tile<T, W> &a, const tile<T, W> &b, pieces_of<T> &to, powers &w, int which, int it, int kb, float tile_on, int along_a, int spread_b)
{
    const int lane = threadIdx.x & 63, before = it - 2 * kb;
    floats P[2] = {(floats)0.0f, (floats)0.0f};
    operand<T> x[2], y[2][2];
    const auto read = [&](int q) {
        x[q & 1] = a.along(along_a, it, q);
#pragma unroll
        for (int half = 0; half < 2; ++half) y[q & 1][half] = b.spread(spread_b, kb, half, q);
    };
    read(0);
#pragma unroll
    for (int q = 0; q < W / 32; ++q) {
        if (q + 1 < W / 32) read(q + 1);
        reads_before_products<EARLY>();
#pragma unroll
        for (int half = 0; half < 2; ++half) P[half] = product(y[q & 1][half], x[q & 1], P[half]);
        reads_before_products<EARLY>();
    }
    if constexpr (sizeof(T) == 4) settle(P);
    const float far = before == 3 ? tile_on : 1.0f;  // 48 rows before: l^16 more than 32
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const floats l = w.p[min(before, 2)][half][lane];
#pragma unroll
        for (int j = 0; j < 4; ++j) P[half][j] *= l[j] * far;
    }
    float down = 1.0f;
    if constexpr (NARROW<T>) {
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(P[i / 4][i % 4]));
        const int e = exponent_for(wave_largest(top));
        down = ldexpf(1.0f, -e);
        if (lane == 0) w.exponent[which][it][kb] = e;
    }
    float z[8];
    operand<T> part[PARTS<T>];
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] = NARROW<T> ? P[i / 4][i % 4] * down : P[i / 4][i % 4];
    in_parts<T>(z, part);
#pragma unroll
    for (int q = 0; q < PARTS<T>; ++q) to.put(it, kb, q, part[q]);
}

// The six pieces of P that are not zero, shared out among the waves.
template <bool EARLY, int WAVES, typename T, int W>
__device__ __forceinline__ void make_pieces(tile<T, W> &a, const tile<T, W> &b, pieces_of<T> &to, powers &w, int which, float tile_on, int along_a, int spread_b, int wave)
{
    const auto piece = [&](int it, int kb) { make_piece<EARLY>(a, b, to, w, which, it, kb, tile_on, along_a, spread_b); };
    if constexpr (WAVES == 4) {
        piece(wave < 2 ? 3 : 2, wave & 1);
        if (wave >= 2) piece(wave - 2, 0);
    } else {
        if (wave < 6) piece(wave < 4 ? 3 - wave / 2 : wave - 4, wave < 4 ? wave & 1 : 0);
    }
}

// The memory behind a chunk: S times `keep`, and the rows of b times those of c.  c is weighed, and what that makes is held to 24 bits as a sum of operands (22
// in float16): the memory is kept in float32, and one rounding to 8 or 11 bits of every row would be left in it.
template <typename T, int W, int NB> __device__ __forceinline__ void remember(floats (&S)[NB], const tile<T, W> &b, const operand<T> (&c)[2], const powers &p, float keep, int across_b)
{
    const int g = (threadIdx.x & 63) >> 4;
    int e = 0;
    float w[2][8];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const floats lo = p.out[8 * t + 2 * g], hi = p.out[8 * t + 2 * g + 1];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[t][i] = (float)c[t][i] * (i < 4 ? lo[i & 3] : hi[i & 3]);
    }
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
    constexpr int KEPT = sizeof(T) == 4 ? 1 : NARROW<T> ? 2 : 3;
    operand<T> part[2][KEPT];
#pragma unroll
    for (int t = 0; t < 2; ++t) in_parts<T>(w[t], part[t]);
#pragma unroll
    for (int bt = 0; bt < NB; ++bt) {
        const operand<T> b0 = b.across_spread(across_b, 0, bt / 2, bt % 2), b1 = b.across_spread(across_b, 1, bt / 2, bt % 2);
        floats x = NARROW<T> ? (floats)0.0f : S[bt];
        if constexpr (!NARROW<T>)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] *= keep;
#pragma unroll
        for (int q = KEPT - 1; q >= 0; --q) {
            x = product(b0, part[0][q], x);
            x = product(b1, part[1][q], x);
        }
        if constexpr (NARROW<T>) {
            const float up = ldexpf(1.0f, e);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = fmaf(S[bt][j], keep, x[j] * up);
        }
        S[bt] = x;
        // Tile after tile: of eight at a time, registers go to memory and back (64000 rows, 8 heads of 128, float16, the gradient 680 us, 532 so).
        if constexpr (W == 128 && sizeof(T) == 2) __builtin_amdgcn_sched_barrier(0);
    }
    if constexpr (sizeof(T) == 4) settle(S);
}

// Results, a wave's 16 columns, transposed: o[it] are rows 16 it, a lane has four entries of a row.  What the memory before the chunk gives them (`weight`: the power of l
// that is missing in the first 16 rows, `tile_on` what is in the next) ...
template <bool EARLY, typename T, int W, typename Part>
__device__ __forceinline__ void from_operands(floats (&o)[4], tile<T, W> &a, Part &&part, float weight, float tile_on, int along_a)
{
    operand<T> s[2][PARTS<T>], x[2][4];
    const auto read = [&](int kb) {
        part(kb, s[kb & 1]);
#pragma unroll
        for (int it = 0; it < 4; ++it) x[kb & 1][it] = a.along(along_a, it, kb);
    };
#pragma unroll
    for (int it = 0; it < 4; ++it) o[it] = (floats)0.0f;
    read(0);
#pragma unroll
    for (int kb = 0; kb < W / 32; ++kb) {
        if (kb + 1 < W / 32) read(kb + 1);
        reads_before_products<EARLY>();
#pragma unroll
        for (int q = PARTS<T> - 1; q >= 0; --q)
#pragma unroll
            for (int it = 0; it < 4; ++it) o[it] = product(s[kb & 1][q], x[kb & 1][it], o[it]);
        reads_before_products<EARLY>();
    }
    if constexpr (sizeof(T) == 4) settle(o);
#pragma unroll
    for (int it = 0; it < 4; ++it) {
#pragma unroll
        for (int j = 0; j < 4; ++j) o[it][j] *= weight;
        weight *= tile_on;
    }
}
template <bool EARLY, typename T, int W, int NB>
__device__ __forceinline__ void from_memory(floats (&o)[4], tile<T, W> &a, const floats (&S)[NB], float weight, float tile_on, int along_a)
{
    const int e = exponent_of<T>(S);
    const float down = NARROW<T> ? ldexpf(1.0f, -e) : 1.0f;
    from_operands<EARLY>(o, a, [&](int kb, operand<T> (&to)[PARTS<T>]) { as_operands<T>(S, kb, down, to); }, NARROW<T> ? ldexpf(weight, e) : weight, tile_on, along_a);
}
// ... and what the rows of the chunk add.
template <typename T>
__device__ __forceinline__ void from_rows(floats &o, const operand<T> (&c)[2], const operand<T> (&P)[2][PARTS<T>], const powers &w, int which, int it)
{
#pragma unroll
    for (int kb = 0; kb <= it / 2; ++kb) {
        floats more = NARROW<T> ? (floats)0.0f : o;
#pragma unroll
        for (int q = PARTS<T> - 1; q >= 0; --q) more = product(c[kb], P[kb][q], more);
        if constexpr (NARROW<T>) {
            const float up = ldexpf(1.0f, w.exponent[which][it][kb]);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] = fmaf(more[j], up, o[j]);
        } else {
            o = more;
        }
    }
    if constexpr (sizeof(T) == 4) settle(o);
}
template <typename T> __device__ __forceinline__ bagel_pack<T, 4> rounded(const floats &o, float scale)
{
    bagel_pack<T, 4> x;
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = (T)(o[j] * scale);
    return x;
}

// Whether results are finite: zero as long as they are.
__device__ __forceinline__ void look_at(float &seen, const floats &o)
{
#pragma unroll
    for (int j = 0; j < 4; ++j) seen = fmaf(o[j], 0.0f, seen);
}

// What a segment's length leaves of the memory before it.
template <typename T> __device__ __forceinline__ float kept(const bagel_attention_pass<T> &p, int state)
{
    return __builtin_amdgcn_exp2f(log2_decay(p, state) * (float)p.segment);
}

// The memory that a segment begins with: joined here, of what the segments before it have added, where that has not been done.
template <typename T, int NB> __device__ __forceinline__ void read_before(floats (&S)[NB], const bagel_attention_pass<T> &p, const place &at, int state, int column)
{
    const int64_t size = (int64_t)p.wb * p.wc, each = p.states * size;
    const float *from = p.first ? p.first + ((int64_t)at.sequence * p.states + state) * size : nullptr;
    const int64_t join = p.join ? at.further : 0;
    if (at.before >= 0) from = p.memories + ((join > 0 ? at.sequence : at.before) * p.states + state) * size;
    read_memory(S, from, p.step_b, p.step_c, column, p.wb, p.wc);
    if (join <= 0) return;
    const float keep = kept(p, state);
    from = p.memories + ((at.before + 1 - join) * p.states + state) * size;
    for (int64_t k = 0; k < join; ++k, from += each) {
        floats add[NB];
        read_memory(add, from, p.step_b, p.step_c, column, p.wb, p.wc);
#pragma unroll
        for (int bt = 0; bt < NB; ++bt)
#pragma unroll
            for (int j = 0; j < 4; ++j) S[bt][j] = fmaf(keep, S[bt][j], add[bt][j]);
    }
}

// A segment once more, row after row, a wave its 16 columns.  By chunks, what is not finite in a row reaches the rows of its chunk that come before it, whose weight is zero:
// zero times those is NaN.  So a wave that has seen results that are not finite makes all of its results again.  (To look at the operands in every step and to leave
// such ones out of the products took 14 to 17 % more time for its registers and branches; to look at the results takes 0 to 3 %.)
//   It needs nothing that the chunks have made, the kernel's arguments are read anew (`which`: of the passes that they hold), so that no register is taken in the loop.
template <typename T, int NB> __device__ __forceinline__ void again(int which)
{
    uint64_t arguments = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(arguments));
    const bagel_attention_pass<T> p = ((const bagel_attention_pass<T> *)arguments)[which];
    const int64_t first = (int64_t)p.sequences * p.states, work = by_dies(p.launched + blockIdx.x, first, first + p.further * p.states), number = work / p.states;
    const int state = (int)(work - number * p.states), column = afresh(threadIdx.x >> 6) * 16 + (threadIdx.x & 15);
    const place at = place_of(p, number);
    const int step = p.back ? -1 : 1, g = (threadIdx.x & 63) >> 4;
    const float decay = __builtin_amdgcn_exp2f(log2_decay(p, state));
    const auto entry = [&](const T *row, int bt, int j) {
        const int r = memory_row<NB>(bt, j);
        return r < p.wb ? (float)row[r] : 0.0f;
    };
    floats S[NB];
    read_before(S, p, at, state, column);
    for (int64_t n = 0; n < at.rows; ++n) {
        const int64_t row = at.base + step * n;
        const float keep = p.back ? 1.0f : decay, after = p.back ? decay : 1.0f;
#pragma unroll
        for (int bt = 0; bt < NB; ++bt)
#pragma unroll
            for (int j = 0; j < 4; ++j) S[bt][j] *= keep;
        for (int h = 0; h < p.ks; ++h) {
            const T *b = p.b.at(row, state * p.ks + h);
            const float c = column < p.wc ? (float)p.c.at(row, state * p.ks + h)[column] * p.scale_b : 0.0f;
#pragma unroll
            for (int bt = 0; bt < NB; ++bt)
#pragma unroll
                for (int j = 0; j < 4; ++j) S[bt][j] = fmaf(entry(b, bt, j), c, S[bt][j]);
        }
        for (int h = 0; h < p.qs; ++h) {
            const T *a = p.a.at(row, state * p.qs + h);
            float o = 0.0f;
#pragma unroll
            for (int bt = 0; bt < NB; ++bt)
#pragma unroll
                for (int j = 0; j < 4; ++j) o = fmaf(entry(a, bt, j), S[bt][j], o);
            o += __shfl_xor(o, 16);
            o += __shfl_xor(o, 32);
            if (g == 0 && column < p.wc) p.out.at(row, state * p.qs + h)[column] = (T)(o * p.scale);
        }
#pragma unroll
        for (int bt = 0; bt < NB; ++bt)
#pragma unroll
            for (int j = 0; j < 4; ++j) S[bt][j] *= after;
    }
}
// All of a workgroup's results are in memory.
__device__ __forceinline__ void all_written()
{
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
}

// Goes through a segment's rows: `ask(tiles, base, h)` asks for the 64 rows from `base` on of head h, ask_few for those that are there of fewer, and `go(tiles,
// h, n, base, next)` takes a step: it puts the tiles away and calls `next`, which asks for those of the steps to come: DEEP of them are on their way.  Behind the
// last ones the same are asked for again, which nobody reads: a branch around the loads would make every wait one for all of them.
template <int DEEP, bool ONE_HEAD, typename Tiles, typename Ask, typename Few, typename Go>
__device__ __forceinline__ void go_through(const place &at, int heads, int step, Tiles (&coming)[DEEP], Ask &&ask, Few &&ask_few, Go &&go)
{
    static_assert(DEEP == 1 || DEEP == 2, "steps on their way");
    const int64_t chunks = at.rows / CHUNK;
    const int rest = (int)(at.rows % CHUNK);
    int64_t ask_chunk = 0, chunk = 0;
    int ask_head = 0, h = 0;
    const auto ask_next = [&](Tiles &to) {
        ask(to, at.base + step * min(ask_chunk * CHUNK, at.rows - CHUNK), ask_head);
        if (ONE_HEAD || ++ask_head == heads) {
            ask_head = 0;
            ++ask_chunk;
        }
    };
    const auto whole_step = [&](const Tiles &come, Tiles &then) {
        go(come, h, CHUNK, at.base + step * (chunk * CHUNK), [&] { ask_next(then); });
        if (ONE_HEAD || ++h == heads) {
            h = 0;
            ++chunk;
        }
    };
    if constexpr (DEEP == 1) {
        if (chunks > 0) ask_next(coming[0]);
        while (chunk < chunks) whole_step(coming[0], coming[0]);
    } else {
        // Two steps to a round, after one on its own where they are odd in number; what is left is then on its way in the first place.
        if ((chunks * heads) & 1) {
            Tiles alone;
            ask_next(alone);
            ask_next(coming[0]);
            whole_step(alone, coming[1]);
        } else if (chunks > 0) {
            ask_next(coming[0]);
            ask_next(coming[1]);
        }
        while (chunk < chunks) {
            whole_step(coming[0], coming[0]);
            whole_step(coming[1], coming[1]);
        }
    }
    if (rest == 0) return;
    // the rows that are left: further heads, or all of them where there are no others, are not on their way yet
    for (h = 0; h < heads; ++h) {
        if (chunks == 0) ask_few(coming[0], h, rest);
        else if (h > 0) ask(coming[0], at.base + step * (at.rows - CHUNK), h);
        go(coming[0], h, rest, at.base + step * (chunks * CHUNK), [] {});
    }
}

// How many heads there are to a memory: one; several of a and out; several of b and c, whose sums are made in turn.
enum heads_kind { ONE, MANY_A, MANY_B };

template <typename T> struct two_passes {
    bagel_attention_pass<T> p[2];
};

// What a segment adds to the memory, or, of the first one of a sequence, the memory behind it.  Segments that are the last of theirs are nobody's to add, so there are
// as many to do as further ones, each of which waits for the one before it.
//   It reads b and c once more than the pass itself: one head of 128 in bf16, 131072 rows, 2 memories, 42 us (134 MB, 3.2 TB/s).
template <typename T, int WB, int WC, bool WHOLE, bool MANY> __global__ __launch_bounds__(4 * WC, 2) void sums_kernel(two_passes<T> both)
{
    bagel_attention_pass<T> p = blockIdx.y ? both.p[1] : both.p[0];
    if constexpr (WHOLE) {
        p.wb = WB;
        p.wc = WC;
    }
    constexpr int THREADS = 4 * WC;
    __shared__ tile<T, WB> sb;
    __shared__ tile<T, WC> sc;
    __shared__ powers w;
    const int64_t work = by_dies(p.launched + blockIdx.x, 0, p.further * p.states), further = work / p.states;
    const int state = (int)(work - further * p.states);
    const place behind_it = place_of(p, p.sequences + further);
    if (!behind_it.there) return;
    place at = behind_it;
    at.rows = p.segment;
    at.base = behind_it.base + (p.back ? p.segment : -p.segment);
    const bool first = behind_it.before < p.sequences;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), column = wave * 16 + (threadIdx.x & 15), step = p.back ? -1 : 1;
    const float l2 = log2_decay(p, state), whole = power(l2, CHUNK);
    floats S[WB / 16];
    const int64_t size = (int64_t)p.wb * p.wc;
    read_memory(S, first && p.first ? p.first + ((int64_t)at.sequence * p.states + state) * size : nullptr, p.step_b, p.step_c, column, p.wb, p.wc);
    w.weigh_out(l2, p.back ? 1 : 0, p.scale_b, CHUNK);
    const lane_parts<T, WB, WC, THREADS> l;
    if constexpr (!WHOLE) {
        clear(sb, p.wb);
        clear(sc, p.wc);
    }
    struct tiles {
        incoming<T, WB, THREADS> b;
        incoming<T, WC, THREADS> c;
    } coming[2];
    const int heads = MANY ? p.ks : 1;
    go_through<2, !MANY>(at, heads, step, coming,
        [&](tiles &to, int64_t base, int h) {
            to.b.load(p.b.at(base, state * heads + h), step * p.b.stride, p.wb);
            to.c.load(p.c.at(base, state * heads + h), step * p.c.stride, p.wc);
        },
        [](tiles &, int, int) {},
        [&](const tiles &come, int h, int n, int64_t, auto &&next) {
            __syncthreads();
            come.b.put(sb, l.pack_b, n, p.wb);
            come.c.put(sc, l.pack_c, n, p.wc);
            __syncthreads();
            next();
            const operand<T> c[2] = {sc.across(l.across_c, 0, wave), sc.across(l.across_c, 1, wave)};
            remember(S, sb, c, w, MANY && h > 0 ? 1.0f : whole, l.across_b);
        });
    write_memory(S, p.memories + (behind_it.before * p.states + state) * size, p.step_b, p.step_c, column, p.wb, p.wc);
}

// What segments have added to the memory, into the memory behind each: a thread to an entry, along its sequence's segments but the last, 16 of which are asked for at
// a time (121 segments of 2 memories of 128 x 128: 14 us).
template <typename T> __global__ __launch_bounds__(256) void memories_kernel(two_passes<T> both, int blocks)
{
    const bagel_attention_pass<T> p = blockIdx.y ? both.p[1] : both.p[0];
    const int size = p.wb * p.wc;
    for (int64_t work = blockIdx.x; work < (int64_t)p.sequences * p.states * blocks; work += gridDim.x) {
        const int state = (int)(work / blocks % p.states), sequence = (int)(work / blocks / p.states);
        int64_t begin, end;
        sequence_rows(p, sequence, begin, end);
        const int64_t first = p.offsets ? begin / p.segment : sequence * further_of_each(p), each = (int64_t)p.states * size;
        const int64_t n = min((end - begin + p.segment - 1) / p.segment - 2, p.further - first);     // segments to join: neither the first nor the last
        if (n < 1) continue;
        const float keep = kept(p, state);
        for (int i = (int)(work % blocks) * 256 + threadIdx.x; i < size; i += blocks * 256) {
            float s = p.memories[((int64_t)sequence * p.states + state) * size + i];
            float *m = p.memories + ((p.sequences + first) * p.states + state) * size + i;
            constexpr int AHEAD = 16;
            for (int64_t k = 0; k < n; k += AHEAD) {
                float add[AHEAD];
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) add[j] = k + j < n ? m[(k + j) * each] : 0.0f;
#pragma unroll
                for (int j = 0; j < AHEAD; ++j)
                    if (k + j < n) m[(k + j) * each] = s = fmaf(keep, s, add[j]);
            }
        }
    }
}

// A pass over a segment.  A wave to 16 columns of a memory, of c and of out, in float32 in its registers.  The rows' products with each other, P, are shared out
// among the waves by pieces (16 rows of it, 32 rows they are multiplied with), and meet in shared memory.
// WHOLE: a and b are as wide as their tiles, and so are c and out.
//   In 16 bits the memory's rate bounds it, and beside it what a step takes between its barriers: 64000 rows, 8 heads of 64, bf16, 59 to 65 us (262 MB, 4.4 to 4.0 TB/s); 131072
// rows, 8 heads of 128 on 2 memories 182 to 202 us (671 MB, 3.7 to 3.3 TB/s).  What brought the former there, in whole calls: one chunk of the next step on its way 175 -> 129 us
// (with other launches), loads without a branch and results in packs -> 79, slots without bank conflicts and two steps on their way -> 62, few segments' memories
// joined by themselves -> 57, memories and P in two operands -> 63.
//   Two waves to a SIMD are all that a lane's 190 to 256 registers leave room for: two workgroups to a compute unit with values of 64, one with 128.  (Their tiles take 50 to 82 KB
// in 16 bits, 66 to 146 with a memory held for several heads, 69 to 117 in 32.)  So what is on its way, not how many waves there are, keeps the memory busy.  In 32 bits
// the matrix instructions have a sixteenth of the rate, and padded widths count as whole.
template <typename T, int WB, int WC, bool WHOLE, heads_kind HEADS> __global__ __launch_bounds__(4 * WC, 2) void chunks_kernel(bagel_attention_pass<T> p)
{
    if constexpr (WHOLE) {
        p.wb = WB;
        p.wc = WC;
    }
    constexpr int WAVES = WC / 16, THREADS = 4 * WC, DEEP = NARROW<T> && WB == 128 && WC == 64 && HEADS == ONE ? 1 : 2;       // steps on their way
    // Results go through shared memory, and from there while the next step's tiles come, so that rows are written in packs; in 32 bits a lane has a pack
    constexpr bool THROUGH = sizeof(T) == 2;
    __shared__ tile<T, WB> sa, sb;
    __shared__ tile<T, WC> sc;
    __shared__ pieces_of<T> sp;
    __shared__ tile<T, THROUGH ? WC : 16> so;
    __shared__ powers w;
    const int64_t first = (int64_t)p.sequences * p.states, all = first + p.further * p.states, group = p.launched + blockIdx.x;
    if (group >= all) return bagel_clear_behind(p, group - all, p.groups - all);
    const int64_t work = by_dies(group, first, all), number = work / p.states;
    const int state = (int)(work - number * p.states);
    const place at = place_of(p, number);
    if (!at.there) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = (threadIdx.x & 63) >> 4, j16 = threadIdx.x & 15, column = wave * 16 + j16;
    const float l2 = log2_decay(p, state);
    const int step = p.back ? -1 : 1, behind = p.back ? 1 : 0;       // of powers of l
    floats S[WB / 16];
    read_before(S, p, at, state, column);
    w.weigh_out(l2, behind, p.scale_b, CHUNK);
    w.weigh_p(l2, p.scale_b);
    const float tile_on = power(l2, 16), weight_in = power(l2, j16 + 1 - behind), whole = power(l2, CHUNK);
    const lane_parts<T, WB, WC, THREADS> l;
    if constexpr (!WHOLE) {
        clear(sa, p.wb);
        clear(sb, p.wb);
        clear(sc, p.wc);
    }
    const int heads = HEADS == MANY_B ? p.ks : HEADS == MANY_A ? p.qs : 1;
    const auto head_a = [&](int h) { return HEADS == MANY_A ? state * heads + h : state; };
    const auto head_b = [&](int h) { return HEADS == MANY_B ? state * heads + h : state; };
    // Two steps are on their way, as one alone would leave too little of the memory's rate in use (float16, 128 x 64, has no registers for two: 64000 rows, 8 heads, 172 us
    // with two, 112 with one).  (What is asked for in every step comes last: what is waited for
    // is counted from there, whether there were others or not.)
    struct tiles {
        incoming<T, WB, THREADS> a, b;
        incoming<T, WC, THREADS> c;
    } coming[DEEP];
    // Several heads of queries read one memory: it becomes operands for the first of them, which the others find in shared memory, a wave its own (131072 rows, 8 heads of 64 on
    // 2 memories, bf16: 127 us made for every head, 119 so).  In 128 x 64 two workgroups of a compute unit would not have the room.
    constexpr bool HELD = HEADS == MANY_A && AHEAD<T, WB, WC>;
    __shared__ operand<T> held[HELD ? WAVES : 1][WB / 32][PARTS<T>][64];
    int exponent = 0;
    floats O[4];
    float seen = 0.0f;
    T *ready = nullptr;                              // where the rows in `so` go, and how many there are
    int ready_rows = 0;
    const auto flush = [&] {
        if constexpr (THROUGH)
            if (ready) write_rows<T, WC, THREADS>(so, l.pack_c, ready, step * p.out.stride, ready_rows, p.wc);
    };
    go_through<DEEP, HEADS == ONE>(at, heads, step, coming,
        [&](tiles &to, int64_t base, int h) {
            const auto ask_a = [&] { to.a.load(p.a.at(base, head_a(h)), step * p.a.stride, p.wb); };
            const auto ask_b = [&] {
                to.b.load(p.b.at(base, head_b(h)), step * p.b.stride, p.wb);
                to.c.load(p.c.at(base, head_b(h)), step * p.c.stride, p.wc);
            };
            if constexpr (HEADS == MANY_B) {
                if (h == 0) ask_a();
                ask_b();
            } else {
                if (h == 0) ask_b();
                ask_a();
            }
        },
        [&](tiles &to, int h, int n) {
            to.a.load_few(p.a.at(at.base, head_a(h)), n, step * p.a.stride, p.wb);
            to.b.load_few(p.b.at(at.base, head_b(h)), n, step * p.b.stride, p.wb);
            to.c.load_few(p.c.at(at.base, head_b(h)), n, step * p.c.stride, p.wc);
        },
        [&](const tiles &come, int h, const int n, int64_t base, auto &&next) {
            __syncthreads();
            flush();
            if (HEADS != MANY_B || h == 0) come.a.put(sa, l.pack_b, n, p.wb);
            if (HEADS == MANY_B || h == 0) {
                come.b.put(sb, l.pack_b, n, p.wb);
                come.c.put(sc, l.pack_c, n, p.wc);
            }
            if (n != CHUNK) w.weigh_out(l2, behind, p.scale_b, n);
            __syncthreads();
            next();
            const bool enter = HEADS != MANY_B || h == 0, leave = HEADS != MANY_B || h == heads - 1;
            const operand<T> c[2] = {sc.across(l.across_c, 0, wave), sc.across(l.across_c, 1, wave)};
            if constexpr (HELD) {
                const int lane = threadIdx.x & 63;
                if (h == 0) {
                    exponent = exponent_of<T>(S);
                    const float down = NARROW<T> ? ldexpf(1.0f, -exponent) : 1.0f;
#pragma unroll
                    for (int kb = 0; kb < WB / 32; ++kb) {
                        operand<T> s[PARTS<T>];
                        as_operands<T>(S, kb, down, s);
#pragma unroll
                        for (int q = 0; q < PARTS<T>; ++q) held[wave][kb][q][lane] = s[q];
                    }
                }
                from_operands<AHEAD<T, WB, WC>>(
                    O, sa,
                    [&](int kb, operand<T> (&to)[PARTS<T>]) {
#pragma unroll
                        for (int q = 0; q < PARTS<T>; ++q) to[q] = held[wave][kb][q][lane];
                    },
                    NARROW<T> ? ldexpf(weight_in, exponent) : weight_in, tile_on, l.along_a);
            } else if (enter && p.out.data) {
                from_memory<AHEAD<T, WB, WC>>(O, sa, S, weight_in, tile_on, l.along_a);
            }
            make_pieces<AHEAD<T, WB, WC>, WAVES>(sa, sb, sp, w, 0, tile_on, l.along_a, l.spread_b, wave);
            if (HEADS == MANY_B || h == heads - 1) remember(S, sb, c, w, HEADS == MANY_B && h > 0 ? 1.0f : n == CHUNK ? whole : power(l2, n), l.across_b);
            __syncthreads();
            if (!p.out.data) return;
            T *const out = p.out.at(base, head_a(h));
            operand<T> P[2][2][PARTS<T>];
            sp.get(P[0], 0);
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                floats &o = O[it];
                if (it < 3) sp.get(P[(it + 1) & 1], it + 1);
                reads_before_products<AHEAD<T, WB, WC>>();
                from_rows(o, c, P[it & 1], w, 0, it);
                if constexpr (HEADS == MANY_B) settle(o);
                if (!leave) continue;
                look_at(seen, o);
                const bagel_pack<T, 4> x = rounded<T>(o, p.scale);
                if constexpr (THROUGH) {
                    so.entries(l.entries_o, it, wave) = x;
                } else {
                    const int from = 16 * wave + 4 * g;
                    if (16 * it + j16 >= n || from >= p.wc) continue;
                    T *to = out + (16 * it + j16) * (step * p.out.stride) + from;
                    if (from + 4 <= p.wc) reinterpret_cast<bagel_loose_pack<T, 4> *>(to)->x = x;
                    else
#pragma unroll
                        for (int j = 0; j < 3; ++j)
                            if (from + j < p.wc) to[j] = x[j];
                }
            }
            ready = leave ? out : nullptr;
            ready_rows = n;
        });
    if constexpr (THROUGH) {
        __syncthreads();
        flush();
    }
    if (at.last && p.last) write_memory(S, p.last + ((int64_t)at.sequence * p.states + state) * p.wb * p.wc, p.step_b, p.step_c, column, p.wb, p.wc);
    all_written();
    if (__any(seen != 0.0f)) again<T, WB / 16>(0);
}

// The gradients of keys and values: two such passes at once, whose memories are each other's transpose, from the same tiles.  Four tiles are read in the place of six
// (64000 rows, 8 heads of 64, bf16: 98 to 108 us for 393 MB, 4.0 to 3.6 TB/s; when it took 92, two passes one after the other took 130).
template <typename T, int W, bool WHOLE, bool MANY> __global__ __launch_bounds__(4 * W, 2) void keys_kernel(bagel_attention_pass<T> p, bagel_attention_pass<T> q)
{
    if constexpr (WHOLE) p.wb = p.wc = q.wb = q.wc = W;
    constexpr int WAVES = W / 16, THREADS = 4 * W;
    constexpr bool EARLY = W == 64;                  // two memories of 128 leave no registers for what is read ahead (8 heads of 100, float16, 712 us with it, 644 without)
    __shared__ tile<T, W> sk, sv, sq, sd, so[2];
    __shared__ pieces_of<T> sp[2];
    __shared__ powers w;
    const int64_t first = (int64_t)p.sequences * p.states, all = first + p.further * p.states, group = p.launched + blockIdx.x;
    if (group >= all) {
        bagel_clear_behind(p, group - all, p.groups - all);
        return bagel_clear_behind(q, group - all, p.groups - all);
    }
    const int64_t work = by_dies(group, first, all), number = work / p.states;
    const int state = (int)(work - number * p.states);
    const place at = place_of(p, number);
    if (!at.there) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), column = wave * 16 + (threadIdx.x & 15);
    const float l2 = log2_decay(p, state);
    floats R[W / 16], Rt[W / 16];
    read_before(R, p, at, state, column);
    read_before(Rt, q, at, state, column);
    w.weigh_out(l2, 1, p.scale_b, CHUNK);
    w.weigh_p(l2, p.scale_b);
    const float tile_on = power(l2, 16), weight_in = power(l2, threadIdx.x & 15), whole = power(l2, CHUNK);
    const lane_parts<T, W, W, THREADS> l;
    if constexpr (!WHOLE) {
        clear(sk, p.wb);
        clear(sq, p.wb);
        clear(sv, p.wc);
        clear(sd, p.wc);
    }
    const int heads = MANY ? p.ks : 1;
    struct tiles {
        incoming<T, W, THREADS> k, v, q, d;
    } coming[1];
    floats O[2][4];
    float seen[2] = {0.0f, 0.0f};
    T *ready[2] = {nullptr, nullptr};
    int ready_rows = 0;
    const auto flush = [&] {
        if (ready[0]) write_rows<T, W, THREADS>(so[0], l.pack_b, ready[0], -p.out.stride, ready_rows, p.wc);
        if (ready[1]) write_rows<T, W, THREADS>(so[1], l.pack_b, ready[1], -q.out.stride, ready_rows, q.wc);
    };
    go_through<1, !MANY>(at, heads, -1, coming,
        [&](tiles &to, int64_t base, int h) {
            if (!MANY || h == 0) {
                to.k.load(p.a.at(base, state), -p.a.stride, p.wb);
                to.v.load(q.a.at(base, state), -q.a.stride, p.wc);
            }
            to.q.load(p.b.at(base, state * heads + h), -p.b.stride, p.wb);
            to.d.load(p.c.at(base, state * heads + h), -p.c.stride, p.wc);
        },
        [&](tiles &to, int h, int n) {
            to.k.load_few(p.a.at(at.base, state), n, -p.a.stride, p.wb);
            to.v.load_few(q.a.at(at.base, state), n, -q.a.stride, p.wc);
            to.q.load_few(p.b.at(at.base, state * heads + h), n, -p.b.stride, p.wb);
            to.d.load_few(p.c.at(at.base, state * heads + h), n, -p.c.stride, p.wc);
        },
        [&](const tiles &come, int h, const int n, int64_t base, auto &&next) {
            __syncthreads();
            flush();
            if (!MANY || h == 0) {
                come.k.put(sk, l.pack_b, n, p.wb);
                come.v.put(sv, l.pack_b, n, p.wc);
            }
            come.q.put(sq, l.pack_b, n, p.wb);
            come.d.put(sd, l.pack_b, n, p.wc);
            if (n != CHUNK) w.weigh_out(l2, 1, p.scale_b, n);
            __syncthreads();
            next();
            const bool enter = !MANY || h == 0, leave = !MANY || h == heads - 1;
            const float keep = MANY && h > 0 ? 1.0f : n == CHUNK ? whole : power(l2, n);
            const operand<T> d[2] = {sd.across(l.across_c, 0, wave), sd.across(l.across_c, 1, wave)}, c[2] = {sq.across(l.across_c, 0, wave), sq.across(l.across_c, 1, wave)};
            if (enter) {
                from_memory<EARLY>(O[0], sk, R, weight_in, tile_on, l.along_a);
                from_memory<EARLY>(O[1], sv, Rt, weight_in, tile_on, l.along_a);
            }
            make_pieces<EARLY, WAVES>(sk, sq, sp[0], w, 0, tile_on, l.along_a, l.spread_b, wave);
            make_pieces<EARLY, WAVES>(sv, sd, sp[1], w, 1, tile_on, l.along_a, l.spread_b, WAVES - 1 - wave);
            remember(R, sq, d, w, keep, l.across_b);
            remember(Rt, sd, c, w, keep, l.across_b);
            __syncthreads();
            const auto results = [&](const operand<T> (&x)[2], int which) {
                operand<T> P[2][2][PARTS<T>];
                sp[which].get(P[0], 0);
#pragma unroll
                for (int it = 0; it < 4; ++it) {
                    floats &o = O[which][it];
                    if (it < 3) sp[which].get(P[(it + 1) & 1], it + 1);
                    reads_before_products<EARLY>();
                    from_rows(o, x, P[it & 1], w, which, it);
                    if constexpr (MANY) settle(o);
                    if (!leave) continue;
                    look_at(seen[which], o);
                    so[which].entries(l.entries_o, it, wave) = rounded<T>(o, 1.0f);
                }
            };
            results(d, 0);
            results(c, 1);
            ready[0] = leave ? p.out.at(base, state) : nullptr;
            ready[1] = leave ? q.out.at(base, state) : nullptr;
            ready_rows = n;
        });
    __syncthreads();
    flush();
    if (at.last && p.last) write_memory(R, p.last + ((int64_t)at.sequence * p.states + state) * p.wb * p.wc, p.step_b, p.step_c, column, p.wb, p.wc);
    all_written();
    if (__any(seen[0] != 0.0f)) again<T, W / 16>(0);
    if (__any(seen[1] != 0.0f)) again<T, W / 16>(1);
}

// f with constants for the widths of the tiles, and whether the rows fill them.
template <typename T, typename F> void by_widths(const bagel_attention_pass<T> &p, F &&f)
{
    const std::integral_constant<int, 64> narrow;
    const std::integral_constant<int, 128> wide;
    const auto filled = [&](auto wb, auto wc) {
        if (p.wb == wb && p.wc == wc) f(wb, wc, std::true_type());
        else f(wb, wc, std::false_type());
    };
    if (p.wb <= 64) p.wc <= 64 ? filled(narrow, narrow) : filled(narrow, wide);
    else p.wc <= 64 ? filled(wide, narrow) : filled(wide, wide);
}

template <typename T> int64_t groups_of(const bagel_attention_pass<T> &p)
{
    return (p.sequences + p.further) * p.states + (p.offsets && p.out.data && p.rows > 0 ? 32 : 0);
}

}  // namespace

template <typename T> hipError_t bagel_launch_attention_memories(const bagel_attention_pass<T> *passes, int n, hipStream_t stream)
{
    two_passes<T> both;
    both.p[0] = passes[0];
    both.p[1] = passes[n - 1];
    const bagel_attention_pass<T> &p = both.p[0];
    const int64_t work = p.further * p.states;
    if (work == 0) return hipSuccess;
    hipError_t e = hipSuccess;
    const bool many = p.ks > 1 || both.p[1].ks > 1;
    by_widths(p, [&](auto wb, auto wc, auto whole) {
        constexpr int WB = decltype(wb)::value, WC = decltype(wc)::value;
        e = bagel_attention_launches(work, [&](unsigned groups, int64_t before) {
            both.p[0].launched = both.p[1].launched = before;
            if (many) sums_kernel<T, WB, WC, decltype(whole)::value, true><<<dim3(groups, n), 4 * WC, 0, stream>>>(both);
            else sums_kernel<T, WB, WC, decltype(whole)::value, false><<<dim3(groups, n), 4 * WC, 0, stream>>>(both);
        });
    });
    if (p.join || e != hipSuccess) return e;
    // some workgroups to a memory where there are few of them
    const int64_t all = (int64_t)p.sequences * p.states, most = (p.wb * p.wc + 255) / 256, wanted = 1024 / all;
    const int blocks = (int)(wanted < 1 ? 1 : wanted < most ? wanted : most);
    memories_kernel<T><<<dim3((unsigned)(all * blocks < 1 << 16 ? all * blocks : 1 << 16), n), 256, 0, stream>>>(both, blocks);
    return hipGetLastError();
}

template <typename T> hipError_t bagel_launch_attention_pass(const bagel_attention_pass<T> &pass, hipStream_t stream)
{
    bagel_attention_pass<T> p = pass;
    p.groups = groups_of(p);
    hipError_t e = hipSuccess;
    by_widths(p, [&](auto wb, auto wc, auto whole) {
        constexpr int WB = decltype(wb)::value, WC = decltype(wc)::value;
        constexpr bool WHOLE = decltype(whole)::value;
        e = bagel_attention_launches(p.groups, [&](unsigned groups, int64_t before) {
            p.launched = before;
            if (p.ks > 1) chunks_kernel<T, WB, WC, WHOLE, MANY_B><<<groups, 4 * WC, 0, stream>>>(p);
            else if (p.qs > 1) chunks_kernel<T, WB, WC, WHOLE, MANY_A><<<groups, 4 * WC, 0, stream>>>(p);
            else chunks_kernel<T, WB, WC, WHOLE, ONE><<<groups, 4 * WC, 0, stream>>>(p);
        });
    });
    return e;
}

template <typename T> hipError_t bagel_launch_attention_keys(const bagel_attention_pass<T> &values, const bagel_attention_pass<T> &keys, hipStream_t stream)
{
    bagel_attention_pass<T> p = values, q = keys;
    p.groups = q.groups = groups_of(p);
    hipError_t e = hipSuccess;
    const auto launch = [&](auto w, auto whole) {
        constexpr int W = decltype(w)::value;
        constexpr bool WHOLE = decltype(whole)::value;
        e = bagel_attention_launches(p.groups, [&](unsigned groups, int64_t before) {
            p.launched = q.launched = before;
            if constexpr (W == 64)
                if (p.ks > 1) return keys_kernel<T, W, WHOLE, true><<<groups, 4 * W, 0, stream>>>(p, q);
            keys_kernel<T, W, WHOLE, false><<<groups, 4 * W, 0, stream>>>(p, q);
        });
    };
    const std::integral_constant<int, 64> narrow;
    const std::integral_constant<int, 128> wide;
    if (p.wb <= 64) p.wb == 64 && p.wc == 64 ? launch(narrow, std::true_type()) : launch(narrow, std::false_type());
    else p.wb == 128 && p.wc == 128 ? launch(wide, std::true_type()) : launch(wide, std::false_type());
    return e;
}
