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

// 64 rows in shared memory, read by rows and by columns.  In 16 bits the slots of 16 bytes of a row are permuted by a number of 3 bits that the row's place among 8
// gives: eight rows' slots of one number (along) and four rows' two slots beside each other (across) are then in different banks.  In 32 bits 16 bytes
// between the rows do.  A lane's part of an address is the same for all tiles of a width and made once; what differs is known to the compiler.
template <typename T, int W> struct tile {
    static constexpr bool PERMUTED = sizeof(T) == 2;
    static constexpr int pitch = PERMUTED ? W : W + 4, row_bytes = pitch * sizeof(T);
    alignas(32) T x[CHUNK * pitch];
    __device__ static __forceinline__ int number(int row) { return (row & 3) << 1 ^ (row & 1) ^ (row >> 2 & 1); }
    __device__ static __forceinline__ int place(int row, int column)     // of an entry
    {
        return row * pitch + (PERMUTED ? ((column >> 3 ^ number(row)) << 3) + (column & 7) : column);
    }
    __device__ static __forceinline__ int bytes(int row, int column) { return place(row, column) * (int)sizeof(T); }
    // `lane_part` (bytes) with `c` columns on, a multiple of 8 that the lane's own column does not carry into
    __device__ static __forceinline__ int on(int lane_part, int c) { return PERMUTED ? (lane_part ^ c % 64 * 2) + c / 64 * 128 : lane_part + c * (int)sizeof(T); }
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
        return in_bytes<operand<T>>((on(lane_part, 32 * t) ^ (PERMUTED ? half * 16 : 0)) + (r * 32 + half * 4) * row_bytes);
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
            const half hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((shared_half *)&in_bytes<half>((from ^ 16) + 4 * row_bytes));
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
    static_assert(apart % 8 == 0, "a thread's rows have the same place among 8");
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

// The wait states between the products in 32 bits and whatever uses their results, ahead of a branch: the compiler may count them along the longer way only.
template <int N> __device__ __forceinline__ void settle(floats (&x)[N])
{
    static_assert(N == 4 || N == 8, "a memory's tiles");
    if constexpr (N == 4) asm volatile("s_nop 9" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]));
    else asm volatile("s_nop 9" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]), "+v"(x[4]), "+v"(x[5]), "+v"(x[6]), "+v"(x[7]));
}

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

// How many heads there are to a memory: one; several of a and out; several of b and c, whose sums are made in turn.
enum heads_kind { ONE, MANY_A, MANY_B };

// A wave to 16 columns of a memory, of c and of out, in float32 in its registers.  The rows' products with each other, P, are shared out
// among the waves by pieces (16 rows of it, 32 rows they are multiplied with), of which six are not zero, and meet in shared memory.
// SUMS: only the memory behind the segment, from zero where it is not the first of its sequence.
// WHOLE: a and b are as wide as their tiles, and so are c and out.
template <typename T, int WB, int WC, bool WHOLE, bool SUMS, heads_kind HEADS, int ON_SIMD>
__global__ __launch_bounds__(4 * WC, ON_SIMD) void chunks_kernel(bagel_attention_pass<T> p)
{
    if constexpr (WHOLE) {
        p.wb = WB;
        p.wc = WC;
    }
    constexpr int NB = WB / 16, KB = WB / 32, WAVES = WC / 16, THREADS = 4 * WC;
    __shared__ tile<T, WB> sb;
    __shared__ tile<T, WC> sc;
    __shared__ tile<T, SUMS ? 16 : WB> sa;
    __shared__ tile<T, SUMS ? 16 : CHUNK> sp;
    // Results go through shared memory, and from there while the next step's tiles come, so that rows are written in packs; in 32 bits a lane has a pack
    constexpr bool THROUGH = !SUMS && sizeof(T) == 2;
    __shared__ tile<T, THROUGH ? WC : 16> so;
    __shared__ int sp_exponent[4][2];
    __shared__ floats weight_out[CHUNK / 4];         // powers of l from the rows to the memory behind the chunk
    __shared__ floats weight_p[SUMS ? 1 : 3][2][64]; // and between rows of a piece of P (a lane's eight entries), that begins 0, 16 and 32 rows before
    const int64_t segments = p.slots * p.states;
    if ((int64_t)blockIdx.x >= segments) return bagel_clear_behind(p, blockIdx.x - segments, gridDim.x - segments);
    // Workgroups go to the eight dies in turn.  Each die takes segments that follow each other, so that the heads of the same rows, which lie side by side in
    // memory, are read by one.
    const int64_t die = blockIdx.x % 8, work = die * (segments / 8) + min(die, segments % 8) + blockIdx.x / 8;
    const int64_t slot = work / p.states;
    const int state = (int)(work - slot * p.states);
    const place at = place_of(p, slot);
    if (!at.there || (SUMS && at.last)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, j16 = lane & 15;
    const int mine = wave * 16 + j16;                                // the lane's column of the memory
    const float l2 = fmaxf(p.log_decay[state], -1e30f) * 1.44269504f;
    const int step = p.back ? -1 : 1, behind = p.back ? 1 : 0;       // of powers of l

    // S[2 kb + half][j]: entry (32 kb + 8 g + 4 half + j, mine) of the memory
    floats S[NB];
    const auto row_of = [&](int bt, int j) { return bt / 2 * 32 + 8 * g + bt % 2 * 4 + j; };
    const int64_t size = (int64_t)p.wb * p.wc, memory = ((int64_t)at.sequence * p.states + state) * size;
    {
        const float *from = at.first ? p.first : SUMS ? nullptr : p.memories + ((slot - 1) * p.states + state) * size;
        const int64_t start = at.first ? memory : 0, step_b = at.first ? p.step_b : p.wc, step_c = at.first ? p.step_c : 1;
#pragma unroll
        for (int bt = 0; bt < NB; ++bt)
#pragma unroll
            for (int j = 0; j < 4; ++j) S[bt][j] = from && row_of(bt, j) < p.wb && mine < p.wc ? from[start + row_of(bt, j) * step_b + mine * step_c] : 0.0f;
    }
    const auto weigh_out = [&](int n) {
        if ((int)threadIdx.x < CHUNK) reinterpret_cast<float *>(weight_out)[threadIdx.x] = power(l2, max(n - 1 - (int)threadIdx.x, 0) + behind) * p.scale_b;
    };
    weigh_out(CHUNK);
    if constexpr (!SUMS)
        for (int i = wave; i < 6; i += WAVES) {
            floats x;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int d = 16 * (i / 2) + j16 - (8 * g + i % 2 * 4 + j);
                x[j] = d >= 0 ? power(l2, d) * p.scale_b : 0.0f;
            }
            weight_p[i / 2][i % 2][lane] = x;
        }
    // 48 rows before: l^16 more than 32.  From a row to the memory before the chunk; over a chunk:
    const float tile_on = power(l2, 16), weight_in = power(l2, j16 + 1 - behind), whole = power(l2, CHUNK);

    // a lane's parts of addresses in shared memory
    const int along_a = tile<T, WB>::lane_along(), along_p = tile<T, CHUNK>::lane_along(), spread_b = tile<T, WB>::lane_spread();
    const int across_b = tile<T, WB>::lane_across(true), across_c = tile<T, WC>::lane_across(false), entries_o = tile<T, WC>::lane_entries();
    const int pack_b = packs_of<T, WB, THREADS>::lane_part(), pack_c = packs_of<T, WC, THREADS>::lane_part();
    if constexpr (!WHOLE) {
        clear(sb, p.wb);
        clear(sc, p.wc);
        if constexpr (!SUMS) clear(sa, p.wb);
    }
    const int heads = HEADS == MANY_B ? p.ks : HEADS == MANY_A && !SUMS ? p.qs : 1;
    const auto head_a = [&](int h) { return HEADS == MANY_A ? state * heads + h : state; };
    const auto head_b = [&](int h) { return HEADS == MANY_B ? state * heads + h : state; };
    // The tiles of a step, on their way: two steps' at a time, as one alone would leave too little of the memory's rate in use
    struct tiles {
        incoming<T, SUMS ? 64 : WB, THREADS> a;
        incoming<T, WB, THREADS> b;
        incoming<T, WC, THREADS> c;
    } coming[2];
    const auto ask = [&](tiles &to, int64_t base, int h) {
        // (those of every step come last: what is waited for is counted from there, whether there were others or not)
        const auto ask_a = [&] {
            if constexpr (!SUMS) to.a.load(p.a.at(base, head_a(h)), step * p.a.stride, p.wb);
        };
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
    };
    const auto ask_few = [&](tiles &to, int h, int n) {
        if constexpr (!SUMS)
            if (HEADS != MANY_B || h == 0) to.a.load_few(p.a.at(at.base, head_a(h)), n, step * p.a.stride, p.wb);
        if (HEADS == MANY_B || h == 0) {
            to.b.load_few(p.b.at(at.base, head_b(h)), n, step * p.b.stride, p.wb);
            to.c.load_few(p.c.at(at.base, head_b(h)), n, step * p.c.stride, p.wc);
        }
    };
    floats O[HEADS == MANY_B ? 4 : 1];
    // One step: head h of the chunk at `base`, of which n rows are there, whose tiles were asked for.  `next` asks for the next one's; `before` takes away what
    // the step before left in `so`.
    const auto go = [&](const tiles &come, int h, const int n, T *out, auto &&before, auto &&next) {
        __syncthreads();
        before();
        if constexpr (!SUMS)
            if (HEADS != MANY_B || h == 0) come.a.put(sa, pack_b, n, p.wb);
        if (HEADS == MANY_B || h == 0) {
            come.b.put(sb, pack_b, n, p.wb);
            come.c.put(sc, pack_c, n, p.wc);
        }
        if (n != CHUNK) weigh_out(n);
        __syncthreads();
        next();

        operand<T> c[2];
#pragma unroll
        for (int t = 0; t < 2; ++t) c[t] = sc.across(across_c, t, wave);
        const bool enter = !SUMS && (HEADS != MANY_B || h == 0), leave = !SUMS && (HEADS != MANY_B || h == heads - 1);
        // the memory before the chunk as operands
        operand<T> s[KB];
        int s_exponent = 0;
        if (enter) {
            float down = 1.0f;
            if constexpr (NARROW<T>) {
                float top = 0.0f;
#pragma unroll
                for (int bt = 0; bt < NB; ++bt)
#pragma unroll
                    for (int j = 0; j < 4; ++j) top = fmaxf(top, fabsf(S[bt][j]));
                s_exponent = exponent_for(wave_largest(top));
                down = ldexpf(1.0f, -s_exponent);
            }
#pragma unroll
            for (int kb = 0; kb < KB; ++kb)
#pragma unroll
                for (int i = 0; i < 8; ++i) s[kb][i] = (T)(NARROW<T> ? S[2 * kb + i / 4][i % 4] * down : S[2 * kb + i / 4][i % 4]);
        }
        if constexpr (!SUMS) {
            // rows 16 it of P by rows 32 kb of b, transposed: a lane has eight entries of a row
            const auto make_piece = [&](int it, int kb) {
                floats P[2] = {(floats)0.0f, (floats)0.0f};
#pragma unroll
                for (int q = 0; q < KB; ++q) {
                    const operand<T> a = sa.along(along_a, it, q);
#pragma unroll
                    for (int half = 0; half < 2; ++half) P[half] = product(sb.spread(spread_b, kb, half, q), a, P[half]);
                }
                const int before = it - 2 * kb;
                const float far = before == 3 ? tile_on : 1.0f;
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const floats w = weight_p[SUMS ? 0 : min(before, 2)][half][lane];
#pragma unroll
                    for (int j = 0; j < 4; ++j) P[half][j] *= w[j] * far;
                }
                float down = 1.0f;
                if constexpr (NARROW<T>) {
                    float top = 0.0f;
#pragma unroll
                    for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(P[i / 4][i % 4]));
                    const int e = exponent_for(wave_largest(top));
                    down = ldexpf(1.0f, -e);
                    if (lane == 0) sp_exponent[it][kb] = e;
                }
                operand<T> x;
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = (T)(NARROW<T> ? P[i / 4][i % 4] * down : P[i / 4][i % 4]);
                sp.along(along_p, it, kb) = x;
            };
            if constexpr (WAVES == 4) {
                make_piece(wave < 2 ? 3 : 2, wave & 1);
                if (wave >= 2) make_piece(wave - 2, 0);
            } else {
                if (wave < 6) make_piece(wave < 4 ? 3 - wave / 2 : wave - 4, wave < 4 ? wave & 1 : 0);
            }
        }
        // The memory behind the chunk.  c is weighed, and what that makes is held to 24 bits as a sum of operands (22 in float16): the memory is kept in
        // float32, and one rounding to 8 or 11 bits of every row would be left in it.
        if (HEADS == MANY_B || h == heads - 1) {
            const float keep = HEADS == MANY_B && h > 0 ? 1.0f : n == CHUNK ? whole : power(l2, n);
            int e = 0;
            float w[2][8];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                const floats lo = weight_out[8 * t + 2 * g], hi = weight_out[8 * t + 2 * g + 1];
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
                const operand<T> b0 = sb.across_spread(across_b, 0, bt / 2, bt % 2), b1 = sb.across_spread(across_b, 1, bt / 2, bt % 2);
                floats x = NARROW<T> ? (floats)0.0f : S[bt];
                if constexpr (!NARROW<T>)
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] *= keep;
#pragma unroll
                for (int q = PARTS - 1; q >= 0; --q) {
                    x = product(b0, part[q][0], x);
                    x = product(b1, part[q][1], x);
                }
                if constexpr (NARROW<T>) {
                    const float up = ldexpf(1.0f, e);
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[j] = fmaf(S[bt][j], keep, x[j] * up);
                }
                S[bt] = x;
            }
            if constexpr (sizeof(T) == 4) settle(S);
        }
        if constexpr (SUMS) return;
        __syncthreads();
        if (!p.out.data) return;
        float w = NARROW<T> ? ldexpf(weight_in, s_exponent) : weight_in;
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            floats &o = O[HEADS == MANY_B ? it : 0];
            if (enter) {
                o = (floats)0.0f;
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) o = product(s[kb], sa.along(along_a, it, kb), o);
#pragma unroll
                for (int j = 0; j < 4; ++j) o[j] *= w;
                w *= tile_on;
            }
#pragma unroll
            for (int kb = 0; kb <= it / 2; ++kb) {
                if constexpr (NARROW<T>) {
                    const floats more = product(c[kb], sp.along(along_p, it, kb), (floats)0.0f);
                    const float up = ldexpf(1.0f, sp_exponent[it][kb]);
#pragma unroll
                    for (int j = 0; j < 4; ++j) o[j] = fmaf(more[j], up, o[j]);
                } else {
                    o = product(c[kb], sp.along(along_p, it, kb), o);
                }
            }
            if (leave) {
                bagel_pack<T, 4> x;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = (T)(o[j] * p.scale);
                if constexpr (THROUGH) {
                    so.entries(entries_o, it, wave) = x;
                } else {
                    const int first = 16 * wave + 4 * g;
                    if (16 * it + j16 >= n || first >= p.wc) continue;
                    T *to = out + (16 * it + j16) * (step * p.out.stride) + first;
                    if (first + 4 <= p.wc) reinterpret_cast<bagel_loose_pack<T, 4> *>(to)->x = x;
                    else
#pragma unroll
                        for (int j = 0; j < 3; ++j)
                            if (first + j < p.wc) to[j] = x[j];
                }
            }
        }
    };
    const int64_t chunks = at.rows / CHUNK;
    const int rest = (int)(at.rows % CHUNK);
    // The steps of whole chunks are asked for, and those of the rows that are left, as the 64 rows up to the last one; behind these the same again, which nobody
    // reads: a branch around the loads would make every wait one for all of them.
    int64_t ask_chunk = 0;
    int ask_head = 0;
    const auto ask_next = [&](tiles &to) {
        ask(to, at.base + step * min(ask_chunk * CHUNK, at.rows - CHUNK), ask_head);
        if (HEADS == ONE || ++ask_head == heads) {
            ask_head = 0;
            ++ask_chunk;
        }
    };
#pragma unroll
    for (int bt = 0; bt < NB; ++bt) asm volatile("" : "+v"(S[bt]));      // the memory is there before anything else is asked for, so that no wait in the loop is one for it
    T *ready = nullptr;                              // where the whole rows in `so` go
    const auto before = [&] {
        if constexpr (THROUGH)
            if (ready) write_rows<T, WC, THREADS>(so, pack_c, ready, step * p.out.stride, CHUNK, p.wc);
    };
    int64_t chunk = 0;
    int h = 0;
    const auto whole_step = [&](const tiles &come, tiles &then) {
        T *out = !SUMS && p.out.data ? p.out.at(at.base + step * (chunk * CHUNK), head_a(h)) : nullptr;
        go(come, h, CHUNK, out, before, [&] { ask_next(then); });
        ready = HEADS == MANY_B && h < heads - 1 ? nullptr : out;
        if (HEADS == ONE || ++h == heads) {
            h = 0;
            ++chunk;
        }
    };
    // Two steps to a round, after one on its own where they are odd in number; what is left is then on its way in the first place.
    if ((chunks * heads) & 1) {
        tiles alone;
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
    if (rest > 0) {                                  // the rows that are left: further heads, or all of them where there are no others, are not on their way yet
        T *out = nullptr;
        for (h = 0; h < heads; ++h) {
            if (chunks == 0) ask_few(coming[0], h, rest);
            else if (h > 0) ask(coming[0], at.base + step * (at.rows - CHUNK), h);
            if (!SUMS && p.out.data) out = p.out.at(at.base + step * (chunks * CHUNK), head_a(h));
            go(coming[0], h, rest, out, before, [] {});
            ready = nullptr;
            if constexpr (THROUGH) {
                __syncthreads();
                if (out && (HEADS != MANY_B || h == heads - 1)) write_rows<T, WC, THREADS>(so, pack_c, out, step * p.out.stride, rest, p.wc);
            }
        }
    } else if constexpr (THROUGH) {
        __syncthreads();
        before();
    }
    float *to = SUMS ? p.memories + (slot * p.states + state) * size : at.last && p.last ? p.last + memory : nullptr;
    if (!to || mine >= p.wc) return;
    int64_t step_b = SUMS ? p.wc : p.step_b, step_c = SUMS ? 1 : p.step_c;
    asm volatile("" : "+s"(step_b));                 // its multiples are not kept from the beginning: they would take all scalar registers
#pragma unroll
    for (int bt = 0; bt < NB; ++bt)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (row_of(bt, j) < p.wb) to[row_of(bt, j) * step_b + mine * step_c] = S[bt][j];
}

// What segments have added to the memory, into the memory behind each: a thread to an entry, along its sequence's segments but the last.
template <typename T> __global__ __launch_bounds__(256) void memories_kernel(bagel_attention_pass<T> p, int blocks)
{
    const int size = p.wb * p.wc;
    for (int64_t work = blockIdx.x; work < (int64_t)p.sequences * p.states * blocks; work += gridDim.x) {
        const int state = (int)(work / blocks % p.states), sequence = (int)(work / blocks / p.states);
        int64_t length = p.each, slot;
        if (!p.offsets) {
            slot = (int64_t)sequence * max((length + p.segment - 1) / p.segment, (int64_t)1);
        } else {
            const int64_t begin = min(max((int64_t)p.offsets[sequence], (int64_t)0), p.rows);
            length = min(max((int64_t)p.offsets[sequence + 1], begin), p.rows) - begin;
            slot = begin / p.segment + sequence;
        }
        const int64_t segments = (length + p.segment - 1) / p.segment, each = (int64_t)p.states * size;
        if (segments < 3) continue;                  // (of two, the first one's is whole)
        const float keep = __builtin_amdgcn_exp2f(fmaxf(p.log_decay[state], -1e30f) * 1.44269504f * (float)p.segment);
        for (int i = (int)(work % blocks) * 256 + threadIdx.x; i < size; i += blocks * 256) {
            float *m = p.memories + (slot * p.states + state) * size + i;
            float s = m[0];
            constexpr int AHEAD = 16;
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
}

template <typename T, int WB, int WC, bool WHOLE, heads_kind HEADS> hipError_t launch_pass(const bagel_attention_pass<T> &p, hipStream_t stream)
{
    constexpr int THREADS = 4 * WC, ON_SIMD = sizeof(T) == 4 && WB == 128 && WC == 64 ? 1 : 2;
    constexpr heads_kind SUMS_HEADS = HEADS == MANY_A ? ONE : HEADS;
    const int64_t work = p.slots * p.states;
    if (p.memories) {
        chunks_kernel<T, WB, WC, WHOLE, true, SUMS_HEADS, ON_SIMD><<<(unsigned)work, THREADS, 0, stream>>>(p);
        // some workgroups to a memory where there are few of them
        const int64_t all = (int64_t)p.sequences * p.states, most = (p.wb * p.wc + 255) / 256, wanted = 1024 / all;
        const int blocks = (int)(wanted < 1 ? 1 : wanted < most ? wanted : most);
        memories_kernel<T><<<(unsigned)(all * blocks < 1 << 16 ? all * blocks : 1 << 16), 256, 0, stream>>>(p, blocks);
    }
    const int64_t clear = p.offsets && p.out.data && p.rows > 0 ? 32 : 0;
    if (work + clear > 0) chunks_kernel<T, WB, WC, WHOLE, false, HEADS, ON_SIMD><<<(unsigned)(work + clear), THREADS, 0, stream>>>(p);
    return hipGetLastError();
}

template <typename T, int WB, int WC, bool WHOLE> hipError_t launch_pass(const bagel_attention_pass<T> &p, hipStream_t stream)
{
    if (p.ks > 1) return launch_pass<T, WB, WC, WHOLE, MANY_B>(p, stream);
    return p.qs > 1 ? launch_pass<T, WB, WC, WHOLE, MANY_A>(p, stream) : launch_pass<T, WB, WC, WHOLE, ONE>(p, stream);
}

template <typename T, int WB, int WC> hipError_t launch_pass(const bagel_attention_pass<T> &p, hipStream_t stream)
{
    return p.wb == WB && p.wc == WC ? launch_pass<T, WB, WC, true>(p, stream) : launch_pass<T, WB, WC, false>(p, stream);
}

}  // namespace

template <typename T> hipError_t bagel_launch_attention_pass(const bagel_attention_pass<T> &p, hipStream_t stream)
{
    if (p.wb <= 64) return p.wc <= 64 ? launch_pass<T, 64, 64>(p, stream) : launch_pass<T, 64, 128>(p, stream);
    return p.wc <= 64 ? launch_pass<T, 128, 64>(p, stream) : launch_pass<T, 128, 128>(p, stream);
}
