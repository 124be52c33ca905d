// The gated linear recurrence of a policy with memory (include/bagel.h) and its gradient.
//
//   q_t = 1 / (1 + exp(f_t + b)),   h_t = h_{t-1} + q_t (x_t - h_{t-1}) = x_t + (1 - q_t) (h_{t-1} - x_t)
// Over several rows h goes to A h + H, with A the product of the (1 - q_t), and the H of two pieces one after the other is A2 H1 + H2.  A
// piece in which a sequence begins does not depend on what was before: it is marked by A = -1, and its A is never multiplied
// (what another sequence left may be infinite).  Backwards, with g_t the gradient of h_t: g_t = dh_t + c_t, dx_t = q_t g_t,
// c_{t-1} = g_t - q_t g_t, df_t = (h_{t-1} - x_t) (1 - q_t) q_t g_t: c is a recurrence of the same kind the other way, and h_{t-1} is
// computed again from the state before the span, which the forward pass kept.  The second form of h_t and 1 - q_t itself are for gates that are nearly open, where
// 1 - q_t is far smaller than a rounding of q_t.
//
// One pass over the data.  A workgroup has a span of rows and 64 V channels, a wave a segment of the span's rows and V channels a lane, all of
// it in registers.  The waves sum up their segments, the workgroup its span, and publishes that; the state before the span comes from
// what the spans before it published, and the rows are gone through once more, in registers, from there.
//   A published sum is one word of 64 bits a channel, A and H: it is whole as soon as it is there, and nothing else has to be ordered with it.
//   Memory is the bound that there has to be: 3 and 5 entries moved for a dozen operations each.  131072 x 1024 in f32 is there (304 us forward and 492 back, 5.3 and
// 5.4 TB/s).  In 16 bits a workgroup moves half as much for the same waits, and a workgroup's life is what bounds it (131072 x 1024 in bf16 209 us and
// 297 us, 3.8 and 4.5 TB/s; of some 12 us forward 3.6 us go by until its rows are there, 2 in its sums, 4.2 in publishing and looking
// back; without looking back the two took 21 and 28 us less).  q, x and the gradient stay in registers in the meantime, which is why two workgroups and no
// more share a compute unit.
//   Spans are handed out by a counter in the order in which they depend on each other.  So a workgroup waits only for spans handed out before
//   its own, to workgroups that run already and publish their sums before they wait for anything: every wait ends.
#include <type_traits>

#include "activations.h"

namespace {

constexpr int SPAN = BAGEL_RECURRENCE_SPAN;
constexpr int WAVES = 8;

template <typename T> struct recurrence_args {
    int rows, width, sequences, each;        // each: rows of a sequence where there are no offsets
    const int32_t *offsets;
    bagel_rows<T> value, forget, hidden, d_hidden, d_value, d_forget;
    const float *bias, *initial, *d_final;
    float *final_state, *carry, *d_initial;
    int spans, groups;                       // of the pass; of channels
    uint64_t *published;                     // [spans][width]
    uint32_t *counter;                       // null: one span, nothing to hand out
    float *bias_sums;                        // [spans][width], null: not wanted
};

// What is published of a span: nothing yet, its A and H, or (CLOSED) the state behind it.  A is never negative, and a NaN among the A is
// made the common one, which is not NOTHING.
constexpr uint32_t NOTHING = 0xFFFFFFFFu;
constexpr float CLOSED = -1.0f;

struct piece {
    float A, H;
};
__device__ __forceinline__ float through(const piece &p, float h) { return p.A == CLOSED ? p.H : fmaf(p.A, h, p.H); }
__device__ __forceinline__ piece joined(const piece &first, const piece &then)
{
    if (then.A == CLOSED) return then;
    return {first.A == CLOSED ? CLOSED : first.A * then.A, fmaf(then.A, first.H, then.H)};
}

__device__ __forceinline__ void publish(uint64_t *to, piece p)
{
    const uint32_t A = p.A != p.A ? 0x7FC00000u : __float_as_uint(p.A);
    __hip_atomic_store(to, (uint64_t)__float_as_uint(p.H) << 32 | A, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t look(const uint64_t *from) { return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Clears what is published, before it is: 5.5 us for 1024 spans of 1024 channels.  (A fill by the runtime inside a captured graph is not to be relied on.)
__global__ __launch_bounds__(256) void nothing_kernel(uint64_t *published, int64_t cells, uint32_t *counter)
{
    const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (first == 0) *counter = 0;
    for (int64_t i = first; i < cells; i += (int64_t)gridDim.x * 256) published[i] = NOTHING;
}

// The state before span number `order` (in the order in which they depend on each other; `spans` is where that of number 0 is, and the next `step`
// cells on).  Spans are in blocks of SPANS.  A span publishes what it is itself, but the last of a block the state behind it, CLOSED.  So the state
// before a span is that before its block, taken through the spans of the block before it: always the same operations, whoever was
// fast, and one wait for another's state in 32 spans, GROUP for each wave.
//   With few channels that chain of states is what a long sequence takes.  Then (DEEP) half of the waves look at spans and half at whole blocks, 16 spans
// to a block and 16 blocks to a state: the last span of a block publishes what its block is, which it knows from the spans before it.
constexpr int GROUP = 4;
template <bool DEEP> struct blocks_of {
    static constexpr int waves = DEEP ? WAVES / 2 : 0;           // that look at blocks
    static constexpr int spans = GROUP * (WAVES - waves), large = DEEP ? spans * GROUP * waves : spans;
    static __device__ __forceinline__ bool ends(int order) { return order % spans == spans - 1; }
    static __device__ __forceinline__ bool ends_large(int order) { return order % large == large - 1; }
};

// `all`, in wave 0, is the span itself, and `to` where it publishes (null: a lane that does not).
template <int V, bool DEEP>
__device__ __forceinline__ void look_back(const uint64_t *spans, int64_t step, int order, int wave, const piece (&all)[V], uint64_t *to,
                                          piece (*seen)[64][V], float (&h)[V])
{
    using in = blocks_of<DEEP>;
    const int lane = threadIdx.x & 63, large = order / in::large * in::large, block = order / in::spans * in::spans;
    const bool blocks = wave < in::waves;
    const int every = blocks ? in::spans : 1, first = (blocks ? wave : wave - in::waves) * GROUP;
    const int count = min((blocks ? (block - large) / in::spans : order - block) - first, GROUP);
    const int from = blocks ? large + (first + 1) * in::spans - 1 : block + first;
    uint64_t word[GROUP + 1][V];
#pragma unroll
    for (int k = 0; k < GROUP; ++k)
        if (k < count)
#pragma unroll
            for (int v = 0; v < V; ++v) word[k][v] = look(spans + (from + k * every) * step + v);
    const bool state = wave == 0 && large > 0;
    if (state)
#pragma unroll
        for (int v = 0; v < V; ++v) word[GROUP][v] = look(spans + (large - 1) * step + v);
    const auto wait = [&] {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            piece p = {1.0f, 0.0f};
            if (state) {
                while (__uint_as_float((uint32_t)word[GROUP][v]) != CLOSED) word[GROUP][v] = look(spans + (large - 1) * step + v);
                p.H = __uint_as_float((uint32_t)(word[GROUP][v] >> 32));
            }
#pragma unroll
            for (int k = 0; k < GROUP; ++k)
                if (k < count) {
                    while ((uint32_t)word[k][v] == NOTHING) word[k][v] = look(spans + (from + k * every) * step + v);
                    p = joined(p, {__uint_as_float((uint32_t)word[k][v]), __uint_as_float((uint32_t)(word[k][v] >> 32))});
                }
            seen[wave][lane][v] = p;
        }
    };
    if constexpr (DEEP) {
        if (!blocks) wait();
        __syncthreads();
        if (in::ends(order) && !in::ends_large(order) && to)     // before it waits for any other block
#pragma unroll
            for (int v = 0; v < V; ++v) {
                piece p = seen[in::waves][lane][v];
#pragma unroll
                for (int k = in::waves + 1; k < WAVES; ++k) p = joined(p, seen[k][lane][v]);
                publish(to + v, joined(p, all[v]));
            }
        if (blocks) wait();
    } else {
        wait();
    }
    __syncthreads();
    const int waves = DEEP ? WAVES : min((order - block + GROUP - 1) / GROUP, WAVES);
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = seen[0][lane][v].H;       // the state before the large block is in it
    for (int k = 1; k < waves; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = through(seen[k][lane][v], h[v]);
    if (in::ends_large(order) && to)
#pragma unroll
        for (int v = 0; v < V; ++v) publish(to + v, {CLOSED, through(all[v], h[v])});
}

// The rows t0 to t0 + S - 1 of a wave: which of them begin a sequence (bit i of `starts` for t0 + i, bit S for the row behind them; the end of the
// last sequence counts as a start), which belong to one at all (begin to end - 1), and the sequence of t0 (-1: it comes before the first).
template <int S> struct segment {
    uint64_t starts;
    int begin, end, sequence;
    static constexpr uint64_t every = (1ull << S) - 1;
    __device__ __forceinline__ bool whole() const { return begin == 0 && end == S; }
    __device__ __forceinline__ bool outside(int i) const { return i < begin || i >= end; }
    __device__ __forceinline__ bool start(int i) const { return !outside(i) && (starts >> i & 1); }
    __device__ __forceinline__ bool last(int i) const { return !outside(i) && (starts >> (i + 1) & 1); }
    // the rows that are not just one more of their sequence
    __device__ __forceinline__ uint64_t special() const { return whole() ? starts | starts >> 1 : every; }
    // whether what is before (behind) the segment does not reach through it
    __device__ __forceinline__ bool closed() const { return !whole() || (starts & every); }
    __device__ __forceinline__ bool closed_back() const { return !whole() || (starts >> 1 & every); }
};

// The first look at the offsets, before the rows are asked for: every lane one, a 64th part of them from the next.
template <typename A> __device__ __forceinline__ int some_offset(const A &a)
{
    const int step = a.sequences / 64 + 1;
    return a.offsets ? a.offsets[min((int)(threadIdx.x & 63) * step, a.sequences)] : 0;
}

template <int S, typename A> __device__ __forceinline__ segment<S> segment_at(const A &a, int t0, int o)
{
    static_assert(S < 64, "one lane to a row");
    const int lane = threadIdx.x & 63, n = a.sequences;
    if (!a.offsets) {
        const int i = t0 / a.each;
        const uint64_t starts = __ballot(lane <= S && (t0 + lane) % a.each == 0);
        return {starts, 0, max(0, min(S, a.rows - t0)), min(i, n - 1)};
    }
    // Down to 64 offsets in a row, o, from number lo on, of which the first is not behind t0 (or is the first of all)
    int lo = 0, step = n / 64 + 1;
    int first, stop;
    if (step == 1) {
        first = __builtin_amdgcn_readlane(o, 0);
        stop = __builtin_amdgcn_readlane(o, n);
    } else {
        first = a.offsets[0];
        stop = a.offsets[n];
    }
    stop = min(stop, a.rows);
    while (step > 1) {
        const int k = __popcll(__ballot((int64_t)lo + (int64_t)lane * step <= n && o <= t0));
        lo += max(k - 1, 0) * step;
        step = (step + 62) / 63;
        o = a.offsets[min((int64_t)lo + (int64_t)lane * step, (int64_t)n)];
    }
    if (lo + lane > n) o = 0x7FFFFFFF;
    const int found = lo + __popcll(__ballot(o <= t0)) - 1;
    uint64_t starts = __ballot(o == t0) ? 1 : 0;
    for (int k = lo;;) {
        for (uint64_t in = __ballot(o > t0 && o <= t0 + S); in; in &= in - 1) starts |= 1ull << (__builtin_amdgcn_readlane(o, __builtin_ctzll(in)) - t0);
        if (__ballot(o <= t0 + S) != ~0ull || (k += 64) > n) break;
        o = k + lane <= n ? a.offsets[k + lane] : 0x7FFFFFFF;
    }
    return {starts, first <= t0 ? 0 : min(S, first - t0), stop <= t0 ? 0 : min(S, stop - t0), min(found, n - 1)};
}

// The sequence of row t, which begins one, from that of the row before it.
template <typename A> __device__ __forceinline__ void to_next(const A &a, int t, int &sequence)
{
    do ++sequence;
    while (sequence < a.sequences - 1 && a.offsets && a.offsets[sequence + 1] <= t);
    sequence = min(sequence, a.sequences - 1);
}
// and that of the row before t.
template <typename A> __device__ __forceinline__ void to_previous(const A &a, int t, int &sequence)
{
    do --sequence;
    while (sequence > 0 && a.offsets && a.offsets[sequence] >= t);
    sequence = max(sequence, 0);
}

// The share q of a forget gate f and bias b.  They are added first: they may be large and cancel, and a rounding of b log2(e) would stay.
// 1 - q is formed from q as long as that leaves enough of it: a unit of q is 8 units of 1 - q at 15/16, but 3 % of it at 1 - e^-13, and from 1 - e^-17 on
// nothing is left.  Of a gate that is open further than 15/16, 1 - q is kept in the place of q, from the exponential, with a minus (also of zero).
constexpr float LOG2E = 1.44269504f, OPEN = 0.9375f;
__device__ __forceinline__ float gate(float f, float b) { return __builtin_amdgcn_exp2f((f + b) * LOG2E); }
__device__ __forceinline__ float share(float f, float b) { return __builtin_amdgcn_rcpf(1.0f + gate(f, b)); }
__device__ __forceinline__ float kept(float q, float f, float b) { return q > OPEN ? -(gate(f, b) * q) : q; }
// a for a gate that is open, else b.  (SOME: whether any of the wave's may be; the results are the same either way.)
// By bits: a comparison for every row would take more scalar registers than there are.
template <bool SOME> __device__ __forceinline__ float where_open(float q, float a, float b)
{
    if constexpr (SOME) asm("v_bfi_b32 %0, %1, %2, %0" : "+v"(b) : "v"(__float_as_int(q) >> 31), "v"(a));
    return b;
}
// h + q (x - h), and where the gate is open x + (1 - q) (h - x): a part of the difference is added to what stays
template <bool SOME> __device__ __forceinline__ float mixed(float q, float x, float h) { return fmaf(q, x - h, where_open<SOME>(q, x, h)); }
// (1 - q) g
template <bool SOME> __device__ __forceinline__ float left(float q, float g) { return fmaf(-q, g, where_open<SOME>(q, 0.0f, g)); }
__device__ __forceinline__ float at(const float *p, int64_t i) { return p ? p[i] : 0.0f; }

// f(special, whether a gate is open) with constants: 0 special rows where there are none, as most segments lie within one sequence and a branch at every row costs
// them a tenth, and no open gates where there are none (131072 x 1024 bf16: 209 and 297 us, and 220 and 309 where many gates are open).
template <typename F> __device__ __forceinline__ void by_rows(uint64_t special, bool open, F &&f)
{
    const std::integral_constant<uint64_t, 0> none;
    if (special != 0 && open) f(special, std::true_type());
    else if (special != 0) f(special, std::false_type());
    else if (open) f(none, std::true_type());
    else f(none, std::false_type());
}

// What is the same in both directions: which span and channels a workgroup has, and its reads.
template <typename T, int V, int S> struct wave_tile {
    using pack = bagel_pack<T, V>;
    static constexpr int rows = S * WAVES;
    int span, wave, lane, t0, ch;            // ch: its first channel.  A lane that has none, or only one of two, takes the last ones: it does once
                                             // more what another lane does.
    bool here;
    __device__ __forceinline__ wave_tile(int work, const recurrence_args<T> &a)
    {
        span = work / a.groups;
        wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        lane = threadIdx.x & 63;
        const int c = (work - span * a.groups) * 64 * V + lane * V;
        here = c < a.width;
        ch = min(c, a.width - V);
    }
    __device__ __forceinline__ void reverse(const recurrence_args<T> &a) { span = a.spans - 1 - span; }
    __device__ __forceinline__ void begin() { t0 = span * rows + wave * S; }
    template <typename Q> __device__ __forceinline__ void load(const bagel_rows<Q> &m, int last, pack (&x)[S]) const
    {
#pragma unroll
        for (int i = 0; i < S; ++i) x[i] = reinterpret_cast<const bagel_loose_pack<T, V> *>(m.row(min(t0 + i, last)) + ch)->x;
    }
    // From here on the packs are what they are and not what they were converted to: the converted ones of two channels in 16 bits would take twice
    // the registers between two passes over the rows.
    static __device__ __forceinline__ void keep_packed(pack (&x)[S])
    {
        if constexpr (sizeof(pack) == 4 && V == 2)
#pragma unroll
            for (int i = 0; i < S; ++i) {
                uint32_t bits = __builtin_bit_cast(uint32_t, x[i]);
                asm volatile("" : "+v"(bits));
                x[i] = __builtin_bit_cast(pack, bits);
            }
    }
    static __device__ __forceinline__ float one(const pack &x, int v)
    {
        if constexpr (V == 1) return (float)x[0];
        else return (float)x[v];
    }
    // Rows that belong to no sequence: a value and a forget gate of which neither is NaN, so that zero stays zero.
    __device__ __forceinline__ void clear_outside(const segment<S> &seg, pack (&f)[S], pack (&x)[S]) const
    {
        if (seg.whole()) return;
#pragma unroll
        for (int i = 0; i < S; ++i)
            if (seg.outside(i)) f[i] = x[i] = (pack)(T)0.0f;
    }
    // h before row i, where that is not what the row before left: `h` of pieces or of states
    __device__ __forceinline__ void enter(const recurrence_args<T> &a, const segment<S> &seg, int i, int &sequence, float (&h)[V]) const
    {
        if (seg.outside(i)) {
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = 0.0f;
        } else if (seg.start(i)) {
            if (i > 0 || sequence < 0) to_next(a, t0 + i, sequence);
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = at(a.initial, (int64_t)sequence * a.width + ch + v);
        }
    }
    __device__ __forceinline__ void enter(const recurrence_args<T> &a, const segment<S> &seg, int i, int &sequence, piece (&p)[V]) const
    {
        float h[V];
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = p[v].H;
        enter(a, seg, i, sequence, h);
#pragma unroll
        for (int v = 0; v < V; ++v) p[v].H = h[v];
    }
    // c behind row i, where that is not what the row behind it left
    __device__ __forceinline__ void enter_back(const recurrence_args<T> &a, const segment<S> &seg, int i, int sequence, float (&c)[V]) const
    {
        if (seg.outside(i) || seg.last(i))
#pragma unroll
            for (int v = 0; v < V; ++v) c[v] = seg.outside(i) ? 0.0f : at(a.d_final, (int64_t)sequence * a.width + ch + v);
    }
    // the shares of the segment's gates; whether any of the wave's is open
    static __device__ __forceinline__ bool shares(const pack (&f)[S], const float (&b)[V], float (&q)[S][V])
    {
        float most = 0.0f;
#pragma unroll
        for (int i = 0; i < S; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                q[i][v] = share(one(f[i], v), b[v]);
                most = fmaxf(most, q[i][v]);
            }
        if (!__any(most > OPEN)) return false;
#pragma unroll
        for (int i = 0; i < S; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) q[i][v] = kept(q[i][v], one(f[i], v), b[v]);
        return true;
    }
    __device__ __forceinline__ void store(const bagel_rows<T> &m, int row, const float (&x)[V]) const { bagel_store<T, V>(m.row(row) + ch, x); }
};

// The number of the work that this workgroup takes.
__device__ __forceinline__ int next_work(uint32_t *counter)
{
    if (!counter) return blockIdx.x;
    __shared__ int work;
    if (threadIdx.x == 0) work = (int)atomicAdd(counter, 1u);
    __syncthreads();
    return __builtin_amdgcn_readfirstlane(work);
}

// What passes through a sequence without a step, by the workgroups behind those of the spans, number `group` and on: a wave to a sequence, at most PASSING
// workgroups (with 64 sequences to each the last workgroups of a call were its longest: 61 sequences of 50021 x 777 f16, 8 of them empty, took
// 99 and 165 us where they take 81 and 135).
constexpr int PASSING = 8192;

template <typename A> __device__ __forceinline__ void pass_through(const A &a, int group, const float *from, float *to)
{
    for (int s = group * WAVES + (threadIdx.x >> 6); s < a.sequences; s += PASSING * WAVES)
        if (a.offsets ? a.offsets[s] >= a.offsets[s + 1] : a.rows == 0)
            for (int ch = threadIdx.x & 63; ch < a.width; ch += 64) to[(int64_t)s * a.width + ch] = at(from, (int64_t)s * a.width + ch);
}

// Forward.  A row is rounded when it is stored and h goes on in 32 bits; what is final and what is carried is in 32 bits.
template <typename T, int V, int S, bool DEEP>
__global__ __launch_bounds__(64 * WAVES, V == 1 && DEEP ? 8 : 4) void recurrence_kernel(recurrence_args<T> a)
{
    __shared__ piece pieces[WAVES][64][V], seen[WAVES][64][V];
    const int work = next_work(a.counter);
    if (work >= a.spans * a.groups) {
        if (a.final_state) pass_through(a, work - a.spans * a.groups, a.initial, a.final_state);
        return;
    }
    using wt = wave_tile<T, V, S>;
    wt w(work, a);
    w.begin();
    typename wt::pack x[S], f[S];
    const int some = some_offset(a);
    w.load(a.forget, a.rows - 1, f);
    w.load(a.value, a.rows - 1, x);
    const segment<S> seg = segment_at<S>(a, w.t0, some);
    const uint64_t special = seg.special();
    w.clear_outside(seg, f, x);
    float q[S][V], h[V], b[V];
    piece mine[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        b[v] = at(a.bias, w.ch + v);
        mine[v] = {1.0f, 0.0f};
    }
    const bool open = wt::shares(f, b, q);
    int sequence = seg.sequence;
    by_rows(special, open, [&](auto special, auto some) {
#pragma unroll
        for (int i = 0; i < S; ++i) {
            if (special >> i & 1) w.enter(a, seg, i, sequence, mine);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                mine[v].H = mixed<some()>(q[i][v], wt::one(x[i], v), mine[v].H);
                mine[v].A = left<some()>(q[i][v], mine[v].A);
            }
        }
    });
    if (seg.closed())
#pragma unroll
        for (int v = 0; v < V; ++v) mine[v].A = CLOSED;
#pragma unroll
    for (int v = 0; v < V; ++v) pieces[w.wave][w.lane][v] = mine[v];
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = 0.0f;
    if (a.spans > 1) {
        uint64_t *to = w.wave == 0 && w.here ? a.published + (int64_t)w.span * a.width + w.ch : nullptr;
        piece all[V];
        if (w.wave == 0)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                all[v] = pieces[0][w.lane][v];
#pragma unroll
                for (int k = 1; k < WAVES; ++k) all[v] = joined(all[v], pieces[k][w.lane][v]);
            }
        if (to && !blocks_of<DEEP>::ends(w.span))
#pragma unroll
            for (int v = 0; v < V; ++v) publish(to + v, all[v]);
        if (w.span > 0) look_back<V, DEEP>(a.published + w.ch, a.width, w.span, w.wave, all, to, seen, h);
    }
    for (int k = 0; k < w.wave; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = through(pieces[k][w.lane][v], h[v]);
    if (!w.here) return;
    if (a.carry && w.t0 % SPAN == 0 && w.t0 < a.rows)
#pragma unroll
        for (int v = 0; v < V; ++v) a.carry[(int64_t)(w.t0 / SPAN) * a.width + w.ch + v] = h[v];
    sequence = seg.sequence;
    by_rows(special, open, [&](auto special, auto some) {
#pragma unroll
        for (int i = 0; i < S; ++i) {
            if (special >> i & 1) {
                if (w.t0 + i >= a.rows) break;
                w.enter(a, seg, i, sequence, h);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = mixed<some()>(q[i][v], wt::one(x[i], v), h[v]);
            if ((special >> i & 1) && a.final_state && seg.last(i))
#pragma unroll
                for (int v = 0; v < V; ++v) a.final_state[(int64_t)sequence * a.width + w.ch + v] = h[v];
            if ((special >> i & 1) && seg.outside(i))
#pragma unroll
                for (int v = 0; v < V; ++v) h[v] = 0.0f;
            w.store(a.hidden, w.t0 + i, h);
        }
    });
}

// Back, spans from the last to the first.  h comes from the carry by the forward pass's operations in 32 bits, not from the rounded rows.
template <typename T, int V, int S, bool DEEP>
__global__ __launch_bounds__(64 * WAVES, V == 1 && DEEP ? 6 : 4) void recurrence_grad_kernel(recurrence_args<T> a)
{
    static_assert(S * WAVES == SPAN, "a span begins with a row of the carry");
    __shared__ piece pieces[WAVES][64][V], back[WAVES][64][V], seen[WAVES][64][V];
    __shared__ float sums[WAVES][64][V];
    const int work = next_work(a.counter);
    if (work >= a.spans * a.groups) {
        if (a.d_initial) pass_through(a, work - a.spans * a.groups, a.d_final, a.d_initial);
        return;
    }
    using wt = wave_tile<T, V, S>;
    wt w(work, a);
    w.reverse(a);
    w.begin();
    typename wt::pack x[S], f[S], d[S];
    const int some = some_offset(a);
    w.load(a.forget, a.rows - 1, f);
    w.load(a.value, a.rows - 1, x);
    w.load(a.d_hidden, a.rows - 1, d);
    float h[V], c[V], q[S][V], b[V], sum[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        h[v] = a.carry[(int64_t)w.span * a.width + w.ch + v];
        b[v] = at(a.bias, w.ch + v);
    }
    const segment<S> seg = segment_at<S>(a, w.t0, some);
    const uint64_t special = seg.special();
    w.clear_outside(seg, f, x);
    w.clear_outside(seg, f, d);
    piece mine[V];
    float reach[V];                          // A and H, of the way back
#pragma unroll
    for (int v = 0; v < V; ++v) {
        mine[v] = {1.0f, 0.0f};
        reach[v] = 0.0f;
    }
    const bool open = wt::shares(f, b, q);
    int sequence = seg.sequence;
    by_rows(special, open, [&](auto special, auto some) {
#pragma unroll
        for (int i = 0; i < S; ++i) {
            if (special >> i & 1) w.enter(a, seg, i, sequence, mine);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                mine[v].H = mixed<some()>(q[i][v], wt::one(x[i], v), mine[v].H);
                mine[v].A = left<some()>(q[i][v], mine[v].A);
            }
        }
    });
    const int last_sequence = sequence;      // of the segment's last row
    by_rows(special, open, [&](auto special, auto some) {
#pragma unroll
        for (int i = S - 1; i >= 0; --i) {
            if (special >> i & 1) w.enter_back(a, seg, i, sequence, reach);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                reach[v] = left<some()>(q[i][v], wt::one(d[i], v) + reach[v]);
            }
            if ((special >> i & 1) && seg.start(i)) to_previous(a, w.t0 + i, sequence);
        }
    });
    w.keep_packed(x);
    w.keep_packed(d);
    piece mine_back[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        mine_back[v] = {seg.closed_back() ? CLOSED : mine[v].A, reach[v]};
        if (seg.closed()) mine[v].A = CLOSED;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        pieces[w.wave][w.lane][v] = mine[v];
        back[w.wave][w.lane][v] = mine_back[v];
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) c[v] = sum[v] = 0.0f;
    if (a.spans > 1) {
        const int order = a.spans - 1 - w.span;
        uint64_t *to = w.wave == 0 && w.here ? a.published + (int64_t)order * a.width + w.ch : nullptr;
        piece all[V];
        if (w.wave == 0)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                all[v] = back[WAVES - 1][w.lane][v];
#pragma unroll
                for (int k = WAVES - 2; k >= 0; --k) all[v] = joined(all[v], back[k][w.lane][v]);
            }
        if (to && !blocks_of<DEEP>::ends(order))
#pragma unroll
            for (int v = 0; v < V; ++v) publish(to + v, all[v]);
        if (order > 0) look_back<V, DEEP>(a.published + w.ch, a.width, order, w.wave, all, to, seen, c);
    }
    // h before every row, less its value
    float hx[S][V];
    for (int k = 0; k < w.wave; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = through(pieces[k][w.lane][v], h[v]);
    sequence = seg.sequence;
    by_rows(special, open, [&](auto special, auto some) {
#pragma unroll
        for (int i = 0; i < S; ++i) {
            if (special >> i & 1) w.enter(a, seg, i, sequence, h);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                hx[i][v] = h[v] - wt::one(x[i], v);
                h[v] = fmaf(-q[i][v], hx[i][v], where_open<some()>(q[i][v], wt::one(x[i], v), h[v]));
            }
        }
    });
    for (int k = WAVES - 1; k > w.wave; --k)
#pragma unroll
        for (int v = 0; v < V; ++v) c[v] = through(back[k][w.lane][v], c[v]);
    const bool write_x = w.here && a.d_value.data, write_f = w.here && a.d_forget.data;
    sequence = last_sequence;
    by_rows(special, open, [&](auto special, auto some) {
#pragma unroll
        for (int i = S - 1; i >= 0; --i) {
            float dx[V], df[V];
            if (special >> i & 1) {
                if (w.t0 + i >= a.rows) continue;
                w.enter_back(a, seg, i, sequence, c);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float part = some() ? fabsf(q[i][v]) : q[i][v], g = wt::one(d[i], v) + c[v], less = part * g, more = fmaf(-part, g, g);
                dx[v] = where_open<some()>(q[i][v], more, less);
                c[v] = where_open<some()>(q[i][v], less, more);
                df[v] = hx[i][v] * fmaf(-part, less, less);
            }
            if (special >> i & 1) {
                if (seg.outside(i))
#pragma unroll
                    for (int v = 0; v < V; ++v) dx[v] = df[v] = 0.0f;
                if (seg.start(i)) {
                    if (a.d_initial && w.here)
#pragma unroll
                        for (int v = 0; v < V; ++v) a.d_initial[(int64_t)sequence * a.width + w.ch + v] = c[v];
                    to_previous(a, w.t0 + i, sequence);
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) sum[v] += df[v];
            if (write_x) w.store(a.d_value, w.t0 + i, dx);
            if (write_f) w.store(a.d_forget, w.t0 + i, df);
        }
    });
    if (!a.bias_sums) return;
#pragma unroll
    for (int v = 0; v < V; ++v) sums[w.wave][w.lane][v] = sum[v];
    __syncthreads();
    if (w.wave > 0 || !w.here) return;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        float s = 0.0f;
#pragma unroll
        for (int k = 0; k < WAVES; ++k) s += sums[k][w.lane][v];
        a.bias_sums[(int64_t)w.span * a.width + w.ch + v] = s;
    }
}

// The sum over the spans in a fixed order, 64 threads to a channel: 6.3 us for 1024 spans of 1024 channels, 4 MB.
__global__ __launch_bounds__(1024) void bias_kernel(const float *sums, int spans, int width, float *d_bias)
{
    __shared__ float part[64][17];
    const int lane = threadIdx.x & 15, slice = threadIdx.x >> 4, ch = blockIdx.x * 16 + lane;
    const int from = (int)((int64_t)spans * slice / 64), to = (int)((int64_t)spans * (slice + 1) / 64);
    float v = 0.0f;
    if (ch < width)
#pragma unroll 8
        for (int k = from; k < to; ++k) v += sums[(int64_t)k * width + ch];
    part[slice][lane] = v;
    __syncthreads();
    if (threadIdx.x >= 16 || ch >= width) return;
    v = 0.0f;
#pragma unroll
    for (int k = 0; k < 64; ++k) v += part[k][lane];
    d_bias[ch] = v;
}

// A row of each of many sequences, a thread to an entry: 2.7 us for 256 x 512 in bf16, all of it latency; 32768 x 4096 347 us in bf16 and f16, 479 us in f32, 131072 x
// 777 bf16 268 us, 5.3 to 5.6 TB/s, which is the rate of a copy: memory bounds it, and wider loads would have nothing to win.
template <typename T>
__global__ __launch_bounds__(256) void step_kernel(int64_t rows, int width, bagel_rows<T> value, bagel_rows<T> forget, bagel_rows<T> hidden,
                                                   const float *bias, float *state)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * width; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / width;
        const int ch = (int)(i - r * width);
        const float f = (float)forget.row(r)[ch], b = at(bias, ch);
        const float h = mixed<true>(kept(share(f, b), f, b), (float)value.row(r)[ch], state[i]);
        state[i] = h;
        if (hidden.data) hidden.row(r)[ch] = (T)h;
    }
}

int span_count(int64_t rows) { return (int)((rows + SPAN - 1) / SPAN); }

template <typename T> recurrence_args<T> args_of(const bagel_gated_recurrence &r, bool grad)
{
    recurrence_args<T> a{};
    a.rows = (int)r.rows;
    a.width = r.width;
    a.sequences = r.sequences;
    a.each = r.sequences > 0 ? (int)(r.rows / r.sequences) : 0;
    a.offsets = r.offsets;
    a.value = bagel_rows_of<T>(r.value);
    a.forget = bagel_rows_of<T>(r.forget);
    a.hidden = bagel_rows_of<T>(r.hidden);
    a.bias = r.bias;
    a.initial = r.initial;
    a.final_state = r.final_state;
    a.carry = r.carry;
    if (grad) {
        a.d_hidden = bagel_rows_of<T>(r.d_hidden);
        a.d_value = bagel_rows_of<T>(r.d_value);
        a.d_forget = bagel_rows_of<T>(r.d_forget);
        a.d_final = r.d_final;
        a.d_initial = r.d_initial;
    }
    return a;
}

template <typename T, int V, int S, bool GRAD> void launch_spans(recurrence_args<T> &a, const bagel_gated_recurrence &r, hipStream_t stream)
{
    static_assert(S * WAVES % SPAN == 0, "the work space has room for a word a channel and SPAN rows");
    a.spans = (int)((r.rows + S * WAVES - 1) / (S * WAVES));
    a.groups = (r.width + 64 * V - 1) / (64 * V);
    const bool empty = r.sequences > 0 && (r.offsets || r.rows == 0) && (GRAD ? r.d_initial : r.final_state);
    const int64_t work = (int64_t)a.spans * a.groups + (empty ? min((r.sequences + WAVES - 1) / WAVES, PASSING) : 0);
    if (work == 0) return;
    const int64_t cells = (int64_t)a.spans * r.width;
    if (a.spans > 1) {
        a.published = (uint64_t *)r.workspace;
        a.counter = (uint32_t *)(a.published + cells);
        const int64_t groups = (cells + 255) / 256;
        nothing_kernel<<<(unsigned)(groups < 4096 ? groups : 4096), 256, 0, stream>>>(a.published, cells, a.counter);
    }
    // Blocks of blocks where there are few groups of channels to hide the chain of states behind, and more than one state.  131072 rows in bf16, forward and
    // back, us, without and with: 64 channels 75 / 87 and 41 / 53, 256 85 / 114 and 71 / 109, 512 126 / 178 and 124 / 179, 1024 212 / 303 and
    // 217 / 308; 64 channels of 3000 rows 12.3 / 20.8 and 12.9 / 21.9, of 9000 14.9 / 24.2 and 13.9 / 23.8.
    const bool deep = a.groups <= 4 && a.spans > blocks_of<false>::spans;
    if constexpr (GRAD) {
        a.bias_sums = !r.d_bias ? nullptr : a.spans == 1 ? r.d_bias : (float *)((char *)r.workspace + cells * 8 + 16);
        (deep ? recurrence_grad_kernel<T, V, S, true> : recurrence_grad_kernel<T, V, S, false>)<<<(unsigned)work, 64 * WAVES, 0, stream>>>(a);
    } else {
        (deep ? recurrence_kernel<T, V, S, true> : recurrence_kernel<T, V, S, false>)<<<(unsigned)work, 64 * WAVES, 0, stream>>>(a);
    }
}

// Two channels a lane in 16 bits, one in 32: a wave reads 256 bytes of a row either way.  (One in 16 bits took 252 and 403 us for 131072 x 1024 where
// two took 220 and 306, two in 32 bits 335 and 682 where one took 311 and 511.)
template <typename T, bool GRAD> hipError_t launch_pass(const bagel_gated_recurrence &r, hipStream_t stream)
{
    recurrence_args<T> a = args_of<T>(r, GRAD);
    if (sizeof(T) == 2 && r.width > 1) launch_spans<T, 4 / sizeof(T), 16, GRAD>(a, r, stream);
    else launch_spans<T, 1, 16, GRAD>(a, r, stream);
    if (GRAD && r.d_bias && a.spans != 1) bias_kernel<<<(r.width + 15) / 16, 1024, 0, stream>>>(a.bias_sums, a.spans, r.width, r.d_bias);
    return hipGetLastError();
}

template <typename T> hipError_t launch_forward(const bagel_gated_recurrence &r, hipStream_t stream) { return launch_pass<T, false>(r, stream); }
template <typename T> hipError_t launch_grad(const bagel_gated_recurrence &r, hipStream_t stream) { return launch_pass<T, true>(r, stream); }

template <typename T> hipError_t launch_step(const bagel_gated_recurrence &r, hipStream_t stream)
{
    const int64_t groups = ((int64_t)r.sequences * r.width + 255) / 256;
    step_kernel<T><<<(unsigned)(groups < 65536 ? groups : 65536), 256, 0, stream>>>(r.sequences, r.width, bagel_rows_of<T>(r.value), bagel_rows_of<T>(r.forget),
                                                                    bagel_rows_of<T>(r.hidden), r.bias, r.state);
    return hipGetLastError();
}

const char *check_sizes(const bagel_gated_recurrence *r)
{
    if (!r) return "null argument";
    if (r->rows < 0 || r->rows >= 1ll << 31) return "rows must be >= 0 and below 2^31";
    if (r->width < 1 || r->width >= 1 << 20) return "width must be >= 1 and below 2^20";
    if (r->sequences < 0) return "sequences must be >= 0";
    if (!bagel_type_ok(r->dtype)) return "unknown dtype";
    return nullptr;
}

const char *check_matrices(const bagel_gated_recurrence *r, int64_t rows, bool grad)
{
    const bagel_matrix forward[] = {r->value, r->forget, r->hidden}, backward[] = {r->d_hidden, r->d_value, r->d_forget};
    for (const bagel_matrix &m : forward)
        if (!bagel_matrix_ok(m, rows, r->width, r->dtype)) return "a matrix has a stride below the width, or an odd start";
    if (grad)
        for (const bagel_matrix &m : backward)
            if (!bagel_matrix_ok(m, rows, r->width, r->dtype)) return "a matrix has a stride below the width, or an odd start";
    return nullptr;
}

// States of all sequences that are read and such that are written: waves read the ones while others write the others.
bool states_overlap(const bagel_gated_recurrence *r, const float *read, const float *written)
{
    const uintptr_t a = (uintptr_t)read, b = (uintptr_t)written, bytes = (uintptr_t)r->sequences * r->width * sizeof(float);
    return read && written && (a < b ? b - a : a - b) < bytes;
}

const char *check_recurrence(const bagel_gated_recurrence *r, bool grad)
{
    if (const char *msg = check_sizes(r)) return msg;
    if (r->rows * (((int64_t)r->width + 63) / 64) >= 1ll << 29) return "rows times groups of 64 channels must be below 2^29";
    if (r->sequences >= 1 << 28) return "sequences must be below 2^28";
    if (r->rows > 0) {
        if (r->sequences < 1) return "rows without a sequence";
        if (!r->offsets && r->rows % r->sequences != 0) return "without offsets, sequences must divide rows";
        if (!r->value.data || !r->forget.data) return "value and forget are needed";
        if (!grad && !r->hidden.data) return "hidden is needed";
        if (grad && !r->d_hidden.data) return "d_hidden is needed";
        if (grad && !r->carry) return "the carry of the forward pass is needed";
        if (!r->workspace) return "a workspace is needed";
    }
    if (!grad && states_overlap(r, r->initial, r->final_state)) return "initial and final_state overlap";
    if (grad && states_overlap(r, r->d_final, r->d_initial)) return "d_final and d_initial overlap";
    if (r->workspace_bytes < bagel_recurrence_workspace(r->rows, r->width)) return "the workspace is too small";
    if ((uintptr_t)r->workspace & 15) return "the workspace must start at a multiple of 16 bytes";
    return check_matrices(r, r->rows, grad);
}

}  // namespace

extern "C" int64_t bagel_recurrence_carry_rows(int64_t rows) { return rows < 0 || rows >= 1ll << 31 ? BAGEL_EINVAL : span_count(rows); }

extern "C" int64_t bagel_recurrence_workspace(int64_t rows, int32_t width)
{
    if (rows < 0 || rows >= 1ll << 31 || width < 1 || width >= 1 << 20) return BAGEL_EINVAL;
    return (int64_t)span_count(rows) * width * (sizeof(uint64_t) + sizeof(float)) + 16;
}

extern "C" int bagel_recurrence(const bagel_gated_recurrence *r, void *hip_stream)
{
    if (const char *msg = check_recurrence(r, false)) return bagel_refuse(BAGEL_EINVAL, "bagel_recurrence: %s", msg);
    const hipError_t e = bagel_by_type(r->dtype, [&](auto t) { return launch_forward<typename decltype(t)::type>(*r, (hipStream_t)hip_stream); });
    if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_recurrence: %s", hipGetErrorString(e));
    return BAGEL_OK;
}

extern "C" int bagel_recurrence_grad(const bagel_gated_recurrence *r, void *hip_stream)
{
    if (const char *msg = check_recurrence(r, true)) return bagel_refuse(BAGEL_EINVAL, "bagel_recurrence_grad: %s", msg);
    const hipError_t e = bagel_by_type(r->dtype, [&](auto t) { return launch_grad<typename decltype(t)::type>(*r, (hipStream_t)hip_stream); });
    if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_recurrence_grad: %s", hipGetErrorString(e));
    return BAGEL_OK;
}

extern "C" int bagel_recurrence_step(const bagel_gated_recurrence *r, void *hip_stream)
{
    const char *msg = check_sizes(r);
    if (!msg && r->sequences > 0 && (!r->value.data || !r->forget.data || !r->state)) msg = "value, forget and state are needed";
    if (!msg && (int64_t)r->sequences * r->width >= 1ll << 38) msg = "sequences times width must be below 2^38";
    if (!msg) msg = check_matrices(r, r->sequences, false);
    if (msg) return bagel_refuse(BAGEL_EINVAL, "bagel_recurrence_step: %s", msg);
    if (r->sequences > 0) {
        const hipError_t e = bagel_by_type(r->dtype, [&](auto t) { return launch_step<typename decltype(t)::type>(*r, (hipStream_t)hip_stream); });
        if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_recurrence_step: %s", hipGetErrorString(e));
    }
    return BAGEL_OK;
}
