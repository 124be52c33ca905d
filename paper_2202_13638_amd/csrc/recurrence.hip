// The gated linear recurrence of a policy with memory (include/bagel.h) and its gradient.
//
//   q_t = 1 / (1 + exp(f_t + b)),   h_t = h_{t-1} + q_t (x_t - h_{t-1})
// Over several rows h goes to A h + H, with A the product of the (1 - q_t), and the H of two pieces one after the other is A2 H1 + H2.  A
// piece in which a sequence begins does not depend on what was before: it is marked by A = -1, and its A is never multiplied
// (what another sequence left may be infinite).  Backwards, with g_t the gradient of h_t: g_t = dh_t + c_t, dx_t = q_t g_t,
// c_{t-1} = g_t - q_t g_t, df_t = (h_{t-1} - x_t) (1 - q_t) q_t g_t: c is a recurrence of the same kind the other way, and h_{t-1} is
// computed again from the state before the span, which the forward pass kept.
//
// One pass over the data.  A workgroup has a span of rows and 64 V channels, a wave a segment of the span's rows and V channels a lane, all of
// it in registers.  The waves sum up their segments, the workgroup its span, and publishes that; the state before the span comes from
// the published sums of the spans before it (looking back until one of them has published its state, which it does as soon as it knows
// it), and the rows are gone through once more, in registers, from there.
//   A published sum is one word of 64 bits a channel, A and H: it is whole as soon as it is there, and nothing else has to be ordered with it.
//   Spans are handed out by a counter in the order in which they depend on each other.  So a workgroup waits only for spans handed out before
//   its own, to workgroups that run already and publish their sums before they wait for anything: every wait ends.
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
__device__ __forceinline__ float through(const piece &p, float h) { return p.A == CLOSED ? p.H : p.A * h + p.H; }
__device__ __forceinline__ piece joined(const piece &first, const piece &then)
{
    if (then.A == CLOSED) return then;
    return {first.A == CLOSED ? CLOSED : first.A * then.A, then.A * first.H + then.H};
}

__device__ __forceinline__ void publish(uint64_t *to, piece p)
{
    const uint32_t A = p.A != p.A ? 0x7FC00000u : __float_as_uint(p.A);
    __hip_atomic_store(to, (uint64_t)__float_as_uint(p.H) << 32 | A, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ uint64_t look(const uint64_t *from) { return __hip_atomic_load(from, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

__global__ __launch_bounds__(256) void nothing_kernel(uint64_t *published, int64_t cells, uint32_t *counter)
{
    const int64_t first = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (first == 0) *counter = 0;
    for (int64_t i = first; i < cells; i += (int64_t)gridDim.x * 256) published[i] = NOTHING;
}

// The state before a span, for one wave's channels: through the published pieces from the nearest (`span`, which goes on by `step`) to the first
// that is closed.  The span that all others come after publishes its state, so that there is one.
template <int V> __device__ __forceinline__ void look_back(const uint64_t *published, int width, int ch, int span, int step, int spans, float (&h)[V])
{
    constexpr int WINDOW = 8 / V;            // spans that are looked at together
    piece all[V];
    bool found[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        all[v] = {1.0f, 0.0f};
        found[v] = false;
    }
    for (;; span += WINDOW * step) {
        uint64_t word[WINDOW][V];
#pragma unroll
        for (int k = 0; k < WINDOW; ++k) {
            const int at = min(max(span + k * step, 0), spans - 1);
#pragma unroll
            for (int v = 0; v < V; ++v) word[k][v] = look(published + (int64_t)at * width + ch + v);
        }
#pragma unroll
        for (int k = 0; k < WINDOW; ++k) {
            const int at = min(max(span + k * step, 0), spans - 1);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                while (!found[v] && (uint32_t)word[k][v] == NOTHING) {
                    __builtin_amdgcn_s_sleep(1);
                    word[k][v] = look(published + (int64_t)at * width + ch + v);
                }
                if (!found[v]) {
                    const piece p = {__uint_as_float((uint32_t)word[k][v]), __uint_as_float((uint32_t)(word[k][v] >> 32))};
                    found[v] = p.A == CLOSED;
                    all[v] = {all[v].A * p.A, all[v].A * p.H + all[v].H};       // (where it is closed, A is of no more use)
                }
            }
        }
        bool every = true;
#pragma unroll
        for (int v = 0; v < V; ++v) every = every && found[v];
        if (__all(every)) break;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = all[v].H;
}

// The rows t0 to t0 + S - 1 of a wave: which of them begin a sequence (bit i of `starts` for t0 + i, bit S for the row behind them; the end of the
// last sequence counts as a start), which belong to one at all (begin to end - 1), and the sequence of t0 (-1: it comes before the first).
template <int S> struct segment {
    uint64_t starts;
    int begin, end, sequence;
    __device__ __forceinline__ bool plain() const { return (starts & ((1ull << S) - 1)) == 0 && begin == 0 && end == S; }
    __device__ __forceinline__ bool outside(int i) const { return i < begin || i >= end; }
    __device__ __forceinline__ bool start(int i) const { return starts >> i & 1; }
    __device__ __forceinline__ bool last(int i) const { return starts >> (i + 1) & 1; }
};

template <int S, typename A> __device__ __forceinline__ segment<S> segment_at(const A &a, int t0)
{
    static_assert(S < 64, "one lane to a row");
    const int lane = threadIdx.x & 63, n = a.sequences;
    if (!a.offsets) {
        const int i = t0 / a.each;
        const uint64_t starts = __ballot(lane <= S && (t0 + lane) % a.each == 0);
        return {starts, 0, max(0, min(S, a.rows - t0)), min(i, n - 1)};
    }
    // the last offset that is not behind t0, by 64 of them at a time
    int lo = 0, count = n + 1, found = -1;
    while (count > 0) {
        const int step = (count + 63) / 64, i = lo + lane * step;
        const bool here = lane * step < count && a.offsets[min(i, n)] <= t0;
        const int k = __popcll(__ballot(here));
        if (k == 0) break;
        found = lo + (k - 1) * step;
        if (step == 1) break;
        count = min(step, count - (k - 1) * step);
        lo = found;
    }
    uint64_t starts = found >= 0 && a.offsets[found] == t0 ? 1 : 0;
    for (int k = found + 1; k <= n; k += 64) {
        const int o = k + lane <= n ? a.offsets[k + lane] : 0x7FFFFFFF;
        for (uint64_t in = __ballot(o > t0 && o <= t0 + S); in; in &= in - 1) starts |= 1ull << (__builtin_amdgcn_readlane(o, __builtin_ctzll(in)) - t0);
        if (__ballot(o <= t0 + S) != ~0ull) break;
    }
    const int begin = a.offsets[0], end = min(a.offsets[n], a.rows);
    return {starts, begin <= t0 ? 0 : min(S, begin - t0), end <= t0 ? 0 : min(S, end - t0), min(found, n - 1)};
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

__device__ __forceinline__ float share(float f) { return __builtin_amdgcn_rcpf(1.0f + __expf(f)); }
__device__ __forceinline__ float at(const float *p, int64_t i) { return p ? p[i] : 0.0f; }

// What is the same in both directions: which span and channels a workgroup has, and its reads.
template <typename T, int V, int S> struct wave_tile {
    using pack = bagel_pack<T, V>;
    static constexpr int rows = S * WAVES;
    int span, wave, lane, t0, ch;            // ch: a channel to read from, also where this lane has none
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
        for (int i = 0; i < S; ++i) x[i] = *reinterpret_cast<const pack *>(m.row(min(t0 + i, last)) + ch);
    }
    static __device__ __forceinline__ float one(const pack &x, int v)
    {
        if constexpr (V == 1) return (float)x[0];
        else return (float)x[v];
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

// What passes through a sequence without a step, by the workgroups behind those of the spans: each has 64 sequences and all channels.
template <typename A> __device__ __forceinline__ void pass_through(const A &a, int group, const float *from, float *to)
{
    const int last = min(a.sequences, group * 64 + 64);
    for (int s = group * 64 + (threadIdx.x >> 6); s < last; s += WAVES)
        if (a.offsets ? a.offsets[s] >= a.offsets[s + 1] : a.rows == 0)
            for (int ch = threadIdx.x & 63; ch < a.width; ch += 64) to[(int64_t)s * a.width + ch] = at(from, (int64_t)s * a.width + ch);
}

template <typename T, int V, int S> __global__ __launch_bounds__(64 * WAVES, 4) void recurrence_kernel(recurrence_args<T> a)
{
    __shared__ piece pieces[WAVES][64][V];
    __shared__ float before[64][V];
    const int work = next_work(a.counter);
    if (work >= a.spans * a.groups) {
        if (a.final_state) pass_through(a, work - a.spans * a.groups, a.initial, a.final_state);
        return;
    }
    using wt = wave_tile<T, V, S>;
    wt w(work, a);
    w.begin();
    typename wt::pack x[S], f[S];
    w.load(a.forget, a.rows - 1, f);
    w.load(a.value, a.rows - 1, x);
    const segment<S> seg = segment_at<S>(a, w.t0);
    const bool plain = seg.plain();
    const auto initial = [&](int sequence, int v) { return at(a.initial, (int64_t)sequence * a.width + w.ch + v); };

    float q[S][V], h[V];
    piece mine[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        const float b = at(a.bias, w.ch + v);
        mine[v] = {1.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < S; ++i) q[i][v] = share(wt::one(f[i], v) + b);
    }
    if (plain) {
#pragma unroll
        for (int i = 0; i < S; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                mine[v].H += q[i][v] * (wt::one(x[i], v) - mine[v].H);
                mine[v].A -= mine[v].A * q[i][v];
            }
    } else {
        int sequence = seg.sequence;
        bool closed = false;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            if (seg.outside(i)) {
                closed = true;
#pragma unroll
                for (int v = 0; v < V; ++v) mine[v].H = 0.0f;
                continue;
            }
            if (seg.start(i)) {
                closed = true;
                if (i > 0 || sequence < 0) to_next(a, w.t0 + i, sequence);
#pragma unroll
                for (int v = 0; v < V; ++v) mine[v].H = initial(sequence, v);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                mine[v].H += q[i][v] * (wt::one(x[i], v) - mine[v].H);
                mine[v].A -= mine[v].A * q[i][v];
            }
        }
        if (closed)
#pragma unroll
            for (int v = 0; v < V; ++v) mine[v].A = CLOSED;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) pieces[w.wave][w.lane][v] = mine[v];
    __syncthreads();
    if (w.wave == 0) {
        piece all[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            all[v] = pieces[0][w.lane][v];
#pragma unroll
            for (int k = 1; k < WAVES; ++k) all[v] = joined(all[v], pieces[k][w.lane][v]);
            h[v] = 0.0f;
        }
        if (a.spans > 1) {
            uint64_t *to = a.published + (int64_t)w.span * a.width + w.ch;
            if (w.span > 0) {
                if (w.here)
#pragma unroll
                    for (int v = 0; v < V; ++v) publish(to + v, all[v]);
                look_back<V>(a.published, a.width, w.ch, w.span - 1, -1, a.spans, h);
            }
            if (w.here)
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (w.span == 0 || all[v].A != CLOSED) publish(to + v, {CLOSED, through(all[v], h[v])});
        }
#pragma unroll
        for (int v = 0; v < V; ++v) before[w.lane][v] = h[v];
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = before[w.lane][v];
    for (int k = 0; k < w.wave; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = through(pieces[k][w.lane][v], h[v]);
    if (!w.here) return;
    if (a.carry && w.t0 % SPAN == 0 && w.t0 < a.rows)
#pragma unroll
        for (int v = 0; v < V; ++v) a.carry[(int64_t)(w.t0 / SPAN) * a.width + w.ch + v] = h[v];
    if (plain) {
#pragma unroll
        for (int i = 0; i < S; ++i) {
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] += q[i][v] * (wt::one(x[i], v) - h[v]);
            w.store(a.hidden, w.t0 + i, h);
        }
        if (seg.last(S - 1) && a.final_state)
#pragma unroll
            for (int v = 0; v < V; ++v) a.final_state[(int64_t)seg.sequence * a.width + w.ch + v] = h[v];
        return;
    }
    int sequence = seg.sequence;
#pragma unroll
    for (int i = 0; i < S; ++i) {
        if (w.t0 + i >= a.rows) break;
        if (seg.outside(i)) {
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = 0.0f;
        } else {
            if (seg.start(i)) {
                if (i > 0 || sequence < 0) to_next(a, w.t0 + i, sequence);
#pragma unroll
                for (int v = 0; v < V; ++v) h[v] = initial(sequence, v);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] += q[i][v] * (wt::one(x[i], v) - h[v]);
            if (seg.last(i) && a.final_state)
#pragma unroll
                for (int v = 0; v < V; ++v) a.final_state[(int64_t)sequence * a.width + w.ch + v] = h[v];
        }
        w.store(a.hidden, w.t0 + i, h);
    }
}

template <typename T, int V, int S> __global__ __launch_bounds__(64 * WAVES, 4) void recurrence_grad_kernel(recurrence_args<T> a)
{
    static_assert(S * WAVES == SPAN, "a span begins with a row of the carry");
    __shared__ piece pieces[WAVES][64][V], back[WAVES][64][V];
    __shared__ float after[64][V], sums[WAVES][64][V];
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
    w.load(a.forget, a.rows - 1, f);
    w.load(a.value, a.rows - 1, x);
    w.load(a.d_hidden, a.rows - 1, d);
    float h[V], c[V], q[S][V], b[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        h[v] = a.carry[(int64_t)w.span * a.width + w.ch + v];
        b[v] = at(a.bias, w.ch + v);
    }
    const segment<S> seg = segment_at<S>(a, w.t0);
    const bool plain = seg.plain(), open = plain && !seg.last(S - 1);            // open: no sequence begins, or ends, in the segment
    const auto initial = [&](int sequence, int v) { return at(a.initial, (int64_t)sequence * a.width + w.ch + v); };
    const auto final = [&](int sequence, int v) { return at(a.d_final, (int64_t)sequence * a.width + w.ch + v); };
    piece mine[V], mine_back[V];
    int last_sequence = seg.sequence;                                            // of the segment's last row
#pragma unroll
    for (int v = 0; v < V; ++v) {
        mine[v] = mine_back[v] = {1.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < S; ++i) q[i][v] = share(wt::one(f[i], v) + b[v]);
    }
    if (open) {
#pragma unroll
        for (int i = 0; i < S; ++i)
#pragma unroll
            for (int v = 0; v < V; ++v) {
                mine[v].H += q[i][v] * (wt::one(x[i], v) - mine[v].H);
                mine[v].A -= mine[v].A * q[i][v];
                const float g = wt::one(d[S - 1 - i], v) + mine_back[v].H;
                mine_back[v].H = g - q[S - 1 - i][v] * g;
            }
#pragma unroll
        for (int v = 0; v < V; ++v) mine_back[v].A = mine[v].A;
    } else {
        bool closed = false;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            if (seg.outside(i)) {
                closed = true;
#pragma unroll
                for (int v = 0; v < V; ++v) mine[v].H = 0.0f;
                continue;
            }
            if (seg.start(i)) {
                closed = true;
                if (i > 0 || last_sequence < 0) to_next(a, w.t0 + i, last_sequence);
#pragma unroll
                for (int v = 0; v < V; ++v) mine[v].H = initial(last_sequence, v);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                mine[v].H += q[i][v] * (wt::one(x[i], v) - mine[v].H);
                mine[v].A -= mine[v].A * q[i][v];
            }
        }
        if (closed)
#pragma unroll
            for (int v = 0; v < V; ++v) mine[v].A = CLOSED;
        closed = false;
        int sequence = last_sequence;
#pragma unroll
        for (int i = S - 1; i >= 0; --i) {
            if (seg.outside(i)) {
                closed = true;
#pragma unroll
                for (int v = 0; v < V; ++v) mine_back[v].H = 0.0f;
                continue;
            }
            if (seg.last(i)) {
                closed = true;
#pragma unroll
                for (int v = 0; v < V; ++v) mine_back[v].H = final(sequence, v);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const float g = wt::one(d[i], v) + mine_back[v].H;
                mine_back[v].H = g - q[i][v] * g;
                mine_back[v].A -= mine_back[v].A * q[i][v];
            }
            if (seg.start(i)) to_previous(a, w.t0 + i, sequence);
        }
        if (closed)
#pragma unroll
            for (int v = 0; v < V; ++v) mine_back[v].A = CLOSED;
    }
#pragma unroll
    for (int v = 0; v < V; ++v) {
        pieces[w.wave][w.lane][v] = mine[v];
        back[w.wave][w.lane][v] = mine_back[v];
    }
    __syncthreads();
    if (w.wave == 0) {
        piece all[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            all[v] = back[WAVES - 1][w.lane][v];
#pragma unroll
            for (int k = WAVES - 2; k >= 0; --k) all[v] = joined(all[v], back[k][w.lane][v]);
            c[v] = 0.0f;
        }
        if (a.spans > 1) {
            uint64_t *to = a.published + (int64_t)w.span * a.width + w.ch;
            if (w.span < a.spans - 1) {
                if (w.here)
#pragma unroll
                    for (int v = 0; v < V; ++v) publish(to + v, all[v]);
                look_back<V>(a.published, a.width, w.ch, w.span + 1, 1, a.spans, c);
            }
            if (w.here)
#pragma unroll
                for (int v = 0; v < V; ++v)
                    if (w.span == a.spans - 1 || all[v].A != CLOSED) publish(to + v, {CLOSED, through(all[v], c[v])});
        }
#pragma unroll
        for (int v = 0; v < V; ++v) after[w.lane][v] = c[v];
    }
    // h before every row, less its value
    float hx[S][V], sum[V];
    for (int k = 0; k < w.wave; ++k)
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = through(pieces[k][w.lane][v], h[v]);
    {
        int sequence = seg.sequence;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            if (!plain && !seg.outside(i) && seg.start(i)) {
                if (i > 0 || sequence < 0) to_next(a, w.t0 + i, sequence);
#pragma unroll
                for (int v = 0; v < V; ++v) h[v] = initial(sequence, v);
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                hx[i][v] = h[v] - wt::one(x[i], v);
                h[v] -= q[i][v] * hx[i][v];
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int v = 0; v < V; ++v) {
        c[v] = after[w.lane][v];
        sum[v] = 0.0f;
    }
    for (int k = WAVES - 1; k > w.wave; --k)
#pragma unroll
        for (int v = 0; v < V; ++v) c[v] = through(back[k][w.lane][v], c[v]);
    const bool write_x = w.here && a.d_value.data, write_f = w.here && a.d_forget.data;
    int sequence = last_sequence;
#pragma unroll
    for (int i = S - 1; i >= 0; --i) {
        float dx[V], df[V];
        if (!open) {
            if (w.t0 + i >= a.rows) continue;
            if (seg.outside(i)) {
#pragma unroll
                for (int v = 0; v < V; ++v) c[v] = dx[v] = 0.0f;
                if (write_x) w.store(a.d_value, w.t0 + i, dx);
                if (write_f) w.store(a.d_forget, w.t0 + i, dx);
                continue;
            }
            if (seg.last(i))
#pragma unroll
                for (int v = 0; v < V; ++v) c[v] = final(sequence, v);
        }
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const float g = wt::one(d[i], v) + c[v];
            dx[v] = q[i][v] * g;
            c[v] = g - dx[v];
            df[v] = hx[i][v] * (dx[v] - q[i][v] * dx[v]);
            sum[v] += df[v];
        }
        if (write_x) w.store(a.d_value, w.t0 + i, dx);
        if (write_f) w.store(a.d_forget, w.t0 + i, df);
        if (!open && seg.start(i)) {
            if (a.d_initial && w.here)
#pragma unroll
                for (int v = 0; v < V; ++v) a.d_initial[(int64_t)sequence * a.width + w.ch + v] = c[v];
            to_previous(a, w.t0 + i, sequence);
        }
    }
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

// The sum over the spans, 16 threads to a channel.
__global__ __launch_bounds__(1024) void bias_kernel(const float *sums, int spans, int width, float *d_bias)
{
    __shared__ float part[16][64];
    const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6, ch = blockIdx.x * 64 + lane;
    const int from = (int)((int64_t)spans * slice / 16), to = (int)((int64_t)spans * (slice + 1) / 16);
    float v = 0.0f;
    if (ch < width)
#pragma unroll 8
        for (int k = from; k < to; ++k) v += sums[(int64_t)k * width + ch];
    part[slice][lane] = v;
    __syncthreads();
    if (slice > 0 || ch >= width) return;
    v = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) v += part[k][lane];
    d_bias[ch] = v;
}

template <typename T>
__global__ __launch_bounds__(256) void step_kernel(int64_t rows, int width, bagel_rows<T> value, bagel_rows<T> forget, bagel_rows<T> hidden,
                                                   const float *bias, float *state)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < rows * width; i += (int64_t)gridDim.x * 256) {
        const int64_t r = i / width;
        const int ch = (int)(i - r * width);
        const float q = share((float)forget.row(r)[ch] + at(bias, ch));
        float h = state[i];
        h += q * ((float)value.row(r)[ch] - h);
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
    a.spans = (int)((r.rows + S * WAVES - 1) / (S * WAVES));
    a.groups = (r.width + 64 * V - 1) / (64 * V);
    const bool empty = r.sequences > 0 && (r.offsets || r.rows == 0) && (GRAD ? r.d_initial : r.final_state);
    const int64_t work = (int64_t)a.spans * a.groups + (empty ? (r.sequences + 63) / 64 : 0);
    if (work == 0) return;
    const int64_t cells = (int64_t)a.spans * r.width;
    if (a.spans > 1) {
        a.published = (uint64_t *)r.workspace;
        a.counter = (uint32_t *)(a.published + cells);
        const int64_t groups = (cells + 255) / 256;
        nothing_kernel<<<(unsigned)(groups < 4096 ? groups : 4096), 256, 0, stream>>>(a.published, cells, a.counter);
    }
    if constexpr (GRAD) {
        a.bias_sums = r.d_bias ? (float *)((char *)r.workspace + cells * 8 + 16) : nullptr;
        recurrence_grad_kernel<T, V, S><<<(unsigned)work, 64 * WAVES, 0, stream>>>(a);
    } else {
        recurrence_kernel<T, V, S><<<(unsigned)work, 64 * WAVES, 0, stream>>>(a);
    }
}

// Two channels a lane where every row of every matrix begins at a multiple of two entries.
template <typename T, bool GRAD> hipError_t launch_pass(const bagel_gated_recurrence &r, hipStream_t stream)
{
    recurrence_args<T> a = args_of<T>(r, GRAD);
    constexpr int S = GRAD ? 16 : 16;
    int pack = r.width % 2 ? 1 : 2;
    const bagel_matrix all[] = {r.value, r.forget, r.hidden, r.d_hidden, r.d_value, r.d_forget};
    for (int i = 0; i < 6; ++i)
        if (GRAD ? i != 2 : i < 3) pack = bagel_matrix_pack(all[i], r.rows, r.dtype, pack);
    if (pack == 2) launch_spans<T, 2, S, GRAD>(a, r, stream);
    else launch_spans<T, 1, S, GRAD>(a, r, stream);
    if (GRAD && r.d_bias) bias_kernel<<<(r.width + 63) / 64, 1024, 0, stream>>>(a.bias_sums, a.spans, r.width, r.d_bias);
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
    bagel_no_error();
    return BAGEL_OK;
}

extern "C" int bagel_recurrence_grad(const bagel_gated_recurrence *r, void *hip_stream)
{
    if (const char *msg = check_recurrence(r, true)) return bagel_refuse(BAGEL_EINVAL, "bagel_recurrence_grad: %s", msg);
    const hipError_t e = bagel_by_type(r->dtype, [&](auto t) { return launch_grad<typename decltype(t)::type>(*r, (hipStream_t)hip_stream); });
    if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_recurrence_grad: %s", hipGetErrorString(e));
    bagel_no_error();
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
    bagel_no_error();
    return BAGEL_OK;
}
