// The join of two blocks (include/bagel.h): norm of the branch, gate, residual sum, norm before the next block, and its gradient.
//
// With m(.) the mean over a row, rz = (m(z^2) + eps)^-1/2 and ro the same of `out`:
//   out = x + c a(g) w n,  n = z rz;   normed = u out ro
// and backwards, with e = u d_normed:
//   dx = d_out + ro e - out ro^3 m(e out)              (= d_resid)
//   k = dx c a w;  dz = rz k - z rz^3 m(k z);  dg = dx c w n a'(g)
//   dw = sum_rows dx c a n,  dc = sum_rows dx a w n,  du = sum_rows d_normed out ro
//
// Memory bounds both, with 5 and 8 entries moved, and the arithmetic is not far behind in 16 bits.  So a row is read once and held in registers until it
// is written, and what is summed over it goes from lane to lane (and from wave to wave through shared memory where a row takes several).  All sums are
// in 32 bits; `out` and `normed` are rounded once, each from the unrounded sum, and the way back starts from the stored `out`.
#include <float.h>

#include "activations.h"

namespace {

template <typename T> struct join_args {
    int64_t rows;
    int width, act;
    float eps;
    bagel_rows<T> branch, gate, resid, out, normed, d_out, d_normed, d_branch, d_gate, d_resid;
    const float *post_weight, *scale, *pre_weight;
    float *sums;                 // [workgroups][2][width]: sums over a workgroup's rows of dx a n (d_post_weight without its factor c, and d_scale
                                 // without w) and of d_normed out ro (d_pre_weight)
};

// act(g) and its derivative.  For an infinite g the logistic function is 0 or 1 exactly and its derivative 0.  silu of minus infinity and its derivative
// are 0, their limits: a gate that is shut for good takes its entry of the branch out.  (silu of plus infinity is infinite, and `out` with it.)  The reciprocal is the
// hardware's, off by one unit in the last place at most: a division takes ten instructions an entry, and in 16 bits these kernels are near the rate of the
// arithmetic (65536 x 4096 back: 844 us with it, 807 without; 20000 x 2500 forward: 131 and 113).
__device__ __forceinline__ float act(int kind, float g, float &slope)
{
    if (kind == BAGEL_ACT_IDENTITY) {
        slope = 1.0f;
        return g;
    }
    const float e = __expf(-fabsf(g)), r = __builtin_amdgcn_rcpf(1.0f + e), s = e * r;         // logistic(|g|) and logistic(-|g|), both without cancellation
    const float sig = g < 0.0f ? s : r, rest = g < 0.0f ? r : s;
    const bool silu = kind == BAGEL_ACT_SILU;
    const float part = fmaxf(g, -FLT_MAX) * sig;             // (NaN stays: sig is NaN too)
    slope = silu ? sig + part * rest : sig * rest;
    return silu ? part : sig;
}

// Sums of N values over the WAVES waves that share a row, in a fixed order.  Two buffers take turns (`turn`), so that one barrier is enough: a
// wave that is ahead writes the other one, and cannot come back to this one before all have read it.
template <int WAVES, int N, int LANES = 64> __device__ __forceinline__ void row_sum(float (&v)[N], float (*shared)[WAVES][4], int &turn)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = LANES == 16 ? bagel_sum_of_16(v[i]) : bagel_wave_sum(v[i]);
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

// A row is held in registers by WAVES waves, K packs of V entries a lane: entry V (64 WAVES k + lane) + i, or (LANES = 16) by a quarter of a wave.  One
// wave or less to a row leaves several rows to a workgroup, which need nothing of each other.  Packs need not be aligned.  One that would reach over the end
// of the row is moved back to end there: its first entries are another pack's, and count as zero here.
template <int V, int K, int WAVES, int LANES = 64> struct tile {
    static_assert(LANES == 64 || (LANES == 16 && WAVES == 1), "a row has whole waves, or 16 lanes of one");
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

// Forward: reads branch, gate and resid, writes out and normed.  The next row waits for this one's end, and other rows of the same compute unit fill the time:
// 64000 x 1024 bf16 123 us, 5.3 TB/s (a copy of this size reaches 5.1); 64000 x 512 f32 120 us, 5.4 TB/s; 16 x 512 3.8 us, all of it latency.
template <typename T, int V, int K, int WAVES, int LANES, bool GATED>
__global__ __launch_bounds__((tile<V, K, WAVES, LANES>::threads)) void join_kernel(join_args<T> a)
{
    using tl = tile<V, K, WAVES, LANES>;
    __shared__ float shared[2][WAVES][4];
    int turn = 0;
    const float per = 1.0f / a.width;
    float cw[K][V], u[K][V];
    tl::product(a.scale, a.post_weight, a.width, cw);
    tl::vector(a.pre_weight, a.width, u);
    for (int64_t r = tl::first_row(); r < a.rows; r += tl::next_row()) {
        float z[K][V], g[K][V], v[K][V], s[1] = {0.0f};
        typename tl::template packed<T> pz, pg, px;
        pz.load(a.branch, r, a.width);
        if (GATED) pg.load(a.gate, r, a.width);
        px.load(a.resid, r, a.width);
        pz.arrived(a.width);
        if (GATED) pg.arrived(a.width);
        px.arrived(a.width);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                z[k][i] = pz(k, i);
                if (GATED) g[k][i] = pg(k, i);
                v[k][i] = px(k, i);
            }
        if (a.branch.data) {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < V; ++i) s[0] += z[k][i] * z[k][i];
            row_sum<WAVES, sizeof(s) / 4, LANES>(s, shared, turn);
            const float rz = 1.0f / sqrtf(s[0] * per + a.eps);
#pragma unroll
            for (int k = 0; k < K; ++k) {
                if (!tl::here(k, a.width)) continue;         // a wave of which nothing is there goes by
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float n = z[k][i] * rz, slope;
                    if (GATED) n *= act(a.act, g[k][i], slope);
                    v[k][i] += cw[k][i] * n;
                }
            }
        }
        if (a.out.data) tl::store(a.out.row(r), a.width, v);
        if (!a.normed.data) continue;
        s[0] = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += v[k][i] * v[k][i];
        row_sum<WAVES, sizeof(s) / 4, LANES>(s, shared, turn);
        const float ro = 1.0f / sqrtf(s[0] * per + a.eps);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) v[k][i] = v[k][i] * ro * u[k][i];
        tl::store(a.normed.row(r), a.width, v);
    }
}

// Back: reads five rows and writes three.  A workgroup keeps its sums for the vectors' gradients in registers over all its rows, so there are few of them, and
// the next row is asked for before this one's sums (without: 65536 x 4096 bf16 1490 us).  That is 808 us, 5.3 TB/s; 64000 x 1024 bf16 213 us,
// 4.9 TB/s; 9973 x 777 f32 47 us, 5.3 TB/s, a quarter of whose lanes have nothing.
// PASS: waves of which nothing is there go by the arithmetic.
template <typename T, int V, int K, int WAVES, int LANES, bool GATED, int ON_SIMD, bool PASS>
__global__ __launch_bounds__((tile<V, K, WAVES, LANES>::threads), ON_SIMD) void join_grad_kernel(join_args<T> a)
{
    using tl = tile<V, K, WAVES, LANES>;
    __shared__ float shared[2][WAVES][4];
    int turn = 0;
    const float per = 1.0f / a.width;
    float cw[K][V], u[K][V], sw[K][V], su[K][V];
    tl::product(a.scale, a.post_weight, a.width, cw);
    tl::vector(a.pre_weight, a.width, u);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) sw[k][i] = su[k][i] = 0.0f;
    struct row {
        typename tl::template packed<T> o, y, z, g, x;
    } next;
    const auto ask = [&](int64_t r) {
        next.o.load(a.out, r, a.width);
        next.y.load(a.d_normed, r, a.width);
        next.z.load(a.branch, r, a.width);
        if (GATED) next.g.load(a.gate, r, a.width);
        next.x.load(a.d_out, r, a.width);
    };
    constexpr bool ahead = WAVES < 16;       // sixteen waves leave 128 registers to a lane: no room for two rows
    if (ahead && tl::first_row() < a.rows) ask(tl::first_row());
    for (int64_t r = tl::first_row(); r < a.rows; r += tl::next_row()) {
        if (!ahead) ask(r);
        row p = next;
        p.o.arrived(a.width);
        p.y.arrived(a.width);
        p.z.arrived(a.width);
        if (GATED) p.g.arrived(a.width);
        p.x.arrived(a.width);
        if (ahead && r + tl::next_row() < a.rows) ask(r + tl::next_row());       // on its way while this row waits for its sums
        float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (PASS && !tl::here(k, a.width)) continue;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s[0] += p.z(k, i) * p.z(k, i);
                s[1] += p.o(k, i) * p.o(k, i);
                s[2] += p.y(k, i) * u[k][i] * p.o(k, i);
            }
        }
        p.o.keep();
        p.y.keep();
        p.z.keep();
        row_sum<WAVES, sizeof(s) / 4, LANES>(s, shared, turn);
        const float rz = 1.0f / sqrtf(s[0] * per + a.eps), ro = 1.0f / sqrtf(s[1] * per + a.eps);
        const float co = s[2] * per * ro * ro;
        float t[1] = {0.0f}, dn[K][V];                               // dn: gradient of R(branch)
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (PASS && !tl::here(k, a.width)) continue;
            float dx[V], dg[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float n = p.o(k, i) * ro, dy = p.y(k, i);
                dx[i] = p.x(k, i) + (ro * (dy * u[k][i]) - n * co);
                su[k][i] += dy * n;
                float av = 1.0f, slope = 0.0f;
                if (GATED) av = act(a.act, p.g(k, i), slope);
                const float zn = p.z(k, i) * rz, x = dx[i] * cw[k][i];
                sw[k][i] += dx[i] * av * zn;                 // times c: d_post_weight, times w: d_scale
                dg[i] = x * zn * slope;
                dn[k][i] = x * av;
                t[0] += dn[k][i] * zn;
            }
            if (a.d_resid.data) tl::store(a.d_resid.row(r), a.width, k, dx);
            if (GATED && a.d_gate.data) tl::store(a.d_gate.row(r), a.width, k, dg);
        }
        p.z.keep();
        if (!a.d_branch.data) continue;
        row_sum<WAVES, 1, LANES>(t, shared, turn);
        const float cz = t[0] * per * rz;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) dn[k][i] = rz * (dn[k][i] - p.z(k, i) * cz);
        tl::store(a.d_branch.row(r), a.width, dn);
    }
    if (!a.sums) return;
    float *sums = a.sums + (size_t)blockIdx.x * 2 * a.width;
    if constexpr (WAVES == 1) {              // several rows' lanes with sums of the same columns: added up in order
        __shared__ float all[2][LANES * K * V];
        for (int row = 0; row < tl::rows; ++row) {
            if ((int)threadIdx.x / LANES == row)
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int j = tl::place(k) + i;
                        all[0][j] = row ? all[0][j] + sw[k][i] : sw[k][i];
                        all[1][j] = row ? all[1][j] + su[k][i] : su[k][i];
                    }
            __syncthreads();
        }
        for (int j = threadIdx.x; j < a.width; j += 256) {
            const int last = a.width - a.width % V;      // from here on the entries of the pack that was moved back
            const int from = j < last ? j : j + V - a.width % V;
#pragma unroll
            for (int q = 0; q < 2; ++q) sums[(size_t)q * a.width + j] = all[q][from];
        }
    } else {
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (tl::here(k, a.width))
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const int j = tl::column(k, a.width) + i;
                    if (i < tl::twice(k, a.width)) continue;
                    sums[j] = sw[k][i];
                    sums[a.width + j] = su[k][i];
                }
    }
}

// Rows that registers do not hold (sixteen waves leave 128 to a lane): three passes over a row, the second and third out of the cache, and the sums
// of a workgroup in its part of the work space, read and written for every row.  8192 x 16384 f32 2200 us, 2.0 TB/s of what has to be moved (1600 us without
// the gradients of the vectors), in bf16 2870 and 1880 us: far from the bound, which is 842 and 421 us.
template <typename T, int V, bool GATED> __global__ __launch_bounds__(1024) void join_grad_wide_kernel(join_args<T> a)
{
    __shared__ float shared[2][16][4];
    int turn = 0;
    const float per = 1.0f / a.width;
    float *sums = a.sums ? a.sums + (size_t)blockIdx.x * 2 * a.width : nullptr;
    const int first = V * threadIdx.x;
    if (sums)
        for (int j = first; j < a.width; j += 1024 * V)
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (j + i < a.width) sums[j + i] = sums[a.width + j + i] = 0.0f;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        const T *branch = a.branch.data ? a.branch.row(r) : nullptr, *d_normed = a.d_normed.data ? a.d_normed.row(r) : nullptr;
        const T *d_out = a.d_out.data ? a.d_out.row(r) : nullptr;
        const auto read = [&](const T *row, int j, float (&v)[V]) {
            const int c = min(j, a.width - V), again = j - c;        // a pack that is moved back to the end of the row: entries before j are zero
            bagel_pack<T, V> x = (bagel_pack<T, V>)(T)0.0f;
            if (row) x = reinterpret_cast<const bagel_loose_pack<T, V> *>(row + c)->x;
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = i < again ? 0.0f : (float)x[i];
        };
        const auto write = [&](const bagel_rows<T> &m, int j, const float (&v)[V]) {
            const int c = min(j, a.width - V), again = j - c;
            bagel_pack<T, V> x;
#pragma unroll
            for (int i = 0; i < V; ++i) x[i] = (T)v[i];
            if (!m.data) return;
            if (!again) reinterpret_cast<bagel_loose_pack<T, V> *>(m.row(r) + c)->x = x;
            else
#pragma unroll
                for (int i = 1; i < V; ++i)
                    if (i >= again) m.row(r)[c + i] = x[i];
        };
        const auto entry = [&](const float *p, int j, int i) { return p ? p[min(j, a.width - V) + i] : 1.0f; };
        float s[3] = {0.0f, 0.0f, 0.0f};
        for (int j = first; j < a.width; j += 1024 * V) {
            float z[V], o[V], dy[V];
            read(branch, j, z);
            read(a.out.row(r), j, o);
            read(d_normed, j, dy);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                s[0] += z[i] * z[i];
                s[1] += o[i] * o[i];
                s[2] += dy[i] * entry(a.pre_weight, j, i) * o[i];
            }
        }
        row_sum<16>(s, shared, turn);
        const float rz = 1.0f / sqrtf(s[0] * per + a.eps), ro = 1.0f / sqrtf(s[1] * per + a.eps);
        const float co = s[2] * per * ro * ro;
        float t[1] = {0.0f};
#pragma unroll 1
        for (int pass = 0; pass < 2; ++pass) {
            const float cz = t[0] * per * rz;
            for (int j = first; j < a.width; j += 1024 * V) {
                float z[V], g[V], o[V], dy[V], dx[V];
                read(branch, j, z);
                if (GATED) read(a.gate.row(r), j, g);
                read(a.out.row(r), j, o);
                read(d_normed, j, dy);
                read(d_out, j, dx);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float n = o[i] * ro, cw = entry(a.scale, j, i) * entry(a.post_weight, j, i);
                    dx[i] += ro * (dy[i] * entry(a.pre_weight, j, i)) - n * co;
                    float av = 1.0f, slope = 0.0f;
                    if (GATED) av = act(a.act, g[i], slope);
                    const float zn = z[i] * rz, x = dx[i] * cw, k = x * av;
                    if (pass == 0) {
                        t[0] += k * zn;
                        continue;
                    }
                    if (sums && i >= j - min(j, a.width - V)) {
                        const int at = min(j, a.width - V) + i;
                        sums[at] += dx[i] * av * zn;
                        sums[a.width + at] += dy[i] * n;
                    }
                    g[i] = x * zn * slope;
                    z[i] = rz * (k - z[i] * cz);
                }
                if (pass == 0) continue;
                write(a.d_resid, j, dx);
                if (GATED) write(a.d_gate, j, g);
                write(a.d_branch, j, z);
            }
            if (pass == 0) row_sum<16>(t, shared, turn);
        }
    }
}

// The gradients of the vectors: sums over the workgroups of the pass over the rows, in a fixed order.  16 threads to a column, each with a part of the
// workgroups: 6.5 us for 512 of them and 4096 columns, 4.7 us for 777: latency.
__global__ __launch_bounds__(1024) void join_sums_kernel(const float *sums, int groups, int width, const float *post, const float *scale, float *d_post,
                                                         float *d_scale, float *d_pre)
{
    __shared__ float part[16][64];
    const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6, i = blockIdx.x * 64 + lane, n = 2 * width;
    float v = 0.0f;
    if (i < n) {
        const int from = groups * slice / 16, to = groups * (slice + 1) / 16;
#pragma unroll 8
        for (int k = from; k < to; ++k) v += sums[(size_t)k * n + i];
    }
    part[slice][lane] = v;
    __syncthreads();
    if (slice > 0 || i >= n) return;
    v = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) v += part[k][lane];
    if (i >= width) {
        if (d_pre) d_pre[i - width] = v;
    } else {
        if (d_post) d_post[i] = scale ? v * scale[i] : v;
        if (d_scale) d_scale[i] = post ? v * post[i] : v;
    }
}

// Workgroups of the backward pass: two to a compute unit, four where rows are short (256 x 262144 in bf16: 262 us with two, 226 with four; 1024 x
// 64000 in f32: 392 and 452).
constexpr int most_groups(int width) { return width <= 256 ? 1024 : 512; }
int grad_groups(int64_t rows, int width) { return (int)(rows < most_groups(width) ? rows : most_groups(width)); }

template <typename T> join_args<T> args_of(const bagel_join &j)
{
    join_args<T> a{};
    a.rows = j.rows;
    a.width = j.width;
    a.act = j.act;
    a.eps = j.eps;
    a.branch = bagel_rows_of<T>(j.branch);
    a.gate = bagel_rows_of<T>(j.gate);
    a.resid = bagel_rows_of<T>(j.resid);
    a.out = bagel_rows_of<T>(j.out);
    a.normed = bagel_rows_of<T>(j.normed);
    a.d_out = bagel_rows_of<T>(j.d_out);
    a.d_normed = bagel_rows_of<T>(j.d_normed);
    a.d_branch = bagel_rows_of<T>(j.d_branch);
    a.d_gate = bagel_rows_of<T>(j.d_gate);
    a.d_resid = bagel_rows_of<T>(j.d_resid);
    a.post_weight = j.post_weight;
    a.scale = j.scale;
    a.pre_weight = j.pre_weight;
    return a;
}

// The number of workgroups.
template <typename T, int V, int K, int WAVES, bool GRAD = true, int ON_SIMD = 1, int LANES = 64, bool PASS = false>
int launch_tile(const join_args<T> &a, bool grad, hipStream_t stream)
{
    using tl = tile<V, K, WAVES, LANES>;
    constexpr int threads = tl::threads, rows = tl::rows;
    const int64_t full = (a.rows + rows - 1) / rows, most = grad ? most_groups(a.width) : 4096;
    const int groups = (int)(full < most ? full : most);
    const bool gated = a.act != BAGEL_ACT_NONE && a.branch.data;
    if (GRAD && grad) {
        if constexpr (GRAD) {
            if (gated) join_grad_kernel<T, V, K, WAVES, LANES, true, ON_SIMD, PASS><<<groups, threads, 0, stream>>>(a);
            else join_grad_kernel<T, V, K, WAVES, LANES, false, ON_SIMD, PASS><<<groups, threads, 0, stream>>>(a);
        }
    } else {
        if (gated) join_kernel<T, V, K, WAVES, LANES, true><<<groups, threads, 0, stream>>>(a);
        else join_kernel<T, V, K, WAVES, LANES, false><<<groups, threads, 0, stream>>>(a);
    }
    return groups;
}

template <typename T, int V> int launch_wide(const join_args<T> &a, hipStream_t stream)
{
    const int groups = grad_groups(a.rows, a.width);
    if (a.act != BAGEL_ACT_NONE && a.branch.data) join_grad_wide_kernel<T, V, true><<<groups, 1024, 0, stream>>>(a);
    else join_grad_wide_kernel<T, V, false><<<groups, 1024, 0, stream>>>(a);
    return groups;
}

// Packs of 16 bytes, single entries where the row is shorter than a pack.  Figures are us, forward / back, in bf16 where no type is said.
//   Up to 16 packs, 16 lanes to a row (200000 x 64: 35 / 69, with a wave to a row 77 / 140; 262144 x 128: 67 / 130, 105 / 193; a wave would have
// few of its lanes at work and four times the rows to go through).
//   Up to 32, a wave and packs of 8 bytes (262144 x 256: 134 / 226, of 16 bytes 172 / 327).
//   Up to 128, a wave, which needs no barrier (64000 x 1024: 124 / 212, by four waves 160 / 379).
//   Up to 256, four waves (32000 x 2048: 131 / 205, by one 140 / 290).
//   Above, back, one pack a lane while eight waves hold the row: with the packs of the next row on their way beside those of this one there is little
// room for more (65536 x 4096, all with a division: 832, two packs on four waves 979); where some of the eight have nothing, four waves on a SIMD at the price
// of a few spilled registers (20000 x 2500: 221, without 278; 65536 x 4096: 891, 832), and up to 320 packs waves without any go by (16384 x 2100: 167, 184;
// 16384 x 3001: 216, 202).  Forward two packs on four waves and one on eight are alike.
//   Up to 1024, two packs on eight waves (16384 x 8192: 257 / 441, one on sixteen 335 / 645; 16384 x 4096 in f32 258 / 409, 246 / 417), which back up
// to 768 go by what is not there (16384 x 4200: 297, 340; 16384 x 6000: 344, 383; 16384 x 8192: 446, 433).
//   Above, what sixteen waves can hold (back only in f32, where a gated tile spills 33 registers: 8192 x 4200 354 us, 3.1 TB/s, 8192 x 8192 500 us, 4.3
// TB/s), and for the way back of wider rows three passes over a row.
template <typename T> int launch_rows(const join_args<T> &a, bool grad, hipStream_t stream)
{
    constexpr int V = 16 / sizeof(T);
    const int packs = (a.width + V - 1) / V;
    if (a.width < V) return launch_tile<T, 1, 1, 1>(a, grad, stream);
    if (packs <= 16) return launch_tile<T, V, 1, 1, true, 1, 16>(a, grad, stream);
    if (packs <= 32) return launch_tile<T, V / 2, 1, 1>(a, grad, stream);
    if (packs <= 64) return launch_tile<T, V, 1, 1>(a, grad, stream);
    if (packs <= 128) return launch_tile<T, V, 2, 1>(a, grad, stream);
    if (packs <= 256) return launch_tile<T, V, 1, 4>(a, grad, stream);
    if (packs <= 320 && grad) return launch_tile<T, V, 1, 8, true, 4, 64, true>(a, true, stream);
    if (packs <= 384 && grad) return launch_tile<T, V, 1, 8, true, 4>(a, true, stream);
    if (packs <= 512) return grad ? launch_tile<T, V, 1, 8>(a, true, stream) : launch_tile<T, V, 2, 4, false>(a, false, stream);
    if (packs <= 768 && grad) return launch_tile<T, V, 2, 8, true, 1, 64, true>(a, true, stream);
    if (packs <= 1024) return launch_tile<T, V, 2, 8>(a, grad, stream);
    if (packs <= 2048 && (V == 4 || !grad)) return launch_tile<T, V, 2, 16, V == 4>(a, grad, stream);
    if (grad) return launch_wide<T, V>(a, stream);
    if constexpr (V == 4) return launch_tile<T, V, 4, 16, false>(a, grad, stream);
    return 0;                                // (16384 entries of 16 bits are 2048 packs)
}

template <typename T> hipError_t launch_join(const bagel_join &j, hipStream_t stream)
{
    launch_rows(args_of<T>(j), false, stream);
    return hipGetLastError();
}

template <typename T> hipError_t launch_join_grad(const bagel_join &j, hipStream_t stream)
{
    join_args<T> a = args_of<T>(j);
    const bool sums = j.d_post_weight || j.d_scale || j.d_pre_weight;
    a.sums = sums ? (float *)j.workspace : nullptr;
    const int groups = j.rows > 0 ? launch_rows(a, true, stream) : 0;
    if (sums)
        join_sums_kernel<<<(2 * j.width + 63) / 64, 1024, 0, stream>>>(a.sums, groups, j.width, j.post_weight, j.scale, j.d_post_weight, j.d_scale, j.d_pre_weight);
    return hipGetLastError();
}

const char *check_join(const bagel_join *j, bool grad)
{
    if (!j) return "null argument";
    if (j->rows < 0 || j->rows >= 1ll << 40) return "rows must be >= 0 and below 2^40";
    if (j->width < 1 || j->width > BAGEL_JOIN_MAX_WIDTH) return "width must be in 1..16384";
    if (!bagel_type_ok(j->dtype)) return "unknown dtype";
    if (j->act < BAGEL_ACT_NONE || j->act > BAGEL_ACT_SILU) return "unknown act";
    if (!(j->eps > 0.0f) || !isfinite(j->eps)) return "eps must be positive";
    if (j->rows > 0) {
        if (j->branch.data && (j->act != BAGEL_ACT_NONE) != (j->gate.data != nullptr)) return "a gate belongs to every act but BAGEL_ACT_NONE";
        if (!grad && !j->resid.data && !j->branch.data) return "resid and branch are both left out";
        if (!grad && !j->out.data && !j->normed.data) return "out and normed are both left out";
        if (grad && !j->out.data) return "out is needed";
        if (grad && !j->branch.data && (j->d_branch.data || j->d_gate.data)) return "d_branch and d_gate need a branch";
        if (grad && j->d_gate.data && j->act == BAGEL_ACT_NONE) return "d_gate needs a gate";
    }
    const bagel_matrix forward[] = {j->branch, j->gate, j->resid, j->out, j->normed};
    const bagel_matrix backward[] = {j->d_out, j->d_normed, j->d_branch, j->d_gate, j->d_resid};
    for (const bagel_matrix &m : forward)
        if (!bagel_matrix_ok(m, j->rows, j->width, j->dtype)) return "a matrix has a stride below the width, or an odd start";
    if (grad)
        for (const bagel_matrix &m : backward)
            if (!bagel_matrix_ok(m, j->rows, j->width, j->dtype)) return "a matrix has a stride below the width, or an odd start";
    if (grad && (j->d_post_weight || j->d_scale || j->d_pre_weight)) {
        if (!j->workspace && j->rows > 0) return "a workspace is needed";
        if (j->workspace_bytes < bagel_block_join_workspace(j->rows, j->width)) return "the workspace is too small";
        if ((uintptr_t)j->workspace & 15) return "the workspace must start at a multiple of 16 bytes";
    }
    return nullptr;
}

}  // namespace

extern "C" int64_t bagel_block_join_workspace(int64_t rows, int32_t width)
{
    if (rows < 0 || width < 1 || width > BAGEL_JOIN_MAX_WIDTH) return BAGEL_EINVAL;
    return (int64_t)grad_groups(rows, width) * 2 * width * sizeof(float);
}

extern "C" int bagel_block_join(const bagel_join *j, void *hip_stream)
{
    if (const char *msg = check_join(j, false)) return bagel_refuse(BAGEL_EINVAL, "bagel_block_join: %s", msg);
    if (j->rows > 0) {
        const hipError_t e = bagel_by_type(j->dtype, [&](auto t) { return launch_join<typename decltype(t)::type>(*j, (hipStream_t)hip_stream); });
        if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_block_join: %s", hipGetErrorString(e));
    }
    return BAGEL_OK;
}

extern "C" int bagel_block_join_grad(const bagel_join *j, void *hip_stream)
{
    if (const char *msg = check_join(j, true)) return bagel_refuse(BAGEL_EINVAL, "bagel_block_join_grad: %s", msg);
    const hipError_t e = bagel_by_type(j->dtype, [&](auto t) { return launch_join_grad<typename decltype(t)::type>(*j, (hipStream_t)hip_stream); });
    if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_block_join_grad: %s", hipGetErrorString(e));
    return BAGEL_OK;
}
