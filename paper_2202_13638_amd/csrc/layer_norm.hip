// Layer norm of rows, or of the equal parts of rows (include/bagel.h), and its gradient.
//
// With m(.) the mean over a part, c = x - m(x), r = (m(c^2) + eps)^-1/2 and n = c r:
//   y = n w + b
// and backwards, with e = w dy:
//   dx = r (e - m(e) - n m(e n)),   dw = sum_rows dy n,   db = sum_rows dy
// The mean is taken off before anything is squared: m(x^2) - m(x)^2 would lose what is small beside the mean.
//
// Memory bounds both, with 2 and 3 entries moved: 64000 x 1024 in 16 parts, float16, 51 us (5.1 TB/s, where a copy of 1 GiB reaches 5.0); the gradient of 65536 x 4096, bf16,
// 335 us (4.8 TB/s, a copy of 4 GiB 4.8), of 9973 x 777, float32, 29 us, of which 24 are the pass over the rows (3.9 TB/s) and 4 the sums.  A part is read once and held in registers until it is written.  Here a "row" of a tile is a part: part
// number s of the call is part s % groups of row s / groups, so that what a workgroup reads at a time lies in one place.  The grid is such that
// a place in it has the same part of all its rows, whose weights it keeps in registers, and the sums for the weights' gradients with them.
#include <numeric>

#include "row_tile.h"

namespace {

template <typename T> struct norm_args {
    int64_t parts;               // of all rows
    int width, groups, each;     // entries of a part; parts of a row; how far on the next part of a place is, in rows (0: there is none)
    float eps;
    bagel_rows<T> x, out, d_out, d_x;
    const float *weight, *bias;
    float *sums;                 // [workgroups][2][min(rows of the tile, groups)][width]: a workgroup's sums of dy n and of dy
};

// Where part number s is: it goes on by whole rows, so the division is done once.
template <typename T, typename tl> struct walk {
    int64_t row, part;           // part: number of the part, of all
    int group;
    __device__ __forceinline__ walk(const norm_args<T> &a) : part(tl::first_row())
    {
        row = part / a.groups;
        group = (int)(part - row * a.groups);
    }
    __device__ __forceinline__ bool there(const norm_args<T> &a) const { return part < a.parts; }
    __device__ __forceinline__ void next(const norm_args<T> &a)
    {
        part += tl::next_row();
        row += a.each;
    }
};

template <typename T> __device__ __forceinline__ bagel_rows<T> part_of(const norm_args<T> &a, const bagel_rows<T> &m, int group)
{
    return {m.data ? m.data + (int64_t)group * a.width : nullptr, m.stride};
}

// c = x - mean: zero in the places that are not of the part, or another pack's
template <typename tl, int V, int K, typename P> __device__ __forceinline__ void centred(const P &x, float mean, int width, bool whole, float (&c)[K][V])
{
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const int from = whole ? 0 : tl::here(k, width) ? tl::twice(k, width) : V;
#pragma unroll
        for (int i = 0; i < V; ++i) c[k][i] = i >= from ? x(k, i) - mean : 0.0f;
    }
}

template <typename T, int V, int K, int WAVES, int LANES>
__global__ __launch_bounds__((tile<V, K, WAVES, LANES>::threads)) void norm_kernel(norm_args<T> a)
{
    using tl = tile<V, K, WAVES, LANES>;
    __shared__ float shared[2][WAVES][4];
    int turn = 0;
    const float per = 1.0f / a.width;
    const bool whole = a.width == V * K * tl::lanes;
    walk<T, tl> at(a);
    float w[K][V], b[K][V];
    tl::vector(a.weight ? a.weight + at.group * a.width : nullptr, a.width, w);
    tl::vector(a.bias ? a.bias + at.group * a.width : nullptr, a.width, b);
    if (!a.bias)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) b[k][i] = 0.0f;
    const bagel_rows<T> from = part_of(a, a.x, at.group), to = part_of(a, a.out, at.group);
    for (; at.there(a); at.next(a)) {
        typename tl::template packed<T> x;
        x.load(from, at.row, a.width);
        x.arrived(a.width);
        float s[1] = {0.0f}, c[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += x(k, i);
        row_sum<WAVES, 1, LANES>(s, shared, turn);
        centred<tl, V, K>(x, s[0] * per, a.width, whole, c);
        s[0] = 0.0f;
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += c[k][i] * c[k][i];
        row_sum<WAVES, 1, LANES>(s, shared, turn);
        const float r = 1.0f / sqrtf(s[0] * per + a.eps);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) c[k][i] = fmaf(c[k][i] * r, w[k][i], b[k][i]);
        tl::store(to.row(at.row), a.width, c);
    }
}

// The number of different parts of a row that a workgroup may have a sum of.
__host__ __device__ constexpr int sum_parts(int rows, int groups) { return rows < groups ? rows : groups; }

template <typename T, int V, int K, int WAVES, int LANES>
__global__ __launch_bounds__((tile<V, K, WAVES, LANES>::threads)) void norm_grad_kernel(norm_args<T> a)
{
    using tl = tile<V, K, WAVES, LANES>;
    __shared__ float shared[2][WAVES][4];
    int turn = 0;
    const float per = 1.0f / a.width;
    const bool whole = a.width == V * K * tl::lanes;
    walk<T, tl> at(a);
    float w[K][V], sw[K][V], sb[K][V];
    tl::vector(a.weight ? a.weight + at.group * a.width : nullptr, a.width, w);
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int i = 0; i < V; ++i) sw[k][i] = sb[k][i] = 0.0f;
    const bagel_rows<T> from = part_of(a, a.x, at.group), dy = part_of(a, a.d_out, at.group), to = part_of(a, a.d_x, at.group);
    struct row {
        typename tl::template packed<T> x, d;
    } next;
    const auto ask = [&](int64_t r) {
        next.x.load(from, r, a.width);
        next.d.load(dy, r, a.width);
    };
    constexpr bool ahead = WAVES < 16;       // sixteen waves leave 128 registers to a lane: no room for two rows
    if (ahead && at.there(a)) ask(at.row);
    for (; at.there(a); at.next(a)) {
        if (!ahead) ask(at.row);
        row now = next;
        typename tl::template packed<T> &x = now.x, &d = now.d;
        x.arrived(a.width);
        d.arrived(a.width);
        if (ahead && at.part + tl::next_row() < a.parts) ask(at.row + a.each);   // on its way while this row waits for its sums
        float s[1] = {0.0f}, t[3] = {0.0f, 0.0f, 0.0f}, c[K][V];
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) s[0] += x(k, i);
        row_sum<WAVES, 1, LANES>(s, shared, turn);
        centred<tl, V, K>(x, s[0] * per, a.width, whole, c);
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float e = d(k, i) * w[k][i];
                t[0] += c[k][i] * c[k][i];
                t[1] += e;
                t[2] += e * c[k][i];
            }
        row_sum<WAVES, 3, LANES>(t, shared, turn);
        const float r = 1.0f / sqrtf(t[0] * per + a.eps), me = t[1] * per, men = t[2] * per * r;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            float dx[V];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float n = c[k][i] * r;
                sw[k][i] += d(k, i) * n;
                sb[k][i] += d(k, i);
                dx[i] = r * (d(k, i) * w[k][i] - me - n * men);
            }
            if (to.data) tl::store(to.row(at.row), a.width, k, dx);
        }
    }
    if (!a.sums) return;
    const int here = sum_parts(tl::rows, a.groups);
    float *sums = a.sums + (size_t)blockIdx.x * 2 * here * a.width;
    if constexpr (WAVES == 1) {              // places with sums of the same part are added up in order
        constexpr int row_places = LANES * K * V;
        __shared__ float all[2][tl::rows * row_places];
        const int mine = threadIdx.x / LANES;
        for (int p = 0; p < tl::rows; ++p) {
            if (mine == p) {
                const bool first = p < here;
                float *const qw = all[0] + (tl::rows <= a.groups ? p : at.group) * row_places, *const qb = qw + tl::rows * row_places;
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        const int j = tl::place(k) + i;
                        qw[j] = first ? sw[k][i] : qw[j] + sw[k][i];
                        qb[j] = first ? sb[k][i] : qb[j] + sb[k][i];
                    }
            }
            __syncthreads();
        }
        const int last = a.width - a.width % V;              // from here on the entries of the pack that was moved back
        for (int j = threadIdx.x; j < here * a.width; j += 256) {
            const int p = j / a.width, c = j - p * a.width, f = p * row_places + (c < last ? c : c + V - a.width % V);
            sums[j] = all[0][f];
            sums[here * a.width + j] = all[1][f];
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
                    sums[a.width + j] = sb[k][i];
                }
    }
}

// The gradients of weight and bias: sums over the workgroups of the pass over the rows, in a fixed order (atomics would have none).  16 threads to an entry, each with a part of the
// workgroups.  With more parts to a row than places in a workgroup, not every workgroup has a part: it is at place (group - rows w) modulo groups of workgroup w.
__global__ __launch_bounds__(1024) void norm_sums_kernel(const float *sums, int workgroups, int rows, int width, int groups, float *d_weight, float *d_bias)
{
    __shared__ float part[16][64];
    const int lane = threadIdx.x & 63, slice = threadIdx.x >> 6, i = blockIdx.x * 64 + lane, all = width * groups, n = 2 * all;
    const int here = sum_parts(rows, groups), from = workgroups * slice / 16, to = workgroups * (slice + 1) / 16;
    const int q = i / all, j = i - q * all;
    const size_t each = (size_t)2 * here * width;
    float v = 0.0f;
    if (i < n) {
        if (here == groups) {
            const float *p = sums + (size_t)q * all + j;
#pragma unroll 8
            for (int k = from; k < to; ++k) v += p[k * each];
        } else {
            const int group = j / width, c = j - group * width;
            for (int k = from; k < to; ++k) {
                const int place = (int)((group + (int64_t)groups * rows - (int64_t)k * rows % groups) % groups);
                if (place < rows) v += sums[k * each + (size_t)(q * here + place) * width + c];
            }
        }
    }
    part[slice][lane] = v;
    __syncthreads();
    if (slice > 0 || i >= n) return;
    v = 0.0f;
#pragma unroll
    for (int k = 0; k < 16; ++k) v += part[k][lane];
    if (q == 0 && d_weight) d_weight[j] = v;
    if (q == 1 && d_bias) d_bias[j] = v;
}

// Workgroups for so many parts, of which a workgroup takes `rows` at a time: with several rounds a multiple of what brings a place back to its part of a row.
int64_t workgroups(int64_t parts, int groups, int rows, int64_t most)
{
    const int64_t all = (parts + rows - 1) / rows, unit = groups / std::gcd(groups, rows);
    if (all <= most || all <= unit) return all;
    return unit * (most / unit > 0 ? most / unit : 1);
}

// Workgroups of the gradient: each keeps sums for the vectors, so more than are needed to keep the memory busy only make more to add up behind them (65536 x 4096 bf16
// by 256, 512 and 1024: 468, 333 and 341 us; 64000 x 512 bf16 by 512, 768 and 1024: 44.6, 42.5 and 42.3; 64000 x 256 f32: 37.2, 36.2 and 38.5).
constexpr int most_groups(int width) { return width <= 512 ? 768 : 512; }

struct pass {
    int64_t workgroups;
    int rows;                    // of the tile
};

// Launches the pass over the rows, or (`launch` false) only says how it would.
template <typename T, int V, int K, int WAVES, int LANES = 64> pass run_tile(norm_args<T> &a, bool grad, bool launch, hipStream_t stream)
{
    using tl = tile<V, K, WAVES, LANES>;
    const pass p = {workgroups(a.parts, a.groups, tl::rows, grad ? most_groups(a.width) : 4096), tl::rows};
    a.each = (int)(p.workgroups * tl::rows / a.groups);      // (what is not whole rows is not gone on by: then there is one round)
    if (launch && grad) norm_grad_kernel<T, V, K, WAVES, LANES><<<(unsigned)p.workgroups, tl::threads, 0, stream>>>(a);
    if (launch && !grad) norm_kernel<T, V, K, WAVES, LANES><<<(unsigned)p.workgroups, tl::threads, 0, stream>>>(a);
    return p;
}

// Packs of 16 bytes, single entries where a part is shorter than a pack.
template <typename T> pass run_rows(norm_args<T> &a, bool grad, bool launch, hipStream_t stream)
{
    constexpr int V = 16 / sizeof(T);
    const int packs = (a.width + V - 1) / V;
    if (a.width < V) return run_tile<T, 1, 1, 1, 16>(a, grad, launch, stream);
    if (packs <= 8) return run_tile<T, V, 1, 1, 8>(a, grad, launch, stream);
    if (packs <= 16) return run_tile<T, V, 1, 1, 16>(a, grad, launch, stream);
    if (packs <= 64) return run_tile<T, V, 1, 1>(a, grad, launch, stream);
    if (packs <= 128) return run_tile<T, V, 2, 1>(a, grad, launch, stream);
    if (packs <= 256) return run_tile<T, V, 1, 4>(a, grad, launch, stream);
    if (packs <= 512) return run_tile<T, V, 1, 8>(a, grad, launch, stream);
    if (packs <= 1024) return run_tile<T, V, 2, 8>(a, grad, launch, stream);
    if constexpr (V == 4) {
        if (packs > 2048) return run_tile<T, V, 4, 16>(a, grad, launch, stream);
    }
    return run_tile<T, V, 2, 16>(a, grad, launch, stream);
}

template <typename T> norm_args<T> args_of(const bagel_norm &n, bool grad)
{
    norm_args<T> a{};
    a.parts = n.rows * n.groups;
    a.width = n.width / n.groups;
    a.groups = n.groups;
    a.eps = n.eps;
    a.x = bagel_rows_of<T>(n.x);
    a.weight = n.weight;
    if (!grad) {
        a.out = bagel_rows_of<T>(n.out);
        a.bias = n.bias;
    } else {
        a.d_out = bagel_rows_of<T>(n.d_out);
        a.d_x = bagel_rows_of<T>(n.d_x);
    }
    return a;
}

template <typename T> hipError_t launch_norm(const bagel_norm &n, hipStream_t stream)
{
    norm_args<T> a = args_of<T>(n, false);
    run_rows(a, false, true, stream);
    return hipGetLastError();
}

template <typename T> hipError_t launch_norm_grad(const bagel_norm &n, hipStream_t stream)
{
    norm_args<T> a = args_of<T>(n, true);
    const bool sums = n.d_weight || n.d_bias;
    a.sums = sums ? (float *)n.workspace : nullptr;
    pass p = {0, 1};
    if (n.rows > 0) p = run_rows(a, true, true, stream);
    if (sums)
        norm_sums_kernel<<<(2 * n.width + 63) / 64, 1024, 0, stream>>>(a.sums, (int)p.workgroups, p.rows, a.width, a.groups, n.d_weight, n.d_bias);
    return hipGetLastError();
}

const char *check_sizes(int64_t rows, int32_t width, int32_t groups)
{
    if (rows < 0 || rows >= 1ll << 40) return "rows must be >= 0 and below 2^40";
    if (width < 1 || width > BAGEL_NORM_MAX_WIDTH) return "width must be in 1..16384";
    if (groups < 1 || width % groups != 0) return "groups must divide the width";
    return nullptr;
}

const char *check_norm(const bagel_norm *n, bool grad)
{
    if (!n) return "null argument";
    if (const char *msg = check_sizes(n->rows, n->width, n->groups)) return msg;
    if (!bagel_type_ok(n->dtype)) return "unknown dtype";
    if (!(n->eps > 0.0f) || !isfinite(n->eps)) return "eps must be positive";
    if (n->rows > 0) {
        if (!n->x.data) return "x is needed";
        if (!grad && !n->out.data) return "out is needed";
        if (grad && !n->d_out.data) return "d_out is needed";
    }
    const bagel_matrix forward[] = {n->x, n->out}, backward[] = {n->x, n->d_out, n->d_x};
    for (const bagel_matrix &m : forward)
        if (!grad && !bagel_matrix_ok(m, n->rows, n->width, n->dtype)) return "a matrix has a stride below the width, or an odd start";
    for (const bagel_matrix &m : backward)
        if (grad && !bagel_matrix_ok(m, n->rows, n->width, n->dtype)) return "a matrix has a stride below the width, or an odd start";
    if (grad && (n->d_weight || n->d_bias)) {
        if (!n->workspace && n->rows > 0) return "a workspace is needed";
        if (n->workspace_bytes < bagel_layer_norm_workspace(n->rows, n->width, n->groups)) return "the workspace is too small";
        if ((uintptr_t)n->workspace & 15) return "the workspace must start at a multiple of 16 bytes";
    }
    return nullptr;
}

// The size of the sums, which goes by the type too: the larger of the two.
template <typename T> int64_t sums_bytes(int64_t rows, int32_t width, int32_t groups)
{
    bagel_norm n{};
    n.rows = rows;
    n.width = width;
    n.groups = groups;
    norm_args<T> a = args_of<T>(n, true);
    const pass p = run_rows(a, true, false, nullptr);
    return p.workgroups * 2 * sum_parts(p.rows, groups) * a.width * (int64_t)sizeof(float);
}

}  // namespace

extern "C" int64_t bagel_layer_norm_workspace(int64_t rows, int32_t width, int32_t groups)
{
    if (check_sizes(rows, width, groups)) return BAGEL_EINVAL;
    const int64_t a = sums_bytes<float>(rows, width, groups), b = sums_bytes<__bf16>(rows, width, groups);
    return a > b ? a : b;
}

extern "C" int bagel_layer_norm(const bagel_norm *n, void *hip_stream)
{
    if (const char *msg = check_norm(n, false)) return bagel_refuse(BAGEL_EINVAL, "bagel_layer_norm: %s", msg);
    if (n->rows > 0) {
        const hipError_t e = bagel_by_type(n->dtype, [&](auto t) { return launch_norm<typename decltype(t)::type>(*n, (hipStream_t)hip_stream); });
        if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_layer_norm: %s", hipGetErrorString(e));
    }
    return BAGEL_OK;
}

extern "C" int bagel_layer_norm_grad(const bagel_norm *n, void *hip_stream)
{
    if (const char *msg = check_norm(n, true)) return bagel_refuse(BAGEL_EINVAL, "bagel_layer_norm_grad: %s", msg);
    const hipError_t e = bagel_by_type(n->dtype, [&](auto t) { return launch_norm_grad<typename decltype(t)::type>(*n, (hipStream_t)hip_stream); });
    if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_layer_norm_grad: %s", hipGetErrorString(e));
    return BAGEL_OK;
}
