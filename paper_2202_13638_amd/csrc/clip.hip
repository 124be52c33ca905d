// The norm of the gradients of many tensors together, and their clipping (include/bagel.h).
//
// Every gradient is read once for the norm, and, where the clipped ones are wanted, once more to be written: the factor is not known before the last
// of them.  Memory bounds both: 33.6 M values in 64 tensors, bf16, take 16.5 us (4.0 TB/s, two launches among them), 402 M, written too, 465 us (5.2 TB/s with the second
// read; 170 of them the norm).  Sums over thousands of workgroups are joined by a kernel of its own, not by atomics, whose order would change the sum.  Squares and their sums are in float64, where neither the largest gradients overflow nor the smallest vanish.
#include <algorithm>
#include <memory>
#include <new>

#include "activations.h"

namespace {

constexpr int TENSORS = 96;                  // 36 bytes each, within the 4 KB of a kernel's arguments
constexpr int PIECE = 8192;                  // entries that a workgroup takes at a time
constexpr int GROUPS = 2048;                 // workgroups of a launch, at most

struct clip_tensor {
    const void *grad;
    void *out;
    int64_t count;
    int dtype;
};

struct clip_args {
    clip_tensor tensor[TENSORS];
    uint32_t first[TENSORS];     // the first piece of each
    uint32_t pieces;             // of all tensors
    int n;
    bool last;                   // whether no launch follows
    int have;                    // sums that launches before this one have left
    double *sums;                // [GROUPS]
};
static_assert(sizeof(clip_args) + 64 <= 4096, "kernel arguments");

// The tensor that a piece is of: the last that does not begin behind it.
__device__ __forceinline__ int tensor_of(const clip_args &a, uint32_t piece)
{
    int k = 0;
    for (int i = (int)(threadIdx.x & 63); i - (int)(threadIdx.x & 63) < a.n; i += 64) k += __popcll(__ballot(i < a.n && a.first[i < a.n ? i : 0] <= piece));
    return k - 1;
}

// The sum over a workgroup, in thread 0.
template <int THREADS> __device__ __forceinline__ double group_sum(double v)
{
    __shared__ double shared[THREADS / 64];
    for (int step = 32; step > 0; step >>= 1) v += __shfl_xor(v, step);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int k = 0; k < THREADS / 64; ++k) v += shared[k];
    return v;
}

// f<type>() for a tensor's type, the same for all threads.
template <typename F> __device__ __forceinline__ void by_type(int dtype, F &&f)
{
    if (dtype == BAGEL_FLOAT32) f(bagel_type<float>());
    else if (dtype == BAGEL_BFLOAT16) f(bagel_type<__bf16>());
    else f(bagel_type<_Float16>());
}

// What threads `lane` of `THREADS` find in pieces number `first`, first + step, ...
template <int THREADS> __device__ __forceinline__ double squares(const clip_args &a, uint32_t first, uint32_t step, int lane)
{
    double sum = 0.0;
    for (uint32_t piece = first; piece < a.pieces; piece += step) {
        const int k = tensor_of(a, piece);
        const int64_t from = (int64_t)(piece - a.first[k]) * PIECE, to = min(from + PIECE, a.tensor[k].count);
        by_type(a.tensor[k].dtype, [&](auto t) {
            using T = typename decltype(t)::type;
            constexpr int V = 16 / sizeof(T);
            const T *g = (const T *)a.tensor[k].grad;
            const int whole = (int)((to - from) / V);
#pragma unroll 8
            for (int i = lane; i < whole; i += THREADS) {
                float v[V];
                bagel_load<T, V>(g + from + V * i, v);
#pragma unroll
                for (int j = 0; j < V; ++j) sum = fma((double)v[j], (double)v[j], sum);
            }
            const int64_t last = from + (int64_t)whole * V + lane;
            if (last < to) sum = fma((double)(float)g[last], (double)(float)g[last], sum);   // (fewer than a pack are left)
        });
    }
    return sum;
}

__global__ __launch_bounds__(256) void squares_kernel(clip_args a)
{
    const double sum = group_sum<256>(squares<256>(a, blockIdx.x, gridDim.x, threadIdx.x));
    if (threadIdx.x == 0) a.sums[blockIdx.x] = (int)blockIdx.x < a.have ? a.sums[blockIdx.x] + sum : sum;
}

struct factor_args {
    const double *sums;
    int count;
    float max_norm, eps;
    const float *grad_scale;
    float *norm, *factor;
};

__device__ __forceinline__ void finish(const factor_args &f, double sum)
{
    const float scale = f.grad_scale ? f.grad_scale[0] : 1.0f, norm = (float)(sqrt(sum) * fabs((double)scale));
    f.norm[0] = norm;
    f.factor[0] = isfinite(norm) ? scale * fminf(1.0f, f.max_norm / (norm + f.eps)) : __builtin_nanf("");
}

__global__ __launch_bounds__(256) void factor_kernel(factor_args f)
{
    double sum = 0.0;
    for (int i = threadIdx.x; i < f.count; i += 256) sum += f.sums[i];
    sum = group_sum<256>(sum);
    if (threadIdx.x == 0) finish(f, sum);
}

// Few values in one launch: a piece to a wave of a single workgroup.
constexpr uint32_t FEW = 32;
__global__ __launch_bounds__(1024) void few_kernel(clip_args a, factor_args f)
{
    const double sum = group_sum<1024>(squares<64>(a, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), 16, threadIdx.x & 63));
    if (threadIdx.x == 0) finish(f, sum);
}

__global__ __launch_bounds__(256) void scale_kernel(clip_args a, const float *factor)
{
    const float f = factor[0];
    if (!isfinite(f)) return;
    for (uint32_t piece = blockIdx.x; piece < a.pieces; piece += gridDim.x) {
        const int k = tensor_of(a, piece);
        const int64_t from = (int64_t)(piece - a.first[k]) * PIECE, to = min(from + PIECE, a.tensor[k].count);
        by_type(a.tensor[k].dtype, [&](auto t) {
            using T = typename decltype(t)::type;
            constexpr int V = 16 / sizeof(T);
            const T *g = (const T *)a.tensor[k].grad;
            T *out = (T *)a.tensor[k].out;
            for (int64_t i = from + V * threadIdx.x; i < to; i += V * 256) {
                if (i + V <= to) {
                    float v[V];
                    bagel_load<T, V>(g + i, v);
#pragma unroll
                    for (int j = 0; j < V; ++j) v[j] *= f;
                    bagel_store<T, V>(out + i, v);
                } else {
                    for (int64_t j = i; j < to; ++j) out[j] = (T)((float)g[j] * f);
                }
            }
        });
    }
}

// Launches f for the tensors, as many at a time as fit the arguments.
template <typename F> hipError_t in_launches(const bagel_clip_tensor *tensors, int32_t n, bool written, F &&f)
{
    clip_args a;
    a.n = 0;
    a.pieces = 0;
    a.have = 0;
    a.sums = nullptr;
    hipError_t e = hipSuccess;
    a.last = false;
    const auto launch = [&] {
        f(a);
        e = hipGetLastError();
        a.n = 0;
        a.pieces = 0;
    };
    for (int i = 0; i < n && e == hipSuccess; ++i) {
        const bagel_clip_tensor &t = tensors[i];
        if (t.count == 0 || (written && !t.out)) continue;
        const uint32_t pieces = (uint32_t)((t.count + PIECE - 1) / PIECE);
        if (a.n == TENSORS || (a.n > 0 && a.pieces + pieces > 1u << 30)) launch();
        if (e != hipSuccess) break;
        a.tensor[a.n] = {t.grad, t.out, t.count, t.dtype};
        a.first[a.n++] = a.pieces;
        a.pieces += pieces;
    }
    a.last = true;
    if (e == hipSuccess && a.n > 0) launch();
    return e;
}

hipError_t launch_clip(const bagel_clip_tensor *tensors, int32_t n, const bagel_clip &o, hipStream_t stream)
{
    factor_args f = {(const double *)o.workspace, 0, o.max_norm, o.eps, o.grad_scale, o.norm, o.factor};
    bool done = false;
    hipError_t e = in_launches(tensors, n, false, [&](clip_args &a) {
        if (f.count == 0 && a.last && a.pieces <= FEW) {
            few_kernel<<<1, 1024, 0, stream>>>(a, f);
            done = true;
            return;
        }
        a.sums = (double *)o.workspace;
        const int groups = (int)(a.pieces < GROUPS ? a.pieces : GROUPS);
        a.have = f.count;
        squares_kernel<<<groups, 256, 0, stream>>>(a);
        f.count = groups > f.count ? groups : f.count;
    });
    if (e != hipSuccess) return e;
    if (!done) factor_kernel<<<1, 256, 0, stream>>>(f);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    return in_launches(tensors, n, true, [&](clip_args &a) {
        scale_kernel<<<(unsigned)(a.pieces < GROUPS ? a.pieces : GROUPS), 256, 0, stream>>>(a, o.factor);
    });
}

// What the pass that writes reads and writes.
struct span {
    uintptr_t begin, end;
    bool written;
};
const char *check_written(const bagel_clip_tensor *tensors, int32_t n)
{
    int written = 0;
    for (int i = 0; i < n; ++i) written += tensors[i].out && tensors[i].count > 0;
    if (written == 0) return nullptr;
    span few[128];
    const std::unique_ptr<span[]> many(written > 64 ? new (std::nothrow) span[2 * (size_t)written] : nullptr);
    if (written > 64 && !many) return "no memory to compare the tensors' places";
    span *const spans = many ? many.get() : few;
    int m = 0;
    for (int i = 0; i < n; ++i) {
        const bagel_clip_tensor &t = tensors[i];
        if (!t.out || t.count == 0) continue;
        const uintptr_t bytes = (uintptr_t)t.count * bagel_type_bytes(t.dtype), grad = (uintptr_t)t.grad, out = (uintptr_t)t.out;
        spans[m++] = {out, out + bytes, true};
        if (out != grad) spans[m++] = {grad, grad + bytes, false};
    }
    std::sort(spans, spans + m, [](const span &x, const span &y) { return x.begin < y.begin; });
    uintptr_t all = 0, outs = 0;                     // where those before end
    for (int i = 0; i < m; ++i) {
        if (spans[i].begin < (spans[i].written ? all : outs)) return "a result overlaps another tensor";
        all = std::max(all, spans[i].end);
        if (spans[i].written) outs = std::max(outs, spans[i].end);
    }
    return nullptr;
}

const char *check_clip(const bagel_clip_tensor *tensors, int32_t n, const bagel_clip *o)
{
    if (n < 0) return "n_tensors must be >= 0";
    if (!o || (n > 0 && !tensors)) return "null argument";
    if (!(o->max_norm >= 0.0f)) return "max_norm must be >= 0";
    if (!(o->eps > 0.0f) || !isfinite(o->eps)) return "eps must be positive";
    if (!o->norm || !o->factor) return "norm and factor are needed";
    for (int i = 0; i < n; ++i) {
        const bagel_clip_tensor &t = tensors[i];
        if (t.count < 0 || t.count >= 1ll << 38) return "count must be >= 0 and below 2^38";
        if (t.count == 0) continue;
        if (!t.grad) return "a tensor has a null argument";
        if (!bagel_type_ok(t.dtype)) return "unknown dtype";
        if (((uintptr_t)t.grad | (uintptr_t)t.out) & (bagel_type_bytes(t.dtype) - 1)) return "a tensor does not start at a multiple of its type";
    }
    if (const char *msg = check_written(tensors, n)) return msg;
    if (!o->workspace) return "a workspace is needed";
    if (o->workspace_bytes < bagel_clip_norm_workspace(n)) return "the workspace is too small";
    if ((uintptr_t)o->workspace & 15) return "the workspace must start at a multiple of 16 bytes";
    return nullptr;
}

}  // namespace

extern "C" int64_t bagel_clip_norm_workspace(int32_t n_tensors) { return n_tensors < 0 ? BAGEL_EINVAL : GROUPS * (int64_t)sizeof(double); }

extern "C" int bagel_clip_norm(const bagel_clip_tensor *tensors, int32_t n_tensors, const bagel_clip *o, void *hip_stream)
{
    if (const char *msg = check_clip(tensors, n_tensors, o)) return bagel_refuse(BAGEL_EINVAL, "bagel_clip_norm: %s", msg);
    const hipError_t e = launch_clip(tensors, n_tensors, *o, (hipStream_t)hip_stream);
    if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_clip_norm: %s", hipGetErrorString(e));
    return BAGEL_OK;
}
