// The join of two blocks (include/bagel.h): norm of the branch, gate, residual sum, norm before the next block, and its gradient.
//
// With m(.) the mean over a row, rz = (m(z^2) + eps)^-1/2 and ro the same of `out`:
//   out = x + c a(g) w n,  n = z rz;   normed = u out ro
// and backwards, with e = u d_normed:
//   dx = d_out + ro e - out ro^3 m(e out)              (= d_resid)
//   k = dx c a w;  dz = rz k - z rz^3 m(k z);  dg = dx c w n a'(g)
//   dw = sum_rows dx c a n,  dc = sum_rows dx a w n,  du = sum_rows d_normed out ro
#include "activations.h"

namespace {

template <typename T> struct join_args {
    int64_t rows;
    int width;
    float eps;
    bagel_rows<T> branch, gate, resid, out, normed, d_out, d_normed, d_branch, d_gate, d_resid;
    const float *post_weight, *scale, *pre_weight;
    float *sums;                 // [workgroups][3][width]: d_post_weight, d_scale, d_pre_weight of a workgroup's rows
};

// act(g) and its derivative.  For an infinite g the logistic function is 0 or 1 exactly, and so is its derivative.
template <int ACT> __device__ __forceinline__ float act(float g, float &slope)
{
    if constexpr (ACT == BAGEL_ACT_NONE) {
        slope = 0.0f;
        return 1.0f;
    } else if constexpr (ACT == BAGEL_ACT_IDENTITY) {
        slope = 1.0f;
        return g;
    } else {
        const float sig = 1.0f / (1.0f + __expf(-g));
        const float rest = 1.0f / (1.0f + __expf(g));        // 1 - sig without cancellation
        if constexpr (ACT == BAGEL_ACT_LOGISTIC) {
            slope = sig * rest;
            return sig;
        }
        slope = sig + g * sig * rest;
        return g * sig;
    }
}

// Sums of N values over a workgroup, in a fixed order.
template <int N> __device__ __forceinline__ void group_sum(float (&v)[N], float (*shared)[N])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = bagel_wave_sum(v[i]);
    __syncthreads();
    if (lane == 0)
#pragma unroll
        for (int i = 0; i < N; ++i) shared[wave][i] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0.0f;
        for (int k = 0; k < waves; ++k) v[i] += shared[k][i];
    }
}

__device__ __forceinline__ float at(const float *p, int i) { return p ? p[i] : 1.0f; }

template <typename T, int ACT> __device__ __forceinline__ float join_out(const join_args<T> &a, int64_t r, int i, float rz)
{
    float v = a.resid.data ? (float)a.resid.row(r)[i] : 0.0f;
    if (a.branch.data) {
        float slope;
        const float g = ACT == BAGEL_ACT_NONE ? 0.0f : (float)a.gate.row(r)[i];
        v += at(a.scale, i) * act<ACT>(g, slope) * ((float)a.branch.row(r)[i] * rz * at(a.post_weight, i));
    }
    return v;
}

template <typename T, int ACT> __global__ __launch_bounds__(256) void join_kernel(join_args<T> a)
{
    __shared__ float shared[4][1];
    extern __shared__ float row_out[];
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        float s[1] = {0.0f};
        if (a.branch.data) {
            for (int i = threadIdx.x; i < a.width; i += 256) {
                const float z = (float)a.branch.row(r)[i];
                s[0] += z * z;
            }
            group_sum(s, shared);
        }
        const float rz = 1.0f / sqrtf(s[0] / a.width + a.eps);
        s[0] = 0.0f;
        for (int i = threadIdx.x; i < a.width; i += 256) {
            const float v = join_out<T, ACT>(a, r, i, rz);
            row_out[i] = v;
            if (a.out.data) a.out.row(r)[i] = (T)v;
            s[0] += v * v;
        }
        if (!a.normed.data) continue;
        group_sum(s, shared);
        const float ro = 1.0f / sqrtf(s[0] / a.width + a.eps);
        for (int i = threadIdx.x; i < a.width; i += 256) a.normed.row(r)[i] = (T)(row_out[i] * ro * at(a.pre_weight, i));
    }
}

template <typename T, int ACT> __global__ __launch_bounds__(256) void join_grad_kernel(join_args<T> a)
{
    __shared__ float shared[4][3];
    float *sums = a.sums ? a.sums + (size_t)blockIdx.x * 3 * a.width : nullptr;
    if (sums)
        for (int i = threadIdx.x; i < 3 * a.width; i += 256) sums[i] = 0.0f;
    for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
        float s[3] = {0.0f, 0.0f, 0.0f};
        for (int i = threadIdx.x; i < a.width; i += 256) {
            const float z = a.branch.data ? (float)a.branch.row(r)[i] : 0.0f, out = (float)a.out.row(r)[i];
            s[0] += z * z;
            s[1] += out * out;
            if (a.d_normed.data) s[2] += (float)a.d_normed.row(r)[i] * at(a.pre_weight, i) * out;
        }
        group_sum(s, shared);
        const float rz = 1.0f / sqrtf(s[0] / a.width + a.eps), ro = 1.0f / sqrtf(s[1] / a.width + a.eps);
        const float co = s[2] / a.width * ro * ro * ro;
        float cz = 0.0f;
        for (int pass = 0; pass < 2; ++pass) {
            float k1[1] = {0.0f};
            for (int i = threadIdx.x; i < a.width; i += 256) {
                const float out = (float)a.out.row(r)[i], dy = a.d_normed.data ? (float)a.d_normed.row(r)[i] : 0.0f;
                const float dx = (a.d_out.data ? (float)a.d_out.row(r)[i] : 0.0f) + ro * dy * at(a.pre_weight, i) - out * co;
                float z = 0.0f, g = 0.0f, slope, k = 0.0f, n = 0.0f, av = 1.0f;
                const float c = at(a.scale, i), w = at(a.post_weight, i);
                if (a.branch.data) {
                    z = (float)a.branch.row(r)[i];
                    if (ACT != BAGEL_ACT_NONE) g = (float)a.gate.row(r)[i];
                    av = act<ACT>(g, slope);
                    n = z * rz;
                    k = dx * c * av * w;
                }
                if (pass == 0) {
                    k1[0] += k * z;
                    continue;
                }
                if (a.branch.data) {
                    if (a.d_branch.data) a.d_branch.row(r)[i] = (T)(rz * k - z * cz);
                    if (ACT != BAGEL_ACT_NONE && a.d_gate.data) a.d_gate.row(r)[i] = (T)(dx * c * w * n * slope);
                }
                if (sums) {
                    sums[i] += dx * c * av * n;
                    sums[a.width + i] += dx * av * w * n;
                    sums[2 * a.width + i] += dy * out * ro;
                }
                if (a.d_resid.data) a.d_resid.row(r)[i] = (T)dx;
            }
            if (pass == 0) {
                group_sum(k1, reinterpret_cast<float (*)[1]>(shared));
                cz = k1[0] / a.width * rz * rz * rz;
                __syncthreads();
            }
        }
    }
}

// The gradients of the vectors: sums over the workgroups of the pass over the rows.
__global__ __launch_bounds__(256) void join_sums_kernel(const float *sums, int groups, int width, float *d_post, float *d_scale, float *d_pre)
{
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i >= 3 * width) return;
    float *to = i < width ? d_post : i < 2 * width ? d_scale : d_pre;
    if (!to) return;
    float v = 0.0f;
    for (int k = 0; k < groups; ++k) v += sums[(size_t)k * 3 * width + i];
    to[i % width] = v;
}

constexpr int JOIN_GROUPS = 1024;
int grad_groups(int64_t rows) { return (int)(rows < JOIN_GROUPS ? rows : JOIN_GROUPS); }

template <typename T> join_args<T> args_of(const bagel_join &j)
{
    join_args<T> a{};
    a.rows = j.rows;
    a.width = j.width;
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

template <typename T> hipError_t launch_join(const bagel_join &j, hipStream_t stream)
{
    const join_args<T> a = args_of<T>(j);
    const int groups = (int)(j.rows < 65536 ? j.rows : 65536);
    const size_t lds = sizeof(float) * j.width;
    switch (j.act) {
    case BAGEL_ACT_NONE: join_kernel<T, BAGEL_ACT_NONE><<<groups, 256, lds, stream>>>(a); break;
    case BAGEL_ACT_IDENTITY: join_kernel<T, BAGEL_ACT_IDENTITY><<<groups, 256, lds, stream>>>(a); break;
    case BAGEL_ACT_LOGISTIC: join_kernel<T, BAGEL_ACT_LOGISTIC><<<groups, 256, lds, stream>>>(a); break;
    default: join_kernel<T, BAGEL_ACT_SILU><<<groups, 256, lds, stream>>>(a);
    }
    return hipGetLastError();
}

template <typename T> hipError_t launch_join_grad(const bagel_join &j, hipStream_t stream)
{
    join_args<T> a = args_of<T>(j);
    const int groups = grad_groups(j.rows);
    const bool sums = j.d_post_weight || j.d_scale || j.d_pre_weight;
    a.sums = sums ? (float *)j.workspace : nullptr;
    if (groups > 0) switch (j.act) {
        case BAGEL_ACT_NONE: join_grad_kernel<T, BAGEL_ACT_NONE><<<groups, 256, 0, stream>>>(a); break;
        case BAGEL_ACT_IDENTITY: join_grad_kernel<T, BAGEL_ACT_IDENTITY><<<groups, 256, 0, stream>>>(a); break;
        case BAGEL_ACT_LOGISTIC: join_grad_kernel<T, BAGEL_ACT_LOGISTIC><<<groups, 256, 0, stream>>>(a); break;
        default: join_grad_kernel<T, BAGEL_ACT_SILU><<<groups, 256, 0, stream>>>(a);
        }
    if (sums)
        join_sums_kernel<<<(3 * j.width + 255) / 256, 256, 0, stream>>>(a.sums, groups, j.width, j.d_post_weight, j.d_scale, j.d_pre_weight);
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
    return (int64_t)grad_groups(rows) * 3 * width * sizeof(float);
}

extern "C" int bagel_block_join(const bagel_join *j, void *hip_stream)
{
    if (const char *msg = check_join(j, false)) return bagel_refuse(BAGEL_EINVAL, "bagel_block_join: %s", msg);
    if (j->rows > 0) {
        const hipError_t e = bagel_by_type(j->dtype, [&](auto t) { return launch_join<typename decltype(t)::type>(*j, (hipStream_t)hip_stream); });
        if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_block_join: %s", hipGetErrorString(e));
    }
    bagel_no_error();
    return BAGEL_OK;
}

extern "C" int bagel_block_join_grad(const bagel_join *j, void *hip_stream)
{
    if (const char *msg = check_join(j, true)) return bagel_refuse(BAGEL_EINVAL, "bagel_block_join_grad: %s", msg);
    const hipError_t e = bagel_by_type(j->dtype, [&](auto t) { return launch_join_grad<typename decltype(t)::type>(*j, (hipStream_t)hip_stream); });
    if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_block_join_grad: %s", hipGetErrorString(e));
    bagel_no_error();
    return BAGEL_OK;
}
