// The gated linear recurrence of a policy with memory (include/bagel.h) and its gradient.
//
//   q_t = 1 / (1 + exp(f_t + b)),   h_t = h_{t-1} + q_t (x_t - h_{t-1})
// Over several rows h goes to A h + H with A the product of the (1 - q_t), and the H of two pieces one after the other is A2 H1 + H2: a
// span of rows is summed up by two numbers a channel, the pieces side by side.  A span in which a sequence begins does not depend on
// what was before, and its A is not used (and not multiplied: what another sequence left may be infinite).
// Backwards, with g_t the gradient of h_t: g_t = dh_t + c_t, dx_t = q_t g_t, c_{t-1} = g_t - q_t g_t, and
// df_t = (h_{t-1} - x_t) (1 - q_t) q_t g_t, where h_{t-1} is computed again from the state before the span.
#include "activations.h"

namespace {

constexpr int SPAN = BAGEL_RECURRENCE_SPAN;

template <typename T> struct recurrence_args {
    int rows, width, sequences;
    const int32_t *offsets;
    bagel_rows<T> value, forget, hidden, d_hidden, d_value, d_forget;
    const float *bias, *initial, *d_final;
    float *final_state, *carry, *d_initial;
    float2 *pieces;              // [spans][width]: A and H of a span; A = -1 where it does not depend on what was before
    float *after;                // [spans][width]: c that comes into a span from behind
    float *bias_sums;            // [spans][width], null: not wanted
};

// The sequence that row t belongs to, as rows [begin, end); index -1 and the rest of the rows where it belongs to none.
struct sequence {
    int index, begin, end;
};
template <typename A> __device__ __forceinline__ sequence sequence_at(const A &a, int t)
{
    if (!a.offsets) {
        const int each = a.rows / a.sequences, i = t / each;
        return {i, i * each, i * each + each};
    }
    int lo = -1, hi = a.sequences;                       // offsets[lo] <= t < offsets[hi + 1]
    while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (a.offsets[mid] <= t) lo = mid;
        else hi = mid - 1;
    }
    if (lo < 0) return {-1, 0, max(t + 1, min(a.rows, a.offsets[0]))};
    if (lo == a.sequences) return {-1, min(t, a.offsets[lo]), a.rows};
    return {lo, a.offsets[lo], max(t + 1, a.offsets[lo + 1])};
}

__device__ __forceinline__ float share(float f) { return 1.0f / (1.0f + __expf(f)); }
__device__ __forceinline__ float at(const float *p, int64_t i) { return p ? p[i] : 0.0f; }

// A and H of every span.
template <typename T> __global__ __launch_bounds__(64) void pieces_kernel(recurrence_args<T> a)
{
    const int ch = blockIdx.y * 64 + threadIdx.x;
    if (ch >= a.width) return;
    const int first = blockIdx.x * SPAN, last = min(a.rows, first + SPAN);
    const float b = at(a.bias, ch);
    float A = 1.0f, H = 0.0f;
    sequence s = sequence_at(a, first);
    for (int t = first; t < last; ++t) {
        if (t >= s.end) s = sequence_at(a, t);
        if (s.index < 0) {
            A = -1.0f;
            H = 0.0f;
            continue;
        }
        if (t == s.begin) {
            A = -1.0f;
            H = at(a.initial, (int64_t)s.index * a.width + ch);
        }
        const float q = share((float)a.forget.row(t)[ch] + b), x = (float)a.value.row(t)[ch];
        H += q * (x - H);
        if (A >= 0.0f) A -= A * q;
    }
    a.pieces[(int64_t)blockIdx.x * a.width + ch] = make_float2(A, H);
}

__global__ __launch_bounds__(64) void join_pieces_kernel(const float2 *pieces, int spans, int width, float *carry)
{
    const int ch = blockIdx.x * 64 + threadIdx.x;
    if (ch >= width) return;
    float h = 0.0f;
    for (int k = 0; k < spans; ++k) {
        const float2 p = pieces[(int64_t)k * width + ch];
        carry[(int64_t)k * width + ch] = h;
        h = p.x == -1.0f ? p.y : p.x * h + p.y;
    }
}

template <typename T> __global__ __launch_bounds__(64) void hidden_kernel(recurrence_args<T> a)
{
    const int ch = blockIdx.y * 64 + threadIdx.x;
    if (ch >= a.width) return;
    const int first = blockIdx.x * SPAN, last = min(a.rows, first + SPAN);
    const float b = at(a.bias, ch);
    float h = a.carry[(int64_t)blockIdx.x * a.width + ch];
    sequence s = sequence_at(a, first);
    for (int t = first; t < last; ++t) {
        if (t >= s.end) s = sequence_at(a, t);
        if (s.index < 0) {
            a.hidden.row(t)[ch] = (T)0.0f;
            continue;
        }
        if (t == s.begin) h = at(a.initial, (int64_t)s.index * a.width + ch);
        const float q = share((float)a.forget.row(t)[ch] + b), x = (float)a.value.row(t)[ch];
        h += q * (x - h);
        a.hidden.row(t)[ch] = (T)h;
        if (t == s.end - 1 && a.final_state) a.final_state[(int64_t)s.index * a.width + ch] = h;
    }
}

// What passes through a sequence without a step.
__global__ __launch_bounds__(64) void empty_kernel(const int32_t *offsets, int rows, int sequences, int width, const float *from, float *to)
{
    const int ch = blockIdx.y * 64 + threadIdx.x;
    if (ch >= width) return;
    for (int s = blockIdx.x; s < sequences; s += gridDim.x)
        if (offsets ? offsets[s] >= offsets[s + 1] : rows == 0) to[(int64_t)s * width + ch] = at(from, (int64_t)s * width + ch);
}

template <typename T> __global__ __launch_bounds__(64) void pieces_grad_kernel(recurrence_args<T> a)
{
    const int ch = blockIdx.y * 64 + threadIdx.x;
    if (ch >= a.width) return;
    const int first = blockIdx.x * SPAN, last = min(a.rows, first + SPAN);
    const float b = at(a.bias, ch);
    float A = 1.0f, c = 0.0f;
    sequence s = sequence_at(a, last - 1);
    for (int t = last - 1; t >= first; --t) {
        if (t < s.begin) s = sequence_at(a, t);
        if (s.index < 0) {
            A = -1.0f;
            c = 0.0f;
            continue;
        }
        if (t == s.end - 1) {
            A = -1.0f;
            c = at(a.d_final, (int64_t)s.index * a.width + ch);
        }
        const float q = share((float)a.forget.row(t)[ch] + b), g = (float)a.d_hidden.row(t)[ch] + c;
        c = g - q * g;
        if (A >= 0.0f) A -= A * q;
    }
    a.pieces[(int64_t)blockIdx.x * a.width + ch] = make_float2(A, c);
}

__global__ __launch_bounds__(64) void join_pieces_grad_kernel(const float2 *pieces, int spans, int width, float *after)
{
    const int ch = blockIdx.x * 64 + threadIdx.x;
    if (ch >= width) return;
    float c = 0.0f;
    for (int k = spans - 1; k >= 0; --k) {
        const float2 p = pieces[(int64_t)k * width + ch];
        after[(int64_t)k * width + ch] = c;
        c = p.x == -1.0f ? p.y : p.x * c + p.y;
    }
}

template <typename T> __global__ __launch_bounds__(64) void grad_kernel(recurrence_args<T> a)
{
    __shared__ float before[SPAN][64];                   // h before each row
    const int ch = blockIdx.y * 64 + threadIdx.x;
    if (ch >= a.width) return;
    const int first = blockIdx.x * SPAN, last = min(a.rows, first + SPAN);
    const float b = at(a.bias, ch);
    float h = a.carry[(int64_t)blockIdx.x * a.width + ch], c = a.after[(int64_t)blockIdx.x * a.width + ch], sum = 0.0f;
    sequence s = sequence_at(a, first);
    for (int t = first; t < last; ++t) {
        if (t >= s.end) s = sequence_at(a, t);
        if (s.index < 0) continue;
        if (t == s.begin) h = at(a.initial, (int64_t)s.index * a.width + ch);
        const float q = share((float)a.forget.row(t)[ch] + b), x = (float)a.value.row(t)[ch];
        before[t - first][threadIdx.x] = h;
        h += q * (x - h);
    }
    s = sequence_at(a, last - 1);
    for (int t = last - 1; t >= first; --t) {
        if (t < s.begin) s = sequence_at(a, t);
        float dx = 0.0f, df = 0.0f;
        if (s.index >= 0) {
            if (t == s.end - 1) c = at(a.d_final, (int64_t)s.index * a.width + ch);
            const float q = share((float)a.forget.row(t)[ch] + b), x = (float)a.value.row(t)[ch], g = (float)a.d_hidden.row(t)[ch] + c;
            dx = q * g;
            c = g - dx;
            df = (before[t - first][threadIdx.x] - x) * (dx - q * dx);
            sum += df;
            if (t == s.begin && a.d_initial) a.d_initial[(int64_t)s.index * a.width + ch] = c;
        }
        if (a.d_value.data) a.d_value.row(t)[ch] = (T)dx;
        if (a.d_forget.data) a.d_forget.row(t)[ch] = (T)df;
    }
    if (a.bias_sums) a.bias_sums[(int64_t)blockIdx.x * a.width + ch] = sum;
}

__global__ __launch_bounds__(64) void bias_kernel(const float *sums, int spans, int width, float *d_bias)
{
    const int ch = blockIdx.x * 64 + threadIdx.x;
    if (ch >= width) return;
    float v = 0.0f;
    for (int k = 0; k < spans; ++k) v += sums[(int64_t)k * width + ch];
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
    a.offsets = r.offsets;
    a.value = bagel_rows_of<T>(r.value);
    a.forget = bagel_rows_of<T>(r.forget);
    a.hidden = bagel_rows_of<T>(r.hidden);
    a.bias = r.bias;
    a.initial = r.initial;
    a.final_state = r.final_state;
    a.carry = r.carry;
    const size_t cells = (size_t)span_count(r.rows) * r.width;
    a.pieces = (float2 *)r.workspace;
    a.after = (float *)(a.pieces + cells);
    if (grad) {
        a.d_hidden = bagel_rows_of<T>(r.d_hidden);
        a.d_value = bagel_rows_of<T>(r.d_value);
        a.d_forget = bagel_rows_of<T>(r.d_forget);
        a.d_final = r.d_final;
        a.d_initial = r.d_initial;
        a.bias_sums = r.d_bias ? a.after + cells : nullptr;
    } else if (!a.carry) {
        a.carry = a.after;
    }
    return a;
}

template <typename T> hipError_t launch_forward(const bagel_gated_recurrence &r, hipStream_t stream)
{
    const recurrence_args<T> a = args_of<T>(r, false);
    const int spans = span_count(r.rows);
    const dim3 groups(spans, (r.width + 63) / 64);
    if (spans > 0) {
        pieces_kernel<T><<<groups, 64, 0, stream>>>(a);
        join_pieces_kernel<<<groups.y, 64, 0, stream>>>(a.pieces, spans, r.width, a.carry);
        hidden_kernel<T><<<groups, 64, 0, stream>>>(a);
    }
    if (r.final_state && r.sequences > 0 && (r.offsets || r.rows == 0))
        empty_kernel<<<dim3(r.sequences < 1024 ? r.sequences : 1024, groups.y), 64, 0, stream>>>(r.offsets, a.rows, r.sequences, r.width, r.initial,
                                                                                               r.final_state);
    return hipGetLastError();
}

template <typename T> hipError_t launch_grad(const bagel_gated_recurrence &r, hipStream_t stream)
{
    const recurrence_args<T> a = args_of<T>(r, true);
    const int spans = span_count(r.rows);
    const dim3 groups(spans, (r.width + 63) / 64);
    if (spans > 0) {
        pieces_grad_kernel<T><<<groups, 64, 0, stream>>>(a);
        join_pieces_grad_kernel<<<groups.y, 64, 0, stream>>>(a.pieces, spans, r.width, a.after);
        grad_kernel<T><<<groups, 64, 0, stream>>>(a);
    }
    if (r.d_bias) bias_kernel<<<groups.y, 64, 0, stream>>>(a.bias_sums, spans, r.width, r.d_bias);
    if (r.d_initial && r.sequences > 0 && (r.offsets || r.rows == 0))
        empty_kernel<<<dim3(r.sequences < 1024 ? r.sequences : 1024, groups.y), 64, 0, stream>>>(r.offsets, a.rows, r.sequences, r.width, r.d_final,
                                                                                               r.d_initial);
    return hipGetLastError();
}

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
    if (r->rows < 0 || r->rows >= (1ll << 31) - SPAN) return "rows must be >= 0 and below 2^31 - 128";
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

extern "C" int64_t bagel_recurrence_carry_rows(int64_t rows) { return rows < 0 || rows >= (1ll << 31) - SPAN ? BAGEL_EINVAL : span_count(rows); }

extern "C" int64_t bagel_recurrence_workspace(int64_t rows, int32_t width)
{
    if (rows < 0 || rows >= (1ll << 31) - SPAN || width < 1 || width >= 1 << 20) return BAGEL_EINVAL;
    return (int64_t)span_count(rows) * width * 4 * sizeof(float);
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
