// Linear attention with a decay for every head (include/bagel.h), its gradient and its single step.
//
// With l the decay of a memory, over the rows t of a sequence,
//   S_t = l S_{t-1} + k_t v_t^T,   o_t = c S_t^T q_t
// and backwards, with R_t the gradient of S_t,
//   R_t = c q_t do_t^T + l R_{t+1},   dq_t = c S_t do_t,   dk_t = R_t v_t,   dv_t = R_t^T k_t,   dS_0 = l R_1
// So every gradient is a linear attention of its own: dq that of do, v, k with the memory S^T; dv that of k, q, do and dk that of v, do, q from the
// last row to the first, with the memories R and R^T.
#include "linear_attention.h"

namespace {

// A pass row after row, for heads that are shorter than a pack: a workgroup to a memory, an entry of its columns in each of 128 threads for half of its rows.
template <typename T> __global__ __launch_bounds__(256) void rows_kernel(bagel_attention_pass<T> p)
{
    constexpr int MOST = BAGEL_ATTENTION_MAX_WIDTH;
    __shared__ float sa[MOST], sb[MOST], sc[MOST], part[MOST];
    const int64_t work = (int64_t)p.sequences * p.states, group = p.launched + blockIdx.x;
    if (group >= work) return bagel_clear_behind(p, group - work, p.groups - work);
    const int state = (int)(group % p.states), sequence = (int)(group / p.states), t = threadIdx.x, column = t & 127, half = t >> 7;
    int64_t begin = (int64_t)sequence * p.each, end = begin + p.each;
    if (p.offsets) {
        begin = min(max((int64_t)p.offsets[sequence], (int64_t)0), p.rows);
        end = min(max((int64_t)p.offsets[sequence + 1], begin), p.rows);
    }
    const float decay = expf(p.log_decay[state]);
    float S[MOST / 2];
    const int64_t memory = ((int64_t)sequence * p.states + state) * p.wb * p.wc;
#pragma unroll
    for (int j = 0; j < MOST / 2; ++j) {
        const int r = half * (MOST / 2) + j;
        S[j] = p.first && r < p.wb && column < p.wc ? p.first[memory + r * p.step_b + column * p.step_c] : 0.0f;
    }
    for (int64_t n = 0; n < end - begin; ++n) {
        const int64_t row = p.back ? end - 1 - n : begin + n;
        if (!p.back)
#pragma unroll
            for (int j = 0; j < MOST / 2; ++j) S[j] *= decay;
        for (int g = 0; g < p.ks; ++g) {
            __syncthreads();
            if (t < MOST) sb[t] = t < p.wb ? (float)p.b.at(row, state * p.ks + g)[t] * p.scale_b : 0.0f;
            else sc[t - MOST] = t - MOST < p.wc ? (float)p.c.at(row, state * p.ks + g)[t - MOST] : 0.0f;
            __syncthreads();
#pragma unroll
            for (int j = 0; j < MOST / 2; ++j) S[j] = fmaf(sb[half * (MOST / 2) + j], sc[column], S[j]);
        }
        for (int g = 0; g < p.qs && p.out.data; ++g) {
            __syncthreads();
            if (t < MOST) sa[t] = t < p.wb ? (float)p.a.at(row, state * p.qs + g)[t] : 0.0f;
            __syncthreads();
            float o = 0.0f;
#pragma unroll
            for (int j = 0; j < MOST / 2; ++j) o = fmaf(sa[half * (MOST / 2) + j], S[j], o);
            if (half) part[column] = o;
            __syncthreads();
            if (!half && column < p.wc) p.out.at(row, state * p.qs + g)[column] = (T)((o + part[column]) * p.scale);
        }
        if (p.back)
#pragma unroll
            for (int j = 0; j < MOST / 2; ++j) S[j] *= decay;
    }
    if (!p.last) return;
#pragma unroll
    for (int j = 0; j < MOST / 2; ++j) {
        const int r = half * (MOST / 2) + j;
        if (r < p.wb && column < p.wc) p.last[memory + r * p.step_b + column * p.step_c] = S[j];
    }
}

// One row of each of many sequences.  A workgroup to a memory: V columns to a thread, whose rows follow each other by as many as there are threads for; the
// memory is read and written once, where no more than HEADS heads share it (more of them read it again, out of the cache).
//   The memories bound it, 8 bytes an entry: 256 sequences of 8 memories of 64 x 64 take 16.2 us (4.2 TB/s) of whole calls, 13 to 15 of the kernel, one sequence 6.8 us, of which
// 5 are the kernel's latency.  Packs of four columns: by single columns 22.6 and 8.7 us.
template <typename T, int V>
__global__ __launch_bounds__(256) void step_kernel(int64_t rows, int states, int each, int wk, int wv, float scale, const float *log_decay, bagel_heads_of<T> q,
                                                   bagel_heads_of<T> k, bagel_heads_of<T> v, bagel_heads_of<T> out, float *state)
{
    constexpr int HEADS = 4, AHEAD = 4, MOST = BAGEL_ATTENTION_MAX_WIDTH;
    __shared__ float sk[MOST], sq[HEADS][MOST], part[HEADS][256 * V];
    const int t = threadIdx.x, columns = wv / V, apart = 256 / columns, c = t % columns * V, first = t / columns;
    const bool here = first < apart;
    for (int64_t i = blockIdx.x; i < rows * states; i += gridDim.x) {
        const int64_t row = i / states;
        const int s = (int)(i - row * states);
        float *S = state + i * wk * wv + c;
        const float decay = expf(log_decay[s]);
        for (int h0 = 0; h0 < each; h0 += HEADS) {
            float x[V], o[HEADS][V];
#pragma unroll
            for (int j = 0; j < V; ++j) {
                x[j] = (float)v.at(row, s)[c + j];
#pragma unroll
                for (int h = 0; h < HEADS; ++h) o[h][j] = 0.0f;
            }
            // the first rows of the memory are on their way while the keys and queries are put where all threads read them
            float m[AHEAD][V];
#pragma unroll
            for (int a = 0; a < AHEAD; ++a)
                if (here && first + a * apart < wk) bagel_load<float, V>(S + (first + a * apart) * wv, m[a]);
            __syncthreads();
            if (t < wk) sk[t] = (float)k.at(row, s)[t];
            for (int j = t; j < HEADS * wk; j += 256) {
                const int h = j / wk;
                sq[h][j - h * wk] = h0 + h < each ? (float)q.at(row, s * each + h0 + h)[j - h * wk] : 0.0f;
            }
            __syncthreads();
            for (int r0 = first; here && r0 < wk; r0 += AHEAD * apart) {
#pragma unroll
                for (int a = 0; a < AHEAD; ++a) {
                    const int r = r0 + a * apart;
                    if (r >= wk) continue;
                    if (r0 != first) bagel_load<float, V>(S + r * wv, m[a]);
                    if (h0 == 0) {
#pragma unroll
                        for (int j = 0; j < V; ++j) m[a][j] = fmaf(sk[r], x[j], m[a][j] * decay);
                        bagel_store<float, V>(S + r * wv, m[a]);
                    }
#pragma unroll
                    for (int h = 0; h < HEADS; ++h)
#pragma unroll
                        for (int j = 0; j < V; ++j) o[h][j] = fmaf(sq[h][r], m[a][j], o[h][j]);
                }
            }
            if (here)
#pragma unroll
                for (int h = 0; h < HEADS; ++h)
#pragma unroll
                    for (int j = 0; j < V; ++j) part[h][first * wv + c + j] = o[h][j];
            __syncthreads();
            for (int j = t; j < min(HEADS, each - h0) * wv; j += 256) {
                const int h = j / wv;
                float sum = 0.0f;
                for (int a = 0; a < apart; ++a) sum += part[h][a * wv + j - h * wv];
                out.at(row, s * each + h0 + h)[j - h * wv] = (T)(sum * scale);
            }
        }
    }
}

// Rows of a segment: as many segments as the card takes at a time, some less, as one more is a round of its own; but no shorter than is worth a memory that is
// written and read.  Where there are sequences enough, they are left whole, and only one that is far longer than the others is shared out.
//   131072 rows in one sequence, bf16, by chunks to a segment: 8 heads of 128 on 2 memories, 16 chunks (258 workgroups, of which 256 fit) 353 us, 17 to 20 (242 to 206
// workgroups) 244, 242, 242 and 244, 24 279; 8 heads of 64 on 8 memories, 32 chunks (520 workgroups, of which 512 fit) 227, 33 to 36 202, 204, 199 and 204, 40 208.
int64_t wanted_groups(const bagel_attention &b) { return b.key_width > 64 || b.value_width > 64 ? 248 : 496; }      // one or two workgroups to a compute unit
int64_t segment_rows(const bagel_attention &b)
{
    constexpr int64_t chunk = BAGEL_ATTENTION_CHUNK;
    // What a segment's steps take is at least what the launches for the memories take: some eight steps of one head in 16 bits, two in 32.  That is for sequences
    // enough (8 heads of 64 on 8 memories, bf16, 20000 rows in 61 sequences: 46 us with eight chunks, 58 with four, 62 with two; f32, 10007 rows in 61, 6 heads of 40 and 77 on 3,
    // 91 with two, 87 with one, 105 with three); one short sequence would do with fewer (8000 rows, bf16: 38 with eight, 27 with four).
    const int64_t step = (int64_t)(b.heads / b.states) * (b.dtype == BAGEL_FLOAT32 ? 4 : 1), least = step < 8 ? 8 / step : 1;
    const int64_t wanted = wanted_groups(b);
    int64_t rows = (b.rows * b.states + wanted - 1) / wanted;
    if (b.sequences > 0 && (int64_t)b.sequences * b.states >= wanted) rows = std::max(rows, 2 * b.rows / b.sequences);
    return chunk * std::max((rows + chunk - 1) / chunk, least);
}

// A segment's rows, and how many numbers there are for segments that are not the first of their sequence.
struct segments {
    int64_t rows, further;
};
segments segments_of(const bagel_attention &b, bool offsets)
{
    const int64_t rows = segment_rows(b), each = b.sequences > 0 ? b.rows / b.sequences : 0;
    return {rows, offsets ? (b.rows > rows ? b.rows / rows : 0) : each > 0 ? (each - 1) / rows * b.sequences : 0};
}
int64_t memories_floats(const bagel_attention &b, const segments &s)
{
    return s.further > 0 ? (b.sequences + s.further) * b.states * b.key_width * b.value_width : 0;
}

// Whether segments join the memories before them themselves, which saves a launch of 5 us: where there can be few, and where there are sequences enough, so that
// mostly there are none.  (Each reads all that its sequence's segments before it have added: 16 of them take as long as the launch.)
bool joined(const bagel_attention &b, int64_t further) { return further <= 16 || (further <= 64 && (int64_t)b.sequences * b.states >= wanted_groups(b)); }

template <typename T> bagel_attention_pass<T> args_of(const bagel_attention &b)
{
    const segments s = segments_of(b, b.offsets);
    bagel_attention_pass<T> p{};
    p.rows = b.rows;
    p.sequences = b.sequences;
    p.each = b.sequences > 0 ? (int)(b.rows / b.sequences) : 0;
    p.states = b.states;
    p.offsets = b.offsets;
    p.log_decay = b.log_decay;
    p.scale = p.scale_b = 1.0f;
    p.segment = s.rows;
    p.further = s.further;
    p.join = joined(b, s.further);
    p.qs = p.ks = 1;
    return p;
}

// S is [key][value]; a pass whose memory is its transpose.
template <typename T> void turned(bagel_attention_pass<T> &p, const bagel_attention &b, bool turned)
{
    p.wb = turned ? b.value_width : b.key_width;
    p.wc = turned ? b.key_width : b.value_width;
    p.step_b = turned ? 1 : b.value_width;
    p.step_c = turned ? b.value_width : 1;
}

// The matrix kernels load packs of 16 bytes; heads that are shorter than that go row by row.
template <typename T> bool by_rows(const bagel_attention &b) { return b.key_width < 16 / (int)sizeof(T) || b.value_width < 16 / (int)sizeof(T); }

template <typename T> hipError_t launch_pass(const bagel_attention_pass<T> &p, const bagel_attention &b, hipStream_t stream)
{
    if (!by_rows<T>(b)) return bagel_launch_attention_pass(p, stream);
    const int64_t work = (int64_t)p.sequences * p.states, clear = p.offsets && p.out.data && p.rows > 0 ? 32 : 0;
    bagel_attention_pass<T> a = p;
    a.groups = work + clear;
    return bagel_attention_launches(a.groups, [&](unsigned groups, int64_t before) {
        a.launched = before;
        rows_kernel<T><<<groups, 256, 0, stream>>>(a);
    });
}

// S along the rows, and R from the last row to the first.
template <typename T> bagel_attention_pass<T> forward_pass(const bagel_attention &b)
{
    bagel_attention_pass<T> p = args_of<T>(b);
    turned(p, b, false);
    p.qs = b.heads / b.states;
    p.scale = b.scale;
    p.a = bagel_heads_from<T>(b.query);
    p.b = bagel_heads_from<T>(b.key);
    p.c = bagel_heads_from<T>(b.value);
    p.out = bagel_heads_from<T>(b.out);
    p.first = b.initial;
    p.last = b.final_state;
    p.memories = (float *)b.workspace;
    return p;
}
template <typename T> bagel_attention_pass<T> backward_pass(const bagel_attention &b, float *memories)
{
    bagel_attention_pass<T> p = args_of<T>(b);
    turned(p, b, false);
    p.back = true;
    p.ks = b.heads / b.states;
    p.scale_b = b.scale;
    p.a = bagel_heads_from<T>(b.key);
    p.b = bagel_heads_from<T>(b.query);
    p.c = bagel_heads_from<T>(b.d_out);
    p.out = bagel_heads_from<T>(b.d_value);
    p.first = b.d_final;
    p.last = b.d_initial;
    p.memories = memories;
    return p;
}

template <typename T> hipError_t launch_attention(const bagel_attention &b, hipStream_t stream)
{
    const bagel_attention_pass<T> p = forward_pass<T>(b);
    if (!by_rows<T>(b))
        if (const hipError_t e = bagel_launch_attention_memories(&p, 1, stream)) return e;
    return launch_pass(p, b, stream);
}

template <typename T> hipError_t launch_attention_grad(const bagel_attention &b, hipStream_t stream)
{
    const bool queries = b.d_query.data, values = b.d_value.data || b.d_initial, keys = b.d_key.data;
    bagel_attention_pass<T> s = forward_pass<T>(b), r = backward_pass<T>(b, (float *)b.workspace + memories_floats(b, segments_of(b, b.offsets)));
    hipError_t e = hipSuccess;
    if (!by_rows<T>(b)) {
        const bagel_attention_pass<T> both[2] = {s, r};
        if (queries && (values || keys)) e = bagel_launch_attention_memories(both, 2, stream);
        else if (queries) e = bagel_launch_attention_memories(&s, 1, stream);
        else if (values || keys) e = bagel_launch_attention_memories(&r, 1, stream);
    }
    if (e == hipSuccess && queries) {
        turned(s, b, true);
        s.a = bagel_heads_from<T>(b.d_out);
        s.b = bagel_heads_from<T>(b.value);
        s.c = bagel_heads_from<T>(b.key);
        s.out = bagel_heads_from<T>(b.d_query);
        s.last = nullptr;
        e = launch_pass(s, b, stream);
    }
    bagel_attention_pass<T> t = r;
    turned(t, b, true);
    t.a = bagel_heads_from<T>(b.value);
    t.b = r.c;
    t.c = r.b;
    t.out = bagel_heads_from<T>(b.d_key);
    t.last = nullptr;
    if constexpr (sizeof(T) == 2) {
        if (e == hipSuccess && keys && b.d_value.data && !by_rows<T>(b) && bagel_attention_keys_fit<T>(b.key_width, b.value_width, r.ks))
            return bagel_launch_attention_keys(r, t, stream);
    }
    if (e == hipSuccess && values) e = launch_pass(r, b, stream);
    if (e == hipSuccess && keys) e = launch_pass(t, b, stream);
    return e;
}

template <typename T> hipError_t launch_step(const bagel_attention &b, hipStream_t stream)
{
    const int64_t groups = b.rows * b.states;
    const auto launch = [&](auto kernel) {
        kernel<<<(unsigned)(groups < 1 << 20 ? groups : 1 << 20), 256, 0, stream>>>(b.rows, b.states, b.heads / b.states, b.key_width, b.value_width, b.scale, b.log_decay,
                                                                                   bagel_heads_from<T>(b.query), bagel_heads_from<T>(b.key),
                                                                                   bagel_heads_from<T>(b.value), bagel_heads_from<T>(b.out), b.state);
    };
    if (b.value_width % 4 == 0) launch(step_kernel<T, 4>);
    else launch(step_kernel<T, 1>);
    return hipGetLastError();
}

const char *check_sizes(const bagel_attention *b)
{
    if (!b) return "null argument";
    if (b->rows < 0 || b->rows >= 1 << 28) return "rows must be >= 0 and below 2^28";
    if (b->sequences < 0 || b->sequences >= 1 << 28) return "sequences must be >= 0 and below 2^28";
    if (b->states < 1 || b->heads < 1 || b->heads > 4096 || b->heads % b->states != 0) return "heads must be in 1..4096, and states divide them";
    if (b->key_width < 1 || b->key_width > BAGEL_ATTENTION_MAX_WIDTH || b->value_width < 1 || b->value_width > BAGEL_ATTENTION_MAX_WIDTH)
        return "key_width and value_width must be in 1..128";
    if ((b->rows + b->sequences) * b->states >= 1ll << 31) return "rows and sequences together, times states, must be below 2^31";
    return nullptr;
}

// Whether heads can be addressed; those of a result may not overlap.
const char *check_heads(const bagel_heads &h, int64_t rows, int heads, int width, int dtype, bool written)
{
    if (!h.data) return nullptr;
    if ((uintptr_t)h.data & (bagel_type_bytes(dtype) - 1)) return "heads do not start at a multiple of their type";
    if (h.stride < 0 || h.head < 0 || h.stride >= 1ll << 40 || h.head >= 1ll << 40) return "a stride of heads or rows must be >= 0 and below 2^40";
    if (rows > 1 && h.stride > (1ll << 60) / rows) return "rows reach past 2^60 entries";
    if (!written) return nullptr;
    const bool side_by_side = (heads <= 1 || h.head >= width) && (rows <= 1 || h.stride >= (heads - 1) * h.head + width);
    const bool one_after_the_other = (rows <= 1 || h.stride >= width) && (heads <= 1 || h.head >= (rows - 1) * h.stride + width);
    return side_by_side || one_after_the_other ? nullptr : "rows or heads of a result overlap: a stride is too small";
}

bool memories_overlap(const bagel_attention *b, const float *read, const float *written)
{
    const uintptr_t x = (uintptr_t)read, y = (uintptr_t)written, bytes = (uintptr_t)b->sequences * b->states * b->key_width * b->value_width * sizeof(float);
    return read && written && (x < y ? y - x : x - y) < bytes;
}

const char *check_inputs(const bagel_attention *b)
{
    if (!bagel_type_ok(b->dtype)) return "unknown dtype";
    if (!isfinite(b->scale)) return "scale must be finite";
    if (!b->log_decay) return "log_decay is needed";
    if (b->rows > 0 && (!b->query.data || !b->key.data || !b->value.data)) return "query, key and value are needed";
    if (const char *msg = check_heads(b->query, b->rows, b->heads, b->key_width, b->dtype, false)) return msg;
    if (const char *msg = check_heads(b->key, b->rows, b->states, b->key_width, b->dtype, false)) return msg;
    return check_heads(b->value, b->rows, b->states, b->value_width, b->dtype, false);
}

const char *check_attention(const bagel_attention *b, bool grad)
{
    if (const char *msg = check_sizes(b)) return msg;
    if (const char *msg = check_inputs(b)) return msg;
    if (b->rows > 0) {
        if (b->sequences < 1) return "rows without a sequence";
        if (!b->offsets && b->rows % b->sequences != 0) return "without offsets, sequences must divide rows";
        if (!grad && !b->out.data) return "out is needed";
        if (grad && !b->d_out.data) return "d_out is needed";
    }
    if (!grad) {
        if (const char *msg = check_heads(b->out, b->rows, b->heads, b->value_width, b->dtype, true)) return msg;
        if (memories_overlap(b, b->initial, b->final_state)) return "initial and final_state overlap";
    } else {
        if (const char *msg = check_heads(b->d_out, b->rows, b->heads, b->value_width, b->dtype, false)) return msg;
        if (const char *msg = check_heads(b->d_query, b->rows, b->heads, b->key_width, b->dtype, true)) return msg;
        if (const char *msg = check_heads(b->d_key, b->rows, b->states, b->key_width, b->dtype, true)) return msg;
        if (const char *msg = check_heads(b->d_value, b->rows, b->states, b->value_width, b->dtype, true)) return msg;
        if (memories_overlap(b, b->d_final, b->d_initial)) return "d_final and d_initial overlap";
    }
    const int64_t need = bagel_linear_attention_workspace(b, grad);
    if (need > 0 && !b->workspace) return "a workspace is needed";
    if (b->workspace_bytes < need) return "the workspace is too small";
    if ((uintptr_t)b->workspace & 15) return "the workspace must start at a multiple of 16 bytes";
    return nullptr;
}

}  // namespace

extern "C" int64_t bagel_linear_attention_workspace(const bagel_attention *b, int32_t grad)
{
    if (check_sizes(b)) return BAGEL_EINVAL;
    // with offsets or without, in 32 bits or 16: which it is may not be known yet
    int64_t most = 0;
    for (int32_t dtype : {BAGEL_FLOAT32, BAGEL_BFLOAT16})
        for (bool offsets : {false, true}) {
            bagel_attention a = *b;
            a.dtype = dtype;
            most = std::max(most, memories_floats(a, segments_of(a, offsets)));
        }
    return most * (grad ? 2 : 1) * (int64_t)sizeof(float);
}

extern "C" int bagel_linear_attention(const bagel_attention *b, void *hip_stream)
{
    if (const char *msg = check_attention(b, false)) return bagel_refuse(BAGEL_EINVAL, "bagel_linear_attention: %s", msg);
    const hipError_t e = bagel_by_type(b->dtype, [&](auto t) { return launch_attention<typename decltype(t)::type>(*b, (hipStream_t)hip_stream); });
    if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_linear_attention: %s", hipGetErrorString(e));
    return BAGEL_OK;
}

extern "C" int bagel_linear_attention_grad(const bagel_attention *b, void *hip_stream)
{
    if (const char *msg = check_attention(b, true)) return bagel_refuse(BAGEL_EINVAL, "bagel_linear_attention_grad: %s", msg);
    const hipError_t e = bagel_by_type(b->dtype, [&](auto t) { return launch_attention_grad<typename decltype(t)::type>(*b, (hipStream_t)hip_stream); });
    if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_linear_attention_grad: %s", hipGetErrorString(e));
    return BAGEL_OK;
}

extern "C" int bagel_linear_attention_step(const bagel_attention *b, void *hip_stream)
{
    const char *msg = check_sizes(b);
    if (!msg && b->sequences != b->rows) msg = "a step has as many rows as sequences";
    if (!msg) msg = check_inputs(b);
    if (!msg && b->rows > 0 && (!b->out.data || !b->state)) msg = "out and state are needed";
    if (!msg) msg = check_heads(b->out, b->rows, b->heads, b->value_width, b->dtype, true);
    if (msg) return bagel_refuse(BAGEL_EINVAL, "bagel_linear_attention_step: %s", msg);
    if (b->rows > 0) {
        const hipError_t e = bagel_by_type(b->dtype, [&](auto t) { return launch_step<typename decltype(t)::type>(*b, (hipStream_t)hip_stream); });
        if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_linear_attention_step: %s", hipGetErrorString(e));
    }
    return BAGEL_OK;
}
