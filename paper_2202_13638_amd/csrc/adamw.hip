// Adam with decoupled weight decay over many tensors at once (include/bagel.h), the moments in 32 bits or in 8 with a scale for
// every 256 values.
//
// A launch takes up to TENSORS tensors by value, with the number of the first piece of each: the table of a thousand tensors needs no
// memory on the device that would have to be filled, kept and waited for.
#include <type_traits>

#include "activations.h"

namespace {

constexpr int TENSORS = 48;                  // 76 bytes each, within the 4 KB of a kernel's arguments
constexpr int BLOCK = BAGEL_ADAMW_BLOCK;
constexpr float LARGEST = 448.0f;            // of float8 e4m3

struct adamw_tensor {
    float *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale;
    void *copy;
    int64_t count;
    float keep;                  // 1 - lr weight_decay
    uint32_t key;                // of its draws
};

struct adamw_args {
    adamw_tensor tensor[TENSORS];
    uint32_t first[TENSORS];     // the first piece of each
    const float *grad_scale;
    int n, grad_dtype, copy_dtype;
    uint32_t pieces;             // of all tensors
    int each;                    // blocks of 256 that a wave takes of a piece: a piece is 4 each
    float beta1, rest1, beta2, rest2, rate, root, eps;       // rate = lr / (1 - beta1^step), root = 1 / sqrt(1 - beta2^step)
};
static_assert(sizeof(adamw_args) <= 4096, "kernel arguments");

// Four entries of a block, in a row (WHOLE: a block of 256, at any alignment) or 64 apart, where those from `rest` on are not there.
template <bool WHOLE> __device__ __forceinline__ int place(int i) { return WHOLE ? 4 * (threadIdx.x & 63) + i : 64 * i + (threadIdx.x & 63); }

template <bool WHOLE, typename T> __device__ __forceinline__ void load_four(const void *p, int64_t from, int64_t rest, float (&v)[4])
{
    const T *q = (const T *)p + from;
    if constexpr (WHOLE) bagel_load<T, 4>(q + place<true>(0), v);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = place<false>(i) < rest ? (float)q[place<false>(i)] : 0.0f;
}

template <bool WHOLE, typename T> __device__ __forceinline__ void store_four(void *p, int64_t from, int64_t rest, const float (&v)[4])
{
    T *q = (T *)p + from;
    if constexpr (WHOLE) bagel_store<T, 4>(q + place<true>(0), v);
    else
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (place<false>(i) < rest) q[place<false>(i)] = (T)v[i];
}

template <bool WHOLE> __device__ __forceinline__ void load_as(const void *p, int64_t from, int64_t rest, int dtype, float (&v)[4])
{
    if (dtype == BAGEL_FLOAT32) load_four<WHOLE, float>(p, from, rest, v);
    else if (dtype == BAGEL_BFLOAT16) load_four<WHOLE, __bf16>(p, from, rest, v);
    else load_four<WHOLE, _Float16>(p, from, rest, v);
}

template <bool WHOLE> __device__ __forceinline__ void store_as(void *p, int64_t from, int64_t rest, int dtype, const float (&v)[4])
{
    if (dtype == BAGEL_FLOAT32) store_four<WHOLE, float>(p, from, rest, v);
    else if (dtype == BAGEL_BFLOAT16) store_four<WHOLE, __bf16>(p, from, rest, v);
    else store_four<WHOLE, _Float16>(p, from, rest, v);
}

struct __attribute__((packed, aligned(1))) loose_int {
    int x;
};

template <bool WHOLE> __device__ __forceinline__ void load_codes(const void *p, int64_t from, int64_t rest, float (&v)[4])
{
    const uint8_t *q = (const uint8_t *)p + from;
    int bytes = 0;
    if constexpr (WHOLE) bytes = reinterpret_cast<const loose_int *>(q + place<true>(0))->x;
    else
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (place<false>(i) < rest) bytes |= (int)q[place<false>(i)] << 8 * i;
    v[0] = __builtin_amdgcn_cvt_f32_fp8(bytes, 0);
    v[1] = __builtin_amdgcn_cvt_f32_fp8(bytes, 1);
    v[2] = __builtin_amdgcn_cvt_f32_fp8(bytes, 2);
    v[3] = __builtin_amdgcn_cvt_f32_fp8(bytes, 3);
}

template <bool WHOLE> __device__ __forceinline__ void store_codes(void *p, int64_t from, int64_t rest, const float (&v)[4])
{
    uint8_t *q = (uint8_t *)p + from;
    int bytes = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    bytes = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], bytes, true);
    if constexpr (WHOLE) reinterpret_cast<loose_int *>(q + place<true>(0))->x = bytes;
    else
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (place<false>(i) < rest) q[place<false>(i)] = (uint8_t)(bytes >> 8 * i);
}

// Two rounds of shift and multiply mix high bits into low ones and back.
__host__ __device__ __forceinline__ uint32_t mixed(uint32_t x)
{
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0x3C6EF373u;
    return x ^ (x >> 16);
}

// 32 random bits for every place of a tensor, which a product with an odd number near 2^32 / golden ratio spreads.  Two keys give the same bits, moved on by
// their difference over that number, so keys have to be far from each other by themselves.
__device__ __forceinline__ uint32_t chance(uint32_t place, uint32_t key) { return mixed(place * 0x9E3779B9u + key); }

// The key of a tensor's draws in one update.  Mixed in one after the other, seed, update and the tensor's number leave no two keys that are near
// each other for a reason.  (A sum of multiples, which a caller that knows its draws gets, makes an update's draws those of the one before, one place on.)
uint32_t key_of(const bagel_adamw &o, int tensor)
{
    if (o.draws == BAGEL_DRAWS_GIVEN) return o.seed * 0xBB67AE85u + (uint32_t)o.step * 0x9E3779B9u;
    return mixed(mixed(mixed(mixed(o.seed + 0x3C6EF372u) ^ (uint32_t)o.step) + (uint32_t)(o.step >> 32)) ^ (uint32_t)tensor);
}

// The magnitude of a code (float8 e4m3) for y in [0, 448], up or down by a chance of 16 bits.  From 2^-6 on a code has 3 bits behind the
// leading one: the chance is added to the 20 bits that go, which carries with the right probability.  Below, codes are the
// multiples of 2^-9.
__device__ __forceinline__ float code_of(float y, uint32_t r)
{
    const float normal = __uint_as_float((__float_as_uint(y) + (r << 4)) & 0xFFF00000u);
    const float small = floorf(y * 512.0f + (float)r * (1.0f / 65536.0f)) * (1.0f / 512.0f);
    return fminf(y >= 1.0f / 64.0f ? normal : small, LARGEST);
}

// The largest magnitude in a wave.  As whole numbers the bits of magnitudes have the same order, and NaN is the largest of all: it is kept.
__device__ __forceinline__ float largest(const float (&v)[4])
{
    const auto bits = [](float x) { return __float_as_uint(x) & 0x7FFFFFFFu; };
    const auto moved = [](uint32_t x, auto move) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(move)::value, 0xF, 0xF, false); };
    uint32_t x = max(max(bits(v[0]), bits(v[1])), max(bits(v[2]), bits(v[3])));
    x = max(x, moved(x, std::integral_constant<int, 0xB1>()));
    x = max(x, moved(x, std::integral_constant<int, 0x4E>()));
    x = max(x, moved(x, std::integral_constant<int, 0x141>()));
    x = max(x, moved(x, std::integral_constant<int, 0x140>()));
    const int i = (int)x;
    return __uint_as_float(max(max((uint32_t)__builtin_amdgcn_readlane(i, 0), (uint32_t)__builtin_amdgcn_readlane(i, 16)),
                               max((uint32_t)__builtin_amdgcn_readlane(i, 32), (uint32_t)__builtin_amdgcn_readlane(i, 48))));
}

// Codes of a block, and its scale in every lane.  ROOT: of roots, of which none above zero becomes zero.
template <bool ROOT> __device__ __forceinline__ float encode_finite(float (&v)[4], const uint32_t (&bits)[4], float top)
{
    if (top < 1e-30f) top = 0.0f;
    const float scale = top > 0.0f ? 1.0f / top * LARGEST : 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float code = code_of(fminf(fabsf(v[i]) * scale, LARGEST), ROOT ? bits[i] >> 16 : bits[i] & 0xFFFFu);
        v[i] = !ROOT ? copysignf(code, v[i]) : v[i] > 0.0f && top > 0.0f ? fmaxf(code, 1.0f / 512.0f) : code;
    }
    return top * (1.0f / LARGEST);
}

// The same where some are not finite: they are kept as NaN in their places.  A scale made of them would take the other 255 along.
template <bool ROOT> __device__ __forceinline__ float encode(float (&v)[4], const uint32_t (&bits)[4])
{
    const float top = largest(v);
    if (isfinite(top)) return encode_finite<ROOT>(v, bits, top);
    float w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = isfinite(v[i]) ? v[i] : 0.0f;
    const float scale = encode_finite<ROOT>(w, bits, largest(w));
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = isfinite(v[i]) ? w[i] : __builtin_nanf("");
    return scale;
}

template <int BITS, bool WHOLE> __device__ __forceinline__ void update_block(const adamw_args &a, const adamw_tensor &w, int64_t block, float gs)
{
    const int64_t from = block * BLOCK, rest = w.count - from;
    float g[4], p[4], m[4], v[4], r[4];
    load_as<WHOLE>(w.grad, from, rest, a.grad_dtype, g);
    load_four<WHOLE, float>(w.param, from, rest, p);
    if (BITS == 32) {
        load_four<WHOLE, float>(w.m, from, rest, m);
        load_four<WHOLE, float>(w.v, from, rest, v);
    } else {
        const float sm = w.m_scale[block], sv = w.v_scale[block];
        load_codes<WHOLE>(w.m, from, rest, m);
        load_codes<WHOLE>(w.v, from, rest, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] *= sm;
            v[i] *= sv;
            v[i] *= v[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        g[i] *= gs;
        m[i] = m[i] * a.beta1 + g[i] * a.rest1;
        v[i] = v[i] * a.beta2 + g[i] * a.rest2 * g[i];
        r[i] = sqrtf(v[i]);
        p[i] = p[i] * w.keep - m[i] * a.rate / (r[i] * a.root + a.eps);
    }
    store_four<WHOLE, float>(w.param, from, rest, p);
    if (w.copy) store_as<WHOLE>(w.copy, from, rest, a.copy_dtype, p);
    if (BITS == 32) {
        store_four<WHOLE, float>(w.m, from, rest, m);
        store_four<WHOLE, float>(w.v, from, rest, v);
    } else {
        uint32_t bits[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) bits[i] = chance((uint32_t)from + place<WHOLE>(i), w.key);
        const float sm = encode<false>(m, bits), sv = encode<true>(r, bits);
        store_codes<WHOLE>(w.m, from, rest, m);
        store_codes<WHOLE>(w.v, from, rest, r);
        if ((threadIdx.x & 63) == 0) {
            w.m_scale[block] = sm;
            w.v_scale[block] = sv;
        }
    }
}

// A wave takes a block of 256 at a time, four entries a lane: the block's largest magnitude is a matter of one wave.  Every byte is read and written once, and
// memory bounds it: 64 tensors, 33.6 million values, 32 bits, gradients and copy in bf16: 179 us, 5.3 TB/s; 404 million values in 8 bits: 1280 us, 5.1
// TB/s.  Six small tensors take 3.9 us, latency.
template <int BITS> __global__ __launch_bounds__(256) void adamw_kernel(adamw_args a)
{
    const float gs = a.grad_scale ? a.grad_scale[0] : 1.0f;
    if (!isfinite(gs)) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t mine = lane < a.n ? a.first[lane] : 0xFFFFFFFFu;
    for (uint32_t piece = blockIdx.x; piece < a.pieces; piece += gridDim.x) {
        const int k = __popcll(__ballot(mine <= piece)) - 1;     // the last tensor that does not begin behind it
        const adamw_tensor &w = a.tensor[k];
        const int64_t blocks = (w.count + BLOCK - 1) / BLOCK;
        int64_t block = (int64_t)(piece - a.first[k]) * 4 * a.each + wave;
        for (int i = 0; i < a.each && block < blocks; ++i, block += 4) {
            if ((block + 1) * BLOCK <= w.count) update_block<BITS, true>(a, w, block, gs);
            else update_block<BITS, false>(a, w, block, gs);
        }
    }
}

const char *check_adamw(const bagel_adamw_tensor *tensors, int32_t n, const bagel_adamw *o)
{
    if (n < 0) return "n_tensors must be >= 0";
    if (!o || (n > 0 && !tensors)) return "null argument";
    if (o->step < 1) return "step must be >= 1";
    if (!(o->lr >= 0.0) || !isfinite(o->lr)) return "lr must be >= 0";
    if (!(o->beta1 >= 0.0 && o->beta1 < 1.0 && o->beta2 >= 0.0 && o->beta2 < 1.0)) return "betas must be in [0, 1)";
    if (!((float)o->eps > 0.0f) || !isfinite((float)o->eps)) return "eps must be positive";
    if (!bagel_type_ok(o->grad_dtype) || !bagel_type_ok(o->copy_dtype)) return "unknown dtype";
    if (o->state_bits != 32 && o->state_bits != 8) return "state_bits must be 32 or 8";
    if (o->draws != BAGEL_DRAWS_MIXED && o->draws != BAGEL_DRAWS_GIVEN) return "unknown draws";
    for (int i = 0; i < n; ++i) {
        const bagel_adamw_tensor &t = tensors[i];
        if (t.count < 0 || t.count >= 1ll << 38) return "count must be >= 0 and below 2^38";
        if (!(t.weight_decay >= 0.0) || !(o->lr * t.weight_decay < 1.0)) return "weight_decay must be >= 0 and lr weight_decay below 1";
        if (t.count == 0) continue;
        if (!t.param || !t.grad || !t.m || !t.v) return "a tensor has a null argument";
        if (o->state_bits == 8 && (!t.m_scale || !t.v_scale)) return "states in 8 bits need m_scale and v_scale";
        const uintptr_t floats = (uintptr_t)t.param | (o->state_bits == 32 ? (uintptr_t)t.m | (uintptr_t)t.v : (uintptr_t)t.m_scale | (uintptr_t)t.v_scale);
        if (floats & 3 || (uintptr_t)t.grad & (bagel_type_bytes(o->grad_dtype) - 1) || (uintptr_t)t.copy & (bagel_type_bytes(o->copy_dtype) - 1))
            return "a tensor does not start at a multiple of its type";
    }
    return nullptr;
}

}  // namespace

extern "C" int bagel_adamw_step(const bagel_adamw_tensor *tensors, int32_t n_tensors, const bagel_adamw *o, void *hip_stream)
{
    if (const char *msg = check_adamw(tensors, n_tensors, o)) return bagel_refuse(BAGEL_EINVAL, "bagel_adamw_step: %s", msg);
    adamw_args a;
    a.grad_scale = o->grad_scale;
    a.grad_dtype = o->grad_dtype;
    a.copy_dtype = o->copy_dtype;
    a.beta1 = (float)o->beta1;
    a.rest1 = (float)(1.0 - o->beta1);
    a.beta2 = (float)o->beta2;
    a.rest2 = (float)(1.0 - o->beta2);
    a.rate = (float)(o->lr / (1.0 - pow(o->beta1, (double)o->step)));
    a.root = (float)(1.0 / sqrt(1.0 - pow(o->beta2, (double)o->step)));
    a.eps = (float)o->eps;
    // A block to a wave, and in 8 bits four one after the other where there are many, whose scales then come together (one tensor, us with one and with four: in
    // 8 bits 4096 blocks 7.6 and 8.9, 65536 58 and 51, 1048576 882 and 836; in 32 bits 65536 67.6 and 70.3, 1048576 1334 and 1411).
    int64_t all = 0;
    for (int i = 0; i < n_tensors; ++i) all += (tensors[i].count + BLOCK - 1) / BLOCK;
    a.each = o->state_bits == 32 || all < 16384 ? 1 : 4;
    a.n = 0;
    a.pieces = 0;
    const auto launch = [&]() {
        const unsigned groups = a.pieces < 1u << 20 ? a.pieces : 1u << 20;
        if (o->state_bits == 8) adamw_kernel<8><<<groups, 256, 0, (hipStream_t)hip_stream>>>(a);
        else adamw_kernel<32><<<groups, 256, 0, (hipStream_t)hip_stream>>>(a);
        a.n = 0;
        a.pieces = 0;
        return hipGetLastError();
    };
    hipError_t e = hipSuccess;
    for (int i = 0; i < n_tensors && e == hipSuccess; ++i) {
        const bagel_adamw_tensor &t = tensors[i];
        if (t.count == 0) continue;
        const uint32_t pieces = (uint32_t)((t.count + 4 * a.each * BLOCK - 1) / (4 * a.each * BLOCK));
        if (a.n == TENSORS || (a.n > 0 && a.pieces + pieces > 1u << 30)) {
            if ((e = launch()) != hipSuccess) break;
        }
        a.tensor[a.n] = {t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.copy, t.count, (float)(1.0 - o->lr * t.weight_decay), key_of(*o, i)};
        a.first[a.n++] = a.pieces;
        a.pieces += pieces;
    }
    if (e == hipSuccess && a.n > 0) e = launch();
    if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_adamw_step: %s", hipGetErrorString(e));
    return BAGEL_OK;
}
