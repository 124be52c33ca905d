// Adam with decoupled weight decay over many tensors at once (include/bagel.h), the moments in 32 bits or in 8 with a scale for
// every 256 values.
//
// A launch takes up to TENSORS tensors by value, with the number of the first block of each: the table of a thousand tensors needs no
// memory on the device that would have to be filled, kept and waited for.
#include "activations.h"

namespace {

constexpr int TENSORS = 48;                  // 72 bytes each, within the 4 KB of a kernel's arguments
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
    uint32_t first;              // its first block of 256
};

struct adamw_args {
    adamw_tensor tensor[TENSORS];
    const float *grad_scale;
    int n, grad_dtype, copy_dtype;
    uint32_t blocks, key;        // of all tensors
    float beta1, rest1, beta2, rest2, rate, root, eps;       // rate = lr / (1 - beta1^step), root = 1 / sqrt(1 - beta2^step)
};
static_assert(sizeof(adamw_args) <= 4096, "kernel arguments");

__device__ __forceinline__ float load_as(const void *p, int64_t i, int dtype)
{
    if (dtype == BAGEL_FLOAT32) return ((const float *)p)[i];
    if (dtype == BAGEL_BFLOAT16) return (float)((const __bf16 *)p)[i];
    return (float)((const _Float16 *)p)[i];
}

__device__ __forceinline__ void store_as(void *p, int64_t i, float v, int dtype)
{
    if (dtype == BAGEL_FLOAT32) ((float *)p)[i] = v;
    else if (dtype == BAGEL_BFLOAT16) ((__bf16 *)p)[i] = (__bf16)v;
    else ((_Float16 *)p)[i] = (_Float16)v;
}

// 32 random bits for every place of a tensor: a product with an odd number near 2^32 / golden ratio spreads the places, two rounds of shift
// and multiply mix high bits into low ones and back.
__device__ __forceinline__ uint32_t chance(uint32_t place, uint32_t key)
{
    uint32_t x = place * 0x9E3779B9u + key;
    x = (x ^ (x >> 16)) * 0x6A09E667u;
    x = (x ^ (x >> 15)) * 0x3C6EF373u;
    return x ^ (x >> 16);
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

__device__ __forceinline__ uint8_t byte_of(float code) { return (uint8_t)__builtin_amdgcn_cvt_pk_fp8_f32(code, code, 0, false); }
__device__ __forceinline__ float value_of(uint8_t byte) { return __builtin_amdgcn_cvt_f32_fp8((int)byte, 0); }

// fmaxf that keeps a NaN
__device__ __forceinline__ float larger(float a, float b) { return a != a || a > b ? a : b; }

__device__ __forceinline__ float group_max(float v, float *shared)
{
#pragma unroll
    for (int i = 32; i > 0; i >>= 1) v = larger(__shfl_xor(v, i), v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    return larger(larger(shared[0], shared[1]), larger(shared[2], shared[3]));
}

template <int BITS> __global__ __launch_bounds__(BLOCK) void adamw_kernel(adamw_args a)
{
    __shared__ float shared[4];
    const float gs = a.grad_scale ? a.grad_scale[0] : 1.0f;
    if (!isfinite(gs)) return;
    for (uint32_t at = blockIdx.x; at < a.blocks; at += gridDim.x) {
        int k = 0;
        for (int i = 1; i < a.n; ++i)
            if (a.tensor[i].first <= at) k = i;
        const adamw_tensor &w = a.tensor[k];
        const int64_t block = at - w.first, i = block * BLOCK + threadIdx.x;
        const bool here = i < w.count;
        float m = 0.0f, v = 0.0f, g = 0.0f, p = 0.0f;
        if (here) {
            g = load_as(w.grad, i, a.grad_dtype) * gs;
            p = w.param[i];
            if (BITS == 32) {
                m = ((const float *)w.m)[i];
                v = ((const float *)w.v)[i];
            } else {
                m = value_of(((const uint8_t *)w.m)[i]) * w.m_scale[block];
                v = value_of(((const uint8_t *)w.v)[i]) * w.v_scale[block];
                v *= v;
            }
        }
        m = m * a.beta1 + g * a.rest1;
        v = v * a.beta2 + g * a.rest2 * g;
        const float r = sqrtf(v);
        p = p * w.keep - m * a.rate / (r * a.root + a.eps);
        if (here) {
            w.param[i] = p;
            if (w.copy) store_as(w.copy, i, p, a.copy_dtype);
        }
        if (BITS == 32) {
            if (here) {
                ((float *)w.m)[i] = m;
                ((float *)w.v)[i] = v;
            }
            continue;
        }
        const uint32_t c = chance((uint32_t)i, a.key);
        float top = group_max(fabsf(m), shared);
        if (top < 1e-30f) top = 0.0f;
        float scale = top > 0.0f ? 1.0f / top * LARGEST : 0.0f;
        float code = code_of(fminf(fabsf(m) * scale, LARGEST), c & 0xFFFFu);
        if (here) ((uint8_t *)w.m)[i] = byte_of(copysignf(code, m));
        if (threadIdx.x == 0) w.m_scale[block] = top * (1.0f / LARGEST);
        top = group_max(r, shared);
        if (top < 1e-30f) top = 0.0f;
        scale = top > 0.0f ? 1.0f / top * LARGEST : 0.0f;
        code = code_of(fminf(r * scale, LARGEST), c >> 16);
        if (r > 0.0f && top > 0.0f) code = fmaxf(code, 1.0f / 512.0f);
        if (here) ((uint8_t *)w.v)[i] = byte_of(code);
        if (threadIdx.x == 0) w.v_scale[block] = top * (1.0f / LARGEST);
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
    a.key = o->seed * 0xBB67AE85u + (uint32_t)o->step * 0x9E3779B9u;
    a.beta1 = (float)o->beta1;
    a.rest1 = (float)(1.0 - o->beta1);
    a.beta2 = (float)o->beta2;
    a.rest2 = (float)(1.0 - o->beta2);
    a.rate = (float)(o->lr / (1.0 - pow(o->beta1, (double)o->step)));
    a.root = (float)(1.0 / sqrt(1.0 - pow(o->beta2, (double)o->step)));
    a.eps = (float)o->eps;
    uint32_t blocks = 0;
    a.n = 0;
    auto launch = [&]() {
        a.blocks = blocks;
        const unsigned groups = blocks < 1u << 20 ? blocks : 1u << 20;
        if (o->state_bits == 8) adamw_kernel<8><<<groups, BLOCK, 0, (hipStream_t)hip_stream>>>(a);
        else adamw_kernel<32><<<groups, BLOCK, 0, (hipStream_t)hip_stream>>>(a);
        a.n = 0;
        blocks = 0;
        return hipGetLastError();
    };
    hipError_t e = hipSuccess;
    for (int i = 0; i < n_tensors && e == hipSuccess; ++i) {
        const bagel_adamw_tensor &t = tensors[i];
        if (t.count == 0) continue;
        const uint32_t more = (uint32_t)((t.count + BLOCK - 1) / BLOCK);
        if (a.n == TENSORS || (a.n > 0 && blocks + more > 1u << 30)) e = launch();
        a.tensor[a.n++] = {t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, t.copy, t.count, (float)(1.0 - o->lr * t.weight_decay), blocks};
        blocks += more;
    }
    if (e == hipSuccess && a.n > 0) e = launch();
    if (e != hipSuccess) return bagel_refuse(BAGEL_EHIP, "bagel_adamw_step: %s", hipGetErrorString(e));
    bagel_no_error();
    return BAGEL_OK;
}
