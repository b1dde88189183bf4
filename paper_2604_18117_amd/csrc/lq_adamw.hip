// An AdamW step over many tensors in one launch for every 64 of them:
//     m = b1 m + (1 - b1) g ;  v = b2 v + (1 - b2) g^2 ;  p = p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// Bound by memory: 28 bytes a value with fp32 states, 16 with states in 8 bits.
// States in 8 bits: E4M3 elements with a power of two as scale for each 256 values, the smallest that brings the block's largest below 448; of v its root is held.
// Elements are rounded up or down with the probabilities that keep the mean (an average that moves by 0.1 % a step would never leave an element of 3 bits of
// mantissa), by bits that come from the seed, the step and the value's place; scales being powers of two, a value that does not change is held as it was.  A root that
// is not zero is not held as zero: m / sqrt(v) stays bounded.
#include "lq_internal.h"

namespace lq {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));

constexpr int TENSORS = 64;  // of a launch: as many as a wavefront looks through at once

struct AdamwArgs {
    void* p[TENSORS];
    float* master[TENSORS];
    const void* g[TENSORS];
    void *m[TENSORS], *v[TENSORS];
    float* scales[TENSORS];
    int64_t n[TENSORS];
    uint32_t end[TENSORS];  // blocks of 256 values up to and with this tensor's
    uint32_t base;          // blocks before the launch's
    int aligned;            // every tensor can be accessed 4 values at a time
    const float *lr_dev, *grad_scale;
    const int32_t* step_dev;
    double beta1, beta2;
    float b1, c1, b2, c2, eps, wd, lr, bias1, bias2;
    uint32_t seed, step;
};
static_assert(sizeof(AdamwArgs) <= 4096, "kernel arguments");

__device__ __forceinline__ double power(double b, uint32_t t)  // b^t by squaring
{
    double r = 1.0;
    for (; t; t >>= 1, b *= b)
        if (t & 1) r *= b;
    return r;
}

// Two 20-bit numbers for a value
__device__ __forceinline__ void random_bits(uint32_t key, uint32_t place, uint32_t& a, uint32_t& b)
{
    uint32_t h = (place ^ key) * 0x9E3779B1u;
    h = (h ^ h >> 16) * 0x6A09E667u;
    h = (h ^ h >> 15) * 0xBB67AE85u;
    h ^= h >> 16;
    a = h & 0xFFFFFu;
    b = h * 0x3C6EF373u >> 12;
}
// 0 <= x <= 448 to one of the E4M3 values next to it.  Below 2^-6 they are 2^-9 apart, as from 2^-6 to 2^-5.
__device__ __forceinline__ float round_e4m3(float x, uint32_t bits)
{
    const float small = x < 0.015625f ? 0.015625f : 0.0f;
    return __uint_as_float((__float_as_uint(x + small) + bits) & 0xFFF00000u) - small;
}
// The smallest power of two that brings amax to 448 or below; 1 for zero, not a number where amax is none or infinite
__device__ __forceinline__ float power_scale(float amax)
{
    const uint32_t bits = __float_as_uint(amax);
    if (bits >= 0x7F800000u) return __uint_as_float(0x7FC00000u);
    const int e = (int)(bits >> 23) - 8 + ((bits & 0x7FFFFFu) > 0x600000u);
    return amax > 0.0f ? __uint_as_float((uint32_t)max(e, 1) << 23) : 1.0f;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x)  // of the bits of numbers without a sign: not a number counts as the largest
{
#pragma unroll
    for (int k = 1; k < 64; k *= 2) x = max(x, (uint32_t)__shfl_xor((int)x, k));
    return x;
}

// Four values of a tensor at i, those from n on zero
template <typename T>
__device__ __forceinline__ void read4(const void* p, int64_t i, int64_t n, bool whole, float (&f)[4])
{
    const T* x = (const T*)p + i;
    if (whole) {
        typedef T V4 __attribute__((ext_vector_type(4)));
        const V4 t = *(const V4*)x;
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = (float)t[k];
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) f[k] = i + k < n ? (float)x[k] : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void write4(void* p, int64_t i, int64_t n, bool whole, const float (&f)[4])
{
    T* x = (T*)p + i;
    if (whole) {
        typedef T V4 __attribute__((ext_vector_type(4)));
        V4 t;
#pragma unroll
        for (int k = 0; k < 4; ++k) t[k] = (T)f[k];
        *(V4*)x = t;
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (i + k < n) x[k] = (T)f[k];
    }
}
__device__ __forceinline__ uint32_t codes4(const void* p, int64_t i, int64_t n, bool whole)
{
    const uint8_t* x = (const uint8_t*)p + i;
    if (whole) return *(const uint32_t*)x;
    uint32_t w = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < n) w |= (uint32_t)x[k] << (8 * k);
    return w;
}
__device__ __forceinline__ void put_codes4(void* p, int64_t i, int64_t n, bool whole, uint32_t w)
{
    uint8_t* x = (uint8_t*)p + i;
    if (whole) {
        *(uint32_t*)x = w;
        return;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < n) x[k] = (uint8_t)(w >> (8 * k));
}
__device__ __forceinline__ void e4m3_values(uint32_t w, float (&f)[4])
{
    f[0] = __builtin_amdgcn_cvt_f32_fp8((int)w, 0);
    f[1] = __builtin_amdgcn_cvt_f32_fp8((int)w, 1);
    f[2] = __builtin_amdgcn_cvt_f32_fp8((int)w, 2);
    f[3] = __builtin_amdgcn_cvt_f32_fp8((int)w, 3);
}
__device__ __forceinline__ uint32_t e4m3_codes(const float (&f)[4])  // of values that are E4M3's
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(f[0], f[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(f[2], f[3], w, true);
}

// A wavefront takes a block of 256 values, four to a lane.
template <typename TP, typename TG, bool EIGHT>
__global__ void __launch_bounds__(256) adamw_kernel(AdamwArgs a)
{
    const int lane = threadIdx.x & 63;
    const uint32_t block = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
    if (block >= a.end[TENSORS - 1]) return;
    const int t = __popcll(__ballot(a.end[lane] <= block));
    const int64_t n = a.n[t], i = (int64_t)(block - (t ? a.end[t - 1] : 0u)) * 256 + lane * 4, at = block - (t ? a.end[t - 1] : 0u);
    const bool whole = a.aligned && i + 4 <= n;
    float p[4], g[4], m[4], v[4];
    uint32_t wm = 0, wv = 0;
    float sm = 1.0f, sv = 1.0f;
    if (a.master[t]) read4<float>(a.master[t], i, n, whole, p);
    else read4<TP>(a.p[t], i, n, whole, p);
    read4<TG>(a.g[t], i, n, whole, g);
    if constexpr (EIGHT) {
        wm = codes4(a.m[t], i, n, whole);
        wv = codes4(a.v[t], i, n, whole);
        sm = a.scales[t][2 * at];
        sv = a.scales[t][2 * at + 1];
    } else {
        read4<float>(a.m[t], i, n, whole, m);
        read4<float>(a.v[t], i, n, whole, v);
    }
    uint32_t step = a.step;
    float bias1 = a.bias1, bias2 = a.bias2;
    if (a.step_dev) {
        step = (uint32_t)max(*a.step_dev, 1);
        bias1 = (float)(1.0 - power(a.beta1, step));
        bias2 = (float)(1.0 - power(a.beta2, step));
    }
    const float lr = a.lr_dev ? *a.lr_dev : a.lr, gs = a.grad_scale ? *a.grad_scale : 1.0f, keep = 1.0f - lr * a.wd;
    if constexpr (EIGHT) {
        e4m3_values(wm, m);
        e4m3_values(wv, v);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            m[k] *= sm;
            v[k] *= sv;
            v[k] *= v[k];
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if (a.grad_scale) g[k] *= gs;
        m[k] = m[k] * a.b1 + g[k] * a.c1;
        v[k] = v[k] * a.b2 + g[k] * a.c2 * g[k];
        p[k] = p[k] * keep - lr * (m[k] / bias1) / (sqrtf(v[k] / bias2) + a.eps);
    }
    if (a.master[t]) write4<float>(a.master[t], i, n, whole, p);
    write4<TP>(a.p[t], i, n, whole, p);
    if constexpr (EIGHT) {
        uint32_t big[2] = {0u, 0u};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v[k] = sqrtf(v[k]);
            big[0] = max(big[0], __float_as_uint(m[k]) & 0x7FFFFFFFu);
            big[1] = max(big[1], __float_as_uint(v[k]) & 0x7FFFFFFFu);
        }
        sm = power_scale(__uint_as_float(wave_max(big[0])));
        sv = power_scale(__uint_as_float(wave_max(big[1])));
        const float im = 1.0f / sm, iv = 1.0f / sv;
        const uint32_t key = a.seed * 0x9E3779B1u + step * 0x6A09E667u, place = (a.base + block) * 256u + lane * 4u;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t rm, rv;
            random_bits(key, place + k, rm, rv);
            m[k] = copysignf(round_e4m3(fabsf(m[k]) * im, rm), m[k]);
            const float r = round_e4m3(v[k] * iv, rv);
            v[k] = v[k] > 0.0f ? fmaxf(r, 0.001953125f) : r;
        }
        put_codes4(a.m[t], i, n, whole, e4m3_codes(m));
        put_codes4(a.v[t], i, n, whole, e4m3_codes(v));
        if (lane == 0) a.scales[t][2 * at] = sm, a.scales[t][2 * at + 1] = sv;
    } else {
        write4<float>(a.m[t], i, n, whole, m);
        write4<float>(a.v[t], i, n, whole, v);
    }
}

hipError_t launch_adamw(const lq_adamw_config* c, const lq_adamw_tensor* tensors, int count, const lq_adamw_args* x, hipStream_t s)
{
    AdamwArgs a{};
    a.lr_dev = x->lr_dev;
    a.grad_scale = x->grad_scale;
    a.step_dev = x->step_dev;
    a.beta1 = c->beta1;
    a.beta2 = c->beta2;
    a.b1 = (float)c->beta1;
    a.c1 = (float)(1.0 - c->beta1);
    a.b2 = (float)c->beta2;
    a.c2 = (float)(1.0 - c->beta2);
    a.eps = (float)c->eps;
    a.wd = (float)c->weight_decay;
    a.lr = (float)x->lr;
    a.step = (uint32_t)x->step;
    double p1 = 1.0, p2 = 1.0, q1 = c->beta1, q2 = c->beta2;
    for (uint32_t t = a.step; t; t >>= 1, q1 *= q1, q2 *= q2)
        if (t & 1) p1 *= q1, p2 *= q2;
    a.bias1 = (float)(1.0 - p1);
    a.bias2 = (float)(1.0 - p2);
    a.seed = c->seed;
    const int pe = c->p_dtype == LQ_F32 ? 4 : 2, ge = c->g_dtype == LQ_F32 ? 4 : 2, se = c->state_bits == 32 ? 4 : 1;
    for (int i = 0; i < count;) {
        int k = 0;
        uint32_t blocks = 0;
        a.aligned = 1;
        for (; i < count && k < TENSORS; ++i) {
            const lq_adamw_tensor& t = tensors[i];
            const uint32_t more = (uint32_t)((t.n + 255) / 256);
            if (more == 0) continue;
            if (blocks + more > (1u << 25)) break;  // (a launch stays below 2^32 threads)
            a.p[k] = t.p;
            a.master[k] = t.master;
            a.g[k] = t.grad;
            a.m[k] = t.m;
            a.v[k] = t.v;
            a.scales[k] = t.scales;
            a.n[k] = t.n;
            a.end[k] = blocks += more;
            a.aligned = a.aligned && (uintptr_t)t.p % (4 * pe) == 0 && (uintptr_t)t.master % 16 == 0 && (uintptr_t)t.grad % (4 * ge) == 0 &&
                        (uintptr_t)t.m % (4 * se) == 0 && (uintptr_t)t.v % (4 * se) == 0;
            ++k;
        }
        if (k == 0) break;
        for (; k < TENSORS; ++k) a.end[k] = blocks;
        const dim3 grid((blocks + 3) / 4), block(256);
        const bool eight = c->state_bits == 8, pf = c->p_dtype == LQ_F32, gf = c->g_dtype == LQ_F32;
#define RUN(TP, TG) \
    if (eight) hipLaunchKernelGGL((adamw_kernel<TP, TG, true>), grid, block, 0, s, a); \
    else hipLaunchKernelGGL((adamw_kernel<TP, TG, false>), grid, block, 0, s, a)
        if (pf && gf) { RUN(float, float); }
        else if (pf) { RUN(float, __bf16); }
        else if (gf) { RUN(__bf16, float); }
        else { RUN(__bf16, __bf16); }
#undef RUN
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.base += blocks;
    }
    return hipSuccess;
}

}  // namespace lq
