// An AdamW step over many tensors in one launch for every 120 of them:
//     m = b1 m + (1 - b1) g ;  v = b2 v + (1 - b2) g^2 ;  p = p (1 - lr wd) - lr (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + eps)
// Bound by memory: 28 bytes a value with fp32 states, 16 with states in 8 bits.
// States in 8 bits: E4M3 elements with a power of two as scale for each 256 values, the smallest that brings the block's largest below 448; of v its root is held.
// Elements are rounded up or down with the probabilities that keep the mean (an average that moves by 0.1 % a step would never leave an element of 3 bits of
// mantissa), by bits that come from the seed, the step and the value's place; scales being powers of two, a value that does not change is held as it was.  A root that
// is not zero is not held as zero: m / sqrt(v) stays bounded.
#include <math.h>

#include "lq_internal.h"

namespace lq {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v4bf __attribute__((ext_vector_type(4)));

// The tensors of a launch: as many as 4 KB of kernel arguments hold.  (With 64 of them, in whole addresses, 229 tensors of 11 M values in 8 bits took four launches and 66 us, of which a
// launch's beginning and end are some 8; with 120 two and 51.)  Addresses are steps of an element from the lowest of their kind.
constexpr int TENSORS = 120, FEW = 8;
struct Entry {
    uint32_t p, master, g, m, v, scales;  // master: NONE without
    uint32_t n;
};
constexpr uint32_t NONE = 0xFFFFFFFFu;
// 1 - lr wd as keep - rest: in fp32 by itself it has none of a decay below 2^-25, and 1e-6 as 1.013e-6, so that what keep lacks is taken off p with the step.  (keep is below the true factor and rest
// below zero: of an infinite parameter both are infinities of one sign, and it stays.  rest is zero where nothing decays.)
struct Decay {
    float keep, rest;
};
__host__ __device__ static inline Decay decay_of(float decay)
{
    Decay d = {1.0f - decay, 0.0f};
    if (decay == 0.0f) return d;
    d.rest = decay - (1.0f - d.keep);
    if (d.rest >= 0.0f && d.keep > 0.0f) {
        d.keep = __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, d.keep) - 1u);  // (the number below)
        d.rest = decay - (1.0f - d.keep);
    }
    return d;
}
template <int CAP>
struct AdamwArgs {
    Entry tensors[CAP];
    uint32_t first[CAP];    // block of 256 values of each in the launch; NONE behind the last
    char *p, *m, *v;
    const char* g;
    float *master, *scales;
    uint32_t blocks;        // of the launch
    uint32_t base;          // before it
    int aligned;            // every tensor can be accessed 4 values at a time
    const float *lr_dev, *grad_scale;
    const int32_t* step_dev;
    double beta1, beta2;
    float b1, c1, b2, c2, eps, wd, lr, correct1, correct2;  // 1 / (1 - beta1^t), 1 / sqrt(1 - beta2^t)
    Decay decay;            // of lr
    uint32_t seed, step;
};
static_assert(sizeof(AdamwArgs<TENSORS>) <= 4096, "kernel arguments");

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
// 0 <= x <= 448 to the code of one of the E4M3 values next to it.  Times 2^-120 the number's fields are E4M3's followed by 20 bits that are cut off: 2^-6, E4M3's smallest normal number, becomes
// fp32's, and what is below stays evenly spaced.  (An answer above 255 stands for not a number.)
__device__ __forceinline__ uint32_t e4m3_code(float x, uint32_t bits) { return (__float_as_uint(x * 0x1p-120f) + bits) >> 20; }
// The smallest power of two that brings amax (its bits) to 448 or below, and its reciprocal; 1 for zero, not a number where amax is none or infinite
__device__ __forceinline__ void power_scale(uint32_t amax, float& scale, float& inverse)
{
    const int e = max((int)((amax + 0x1FFFFFu) >> 23) - 8, 1);  // (448 is 1.75 times a power of two)
    const bool number = amax < 0x7F800000u;
    scale = __uint_as_float(!number ? 0x7FC00000u : amax ? (uint32_t)e << 23 : 0x3F800000u);
    inverse = __uint_as_float(!number ? 0x7FC00000u : amax ? (uint32_t)(254 - e) << 23 : 0x3F800000u);
}
template <int CTRL>
__device__ __forceinline__ uint32_t max_dpp(uint32_t v)
{
    return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v)  // of the bits of numbers without a sign: not a number counts as the largest
{
    v = max_dpp<0xB1>(v);   // quad_perm [1,0,3,2]
    v = max_dpp<0x4E>(v);   // quad_perm [2,3,0,1]
    v = max_dpp<0x141>(v);  // row_half_mirror
    v = max_dpp<0x140>(v);  // row_mirror
    const auto s = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = max(s[0], s[1]);
    const auto t = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (uint32_t)__builtin_amdgcn_readfirstlane((int)max(t[0], t[1]));
}

// The nearest number to the root of x >= 0 by Goldschmidt's iteration with a last step by the residual: from an estimate y of 1 / sqrt(x), s = x y and h = y / 2 go to the root and to half of its reciprocal
// together (e = 1/2 - h s; s += s e; h += h e), then s += (x - s^2) h, each step by fused operations (9 instructions, the library's 15).  Outside the estimate's range the
// library's.
__device__ __forceinline__ float nearest_root(float x)
{
    const float y = __builtin_amdgcn_rsqf(x);
    float s = x * y, h = 0.5f * y;
    const float e = fmaf(-h, s, 0.5f);
    s = fmaf(s, e, s);
    h = fmaf(h, e, h);
    s = fmaf(fmaf(-s, s, x), h, s);
    if (!(x >= 1e-30f && x <= 1e30f)) s = sqrtf(x);
    return s;
}
// Four values of a tensor at i, those from n on zero
template <typename T>
__device__ __forceinline__ void read4(const void* p, int i, int n, bool whole, float (&f)[4])
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
__device__ __forceinline__ void write4(void* p, int i, int n, bool whole, const float (&f)[4])
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
__device__ __forceinline__ uint32_t codes4(const void* p, int i, int n, bool whole)
{
    const uint8_t* x = (const uint8_t*)p + i;
    if (whole) return *(const uint32_t*)x;
    uint32_t w = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (i + k < n) w |= (uint32_t)x[k] << (8 * k);
    return w;
}
__device__ __forceinline__ void put_codes4(void* p, int i, int n, bool whole, uint32_t w)
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
__device__ __forceinline__ uint32_t bytes4(const uint32_t (&c)[4])  // the lowest byte of each
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[3], c[2], 0x0C0C0400u), __builtin_amdgcn_perm(c[1], c[0], 0x0C0C0400u), 0x05040100u);
}

// A wavefront takes a block of 256 values, four to a lane (two or four blocks to a wavefront, requested at once: 2 to 25 % slower).  Bound by memory, in 8 bits nearly as much by its
// arithmetic (some 85 instructions a value): what 1 - beta^t divides is multiplied, and the new root of v serves its code and the step.  One tensor of 12 M values: 67 us in 32 bits (5.0 TB/s), 44 in 8
// (4.4).  Wavefronts that stay, with the next block asked for ahead of this one's arithmetic, change nothing (11.4 M values of 229 tensors, 8 bits: 48.8 us with 8192 of them, 48.6 with one for each block).
template <typename TP, typename TG, bool EIGHT, int CAP>
__global__ void __launch_bounds__(256) adamw_kernel(AdamwArgs<CAP> a)
{
    const int lane = threadIdx.x & 63;
    const uint32_t block = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
    if (block >= a.blocks) return;
    int t = __popcll(__ballot(lane < CAP && a.first[min(lane, CAP - 1)] <= block)) - 1;
    if (CAP > 64 && t == 63) t += __popcll(__ballot(lane < CAP - 64 && a.first[min(64 + lane, CAP - 1)] <= block));
    t = __builtin_amdgcn_readfirstlane(t);
    const Entry e = a.tensors[t];
    const uint32_t at = block - a.first[t];
    const size_t o = (size_t)at * 256;  // of the block; the same for the wavefront, so that a lane adds its place alone
    const int n = (int)min((uint32_t)(e.n - at * 256u), 256u), i = lane * 4;
    const bool whole = a.aligned && i + 4 <= n;
    void* const pp = a.p + (e.p + o) * sizeof(TP);
    float *const master = e.master != NONE ? a.master + (e.master + o) : nullptr, *const scales = a.scales + (e.scales + 2 * (size_t)at);
    void *const pm = a.m + (e.m + o) * (EIGHT ? 1 : 4), *const pv = a.v + (e.v + o) * (EIGHT ? 1 : 4);
    float p[4], g[4], m[4], v[4], root[4], step_of[4];
    uint32_t wm = 0, wv = 0;
    float sm = 1.0f, sv = 1.0f;
    if (master) read4<float>(master, i, n, whole, p);
    else read4<TP>(pp, i, n, whole, p);
    read4<TG>(a.g + (e.g + o) * sizeof(TG), i, n, whole, g);
    if constexpr (EIGHT) {
        wm = codes4(pm, i, n, whole);
        wv = codes4(pv, i, n, whole);
        sm = scales[0];
        sv = scales[1];
    } else {
        read4<float>(pm, i, n, whole, m);
        read4<float>(pv, i, n, whole, v);
    }
    uint32_t step = a.step;
    float correct1 = a.correct1, correct2 = a.correct2;
    if (a.step_dev) {
        step = (uint32_t)max(*a.step_dev, 1);
        correct1 = (float)(1.0 / (1.0 - power(a.beta1, step)));
        correct2 = (float)sqrt(1.0 / (1.0 - power(a.beta2, step)));
    }
    const float lr = a.lr_dev ? *a.lr_dev : a.lr, gs = a.grad_scale ? *a.grad_scale : 1.0f, rate = lr * correct1;
    Decay d = a.decay;
    if (a.lr_dev) d = decay_of(lr * a.wd);
    if constexpr (EIGHT) {
        e4m3_values(wm, m);
        e4m3_values(wv, v);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (EIGHT) {
            m[k] *= sm;
            v[k] *= sv;
            v[k] *= v[k];
        }
        if (a.grad_scale) g[k] *= gs;
        m[k] = m[k] * a.b1 + g[k] * a.c1;
        v[k] = v[k] * a.b2 + g[k] * a.c2 * g[k];
        root[k] = nearest_root(v[k]);
        step_of[k] = (m[k] * rate) * __builtin_amdgcn_rcpf(fmaf(root[k], correct2, a.eps));
    }
    if (__builtin_amdgcn_readfirstlane(__float_as_int(d.rest)) != 0) {
#pragma unroll
        for (int k = 0; k < 4; ++k) step_of[k] = fmaf(p[k], d.rest, step_of[k]);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) p[k] = fmaf(p[k], d.keep, -step_of[k]);
    if (master) write4<float>(master, i, n, whole, p);
    write4<TP>(pp, i, n, whole, p);
    if constexpr (EIGHT) {
        uint32_t big[2] = {0u, 0u}, cm[4], cv[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            big[0] = max(big[0], __float_as_uint(m[k]) & 0x7FFFFFFFu);
            big[1] = max(big[1], __float_as_uint(root[k]) & 0x7FFFFFFFu);
        }
        float im, iv;
        power_scale(wave_max(big[0]), sm, im);
        power_scale(wave_max(big[1]), sv, iv);
        const uint32_t key = a.seed * 0x9E3779B1u + step * 0x6A09E667u, place = (a.base + block) * 256u + lane * 4u;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            uint32_t rm, rv;
            random_bits(key, place + k, rm, rv);
            cm[k] = e4m3_code(fabsf(m[k]) * im, rm) | (__float_as_uint(m[k]) >> 24 & 0x80u);
            cv[k] = max(e4m3_code(root[k] * iv, rv), min(__float_as_uint(root[k]), 1u));  // (not zero for what is not)
        }
        put_codes4(pm, i, n, whole, bytes4(cm));
        put_codes4(pv, i, n, whole, bytes4(cv));
        if (lane == 0) scales[0] = sm, scales[1] = sv;
    } else {
        write4<float>(pm, i, n, whole, m);
        write4<float>(pv, i, n, whole, v);
    }
}

// The lowest address of a kind and how far the others are from it, in elements of 2^log2 bytes: whether one more fits.  (Shifts: a division of the host's costs as much as all else that
// it does for a pointer.)
struct Window {
    int log2;
    uintptr_t low = ~(uintptr_t)0, high = 0;
    bool take(const void* p)
    {
        const uintptr_t x = (uintptr_t)p, l = x < low ? x : low, h = x > high ? x : high;
        if ((h - l) >> log2 >= NONE) return false;
        low = l;
        high = h;
        return true;
    }
    uint32_t step(const void* p) const { return (uint32_t)(((uintptr_t)p - low) >> log2); }
};

template <int CAP>
static hipError_t adamw_run(const lq_adamw_config* c, const lq_adamw_tensor* tensors, int count, const lq_adamw_args* x, hipStream_t s)
{
    AdamwArgs<CAP> a{};
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
    a.decay = decay_of(a.lr * a.wd);
    a.step = (uint32_t)x->step;
    double p1 = 1.0, p2 = 1.0, q1 = c->beta1, q2 = c->beta2;
    for (uint32_t t = a.step; t; t >>= 1, q1 *= q1, q2 *= q2)
        if (t & 1) p1 *= q1, p2 *= q2;
    a.correct1 = (float)(1.0 / (1.0 - p1));
    a.correct2 = (float)sqrt(1.0 / (1.0 - p2));
    a.seed = c->seed;
    const bool eight = c->state_bits == 8, pf = c->p_dtype == LQ_F32, gf = c->g_dtype == LQ_F32;
    const int pl = pf ? 2 : 1, gl = gf ? 2 : 1, sl = eight ? 0 : 2;  // log2 of an element's bytes
    for (int i = 0; i < count;) {
        const lq_adamw_tensor* of[CAP];
        int k = 0;
        Window wp{pl}, wmaster{2}, wg{gl}, wm{sl}, wv{sl}, ws{2};
        uintptr_t odd = 0;  // what keeps four values from being one access
        a.blocks = 0;
        for (; i < count && k < CAP; ++i) {
            const lq_adamw_tensor& t = tensors[i];
            const uint32_t more = (uint32_t)((t.n + 255) / 256);
            if (more == 0) continue;
            if (a.blocks + more > (1u << 25)) break;  // (a launch stays below 2^32 threads)
            const Window before[6] = {wp, wmaster, wg, wm, wv, ws};
            if (!wp.take(t.p) || (t.master && !wmaster.take(t.master)) || !wg.take(t.grad) || !wm.take(t.m) || !wv.take(t.v) || (eight && !ws.take(t.scales))) {
                wp = before[0], wmaster = before[1], wg = before[2], wm = before[3], wv = before[4], ws = before[5];
                break;  // (its launch is the next one)
            }
            a.tensors[k].n = (uint32_t)t.n;
            a.first[k] = a.blocks;
            a.blocks += more;
            odd |= ((uintptr_t)t.p & ((4u << pl) - 1)) | ((uintptr_t)t.master & 15) | ((uintptr_t)t.grad & ((4u << gl) - 1)) | (((uintptr_t)t.m | (uintptr_t)t.v) & ((4u << sl) - 1));
            of[k++] = &t;
        }
        if (k == 0) break;
        a.aligned = odd == 0;
        for (int j = 0; j < k; ++j) {
            const lq_adamw_tensor& t = *of[j];
            Entry& e = a.tensors[j];
            e.p = wp.step(t.p);
            e.master = t.master ? wmaster.step(t.master) : NONE;
            e.g = wg.step(t.grad);
            e.m = wm.step(t.m);
            e.v = wv.step(t.v);
            e.scales = eight ? ws.step(t.scales) : 0;
        }
        for (; k < CAP; ++k) a.first[k] = NONE;
        a.p = (char*)wp.low;
        a.master = (float*)wmaster.low;
        a.g = (const char*)wg.low;
        a.m = (char*)wm.low;
        a.v = (char*)wv.low;
        a.scales = (float*)ws.low;
        const dim3 grid((a.blocks + 3) / 4), block(256);
#define RUN(TP, TG) \
    if (eight) hipLaunchKernelGGL((adamw_kernel<TP, TG, true, CAP>), grid, block, 0, s, a); \
    else hipLaunchKernelGGL((adamw_kernel<TP, TG, false, CAP>), grid, block, 0, s, a)
        if (pf && gf) { RUN(float, float); }
        else if (pf) { RUN(float, __bf16); }
        else if (gf) { RUN(__bf16, float); }
        else { RUN(__bf16, __bf16); }
#undef RUN
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        a.base += a.blocks;
    }
    return hipSuccess;
}

// A few tensors: fewer arguments to bring to the card (us, with room for 8 / 120: one tensor of 1152 values 3.9 / 5.3, eight of 0.6 M 5.4 / 5.9)
hipError_t launch_adamw(const lq_adamw_config* c, const lq_adamw_tensor* tensors, int count, const lq_adamw_args* x, hipStream_t s)
{
    return count <= FEW ? adamw_run<FEW>(c, tensors, count, x, s) : adamw_run<TENSORS>(c, tensors, count, x, s);
}

}  // namespace lq
