// Product of a few rows with 4-bit weights in groups along K, and its transpose:
//     Y[m,n] = bias[n] + sum_g s[n,g] sum_{k in g} X[m,k] c[n,k] ;   dX[m,k] = sum_n dY[m,n] s[n,g(k)] c[n,k]
// Codes are small integers, exact in bf16; group sums and everything after them are held in fp32.  Bound by the read of the codes (half a byte a weight), in
// small layers by latency.
#include "lq_internal.h"

namespace lq {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// ---- layout -------------------------------------------------------------------------------------
// codes:  [tile of 16 channels][block of 128 of K][lane = n%16 + 16 q][16 bytes]: dword j of lane (n, q) holds k = 32 j + 8 q .. + 7 of the block, so that product
//         j of the matrix core takes 32 consecutive k, which belong to one group.  Value i < 4 of a dword is the low nibble of byte i, value 4 + i its high
//         nibble; a nibble is sign and magnitude.  What lies past N or K is zero.
// scales: [tile][block][n%16][128 / group] fp32
struct W4Shape {
    int64_t N, K;
    int tiles, blocks, per;  // tiles of N, blocks of K, groups of a block
};
static W4Shape w4_shape(const lq_w4_config* c)
{
    return {c->N, c->K, (int)((c->N + 15) / 16), (int)((c->K + 127) / 128), 128 / c->group};
}
static size_t w4_code_bytes(const W4Shape& s) { return (size_t)s.tiles * s.blocks * 1024; }
size_t w4_packed_bytes(const lq_w4_config* c)
{
    const W4Shape s = w4_shape(c);
    return w4_code_bytes(s) + (size_t)s.tiles * s.blocks * 16 * s.per * 4;
}

// ---- packing ------------------------------------------------------------------------------------

__device__ __forceinline__ uint32_t w4_nibble(int code)  // sign and magnitude
{
    const int m = min(abs(code), 7);
    return (uint32_t)m | (code < 0 && m ? 8u : 0u);
}
__device__ __forceinline__ int w4_code(uint32_t dword, int i)
{
    const uint32_t v = dword >> (8 * (i & 3) + (i & 4)) & 15u;
    return v & 8u ? -(int)(v & 7u) : (int)(v & 7u);
}

// A wavefront packs a block of a tile.  W: values, quantised by the INT family's rule (scale = amax / 7, code = rint(v 7 / amax), 1 for a group of zeros); or codes
// and scales that are there.
__global__ void __launch_bounds__(64) w4_pack_kernel(const float* W, const int8_t* codes, const float* scales, W4Shape s, uint8_t* out, float* sout)
{
    const int tile = blockIdx.x / s.blocks, block = blockIdx.x % s.blocks, lane = threadIdx.x, q = lane >> 4;
    const int64_t n = (int64_t)tile * 16 + (lane & 15), k0 = (int64_t)block * 128 + 8 * q;
    const int groups = (int)((s.K + 128 / s.per - 1) / (128 / s.per));
    uint32_t word[4];
    float sc[4];
    if (W) {
        float v[4][8], amax[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            amax[j] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t k = k0 + 32 * j + i;
                v[j][i] = n < s.N && k < s.K ? W[n * s.K + k] : 0.0f;
                amax[j] = fmaxf(amax[j], fabsf(v[j][i]));
            }
            amax[j] = fmaxf(amax[j], __shfl_xor(amax[j], 16));
            amax[j] = fmaxf(amax[j], __shfl_xor(amax[j], 32));
        }
        if (s.per <= 2) amax[0] = amax[1] = fmaxf(amax[0], amax[1]), amax[2] = amax[3] = fmaxf(amax[2], amax[3]);
        if (s.per == 1) amax[0] = amax[1] = amax[2] = amax[3] = fmaxf(amax[0], amax[2]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float inv = amax[j] == 0.0f ? 1.0f : 7.0f / amax[j];
            sc[j] = amax[j] == 0.0f ? 1.0f : amax[j] / 7.0f;
            word[j] = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) word[j] |= w4_nibble((int)fminf(fmaxf(rintf(v[j][i] * inv), -7.0f), 7.0f)) << (8 * (i & 3) + (i & 4));
        }
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int g = block * s.per + j * s.per / 4;
            sc[j] = n < s.N && g < groups ? scales[n * groups + g] : 1.0f;
            word[j] = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int64_t k = k0 + 32 * j + i;
                word[j] |= w4_nibble(n < s.N && k < s.K ? codes[n * s.K + k] : 0) << (8 * (i & 3) + (i & 4));
            }
        }
    }
    ((v4i*)out)[(size_t)blockIdx.x * 64 + lane] = v4i{(int)word[0], (int)word[1], (int)word[2], (int)word[3]};
    if (q == 0) {
        float* p = sout + ((size_t)blockIdx.x * 16 + lane) * s.per;
        if (s.per == 4) p[0] = sc[0], p[1] = sc[1], p[2] = sc[2], p[3] = sc[3];
        else if (s.per == 2) p[0] = sc[0], p[1] = sc[2];
        else p[0] = sc[0];
    }
}

__global__ void __launch_bounds__(64) w4_unpack_kernel(const uint8_t* in, const float* sin, W4Shape s, int8_t* codes, float* scales)
{
    const int tile = blockIdx.x / s.blocks, block = blockIdx.x % s.blocks, lane = threadIdx.x, q = lane >> 4;
    const int64_t n = (int64_t)tile * 16 + (lane & 15), k0 = (int64_t)block * 128 + 8 * q;
    const int groups = (int)((s.K + 128 / s.per - 1) / (128 / s.per));
    if (n >= s.N) return;
    const v4i w = ((const v4i*)in)[(size_t)blockIdx.x * 64 + lane];
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (codes && k0 + 32 * j + i < s.K) codes[n * s.K + k0 + 32 * j + i] = (int8_t)w4_code((uint32_t)w[j], i);
    if (q == 0 && scales)
        for (int g = 0; g < s.per; ++g)
            if (block * s.per + g < groups) scales[n * groups + block * s.per + g] = sin[((size_t)blockIdx.x * 16 + lane) * s.per + g];
}

// ---- codes to numbers -----------------------------------------------------------------------------

// Eight codes as bf16: the bytes of the eight magnitudes 0 .. 7 are two registers each, from which v_perm picks four at a time by the nibbles.  14 instructions,
// exact; the usual trick (nibbles into the mantissa of a larger number, which is subtracted from the sums) costs 7 and several bits of sums of one sign.
__device__ __forceinline__ v4i w4_bf16(uint32_t w)
{
    const uint32_t lo = w & 0x07070707u, hi = w >> 4 & 0x07070707u;
    uint32_t top[2], low[2];
    top[0] = __builtin_amdgcn_perm(0x40404040u, 0x40403F00u, lo) | (w << 4 & 0x80808080u);
    top[1] = __builtin_amdgcn_perm(0x40404040u, 0x40403F00u, hi) | (w & 0x80808080u);
    low[0] = __builtin_amdgcn_perm(0xE0C0A080u, 0x40008000u, lo);
    low[1] = __builtin_amdgcn_perm(0xE0C0A080u, 0x40008000u, hi);
    v4i r;
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        r[2 * h] = (int)__builtin_amdgcn_perm(top[h], low[h], 0x05010400u);
        r[2 * h + 1] = (int)__builtin_amdgcn_perm(top[h], low[h], 0x07030602u);
    }
    return r;
}
__device__ __forceinline__ v4f mfma(v4i a, v4i b, v4f c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}
// An fp32 number as three bf16 terms, each the leading bits of what the ones before leave: all 24 bits of it.  Of an infinity the first term is one and nothing
// is left.
__device__ __forceinline__ float cut(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t tops(float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u); }
__device__ __forceinline__ void split8(const float (&v)[8], v4i (&t)[3])
{
    float r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = v[j];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
#pragma unroll
        for (int d = 0; d < 4; ++d) t[k][d] = (int)tops(r[2 * d], r[2 * d + 1]);
#pragma unroll
        for (int j = 0; j < 8; ++j) r[j] = k == 0 && __builtin_isinf(r[j]) ? 0.0f : r[j] - cut(r[j]);
    }
}

// ---- forward ------------------------------------------------------------------------------------

struct W4Args {
    const uint8_t* codes;
    const float* scales;
    const void* X;  // rows that come in
    int64_t ldx;
    const float* bias;
    void* Y;        // rows that go out
    int64_t ldy;
    int64_t M, N, K;
    int tiles, blocks;
    int vec;        // rows of X can be read 16 bytes at a time
    int out_f32;
    int splits;     // backward: parts of N
    float* part;
};

// Eight values of a row of X from k on, as they lie in memory
template <bool F32>
struct Eight {
    v4i v[F32 ? 2 : 1];
    __device__ __forceinline__ void fetch(const void* row, int64_t k, int64_t K, bool vec)
    {
#pragma unroll
        for (int h = 0; h < (F32 ? 2 : 1); ++h) v[h] = v4i{0, 0, 0, 0};
        if (!row) return;
        if (vec && k + 8 <= K) {
#pragma unroll
            for (int h = 0; h < (F32 ? 2 : 1); ++h) v[h] = ((const v4i*)((const char*)row + k * (F32 ? 4 : 2)))[h];
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (k + i < K) {
                    if constexpr (F32) v[i / 4][i % 4] = ((const int*)row)[k + i];
                    else v[0][i / 2] |= (int)((uint32_t)((const uint16_t*)row)[k + i] << (16 * (i & 1)));
                }
            }
        }
    }
    __device__ __forceinline__ void terms(v4i (&t)[F32 ? 3 : 1]) const
    {
        if constexpr (F32) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = __int_as_float(v[i / 4][i % 4]);
            split8(f, t);
        } else {
            t[0] = v[0];
        }
    }
};

// A workgroup makes 16 MT rows of NT tiles; its wavefronts share K out block by block and join their sums in the LDS.
template <bool F32, int MT, int NT, int PER>
__global__ void __launch_bounds__(512) w4_fwd_kernel(W4Args a)
{
    extern __shared__ float joined[];  // [wavefront][MT][NT][4][64]
    constexpr int TERMS = F32 ? 3 : 1;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
    const int q = lane >> 4, tile0 = blockIdx.x * NT;
    const int64_t m0 = (int64_t)blockIdx.y * (16 * MT);
    const void* row[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int64_t m = m0 + 16 * mt + (lane & 15);
        row[mt] = m < a.M ? (const char*)a.X + m * a.ldx * (F32 ? 4 : 2) : nullptr;
    }
    v4f sum[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[mt][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    for (int b = wave; b < a.blocks; b += waves) {
        v4i code[NT];
        float sc[NT][PER];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const size_t at = (size_t)min(tile0 + t, a.tiles - 1) * a.blocks + b;
            code[t] = ((const v4i*)a.codes)[at * 64 + lane];
#pragma unroll
            for (int g = 0; g < PER; ++g) sc[t][g] = a.scales[(at * 16 + (lane & 15)) * PER + g];
        }
        Eight<F32> x[MT][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int j = 0; j < 4; ++j) x[mt][j].fetch(row[mt], (int64_t)b * 128 + 32 * j + 8 * q, a.K, a.vec);
#pragma unroll
        for (int g = 0; g < PER; ++g) {
            v4f acc[MT][NT];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int t = 0; t < NT; ++t) acc[mt][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int j = g * 4 / PER; j < (g + 1) * 4 / PER; ++j) {
                v4i w[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) w[t] = w4_bf16((uint32_t)code[t][j]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    v4i xt[TERMS];
                    x[mt][j].terms(xt);
#pragma unroll
                    for (int k = TERMS - 1; k >= 0; --k)
#pragma unroll
                        for (int t = 0; t < NT; ++t) acc[mt][t] = mfma(xt[k], w[t], acc[mt][t]);
                }
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[mt][t][r] = fmaf(sc[t][g], acc[mt][t][r], sum[mt][t][r]);
        }
    }
    constexpr int S = MT * NT * 256;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) joined[wave * S + ((mt * NT + t) * 4 + r) * 64 + lane] = sum[mt][t][r];
    __syncthreads();
    // value (mt, t, r, lane): row 16 mt + 4 (lane / 16) + r, channel lane % 16 of tile t
    for (int o = threadIdx.x; o < S; o += blockDim.x) {
        const int l = o & 63, r = o >> 6 & 3, u = o >> 8, t = u % NT, mt = u / NT;
        const int64_t m = m0 + 16 * mt + 4 * (l >> 4) + r, n = (int64_t)(tile0 + t) * 16 + (l & 15);
        if (m >= a.M || n >= a.N) continue;
        float y = joined[o];
        for (int w = 1; w < waves; ++w) y += joined[w * S + o];
        if (a.bias) y += a.bias[n];
        if (a.out_f32) ((float*)a.Y)[m * a.ldy + n] = y;
        else ((__bf16*)a.Y)[m * a.ldy + n] = (__bf16)y;
    }
}

// ---- gradient ------------------------------------------------------------------------------------

// dX of R rows: a lane's 32 columns of a block, over the 16 channels of a tile in 16 lanes; tiles are dealt to the workgroup's wavefronts and to the parts of N.  The
// 16 lanes' sums are joined by halving what each keeps, the wavefronts' in the LDS, the parts' by w4_join.
template <bool F32, int R, int PER>
__global__ void __launch_bounds__(256) w4_bwd_kernel(W4Args a)
{
    __shared__ float joined[4][R][128];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, q = lane >> 4;
    const int block = blockIdx.x, split = blockIdx.y;
    const int64_t m0 = (int64_t)blockIdx.z * R;
    float acc[R][32];
#pragma unroll
    for (int m = 0; m < R; ++m)
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[m][i] = 0.0f;
    for (int t = split * 4 + wave; t < a.tiles; t += 4 * a.splits) {
        const size_t at = (size_t)t * a.blocks + block;
        const v4i code = ((const v4i*)a.codes)[at * 64 + lane];
        float sc[PER], g[R];
#pragma unroll
        for (int i = 0; i < PER; ++i) sc[i] = a.scales[(at * 16 + c) * PER + i];
        const int64_t n = (int64_t)t * 16 + c;
#pragma unroll
        for (int m = 0; m < R; ++m) {
            g[m] = 0.0f;
            if (n < a.N && m0 + m < a.M) {
                if constexpr (F32) g[m] = ((const float*)a.X)[(m0 + m) * a.ldx + n];
                else g[m] = (float)((const __bf16*)a.X)[(m0 + m) * a.ldx + n];
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const v4i w = w4_bf16((uint32_t)code[j]);
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(i & 1 ? (uint32_t)w[i / 2] & 0xFFFF0000u : (uint32_t)w[i / 2] << 16);
#pragma unroll
            for (int m = 0; m < R; ++m) {
                const float u = g[m] * sc[j * PER / 4];
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[m][8 * j + i] = fmaf(u, f[i], acc[m][8 * j + i]);
            }
        }
    }
#pragma unroll
    for (int m = 0; m < R; ++m) {
#pragma unroll
        for (int half = 16; half >= 2; half /= 2) {
            const int bit = half / 2;
            const bool up = c & bit;
#pragma unroll
            for (int i = 0; i < half; ++i) {
                const float give = up ? acc[m][i] : acc[m][i + half], keep = up ? acc[m][i + half] : acc[m][i];
                acc[m][i] = keep + __shfl_xor(give, bit);
            }
        }
        // two values are left: columns 2 c, 2 c + 1 of the 32
        const int i = 2 * c;
        joined[wave][m][32 * (i >> 3) + 8 * q + (i & 7)] = acc[m][0];
        joined[wave][m][32 * (i >> 3) + 8 * q + (i & 7) + 1] = acc[m][1];
    }
    __syncthreads();
    for (int o = threadIdx.x; o < R * 128; o += 256) {
        const int m = o >> 7, k = o & 127;
        const int64_t kk = (int64_t)block * 128 + k;
        if (m0 + m >= a.M || kk >= a.K) continue;
        const float v = (joined[0][m][k] + joined[1][m][k]) + (joined[2][m][k] + joined[3][m][k]);
        if (a.part) a.part[((size_t)split * a.M + m0 + m) * a.K + kk] = v;
        else if (a.out_f32) ((float*)a.Y)[(m0 + m) * a.ldy + kk] = v;
        else ((__bf16*)a.Y)[(m0 + m) * a.ldy + kk] = (__bf16)v;
    }
}

// Sum of the parts, in a fixed order: four shares of them, 64 values to a workgroup
__global__ void __launch_bounds__(256) w4_join(W4Args a)
{
    __shared__ float sh[4][64];
    const int64_t o = (int64_t)blockIdx.x * 64 + (threadIdx.x & 63), total = a.M * a.K;
    const int r = threadIdx.x >> 6;
    float t = 0.0f;
    if (o < total)
#pragma unroll 8
        for (int i = r; i < a.splits; i += 4) t += a.part[i * total + o];
    sh[r][threadIdx.x & 63] = t;
    __syncthreads();
    if (r == 0 && o < total) {
        const int c = threadIdx.x;
        t = (sh[0][c] + sh[1][c]) + (sh[2][c] + sh[3][c]);
        const int64_t m = o / a.K, k = o - m * a.K;
        if (a.out_f32) ((float*)a.Y)[m * a.ldy + k] = t;
        else ((__bf16*)a.Y)[m * a.ldy + k] = (__bf16)t;
    }
}

// ---- host ---------------------------------------------------------------------------------------

hipError_t launch_w4_pack(const lq_w4_config* c, const float* W, const int8_t* codes, const float* scales, uint8_t* packed, hipStream_t s)
{
    const W4Shape sh = w4_shape(c);
    hipLaunchKernelGGL(w4_pack_kernel, dim3((unsigned)(sh.tiles * sh.blocks)), dim3(64), 0, s, W, codes, scales, sh, packed, (float*)(packed + w4_code_bytes(sh)));
    return hipGetLastError();
}

hipError_t launch_w4_unpack(const lq_w4_config* c, const uint8_t* packed, int8_t* codes, float* scales, hipStream_t s)
{
    const W4Shape sh = w4_shape(c);
    hipLaunchKernelGGL(w4_unpack_kernel, dim3((unsigned)(sh.tiles * sh.blocks)), dim3(64), 0, s, packed, (const float*)(packed + w4_code_bytes(sh)), sh, codes, scales);
    return hipGetLastError();
}

template <bool F32, int MT, int NT>
static void w4_fwd_per(const W4Args& a, int per, dim3 grid, int waves, hipStream_t s)
{
    const size_t lds = (size_t)waves * MT * NT * 1024;
    if (per == 1) hipLaunchKernelGGL((w4_fwd_kernel<F32, MT, NT, 1>), grid, dim3(64 * waves), lds, s, a);
    else if (per == 2) hipLaunchKernelGGL((w4_fwd_kernel<F32, MT, NT, 2>), grid, dim3(64 * waves), lds, s, a);
    else hipLaunchKernelGGL((w4_fwd_kernel<F32, MT, NT, 4>), grid, dim3(64 * waves), lds, s, a);
}
template <bool F32>
static void w4_fwd_rows(const W4Args& a, int per, hipStream_t s)
{
    const int waves = a.blocks < 8 ? a.blocks : 8;
    if (a.M <= 16) w4_fwd_per<F32, 1, 1>(a, per, dim3(a.tiles, 1), waves, s);
    else if (a.M <= 32) w4_fwd_per<F32, 2, 1>(a, per, dim3(a.tiles, 1), waves, s);
    else w4_fwd_per<F32, 4, 2>(a, per, dim3((a.tiles + 1) / 2, (unsigned)((a.M + 63) / 64)), waves, s);
}

static W4Args w4_args(const lq_w4_config* c, const uint8_t* packed, const void* in, int64_t ldin, int in_elem, void* out, int64_t ldout, int64_t M)
{
    const W4Shape sh = w4_shape(c);
    W4Args a{};
    a.codes = packed;
    a.scales = (const float*)(packed + w4_code_bytes(sh));
    a.X = in;
    a.ldx = ldin;
    a.Y = out;
    a.ldy = ldout;
    a.M = M;
    a.N = c->N;
    a.K = c->K;
    a.tiles = sh.tiles;
    a.blocks = sh.blocks;
    a.vec = (uintptr_t)in % 16 == 0 && (M < 2 || ldin * in_elem % 16 == 0);
    return a;
}

hipError_t launch_w4_fwd(const lq_w4_config* c, const uint8_t* packed, const void* X, int64_t ldx, const float* bias, void* Y, int64_t ldy, int64_t M, hipStream_t s)
{
    W4Args a = w4_args(c, packed, X, ldx, c->x_dtype == LQ_F32 ? 4 : 2, Y, ldy, M);
    a.bias = bias;
    a.out_f32 = c->y_dtype == LQ_F32;
    if (c->x_dtype == LQ_F32) w4_fwd_rows<true>(a, 128 / c->group, s);
    else w4_fwd_rows<false>(a, 128 / c->group, s);
    return hipGetLastError();
}

// Rows of a workgroup of the gradient, and parts of N: two workgroups to a compute unit, each wavefront with two tiles or more
static int w4_bwd_rows(int64_t M) { return M == 1 ? 1 : M == 2 ? 2 : 4; }
static int w4_bwd_splits(const W4Shape& s, int64_t M)
{
    const int R = w4_bwd_rows(M);
    const int64_t others = (int64_t)s.blocks * ((M + R - 1) / R), want = (512 + others - 1) / others, most = (s.tiles + 7) / 8;
    return (int)(want < 1 ? 1 : want < most ? want : most);
}
size_t w4_work_bytes(const lq_w4_config* c, int64_t M)
{
    const int splits = M ? w4_bwd_splits(w4_shape(c), M) : 1;
    return splits > 1 ? align256((size_t)splits * M * c->K * 4) : 0;
}

template <bool F32, int R>
static void w4_bwd_per(const W4Args& a, int per, dim3 grid, hipStream_t s)
{
    if (per == 1) hipLaunchKernelGGL((w4_bwd_kernel<F32, R, 1>), grid, dim3(256), 0, s, a);
    else if (per == 2) hipLaunchKernelGGL((w4_bwd_kernel<F32, R, 2>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((w4_bwd_kernel<F32, R, 4>), grid, dim3(256), 0, s, a);
}
template <bool F32>
static void w4_bwd_all(const W4Args& a, int per, hipStream_t s)
{
    const int R = w4_bwd_rows(a.M);
    const dim3 grid(a.blocks, a.splits, (unsigned)((a.M + R - 1) / R));
    if (R == 1) w4_bwd_per<F32, 1>(a, per, grid, s);
    else if (R == 2) w4_bwd_per<F32, 2>(a, per, grid, s);
    else w4_bwd_per<F32, 4>(a, per, grid, s);
}
hipError_t launch_w4_bwd(const lq_w4_config* c, const uint8_t* packed, const void* dY, int64_t lddy, void* dX, int64_t lddx, int64_t M, uint8_t* work, hipStream_t s)
{
    W4Args a = w4_args(c, packed, dY, lddy, c->y_dtype == LQ_F32 ? 4 : 2, dX, lddx, M);
    a.out_f32 = c->x_dtype == LQ_F32;
    a.splits = w4_bwd_splits(w4_shape(c), M);
    a.part = a.splits > 1 ? (float*)work : nullptr;
    if (c->y_dtype == LQ_F32) w4_bwd_all<true>(a, 128 / c->group, s);
    else w4_bwd_all<false>(a, 128 / c->group, s);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !a.part) return e;
    hipLaunchKernelGGL(w4_join, dim3((unsigned)((M * c->K + 63) / 64)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace lq
