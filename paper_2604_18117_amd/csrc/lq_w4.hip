// Product of a few rows with 4-bit weights in groups along K, and its transpose:
//     Y[m,n] = bias[n] + sum_g s[n,g] sum_{k in g} X[m,k] c[n,k] ;   dX[m,k] = sum_n dY[m,n] s[n,g(k)] c[n,k]
// Codes are small integers, exact in bf16; group sums and everything after them are held in fp32.  Bound by the read of the codes (half a byte a weight), in
// small layers by latency.
#include "lq_internal.h"
#include <type_traits>

namespace lq {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

// ---- layout -------------------------------------------------------------------------------------
// header: BLOB_HEADER bytes, w4_tag and zeros
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
    return BLOB_HEADER + w4_code_bytes(s) + (size_t)s.tiles * s.blocks * 16 * s.per * 4;
}
static const uint8_t* w4_codes(const uint8_t* packed) { return packed + BLOB_HEADER; }
static const float* w4_scales(const uint8_t* packed, const W4Shape& s) { return (const float*)(packed + BLOB_HEADER + w4_code_bytes(s)); }

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
// and scales that are there.  Done once for a layer: 11200 x 2240 49 us, 2.3 TB/s (a lane's eight values lie together, its neighbours' in other rows).
__global__ void __launch_bounds__(64) w4_pack_kernel(const float* W, const int8_t* codes, const float* scales, W4Shape s, BlobTag tag, uint32_t* header, uint8_t* out, float* sout)
{
    static_assert(BLOB_HEADER == 64 * 4, "a dword to a lane");
    const int tile = blockIdx.x / s.blocks, block = blockIdx.x % s.blocks, lane = threadIdx.x, q = lane >> 4;
    if (blockIdx.x == 0) header[lane] = lane < 8 ? tag.w[lane & 7] : 0u;
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
            const float up = amax[j] < 0x1p-100f ? 0x1p100f : 1.0f;  // (below 2^-125 the quotient would be infinite)
            const float inv = amax[j] == 0.0f ? 1.0f : 7.0f / (amax[j] * up);
            sc[j] = amax[j] == 0.0f ? 1.0f : amax[j] / 7.0f;
            word[j] = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) word[j] |= w4_nibble((int)fminf(fmaxf(rintf(v[j][i] * up * inv), -7.0f), 7.0f)) << (8 * (i & 3) + (i & 4));
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
// An fp32 number as three bf16 terms, each the leading bits of what the ones before leave: all 24 bits of it from 2^-110 on, below that all down to 2^-133, bf16's smallest number.  Of an infinity the
// first term is one and nothing is left.
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

__device__ __forceinline__ void split4(v4i v, uint2 (&t)[3])  // ... of four, as packed pairs
{
    float r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = __int_as_float(v[j]);
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        t[k] = make_uint2(tops(r[0], r[1]), tops(r[2], r[3]));
#pragma unroll
        for (int j = 0; j < 4; ++j) r[j] = k == 0 && __builtin_isinf(r[j]) ? 0.0f : r[j] - cut(r[j]);
    }
}

// Between a wavefront's stores to its LDS and other lanes' loads of them or stores over them, and between loads and the next stores: neither moves across.  (The LDS takes a wavefront's accesses in their order, so that this is no
// instruction.)
__device__ __forceinline__ void wave_lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
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
    int out_f32;
    int splits;     // backward: parts of N
    float* part;
};

constexpr int w4_fwd_lds(bool f32, int mt, int nt)  // bytes of a wavefront: its block of X (of fp32 values three terms), then its sums
{
    const int x = (f32 ? 3 : 1) * 16 * mt * 272, sums = mt * nt * 1024;
    return x > sums ? x : sums;
}

// Eight values of a row, as they lie in memory (of any alignment: the card reads 16 bytes from wherever they start)
template <bool F32>
struct Eight {
    typedef v4i Access __attribute__((aligned(2)));
    static constexpr int H = F32 ? 2 : 1;
    v4i v[H];
    __device__ __forceinline__ void read(const char* row, int k)
    {
#pragma unroll
        for (int h = 0; h < H; ++h) v[h] = ((const Access*)(row + (size_t)k * (F32 ? 4 : 2)))[h];
    }
    // Where a row may end among them: zeros from `end` on.  The row's last eight values are read and moved to their places; with a read of its own for every value, or a branch for
    // every read, the end of a row cost more than the rest of it.
    __device__ __forceinline__ void read_end(const char* row, int k, int end)
    {
        if (end < 8) {
#pragma unroll
            for (int h = 0; h < H; ++h) v[h] = v4i{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (k + i < end) {
                    if constexpr (F32) v[i / 4][i % 4] = ((const int*)row)[k + i];
                    else v[0][i / 2] |= (int)((uint32_t)((const uint16_t*)row)[k + i] << (16 * (i & 1)));
                }
            return;
        }
        const int first = min(k, end - 8), past = min(k - first, 8);
        read(row, first);
#pragma unroll
        for (int step = 8; step >= 1; step /= 2) {
            const bool on = past & step;
#pragma unroll
            for (int d = 0; d < 4 * H; ++d) {
                int moved;
                if (!F32 && step == 1) {
                    moved = (int)((uint32_t)v[0][d] >> 16) | (d < 3 ? v[0][d < 3 ? d + 1 : 0] << 16 : 0);
                } else {
                    const int from = d + (F32 ? step : step / 2);
                    moved = from < 4 * H ? v[from / 4 < H ? from / 4 : 0][from % 4] : 0;
                }
                v[d / 4][d % 4] = on ? moved : v[d / 4][d % 4];
            }
        }
    }
    __device__ __forceinline__ void values(float (&f)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = __int_as_float(F32 ? v[F32 ? i / 4 : 0][i % 4] : i & 1 ? v[0][i / 2] & (int)0xFFFF0000 : v[0][i / 2] << 16);
    }
};

// A workgroup makes 16 MT rows of NT tiles; its wavefronts share K out block by block and join their sums in the LDS.  A wavefront brings its block of X through LDS of its own: 16 lanes
// read a row's 256 bytes (32 lanes 512), where the product's order, 16 rows in 16 lanes, is a piece of a cache line in every lane.  The next block is requested ahead of the products of
// this one (codes two blocks ahead: 64 x 2240 -> 11200 13.4 us for 13.1).  64 x 2240 -> 11200 takes 13-14 us, 2 x 1152 -> 6912 4.0, of which 3.2 are any launch's.  In the first 31 MB come
// past the L2s, the codes twice, once for each 32 rows; 1.4 wavefronts a SIMD wait 43 % of their cycles, the vector unit has 25 %.  Tried there: 64 rows to a workgroup 16.5, four tiles 16.1; the
// workgroups of a tile one after another on one XCD, where the second finds the codes, 13.1, but then 48 x 1152 -> 6912 takes 7.1 for 6.3.  Rows past M repeat the last one and are not stored.  In the block where rows end, pieces of 16 bytes past the end are zero; the one in which they end is brought value by value.
template <bool F32, int MT, int NT, int PER>
__global__ void __launch_bounds__(512) w4_fwd_kernel(W4Args a)
{
    extern __shared__ v4i shared[];
    typedef v4i Piece __attribute__((aligned(2)));
    typedef typename std::conditional<F32, uint32_t, uint16_t>::type Bits;
    float* joined = (float*)shared;  // [wavefront][MT][NT][4][64]
    constexpr int TERMS = F32 ? 3 : 1, EB = F32 ? 4 : 2, LANES = 8 * EB, ROWS = 64 / LANES, N = 16 * MT / ROWS, STRIDE = 272, TERM = 16 * MT * STRIDE;  // lanes of a row; rows at a time; bytes of a row and of a term in the LDS
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    const int q = lane >> 4, tile0 = blockIdx.x * NT, m0 = blockIdx.y * (16 * MT), end = (int)a.K * EB;
    char* mine = (char*)shared + wave * w4_fwd_lds(F32, MT, NT);
    const char* X = (const char*)a.X + (int64_t)m0 * a.ldx * EB;
    const unsigned pitch = (unsigned)a.ldx * EB;
    const int part = lane % LANES * 16, last = (int)a.M - 1 - m0;
    unsigned at[N];  // of the lane's rows
#pragma unroll
    for (int i = 0; i < N; ++i) at[i] = (unsigned)min(i * ROWS + lane / LANES, last) * pitch;
    v4f sum[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < NT; ++t) sum[mt][t] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    v4i next[NT], x[N];
    float next_sc[NT][PER];
    auto request = [&](int b) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const size_t o = (size_t)min(tile0 + t, a.tiles - 1) * a.blocks + b;
            next[t] = ((const v4i*)a.codes)[o * 64 + lane];
#pragma unroll
            for (int g = 0; g < PER; ++g) next_sc[t][g] = a.scales[(o * 16 + (lane & 15)) * PER + g];
        }
        if (end >= 16) {
            const unsigned k = (unsigned)min(b * (128 * EB) + part, end - 16);
#pragma unroll
            for (int i = 0; i < N; ++i)
                if (i * ROWS <= last) x[i] = *(const Piece*)(X + (at[i] + k));  // (the same for the wavefront)
        }
    };
    request(wave);  // (there are no more wavefronts than blocks)
    for (int b = wave; b < a.blocks; b += waves) {
        const int k0 = b * (128 * EB);
        if (k0 + 128 * EB > end) {
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = k0 + part + 16 <= end ? x[i] : v4i{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i * ROWS <= last) {
                char* to = mine + (i * ROWS + lane / LANES) * STRIDE + part * 2 / EB;
                if constexpr (F32) {
                    uint2 t[3];
                    split4(x[i], t);
#pragma unroll
                    for (int k = 0; k < 3; ++k) *(uint2*)(to + k * TERM) = t[k];
                } else {
                    *(v4i*)to = x[i];
                }
            }
        if (k0 + 128 * EB > end && end % 16) {
            wave_lds_order();  // (the zeros of that piece were another lane's)
            Bits v[2 * MT];  // eight rows of eight values (f32: of four) at a time
            const int k = end / 16 * 16 + (lane & 7) * EB;
#pragma unroll
            for (int i = 0; i < 2 * MT; ++i) v[i] = k < end ? *(const Bits*)(X + (int64_t)min(8 * i + (lane >> 3), last) * pitch + k) : (Bits)0;
#pragma unroll
            for (int i = 0; i < 2 * MT; ++i)
                if ((lane & 7) * EB < 16) {
                    char* to = mine + (8 * i + (lane >> 3)) * STRIDE + (k - k0) * 2 / EB;
                    if constexpr (F32) {
                        uint2 t[3];
                        split4(v4i{(int)v[i], 0, 0, 0}, t);
#pragma unroll
                        for (int k = 0; k < 3; ++k) *(uint16_t*)(to + k * TERM) = (uint16_t)t[k].x;
                    } else {
                        *(uint16_t*)to = v[i];
                    }
                }
        }
        wave_lds_order();
        v4i code[NT];
        float sc[NT][PER];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            code[t] = next[t];
#pragma unroll
            for (int g = 0; g < PER; ++g) sc[t][g] = next_sc[t][g];
        }
        if (b + waves < a.blocks) request(b + waves);
#pragma unroll
        for (int g = 0; g < PER; ++g) {
            v4f acc[MT][NT];
#pragma unroll
            for (int j = g * 4 / PER; j < (g + 1) * 4 / PER; ++j) {
                v4i w[NT];
#pragma unroll
                for (int t = 0; t < NT; ++t) w[t] = w4_bf16((uint32_t)code[t][j]);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) {
                    v4i xt[TERMS];
#pragma unroll
                    for (int k = 0; k < TERMS; ++k) xt[k] = *(const v4i*)(mine + k * TERM + (16 * mt + (lane & 15)) * STRIDE + (32 * j + 8 * q) * 2);
#pragma unroll
                    for (int k = TERMS - 1; k >= 0; --k)
#pragma unroll
                        for (int t = 0; t < NT; ++t) acc[mt][t] = mfma(xt[k], w[t], j == g * 4 / PER && k == TERMS - 1 ? v4f{0.0f, 0.0f, 0.0f, 0.0f} : acc[mt][t]);
                }
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int r = 0; r < 4; ++r) sum[mt][t][r] = fmaf(sc[t][g], acc[mt][t][r], sum[mt][t][r]);
        }
        wave_lds_order();
    }
    __syncthreads();
    constexpr int S = MT * NT * 256;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) joined[wave * (w4_fwd_lds(F32, MT, NT) / 4) + ((mt * NT + t) * 4 + r) * 64 + lane] = sum[mt][t][r];
    __syncthreads();
    // value (mt, t, r, lane): row 16 mt + 4 (lane / 16) + r, channel lane % 16 of tile t
    for (int o = threadIdx.x; o < S; o += blockDim.x) {
        const int l = o & 63, r = o >> 6 & 3, u = o >> 8, t = u % NT, mt = u / NT;
        const int64_t m = m0 + 16 * mt + 4 * (l >> 4) + r, n = (int64_t)(tile0 + t) * 16 + (l & 15);
        if (m >= a.M || n >= a.N) continue;
        float y = joined[o];
        for (int w = 1; w < waves; ++w) y += joined[w * (w4_fwd_lds(F32, MT, NT) / 4) + o];
        if (a.bias) y += a.bias[n];
        if (a.out_f32) ((float*)a.Y)[m * a.ldy + n] = y;
        else ((__bf16*)a.Y)[m * a.ldy + n] = (__bf16)y;
    }
}

// ---- gradient ------------------------------------------------------------------------------------

// Nibble p(r) of dword i from nibble p(i) of dword r, eight by eight (p: the place of a value in a dword): bit by bit of the two numbers, 32 instructions
__device__ __forceinline__ void turn_nibbles(uint32_t (&d)[8])
{
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const uint32_t x = d[r], y = d[r + 4];
        d[r] = (x & 0x0F0F0F0Fu) | (y << 4 & 0xF0F0F0F0u);
        d[r + 4] = (x >> 4 & 0x0F0F0F0Fu) | (y & 0xF0F0F0F0u);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const int r = k & 1 | (k & 2) << 1;
        const uint32_t x = d[r], y = d[r + 2];
        d[r] = __builtin_amdgcn_perm(y, x, 0x05040100u);
        d[r + 2] = __builtin_amdgcn_perm(y, x, 0x07060302u);
    }
#pragma unroll
    for (int r = 0; r < 8; r += 2) {
        const uint32_t x = d[r], y = d[r + 1];
        d[r] = __builtin_amdgcn_perm(y, x, 0x06020400u);
        d[r + 1] = __builtin_amdgcn_perm(y, x, 0x07030501u);
    }
}

// dX of 16 rows and a block of 128 columns.  A wavefront takes 32 channels at a time (two tiles), which it brings through LDS of its own so that lane (c, q) holds eight channels
// 8 q .. + 7 of the eight columns 8 c .. + 7; turned, they are the operands of eight products, product i with the columns 8 c + i.  The channels' scales go into dY (fp32, three terms);
// where a block has several groups, a product is made for each and a lane keeps that of its own columns.  The wavefronts' sums are joined in the LDS, those of the parts of N by w4_join.
// 16 x 2240 -> 13440: 11 us (at 0.9 wavefronts a SIMD, which wait 45 % of their cycles; vector unit 24 %) and 3.5 for the join; 2 x 1152 -> 6912: 6 and 3.9.
constexpr int w4_bwd_waves(int per) { return per == 4 ? 4 : 8; }  // (sums for four groups are 128 registers)
template <bool F32, int PER>
__global__ void __launch_bounds__(64 * w4_bwd_waves(PER)) w4_bwd_kernel(W4Args a)
{
    extern __shared__ v4i shared[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, c = lane & 15, q = lane >> 4;
    const int block = blockIdx.x, split = blockIdx.y, steps = (a.tiles + 1) / 2;
    const int64_t m0 = (int64_t)blockIdx.z * 16;
    const char* row = (const char*)a.X + min(m0 + c, a.M - 1) * a.ldx * (F32 ? 4 : 2);
    char* mine = (char*)shared + wave * 2176;  // [2 tiles][4][16 channels + 1][16 bytes]: every read finds 64 banks
    v4f acc[PER][8];
#pragma unroll
    for (int g = 0; g < PER; ++g)
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[g][i] = v4f{0.0f, 0.0f, 0.0f, 0.0f};
    v4i next[2];
    float next_sc[8 * PER];
    Eight<F32> next_dy;
    auto request = [&](int s) {
#pragma unroll
        for (int t = 0; t < 2; ++t) next[t] = ((const v4i*)a.codes)[((size_t)min(2 * s + t, a.tiles - 1) * a.blocks + block) * 64 + lane];
        const float* sc = a.scales + (((size_t)min(2 * s + (q >> 1), a.tiles - 1) * a.blocks + block) * 16 + 8 * (q & 1)) * PER;
#pragma unroll
        for (int i = 0; i < 2 * PER; ++i) {
            const v4f v = ((const v4f*)sc)[i];
#pragma unroll
            for (int e = 0; e < 4; ++e) next_sc[4 * i + e] = v[e];
        }
        if ((s + 1) * 32 <= a.N) next_dy.read(row, s * 32 + 8 * q);
        else next_dy.read_end(row, s * 32 + 8 * q, (int)a.N);
    };
    const int first = split * waves + wave, stride = a.splits * waves;
    if (first < steps) request(first);
    for (int s = first; s < steps; s += stride) {
#pragma unroll
        for (int t = 0; t < 2; ++t) *(v4i*)(mine + t * 1088 + q * 272 + c * 16) = next[t];
        wave_lds_order();
        float dy[8], sc[8 * PER];
        next_dy.values(dy);
#pragma unroll
        for (int i = 0; i < 8 * PER; ++i) sc[i] = next_sc[i];
        if (s + stride < steps) request(s + stride);
        uint32_t d[8];
#pragma unroll
        for (int r = 0; r < 8; ++r) d[r] = *(const uint32_t*)(mine + (q >> 1) * 1088 + (c & 3) * 272 + (8 * (q & 1) + r) * 16 + (c >> 2) * 4);
        wave_lds_order();
        turn_nibbles(d);
        v4i up[PER][3];
#pragma unroll
        for (int g = 0; g < PER; ++g) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = dy[i] * sc[i * PER + g];
            split8(f, up[g]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const v4i w = w4_bf16(d[i]);
#pragma unroll
            for (int k = 2; k >= 0; --k)
#pragma unroll
                for (int g = 0; g < PER; ++g) acc[g][i] = mfma(up[g][k], w, acc[g][i]);
        }
    }
    float* joined = (float*)shared;  // [wavefront][16][128]
    __syncthreads();
    // sum r of product i: row 4 q + r, column 8 c + i
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v4f v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[e] = acc[0][4 * h + e][r];
#pragma unroll
                for (int g = 1; g < PER; ++g) v[e] = c * PER / 16 == g ? acc[g][4 * h + e][r] : v[e];
            }
            *(v4f*)(joined + (wave * 16 + 4 * q + r) * 128 + 8 * c + 4 * h) = v;
        }
    __syncthreads();
    for (int o = threadIdx.x; o < 16 * 128; o += blockDim.x) {
        const int m = o >> 7, k = o & 127;
        const int64_t kk = (int64_t)block * 128 + k;
        if (m0 + m >= a.M || kk >= a.K) continue;
        float v = joined[m * 128 + k];
        for (int w = 1; w < waves; ++w) v += joined[(w * 16 + m) * 128 + k];
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
    hipLaunchKernelGGL(w4_pack_kernel, dim3((unsigned)(sh.tiles * sh.blocks)), dim3(64), 0, s, W, codes, scales, sh, w4_tag(c), (uint32_t*)packed, (uint8_t*)w4_codes(packed),
                       (float*)w4_scales(packed, sh));
    return hipGetLastError();
}

hipError_t launch_w4_unpack(const lq_w4_config* c, const uint8_t* packed, int8_t* codes, float* scales, hipStream_t s)
{
    const W4Shape sh = w4_shape(c);
    hipLaunchKernelGGL(w4_unpack_kernel, dim3((unsigned)(sh.tiles * sh.blocks)), dim3(64), 0, s, w4_codes(packed), w4_scales(packed, sh), sh, codes, scales);
    return hipGetLastError();
}

template <bool F32, int MT, int NT, int PER>
static hipError_t w4_fwd_run(const W4Args& a, int waves, hipStream_t s)
{
    const int lds = waves * w4_fwd_lds(F32, MT, NT);
    if (lds > 65536) {
        const hipError_t e = allow_lds<w4_fwd_kernel<F32, MT, NT, PER>>(8 * w4_fwd_lds(F32, MT, NT));
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((w4_fwd_kernel<F32, MT, NT, PER>), dim3((a.tiles + NT - 1) / NT, (unsigned)((a.M + 16 * MT - 1) / (16 * MT))), dim3(64 * waves), lds, s, a);
    return hipGetLastError();
}
template <bool F32, int MT, int NT>
static hipError_t w4_fwd_per(const W4Args& a, int per, int waves, hipStream_t s)
{
    return per == 1 ? w4_fwd_run<F32, MT, NT, 1>(a, waves, s) : per == 2 ? w4_fwd_run<F32, MT, NT, 2>(a, waves, s) : w4_fwd_run<F32, MT, NT, 4>(a, waves, s);
}
// Rows and channels of a workgroup, and the wavefronts that share K out.  bf16: one tile and up to 16 rows, from more than 16 rows on 32, with two tiles (what is unpacked and what is read of X are
// shared) where one would leave more than two workgroups to a compute unit, three where two would leave more than the three that it holds (us, one / two tiles: 64 x 2240 -> 11200 16.5 / 13.4,
// 64 x 1152 -> 1152 4.3 / 5.1; two / three: 64 x 4608 -> 13440 27.3 / 24.0, 64 x 2240 -> 11200 13.4 / 13.9).  Eight wavefronts where there is a workgroup to a compute unit at most, four elsewhere (us, 8 / 4:
// 16 x 4608 -> 2240 5.2 / 5.9, 64 x 2240 -> 11200 16.6 / 12.9).  fp32 rows, which are split into three terms for every workgroup and take three times the LDS: 16 rows, and up to four tiles that
// leave one workgroup of eight wavefronts to a compute unit (us, against one tile and four: 16 x 2240 -> 11200 9.5 / 13.3, 6 x 3992 -> 5760 8.7 / 11.4, 64 x 1152 -> 1152 6.1 / 7.0; against two and four, 16 x 2240 -> 15000 10.8 / 13.7, 64 x 1152 -> 3456 7.5 / 8.4); where more than
// four would do that, two or three and four wavefronts (33 x 1152 -> 6912, two / three: 8.7 / 9.8; 64 x 2240 -> 11200 29.7 / 26.5).
template <bool F32>
static hipError_t w4_fwd_rows(const W4Args& a, int per, hipStream_t s)
{
    const int MT = !F32 && a.M > 16 ? 2 : 1;
    const int64_t groups = a.tiles * ((a.M + 16 * MT - 1) / (16 * MT));
    int NT = 1;
    if (F32) NT = a.blocks >= 8 && groups <= 1024 ? (int)((groups + 255) / 256) : groups <= 768 ? 1 : groups <= 1536 ? 2 : 3;
    else if (MT == 2) NT = groups <= 512 ? 1 : groups <= 1536 ? 2 : 3;
    const int most = (groups + NT - 1) / NT <= 256 ? 8 : 4, waves = a.blocks < most ? a.blocks : most;
    if constexpr (F32) {
        if (NT == 1) return w4_fwd_per<F32, 1, 1>(a, per, waves, s);
        if (NT == 2) return w4_fwd_per<F32, 1, 2>(a, per, waves, s);
        return NT == 3 ? w4_fwd_per<F32, 1, 3>(a, per, waves, s) : w4_fwd_per<F32, 1, 4>(a, per, waves, s);
    } else {
        if (MT == 1) return w4_fwd_per<F32, 1, 1>(a, per, waves, s);
        if (NT == 1) return w4_fwd_per<F32, 2, 1>(a, per, waves, s);
        return NT == 2 ? w4_fwd_per<F32, 2, 2>(a, per, waves, s) : w4_fwd_per<F32, 2, 3>(a, per, waves, s);
    }
}

static W4Args w4_args(const lq_w4_config* c, const uint8_t* packed, const void* in, int64_t ldin, void* out, int64_t ldout, int64_t M)
{
    const W4Shape sh = w4_shape(c);
    W4Args a{};
    a.codes = w4_codes(packed);
    a.scales = w4_scales(packed, sh);
    a.X = in;
    a.ldx = ldin;
    a.Y = out;
    a.ldy = ldout;
    a.M = M;
    a.N = c->N;
    a.K = c->K;
    a.tiles = sh.tiles;
    a.blocks = sh.blocks;
    return a;
}

hipError_t launch_w4_fwd(const lq_w4_config* c, const uint8_t* packed, const void* X, int64_t ldx, const float* bias, void* Y, int64_t ldy, int64_t M, hipStream_t s)
{
    W4Args a = w4_args(c, packed, X, ldx, Y, ldy, M);
    a.bias = bias;
    a.out_f32 = c->y_dtype == LQ_F32;
    return c->x_dtype == LQ_F32 ? w4_fwd_rows<true>(a, 128 / c->group, s) : w4_fwd_rows<false>(a, 128 / c->group, s);
}

// Parts of N of the gradient: a workgroup to a compute unit (us by their number, 16 x 2240 -> 13440 / 2 x 1152 -> 6912: 128 15.9 / 9.8, 256 12.8 / 9.0, 512 15.0 / 8.8, 1024 18.1 / 9.4)
static int w4_bwd_splits(const W4Shape& s, int64_t M)
{
    const int64_t others = (int64_t)s.blocks * ((M + 15) / 16), want = 256 / others, waves = w4_bwd_waves(s.per), most = ((s.tiles + 1) / 2 + waves - 1) / waves;
    if (most <= 2) return 1;  // (two steps of a wavefront cost less than a second launch: 3 x 359 -> 256 4.5 us for 6.2)
    return (int)(want < 1 ? 1 : want < most ? want : most);
}
size_t w4_work_bytes(const lq_w4_config* c, int64_t M)
{
    const W4Shape s = w4_shape(c);
    int64_t rows = 0;  // of all parts: the most that a batch of up to M needs, so that a workspace serves smaller ones
    for (int64_t m = 16; m - 16 < M; m += 16) {
        const int64_t n = m < M ? m : M, splits = w4_bwd_splits(s, n);
        if (splits == 1) break;  // (more rows have no more parts)
        if (splits * n > rows) rows = splits * n;
    }
    return align256((size_t)rows * c->K * 4);
}

template <bool F32, int PER>
static hipError_t w4_bwd_run(const W4Args& a, hipStream_t s)
{
    constexpr int waves = w4_bwd_waves(PER);
    hipLaunchKernelGGL((w4_bwd_kernel<F32, PER>), dim3(a.blocks, a.splits, (unsigned)((a.M + 15) / 16)), dim3(64 * waves), waves * 8192, s, a);
    return hipGetLastError();
}
template <bool F32>
static hipError_t w4_bwd_all(const W4Args& a, int per, hipStream_t s)
{
    return per == 1 ? w4_bwd_run<F32, 1>(a, s) : per == 2 ? w4_bwd_run<F32, 2>(a, s) : w4_bwd_run<F32, 4>(a, s);
}
hipError_t launch_w4_bwd(const lq_w4_config* c, const uint8_t* packed, const void* dY, int64_t lddy, void* dX, int64_t lddx, int64_t M, uint8_t* work, hipStream_t s)
{
    W4Args a = w4_args(c, packed, dY, lddy, dX, lddx, M);
    a.out_f32 = c->x_dtype == LQ_F32;
    a.splits = w4_bwd_splits(w4_shape(c), M);
    a.part = a.splits > 1 ? (float*)work : nullptr;
    const hipError_t e = c->y_dtype == LQ_F32 ? w4_bwd_all<true>(a, 128 / c->group, s) : w4_bwd_all<false>(a, 128 / c->group, s);
    if (e != hipSuccess || !a.part) return e;
    hipLaunchKernelGGL(w4_join, dim3((unsigned)((M * c->K + 63) / 64)), dim3(256), 0, s, a);
    return hipGetLastError();
}

}  // namespace lq
