// What lies between two blocks of a transformer, in one pass over the rows, and its gradient:
//     h' = alpha h + gate[s] post(y) w_post ;   x = pre(h') w_pre (1 + scale[s]) + shift[s]          (s: the row's sequence)
// Bound by memory in large batches.  A row belongs to one to sixteen wavefronts; a lane holds the same columns of every row it meets, so that the factors
//     a = w_pre (1 + scale[s]) ,  b = gate[s] w_post
// and, in the gradient, the sums over rows stay in registers for as long as the sequence lasts.  Means, variances (of differences from the mean) and everything
// else are held in fp32; outputs are rounded once.
#include "lq_internal.h"

namespace lq {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

template <int CTRL>
__device__ __forceinline__ float add_dpp(float v)
{
    return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float sum_wave(float v)  // over 64 lanes, in all of them
{
    v = add_dpp<0xB1>(v);   // quad_perm [1,0,3,2]
    v = add_dpp<0x4E>(v);   // quad_perm [2,3,0,1]
    v = add_dpp<0x141>(v);  // row_half_mirror
    v = add_dpp<0x140>(v);  // row_mirror
    const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(t[0]) + __uint_as_float(t[1]);
}

// Sums over the W wavefronts of a row.  Two sets of slots are used in turn, so that one barrier serves a sum: who writes a set again has passed the barrier of the
// other one, behind which nobody reads the first.
template <bool MULTI>
struct RowSum {
    float* slot;  // [2][wavefronts of the workgroup][2]
    int waves, first, wave, W, turn = 0;
    __device__ __forceinline__ void operator()(float& u, float& v)
    {
        u = sum_wave(u);
        v = sum_wave(v);
        if constexpr (MULTI) {
            float* p = slot + turn * waves * 2;
            turn ^= 1;
            if ((threadIdx.x & 63) == 0) p[wave * 2] = u, p[wave * 2 + 1] = v;
            __syncthreads();
            u = v = 0.0f;
            for (int w = 0; w < W; ++w) u += p[(first + w) * 2], v += p[(first + w) * 2 + 1];
        }
    }
    __device__ __forceinline__ void operator()(float& u)
    {
        float v = 0.0f;
        operator()(u, v);
    }
};

// N values at p: 1, or 8 in 16-byte accesses
template <int VEC>
__device__ __forceinline__ void read(const float* p, float (&v)[VEC])
{
    if constexpr (VEC == 1) {
        v[0] = *p;
    } else {
#pragma unroll
        for (int h = 0; h < VEC / 4; ++h) {
            const v4f t = ((const v4f*)p)[h];
#pragma unroll
            for (int i = 0; i < 4; ++i) v[4 * h + i] = t[i];
        }
    }
}
// ... of a row, as they lie in memory
template <typename T, int VEC>
struct Raw {
    T v;
    __device__ __forceinline__ void fetch(const T* p) { v = *p; }
    __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = (float)v; }
    static __device__ __forceinline__ void put(T* p, const float (&f)[1]) { *p = (T)f[0]; }
};
template <>
struct Raw<__bf16, 8> {
    v8bf v;
    __device__ __forceinline__ void fetch(const __bf16* p) { v = *(const v8bf*)p; }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)v[i];
    }
    static __device__ __forceinline__ void put(__bf16* p, const float (&f)[8])
    {
        v8bf t;
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = (__bf16)f[i];
        *(v8bf*)p = t;
    }
};
template <>
struct Raw<float, 8> {
    v4f v[2];
    __device__ __forceinline__ void fetch(const float* p) { v[0] = ((const v4f*)p)[0], v[1] = ((const v4f*)p)[1]; }
    __device__ __forceinline__ void get(float (&f)[8]) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = v[i / 4][i % 4];
    }
    static __device__ __forceinline__ void put(float* p, const float (&f)[8])
    {
        ((v4f*)p)[0] = v4f{f[0], f[1], f[2], f[3]};
        ((v4f*)p)[1] = v4f{f[4], f[5], f[6], f[7]};
    }
};

// The sequence of a row: how many of the S ends are at or before it, a wavefront looking at 64 of them at a time.  Bounded and inside [0, S] whatever they hold.
__device__ __forceinline__ int sequence_of(const int32_t* ends, int S, int row)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = S;
    while (n > 0) {
        const int step = (n + 63) >> 6, i = lane * step + step - 1;
        const int k = __popcll(__ballot(i < n && ends[lo + (i < n ? i : 0)] <= row));
        lo += k * step;
        n = min(step - 1, n - k * step);
    }
    return __builtin_amdgcn_readfirstlane(lo);
}
// Sequence s and its rows from `row` on: [row, end), cut to the limit; s < 0: rows of no sequence.
struct Segment {
    int s, end;
    __device__ __forceinline__ Segment(const BlockTensors& t, int row, int limit)
    {
        if (!t.offsets) {
            s = 0;
            end = limit;
            return;
        }
        const int start = t.offsets[0];
        if (row < start) {
            s = -1;
            end = min(start, limit);
            return;
        }
        s = sequence_of(t.offsets + 1, t.S, row);
        end = s < t.S ? min(t.offsets[s + 1], limit) : limit;
        if (s >= t.S) s = -1;
        if (end <= row) end = row + 1;  // (ends that do not rise)
    }
};

// What a lane knows of its NV vectors of columns
template <int VEC, int NV>
struct Columns {
    bool has[NV];
    int at[NV];
    __device__ __forceinline__ Columns(int dim, int lane, int lanes)
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            at[v] = (lane + v * lanes) * VEC;
            has[v] = at[v] < dim;
            at[v] = has[v] ? at[v] : 0;
        }
    }
};

// Normalises the values of a row in place; returns 1 / deviation.
template <int VEC, int NV, bool MULTI>
__device__ __forceinline__ float normalise(int kind, float (&x)[NV][VEC], const Columns<VEC, NV>& c, RowSum<MULTI>& sum, const BlockArgs& a)
{
    if (kind == LQ_NORM_LAYER) {
        float m = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i) m += c.has[v] ? x[v][i] : 0.0f;
        sum(m);
        m *= a.inv_dim;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[v][i] -= m;
    }
    float ss = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < VEC; ++i) t = fmaf(x[v][i], x[v][i], t);
        ss += c.has[v] ? t : 0.0f;
    }
    sum(ss);
    const float r = 1.0f / sqrtf(fmaf(ss, a.inv_dim, a.eps));
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[v][i] *= r;
    return r;
}

// a, b of the header, and shift, of sequence s
template <int VEC, int NV>
__device__ __forceinline__ void factors(const BlockTensors& t, const Columns<VEC, NV>& c, int s, float (&a)[NV][VEC], float (&b)[NV][VEC], float (*shift)[VEC])
{
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        float w[VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) a[v][i] = b[v][i] = 1.0f;
        if (t.scale.p) {
            read<VEC>(t.scale.p + s * t.scale.ld + c.at[v], w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) a[v][i] = 1.0f + w[i];
        }
        if (t.w_pre) {
            read<VEC>(t.w_pre + c.at[v], w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) a[v][i] *= w[i];
        }
        if (t.gate.p) read<VEC>(t.gate.p + s * t.gate.ld + c.at[v], b[v]);
        if (t.w_post) {
            read<VEC>(t.w_post + c.at[v], w);
#pragma unroll
            for (int i = 0; i < VEC; ++i) b[v][i] *= w[i];
        }
        if (shift) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) shift[v][i] = 0.0f;
            if (t.shift.p) read<VEC>(t.shift.p + s * t.shift.ld + c.at[v], shift[v]);
        }
    }
}

// Forward.  A group of W wavefronts takes `chunk` rows one after another, the next row already requested.  MULTI: the group is the workgroup; otherwise a workgroup
// has four of one wavefront.
template <typename TH, typename TY, int VEC, int NV, bool MULTI>
__global__ void __launch_bounds__(MULTI ? 1024 : 256) block_fwd_kernel(BlockArgs a)
{
    __shared__ float slots[MULTI ? 64 : 1];
    const BlockTensors& t = a.t;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const Columns<VEC, NV> c(a.dim, MULTI ? threadIdx.x : lane, MULTI ? blockDim.x : 64);
    const int group = MULTI ? blockIdx.x : blockIdx.x * 4 + wave;
    RowSum<MULTI> sum{slots, waves, 0, wave, waves};
    int row = group * a.chunk;
    const int limit = min(row + a.chunk, (int)a.M);
    if (row >= limit) return;
    Raw<TH, VEC> rh[NV];
    Raw<TY, VEC> ry[NV];
    auto request = [&](int m) {
        const TH* h = (const TH*)t.h + m * t.ldh;
        const TY* y = (const TY*)t.y + m * t.ldy;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            rh[v].fetch(h + c.at[v]);
            if (t.y) ry[v].fetch(y + c.at[v]);
        }
    };
    request(row);
    while (row < limit) {
        const Segment seg(t, row, limit);
        if (seg.s < 0) {
            row = seg.end;
            if (row < limit) request(row);
            continue;
        }
        float fa[NV][VEC], fb[NV][VEC], fs[NV][VEC];
        factors<VEC, NV>(t, c, seg.s, fa, fb, fs);
        for (; row < seg.end; ++row) {
            float h[NV][VEC], y[NV][VEC];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                rh[v].get(h[v]);
                if (t.y) ry[v].get(y[v]);
            }
            if (row + 1 < limit) request(row + 1);
            if (t.y) {
                if (a.post != LQ_NORM_NONE) normalise<VEC, NV, MULTI>(a.post, y, c, sum, a);
                TH* o = (TH*)t.ho + row * t.ldho;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) h[v][i] = fmaf(a.alpha, h[v][i], fb[v][i] * y[v][i]);
                    if (c.has[v]) Raw<TH, VEC>::put(o + c.at[v], h[v]);
                }
            }
            if (t.x) {
                if (a.pre != LQ_NORM_NONE) normalise<VEC, NV, MULTI>(a.pre, h, c, sum, a);
                TY* o = (TY*)t.x + row * t.ldx;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) h[v][i] = fmaf(h[v][i], fa[v][i], fs[v][i]);
                    if (c.has[v]) Raw<TY, VEC>::put(o + c.at[v], h[v]);
                }
            }
        }
    }
}

// Gradient.  With n = pre(h'), p = post(y) before their weights, r the reciprocal deviations:
//     G = dh' + r (dx a - mean(dx a) - n mean(dx a n)) ;  dh = alpha G ;  dy = r_y (G b - mean(G b) - p mean(G b p))       (the plain means with LQ_NORM_LAYER only)
// and the sums over the rows of a sequence of dx, dx n and G p, from which block_sums makes the gradients of modulation and weights.  A workgroup takes a chunk of rows,
// its groups of W wavefronts in turn; at the end of a sequence or of the chunk the groups' sums are joined in the LDS and written to place chunk + s of the parts,
// which no other pair of chunk and sequence has (both rise from one pair to the next).
template <typename TH, typename TY, int VEC, int NV, bool MULTI, int THREADS>
__global__ void __launch_bounds__(THREADS) block_bwd_kernel(BlockArgs a)
{
    extern __shared__ float joined[];  // [groups][dim]
    __shared__ float slots[64];
    const BlockTensors& t = a.t;
    const int wave = threadIdx.x >> 6, waves = blockDim.x >> 6, W = a.waves, group = wave / W, groups = waves / W;
    const Columns<VEC, NV> c(a.dim, threadIdx.x - group * W * 64, W * 64);
    RowSum<MULTI> sum{slots, waves, group * W, wave, W};
    int first = blockIdx.x * a.chunk;
    const int limit = min(first + a.chunk, (int)a.M);
    const bool has_dx = t.dx, has_y = t.y, has_dho = t.dho;
    Raw<TH, VEC> rh[NV], rg[NV];
    Raw<TY, VEC> ry[NV], rx[NV];
    auto request = [&](int m) {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            if (has_dx) {
                rh[v].fetch((const TH*)t.h + m * t.ldh + c.at[v]);
                rx[v].fetch((const TY*)t.dx + m * t.lddx + c.at[v]);
            }
            if (has_y) ry[v].fetch((const TY*)t.y + m * t.ldy + c.at[v]);
            if (has_dho) rg[v].fetch((const TH*)t.dho + m * t.lddho + c.at[v]);
        }
    };
    while (first < limit) {
        const Segment seg(t, first, limit);
        if (seg.s < 0) {
            first = seg.end;
            continue;
        }
        float fa[NV][VEC], fb[NV][VEC], s1[NV][VEC], s2[NV][VEC], s3[NV][VEC];
        if (first + group < seg.end) request(first + group);
        factors<VEC, NV>(t, c, seg.s, fa, fb, nullptr);
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s1[v][i] = s2[v][i] = s3[v][i] = 0.0f;
        for (int base = first; base < seg.end; base += groups) {
            const int row = base + group;
            const bool on = row < seg.end;  // (of a row: all its wavefronts)
            if (!MULTI && !on) break;
            float n[NV][VEC], p[NV][VEC], dx[NV][VEC], g[NV][VEC];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) n[v][i] = p[v][i] = dx[v][i] = g[v][i] = 0.0f;
                if (on) {
                    if (has_dx) rh[v].get(n[v]), rx[v].get(dx[v]);
                    if (has_y) ry[v].get(p[v]);
                    if (has_dho) rg[v].get(g[v]);
                }
            }
            if (row + groups < seg.end) request(row + groups);
            if (has_dx) {
                float r = 1.0f;
                if (a.pre != LQ_NORM_NONE) r = normalise<VEC, NV, MULTI>(a.pre, n, c, sum, a);
                float dn[NV][VEC], u = 0.0f, w = 0.0f;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float tu = 0.0f, tw = 0.0f;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        s1[v][i] += dx[v][i];
                        s2[v][i] = fmaf(dx[v][i], n[v][i], s2[v][i]);
                        dn[v][i] = dx[v][i] * fa[v][i];
                        tu = fmaf(dn[v][i], n[v][i], tu);
                        tw += dn[v][i];
                    }
                    u += c.has[v] ? tu : 0.0f;
                    w += c.has[v] ? tw : 0.0f;
                }
                if (a.pre != LQ_NORM_NONE) {
                    sum(u, w);
                    u *= a.inv_dim;
                    w = a.pre == LQ_NORM_LAYER ? w * a.inv_dim : 0.0f;
                } else {
                    u = w = 0.0f;
                }
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) g[v][i] = fmaf(r, fmaf(-n[v][i], u, dn[v][i] - w), g[v][i]);
            }
            if (t.dh && on) {
                TH* o = (TH*)t.dh + row * t.lddh;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float d[VEC];
#pragma unroll
                    for (int i = 0; i < VEC; ++i) d[i] = a.alpha * g[v][i];
                    if (c.has[v]) Raw<TH, VEC>::put(o + c.at[v], d);
                }
            }
            if (has_y) {
                float r = 1.0f;
                if (a.post != LQ_NORM_NONE) r = normalise<VEC, NV, MULTI>(a.post, p, c, sum, a);
                float u = 0.0f, w = 0.0f;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float tu = 0.0f, tw = 0.0f;
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        s3[v][i] = fmaf(g[v][i], p[v][i], s3[v][i]);
                        g[v][i] *= fb[v][i];
                        tu = fmaf(g[v][i], p[v][i], tu);
                        tw += g[v][i];
                    }
                    u += c.has[v] ? tu : 0.0f;
                    w += c.has[v] ? tw : 0.0f;
                }
                if (a.post != LQ_NORM_NONE) {
                    sum(u, w);
                    u *= a.inv_dim;
                    w = a.post == LQ_NORM_LAYER ? w * a.inv_dim : 0.0f;
                } else {
                    u = w = 0.0f;
                }
                if (t.dy && on) {
                    TY* o = (TY*)t.dy + row * t.lddy;
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
                        float d[VEC];
#pragma unroll
                        for (int i = 0; i < VEC; ++i) d[i] = r * fmaf(-p[v][i], u, g[v][i] - w);
                        if (c.has[v]) Raw<TY, VEC>::put(o + c.at[v], d);
                    }
                }
            }
        }
        if (a.part) {
            float* out = a.part + (size_t)(blockIdx.x + seg.s) * 3 * a.dim;
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                float* mine = groups == 1 ? out + k * a.dim : joined + group * a.dim;
#pragma unroll
                for (int v = 0; v < NV; ++v)
                    if (c.has[v])
#pragma unroll
                        for (int i = 0; i < VEC; ++i) mine[c.at[v] + i] = k == 0 ? s1[v][i] : k == 1 ? s2[v][i] : s3[v][i];
                if (groups == 1) continue;
                __syncthreads();
                for (int o = threadIdx.x; o < a.dim; o += blockDim.x) {
                    float y = joined[o];
                    for (int w = 1; w < groups; ++w) y += joined[w * a.dim + o];
                    out[k * a.dim + o] = y;
                }
                __syncthreads();
            }
        }
        first = seg.end;
    }
}

// Sums over a sequence's parts in a fixed order; 64 columns of one of the three sums to a workgroup, its wavefronts take parts in turn and are joined in a tree.
//     dshift = sum dx ;  dscale = w_pre sum dx n ;  dgate = w_post sum G p
// raw: the last two without the weights, for those of the weights.
__global__ void __launch_bounds__(1024) block_sums(BlockArgs a, float* raw)
{
    __shared__ float sh[16][64];
    const BlockTensors& t = a.t;
    const int k = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, col = blockIdx.x * 64 + lane;
    for (int s = blockIdx.z; s < t.S; s += gridDim.z) {
        int begin = 0, end = (int)a.M;
        if (t.offsets) {
            begin = max(t.offsets[s], 0);
            end = min(t.offsets[s + 1], (int)a.M);
        }
        const int c0 = begin / a.chunk, c1 = begin < end ? (end - 1) / a.chunk + 1 : c0;
        float y = 0.0f;
        if (col < a.dim) {
            const float* p = a.part + (size_t)s * 3 * a.dim + k * a.dim + col;
#pragma unroll 8
            for (int i = c0 + wave; i < c1; i += waves) y += p[(size_t)i * 3 * a.dim];
        }
        sh[wave][lane] = y;
        __syncthreads();
        for (int half = waves / 2; half > 0; half /= 2) {
            if (wave < half) sh[wave][lane] += sh[wave + half][lane];
            __syncthreads();
        }
        if (wave == 0 && col < a.dim) {
            y = sh[0][lane];
            const lq_mod_out& o = k == 0 ? t.dshift : k == 1 ? t.dscale : t.dgate;
            const float* w = k == 0 ? nullptr : k == 1 ? t.w_pre : t.w_post;
            if (o.p) o.p[s * o.ld + col] = w ? y * w[col] : y;
            if (raw && k) raw[((size_t)s * 2 + k - 1) * a.dim + col] = y;
        }
        __syncthreads();
    }
}
// dw_pre = sum over sequences of (1 + scale) sum dx n ;  dw_post = sum of gate sum G p
__global__ void __launch_bounds__(1024) block_weight_sums(BlockArgs a, const float* raw)
{
    __shared__ float sh[16][64];
    const BlockTensors& t = a.t;
    const int k = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
    const lq_mod& f = k == 0 ? t.scale : t.gate;
    float* out = k == 0 ? t.dw_pre : t.dw_post;
    float y = 0.0f;
    if (col < a.dim && out)
#pragma unroll 4
        for (int s = wave; s < t.S; s += 16) {
            const float u = raw[((size_t)s * 2 + k) * a.dim + col];
            y += f.p ? u * (k == 0 ? 1.0f + f.p[s * f.ld + col] : f.p[s * f.ld + col]) : u;
        }
    sh[wave][lane] = y;
    __syncthreads();
    for (int half = 8; half > 0; half /= 2) {
        if (wave < half) sh[wave][lane] += sh[wave + half][lane];
        __syncthreads();
    }
    if (wave == 0 && col < a.dim && out) out[col] = sh[0][lane];
}

// ---- host ---------------------------------------------------------------------------------------

// Vectors of columns to a lane, and wavefronts to a row
struct BlockShape {
    int vec, NV, W;
};
static BlockShape block_shape(int dim, bool wide, int most)
{
    if (wide) {
        const int vectors = dim / 8, W = (vectors + 64 * most - 1) / (64 * most);
        return {8, (vectors + 64 * W - 1) / (64 * W), W};
    }
    const int W = (dim + 1023) / 1024;
    return {1, dim <= 256 ? 4 : 16, W};
}
static bool fits(const void* p, int64_t ld, int64_t rows, int elem) { return (uintptr_t)p % 16 == 0 && (rows < 2 || ld * elem % 16 == 0); }
static bool block_wide(const lq_block_config* c, const BlockTensors& t, int64_t M)
{
    const int he = c->h_dtype == LQ_F32 ? 4 : 2, ye = c->y_dtype == LQ_F32 ? 4 : 2;
    return c->dim % 8 == 0 && fits(t.h, t.ldh, M, he) && fits(t.y, t.ldy, M, ye) && fits(t.ho, t.ldho, M, he) && fits(t.x, t.ldx, M, ye) && fits(t.dho, t.lddho, M, he) &&
           fits(t.dx, t.lddx, M, ye) && fits(t.dh, t.lddh, M, he) && fits(t.dy, t.lddy, M, ye) && fits(t.gate.p, t.gate.ld, t.S, 4) &&
           fits(t.scale.p, t.scale.ld, t.S, 4) && fits(t.shift.p, t.shift.ld, t.S, 4) && fits(t.w_pre, 0, 1, 4) && fits(t.w_post, 0, 1, 4);
}
static BlockArgs block_args(const lq_block_config* c, const BlockTensors& t, int64_t M)
{
    BlockArgs a{};
    a.t = t;
    a.M = M;
    a.dim = c->dim;
    a.post = c->post;
    a.pre = c->pre;
    a.eps = c->eps;
    a.inv_dim = 1.0f / (float)c->dim;
    a.alpha = t.y ? c->res_scale : 1.0f;
    return a;
}

template <typename TH, typename TY, int VEC, int NV>
static void block_fwd_run(const BlockArgs& a, int W, hipStream_t s)
{
    const int64_t groups = (a.M + a.chunk - 1) / a.chunk;
    if (W > 1) hipLaunchKernelGGL((block_fwd_kernel<TH, TY, VEC, NV, true>), dim3((unsigned)groups), dim3(64 * W), 0, s, a);
    else hipLaunchKernelGGL((block_fwd_kernel<TH, TY, VEC, NV, false>), dim3((unsigned)((groups + 3) / 4)), dim3(256), 0, s, a);
}
template <typename TH, typename TY>
static void block_fwd_types(const BlockArgs& a, const BlockShape& sh, hipStream_t s)
{
    if (sh.vec == 8) {
        if (sh.NV == 1) block_fwd_run<TH, TY, 8, 1>(a, sh.W, s);
        else if (sh.NV == 2) block_fwd_run<TH, TY, 8, 2>(a, sh.W, s);
        else block_fwd_run<TH, TY, 8, 3>(a, sh.W, s);
    } else {
        if (sh.NV == 4) block_fwd_run<TH, TY, 1, 4>(a, sh.W, s);
        else block_fwd_run<TH, TY, 1, 16>(a, sh.W, s);
    }
}
hipError_t launch_block_fwd(const lq_block_config* c, const BlockTensors& t, int64_t M, hipStream_t s)
{
    const BlockShape sh = block_shape(c->dim, block_wide(c, t, M), 3);
    BlockArgs a = block_args(c, t, M);
    // rows one after another while every SIMD has two wavefronts
    const int64_t chunk = M * sh.W / 2048;
    a.chunk = (int)(chunk < 1 ? 1 : chunk > 16 ? 16 : chunk);
    if (c->h_dtype == LQ_BF16) block_fwd_types<__bf16, __bf16>(a, sh, s);
    else if (c->y_dtype == LQ_BF16) block_fwd_types<float, __bf16>(a, sh, s);
    else block_fwd_types<float, float>(a, sh, s);
    return hipGetLastError();
}

// Rows of a workgroup of the gradient, each of which leaves parts of the sums
static int block_bwd_chunk(int64_t M)
{
    const int64_t t = (M + 511) / 512;
    return (int)(t < 8 ? 8 : t);
}
static size_t block_parts(const lq_block_config* c, int64_t M, int64_t S)
{
    const int chunk = block_bwd_chunk(M);
    return (size_t)((M + chunk - 1) / chunk + S) * 3 * c->dim;
}
size_t block_work_bytes(const lq_block_config* c, int64_t M, int64_t S)
{
    return align256(block_parts(c, M, S) * 4) + align256((size_t)S * 2 * c->dim * 4);
}

template <typename TH, typename TY, int VEC, int NV>
static void block_bwd_run(const BlockArgs& a, hipStream_t s)
{
    const int W = a.waves, groups = W > 4 ? 1 : 8 / W;
    const dim3 grid((unsigned)((a.M + a.chunk - 1) / a.chunk)), block(64 * W * groups);
    const size_t lds = groups > 1 ? (size_t)groups * a.dim * 4 : 0;
    if (W == 1) hipLaunchKernelGGL((block_bwd_kernel<TH, TY, VEC, NV, false, 512>), grid, block, lds, s, a);
    else if (W <= 8) hipLaunchKernelGGL((block_bwd_kernel<TH, TY, VEC, NV, true, 512>), grid, block, lds, s, a);
    else hipLaunchKernelGGL((block_bwd_kernel<TH, TY, VEC, NV, true, 1024>), grid, block, lds, s, a);
}
template <typename TH, typename TY>
static void block_bwd_types(const BlockArgs& a, const BlockShape& sh, hipStream_t s)
{
    if (sh.vec == 8) {
        if (sh.NV == 1) block_bwd_run<TH, TY, 8, 1>(a, s);
        else block_bwd_run<TH, TY, 8, 2>(a, s);
    } else {
        if (sh.NV == 4) block_bwd_run<TH, TY, 1, 4>(a, s);
        else block_bwd_run<TH, TY, 1, 16>(a, s);
    }
}
hipError_t launch_block_bwd(const lq_block_config* c, const BlockTensors& t, int64_t M, uint8_t* work, hipStream_t s)
{
    const bool sums = t.dgate.p || t.dscale.p || t.dshift.p || t.dw_pre || t.dw_post, weights = t.dw_pre || t.dw_post;
    BlockArgs a = block_args(c, t, M);
    a.chunk = block_bwd_chunk(M);
    a.part = sums ? (float*)work : nullptr;
    hipError_t e = hipSuccess;
    if (M > 0) {
        const BlockShape sh = block_shape(c->dim, block_wide(c, t, M), 2);
        a.waves = sh.W;
        if (c->h_dtype == LQ_BF16) block_bwd_types<__bf16, __bf16>(a, sh, s);
        else if (c->y_dtype == LQ_BF16) block_bwd_types<float, __bf16>(a, sh, s);
        else block_bwd_types<float, float>(a, sh, s);
        e = hipGetLastError();
    }
    if (e != hipSuccess || !sums) return e;
    float* raw = weights ? (float*)(work + align256(block_parts(c, M, t.S) * 4)) : nullptr;
    const int64_t each = (M + a.chunk - 1) / a.chunk / t.S;  // parts of a sequence
    const unsigned cols = (unsigned)((c->dim + 63) / 64);
    hipLaunchKernelGGL(block_sums, dim3(cols, 3, (unsigned)(t.S < 4096 ? t.S : 4096)), dim3(each >= 32 ? 1024 : 256), 0, s, a, raw);
    e = hipGetLastError();
    if (e != hipSuccess || !weights) return e;
    hipLaunchKernelGGL(block_weight_sums, dim3(cols, 2), dim3(1024), 0, s, a, (const float*)raw);
    return hipGetLastError();
}

}  // namespace lq
