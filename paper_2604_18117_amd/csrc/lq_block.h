// What lies between two blocks of a transformer, in one pass over the rows, and its gradient:
//     h' = alpha h + gate[s] post(y) w_post ;   x = pre(h') w_pre (1 + scale[s]) + shift[s]          (s: the row's sequence)
// Bound by memory in large batches.  A row belongs to one to sixteen wavefronts; a lane holds the same columns of every row it meets, so that the factors
//     a = w_pre (1 + scale[s]) ,  b = gate[s] w_post
// and, in the gradient, the sums over rows stay in registers for as long as the sequence lasts.  Means, variances (of differences from the mean) and everything
// else are held in fp32; outputs are rounded once.
#pragma once
#include <utility>

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
        __builtin_amdgcn_sched_barrier(0);  // (what follows a sum is not begun before it: its values would be held beside all others)
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

// VEC consecutive values in memory.  ANY: of any alignment, and rows may end among them.
template <typename T, int VEC, bool ANY>
struct Raw {
    typedef T Value __attribute__((ext_vector_type(VEC)));
    typedef Value Access __attribute__((aligned(ANY ? sizeof(T) : sizeof(T) * VEC > 16 ? 16 : sizeof(T) * VEC)));
    Value v;
    __device__ __forceinline__ void fetch(const T* p) { v = *(const Access*)p; }
    // Where the row of `dim` values may end before or among them: zeros from there on.  ANY: the row's last VEC values are read and moved to their places.
    __device__ __forceinline__ void fetch_end(const T* row, int at, int dim)
    {
        if constexpr (!ANY) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = (T)0.0f;
            if (at < dim) fetch(row + at);
        } else if (dim < VEC) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = at + i < dim ? row[at + i] : (T)0.0f;
        } else {
            const int first = min(at, dim - VEC), past = min(at - first, VEC);
            fetch(row + first);
#pragma unroll
            for (int step = VEC; step >= 1; step /= 2)
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[i] = past & step ? (i + step < VEC ? v[i + step < VEC ? i + step : 0] : (T)0.0f) : v[i];
        }
    }
    __device__ __forceinline__ void get(float (&f)[VEC]) const
    {
#pragma unroll
        for (int i = 0; i < VEC; ++i) f[i] = (float)v[i];
    }
    static __device__ __forceinline__ void put(T* p, const float (&f)[VEC])
    {
        Value t;
#pragma unroll
        for (int i = 0; i < VEC; ++i) t[i] = (T)f[i];
        *(Access*)p = t;
    }
    static __device__ __forceinline__ void put_end(T* row, int at, int dim, const float (&f)[VEC])
    {
        if (at + (ANY ? VEC : 1) <= dim) {
            put(row + at, f);
        } else if constexpr (ANY) {
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (at + i < dim) row[at + i] = (T)f[i];
        }
    }
};
template <int VEC, bool ANY>
__device__ __forceinline__ void read(const float* row, int at, int dim, float (&f)[VEC], bool whole = false)  // whole: the row does not end before or among them
{
    Raw<float, VEC, ANY> r;
    if (whole) r.fetch(row + at);
    else r.fetch_end(row, at, dim);
    r.get(f);
}

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
// The sequences as a wavefront knows them: up to 64 ends lie in its lanes, so that they cost one round trip, whose load is the first of all.
struct Sequences {
    const int32_t* offsets;
    int S, start, mine;  // first row of the first; lane's end
    __device__ __forceinline__ Sequences(const BlockTensors& t) : offsets(t.offsets), S(t.S), start(0), mine(0)
    {
        const int lane = threadIdx.x & 63;
        if (!offsets) return;
        start = offsets[0];
        if (S <= 64) mine = offsets[1 + min(lane, S - 1)];
    }
    // the sequence of `row` (-1: none) and the end of its rows from there on, not past `limit`
    __device__ __forceinline__ int find(int row, int limit, int& end) const
    {
        end = limit;
        if (!offsets) return 0;
        const int first = __builtin_amdgcn_readfirstlane(start);
        if (row < first) {
            end = min(first, limit);
            return -1;
        }
        int s, e;
        if (S <= 64) {
            s = __popcll(__ballot((int)(threadIdx.x & 63) < S && mine <= row));
            e = __builtin_amdgcn_readlane(mine, s < 63 ? s : 63);
        } else {
            s = sequence_of(offsets + 1, S, row);
            e = s < S ? __builtin_amdgcn_readfirstlane(offsets[1 + s]) : 0;
        }
        if (s >= S) return -1;
        end = min(e, limit);
        if (end <= row) end = row + 1;  // (ends that do not rise)
        return s;
    }
};

// A lane's NV vectors of columns: the first at `at`, each `step` values from the one before, so that with the row's address in scalar registers one offset serves all.  All but the last
// are there in every lane; a last one past the row's end is zero and left out of sums.
template <int VEC, int NV, bool ANY>
struct Columns {
    int at, step, dim;
    __device__ __forceinline__ Columns(int dim_, int lane, int lanes) : at(lane * VEC), step(lanes * VEC), dim(dim_) {}
    __device__ __forceinline__ int have(int v) const { return v < NV - 1 ? VEC : dim - (at + v * step); }
    __device__ __forceinline__ float counted(int v, float sum) const { return v < NV - 1 || have(v) > 0 ? sum : 0.0f; }
    template <typename T>
    __device__ __forceinline__ void fetch(const T* row, Raw<T, VEC, ANY> (&r)[NV]) const
    {
#pragma unroll
        for (int v = 0; v < NV - 1; ++v) r[v].fetch(row + v * step + at);
        r[NV - 1].fetch_end(row, (NV - 1) * step + at, dim);
    }
    template <typename T>
    __device__ __forceinline__ void put(T* row, int v, const float (&f)[VEC]) const
    {
        if (v < NV - 1) Raw<T, VEC, ANY>::put(row + v * step + at, f);
        else Raw<T, VEC, ANY>::put_end(row, v * step + at, dim, f);
    }
};

// Normalises the values of a row in place; returns 1 / deviation.
template <int VEC, int NV, bool ANY, bool MULTI>
__device__ __forceinline__ float normalise(int kind, float (&x)[NV][VEC], const Columns<VEC, NV, ANY>& c, RowSum<MULTI>& sum, const BlockArgs& a)
{
    if (kind == LQ_NORM_LAYER) {
        float m = 0.0f;
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            float t = 0.0f;
#pragma unroll
            for (int i = 0; i < VEC; ++i) t += x[v][i];
            m += c.counted(v, t);
        }
        sum(m);
        m *= a.inv_dim;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i) x[v][i] = ANY && i >= c.have(v) ? 0.0f : x[v][i] - m;
    }
    float ss = 0.0f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < VEC; ++i) t = fmaf(x[v][i], x[v][i], t);
        ss += c.counted(v, t);
    }
    sum(ss);
    const float r = 1.0f / sqrtf(fmaf(ss, a.inv_dim, a.eps));
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int i = 0; i < VEC; ++i) x[v][i] *= r;
    return r;
}

// a, b of the header, and shift, of sequence s, at a column
template <int VEC, bool ANY>
__device__ __forceinline__ void factor_a(const BlockTensors& t, int at, int dim, int s, float (&a)[VEC], bool whole = false)
{
    float w[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) a[i] = 1.0f;
    if (t.scale.p) {
        read<VEC, ANY>(t.scale.p + s * t.scale.ld, at, dim, w, whole);
#pragma unroll
        for (int i = 0; i < VEC; ++i) a[i] = 1.0f + w[i];
    }
    if (t.w_pre) {
        read<VEC, ANY>(t.w_pre, at, dim, w, whole);
#pragma unroll
        for (int i = 0; i < VEC; ++i) a[i] *= w[i];
    }
}
template <int VEC, bool ANY>
__device__ __forceinline__ void factor_b(const BlockTensors& t, int at, int dim, int s, float (&b)[VEC], bool whole = false)
{
    float w[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) b[i] = 1.0f;
    if (t.gate.p) read<VEC, ANY>(t.gate.p + s * t.gate.ld, at, dim, b, whole);
    if (t.w_post) {
        read<VEC, ANY>(t.w_post, at, dim, w, whole);
#pragma unroll
        for (int i = 0; i < VEC; ++i) b[i] *= w[i];
    }
}

// ---- host ---------------------------------------------------------------------------------------

// Vectors of four columns to a lane (up to five), and wavefronts to a row: the fewest; `wide` (forward, small batches): one more where lanes would be idle otherwise (us, 16384 rows of 2240, fp32 stream and both norms / bf16
// and one: two wavefronts with five vectors, 12 % of them past the end, 102.8 / 67.6, three with three 93.8 / 63.9; 8192 rows of 4608: four with five 66.0, six with three 70.7;
// gradient of 8192 rows of 2240: two with five 67.0, three with three 73.7, of 500 24.0 / 21.2)
struct BlockShape {
    bool any;
    int NV, W;
};
static inline BlockShape block_shape(int dim, bool any, bool wide)
{
    const int vectors = (dim + 3) / 4;
    BlockShape s{any, 0, (vectors + 319) / 320};
    if (s.W > 8) s.W = 16;  // (1024 threads have 128 registers each, of which every vector takes some 30)
    s.NV = (vectors + 64 * s.W - 1) / (64 * s.W);
    const int more = (vectors + 64 * (s.W + 1) - 1) / (64 * (s.W + 1));
    if (wide && s.W > 1 && s.W < 8 && vectors * 10 < s.NV * 64 * s.W * 9 && more >= 3 && more * (s.W + 1) < s.NV * s.W) s.NV = more, ++s.W;
    return s;
}
static inline bool fits(const void* p, int64_t ld, int64_t rows, int bytes, int elem) { return (uintptr_t)p % bytes == 0 && (rows < 2 || ld * elem % bytes == 0); }
// Whether every row can be read four values at a time
static inline bool block_fours(const lq_block_config* c, const BlockTensors& t, int64_t M)
{
    const int he = c->h_dtype == LQ_F32 ? 4 : 2, ye = c->y_dtype == LQ_F32 ? 4 : 2;
    bool ok = c->dim % 4 == 0;
    for (const auto& r : {std::pair<const void*, int64_t>(t.h, t.ldh), {t.ho, t.ldho}, {t.dho, t.lddho}, {t.dh, t.lddh}}) ok = ok && fits(r.first, r.second, M, 4 * he, he);
    for (const auto& r : {std::pair<const void*, int64_t>(t.y, t.ldy), {t.x, t.ldx}, {t.dx, t.lddx}, {t.dy, t.lddy}}) ok = ok && fits(r.first, r.second, M, 4 * ye, ye);
    for (const lq_mod& m : {t.gate, t.scale, t.shift}) ok = ok && fits(m.p, m.ld, t.S, 16, 4);
    return ok && (uintptr_t)t.w_pre % 16 == 0 && (uintptr_t)t.w_post % 16 == 0;
}
static inline BlockArgs block_args(const lq_block_config* c, const BlockTensors& t, int64_t M)
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

}  // namespace lq
