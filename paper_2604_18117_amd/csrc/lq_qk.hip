// Norm of queries and keys for each head with the rotation by positions of several axes, and its gradient, one pass over the heads each:
//     n = x rsqrt(mean x^2 + eps) w ;  (n_a, n_b) -> (n_a cos t - n_b sin t, n_a sin t + n_b cos t) ,  t = pos[axis] inv_freq
// Bound by memory in large batches: two bytes moved per byte of heads, three in the gradient.  A workgroup takes a few tokens; it computes their cosines and
// sines once, into the LDS, for all heads.  A head belongs to a group of 2^k lanes; a lane holds the same V pairs of every head it meets, so that
// its weights, and its sums of dw, stay in registers.  Sums, angles and the rotation are in fp32 (whole turns of the angles in 64 bits); outputs are rounded once.
#include "lq_internal.h"

namespace lq {

typedef float v4f __attribute__((ext_vector_type(4)));

struct QkArgs {
    QkTensors t;
    int64_t M;
    int heads[2], dim, pairs, axes;
    int axis_end[4];  // first pair past each axis
    int lanes_log2;   // lanes of a head
    int tokens;       // of a workgroup at a time
    int turn_k[2], turn_h[2];  // tokens and heads from one turn of a lane to its next
    unsigned magic[2], half_magic;  // 2^32 / heads, 2^32 / (dim / 2), rounded up: quotients of small numbers
    float eps, inv_dim;
    float* part;      // [workgroup][2][dim] sums of dw
};

__device__ __forceinline__ int quotient(int i, unsigned magic) { return magic ? (int)__umulhi((unsigned)i, magic) : i; }

// cos and sin of the angle of pair p (ones and zeros for the values that are not rotated).  The product of two fp32 numbers is exact in 64 bits; whole
// turns are taken off there, what is left fits 32.
__device__ __forceinline__ float2 turn(const QkArgs& a, unsigned row, int p)
{
    float2 v = make_float2(1.0f, 0.0f);
    if (p < a.pairs) {
        const int axis = (p >= a.axis_end[0]) + (p >= a.axis_end[1]) + (p >= a.axis_end[2]);
        const double turns = (double)a.t.pos[(size_t)row * a.axes + axis] * (double)a.t.inv_freq[p] * 0.15915494309189533577;
        const float r = (float)(turns - rint(turns));
        sincospif(2.0f * r, &v.y, &v.x);
    }
    return v;
}
// row of pos of token m0 + k; first = m0 % pos_rows
__device__ __forceinline__ unsigned pos_row(const QkArgs& a, unsigned first, int k)
{
    const unsigned row = first + k;
    return row < (unsigned)a.t.pos_rows ? row : row % (unsigned)a.t.pos_rows;
}
__device__ __forceinline__ unsigned first_pos(const QkArgs& a, int m0) { return a.pairs ? (unsigned)m0 % (unsigned)a.t.pos_rows : 0u; }

template <int CTRL>
__device__ __forceinline__ float add_dpp(float v)
{
    return v + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), CTRL, 0xF, 0xF, true));
}
// sum over groups of 2^k lanes, in all of them
__device__ __forceinline__ float sum_lanes(float v, int k)
{
    if (k > 0) v = add_dpp<0xB1>(v);   // quad_perm [1,0,3,2]
    if (k > 1) v = add_dpp<0x4E>(v);   // quad_perm [2,3,0,1]
    if (k > 2) v = add_dpp<0x141>(v);  // row_half_mirror
    if (k > 3) v = add_dpp<0x140>(v);  // row_mirror
    if (k > 4) v += __shfl_xor(v, 16);
    if (k > 5) v += __shfl_xor(v, 32);
    return v;
}

// Each of N values: the sum over the lanes of a wavefront with the same place in their group of 2^k, valid in the first group.  (Values inside, steps
// outside: a uniform branch per step, not per step and value.)
template <int N>
__device__ __forceinline__ void sum_groups(float (&v)[N], int k)
{
#define STEP(K, EXPR) \
    if (k < K) { \
        _Pragma("unroll") for (int i = 0; i < N; ++i) v[i] = EXPR; \
    }
    STEP(1, add_dpp<0xB1>(v[i]))
    STEP(2, add_dpp<0x4E>(v[i]))
    STEP(3, add_dpp<0x124>(v[i]))  // row_ror:4
    STEP(4, add_dpp<0x128>(v[i]))  // row_ror:8
#undef STEP
    if (k < 5) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i]), false, false);
            v[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
        }
    }
    if (k < 6) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v[i]), __float_as_uint(v[i]), false, false);
            v[i] = __uint_as_float(s[0]) + __uint_as_float(s[1]);
        }
    }
}

// What an access of V pairs is aligned to, in bytes: the whole of it up to 16, and nothing but its values where V = 1 (of adjacent pairs two at once, which any
// strides may put anywhere).  The host's choice of V keeps to it.
constexpr int access_align(int V, bool half, int elem)
{
    const int bytes = V == 1 ? elem : half ? V * elem : 2 * V * elem;
    return bytes > 16 ? 16 : bytes;
}
// N consecutive values
template <typename T, int N>
struct Vec {
    typedef T type __attribute__((ext_vector_type(N)));
};
template <typename T>
struct Vec<T, 1> {
    typedef T type;
};
template <int V, typename VT>
__device__ __forceinline__ float part(const VT& v, int j)
{
    if constexpr (V == 1) return (float)v;
    else return (float)v[j];
}

// The members a, b of V pairs of a head as they lie in memory: two vectors of V (halves), or one of 2 V
template <typename T, int V, bool HALF>
struct Raw {
    typedef typename Vec<T, HALF ? V : 2 * V>::type Value;
    typedef Value Access __attribute__((aligned(access_align(V, HALF, sizeof(T)))));
    Value v[HALF ? 2 : 1];
    __device__ __forceinline__ void fetch(const T* x, int oa, int ob)
    {
        v[0] = *(const Access*)(x + oa);
        if constexpr (HALF) v[1] = *(const Access*)(x + ob);
    }
    __device__ __forceinline__ void get(float (&a)[V], float (&b)[V]) const
    {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if constexpr (HALF) a[j] = part<V>(v[0], j), b[j] = part<V>(v[1], j);
            else a[j] = part<2 * V>(v[0], 2 * j), b[j] = part<2 * V>(v[0], 2 * j + 1);
        }
    }
};
template <typename T, int V, bool HALF>
__device__ __forceinline__ void put(T* x, int oa, int ob, const float (&a)[V], const float (&b)[V])
{
    if constexpr (HALF && V == 1) {
        x[oa] = (T)a[0];
        x[ob] = (T)b[0];
    } else if constexpr (HALF) {
        typename Raw<T, V, HALF>::Value va, vb;
#pragma unroll
        for (int j = 0; j < V; ++j) va[j] = (T)a[j], vb[j] = (T)b[j];
        *(typename Raw<T, V, HALF>::Access*)(x + oa) = va;
        *(typename Raw<T, V, HALF>::Access*)(x + ob) = vb;
    } else {
        typename Raw<T, V, HALF>::Value w;
#pragma unroll
        for (int j = 0; j < V; ++j) w[2 * j] = (T)a[j], w[2 * j + 1] = (T)b[j];
        *(typename Raw<T, V, HALF>::Access*)(x + oa) = w;
    }
}

// A lane's way through the heads of a chunk of tokens: head h of token k, in the same steps at every turn, so that a turn costs no division and
// no product.  at: offset of the head in a tensor, or of the token's cosines in their table.
struct Walk {
    int h;
    int64_t at, turn, wrap;  // of a turn; what is added where the next token begins
    __device__ __forceinline__ Walk(int h0, int k0, int dh, int dk, int H, int64_t ld, int64_t hs)
        : h(h0), at(k0 * ld + h0 * hs), turn(dk * ld + dh * hs), wrap(ld - H * hs)
    {
    }
    __device__ __forceinline__ void next(int dh, int H)
    {
        h += dh;
        at += turn;
        if (h >= H) h -= H, at += wrap;
    }
};

// What a lane knows of its NV pair vectors: offsets of the members in a head, first pair; lanes past the head's end repeat vector 0 and store nothing.
template <int V, int NV, bool HALF>
struct Lane {
    static constexpr int WS = HALF ? 1 : 2;  // from one member to the next of its kind
    bool has[NV];
    int oa[NV], ob[NV], oc[NV];
    __device__ __forceinline__ Lane(const QkArgs& a, int lane, int ln)
    {
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int t = lane + v * ln;
            has[v] = t < a.dim / (2 * V);
            const int u = has[v] ? t : 0;
            const bool rot = HALF && u * V < a.pairs;
            oa[v] = rot ? u * V : 2 * u * V;
            ob[v] = rot ? a.pairs + u * V : 2 * u * V + (HALF ? V : 1);
            oc[v] = u * V;
        }
    }
};

// Forward.  The table holds, for queries and for keys, {cos wa, sin wb, sin wa, cos wb} of every pair: a pair is then four products, and
// the norm's factor two.  A lane works on one head of the queries and one of the keys at a time, with the next ones already requested; the first are
// requested before the table is made.  us and TB/s, bf16: 8192 tokens of 16 + 16 heads of 72 19.4 and 3.9, 16380 of 20 + 20 of 112 in adjacent pairs 61.9 and 4.7 (a strided
// copy of the first's bytes: 17.5); one token 4.2, the launch and a few round trips.  One vector to a lane for heads of 72 leaves 7 of 16 lanes idle and
// is bound by the vector ALU (35).
template <typename T, int V, int NV, bool HALF, bool NORM>
__global__ void __launch_bounds__(256) qk_fwd_kernel(QkArgs a)
{
    extern __shared__ v4f table[];  // [queries, keys][token][pair]
    const int ln = 1 << a.lanes_log2, lane = threadIdx.x & (ln - 1), group = threadIdx.x >> a.lanes_log2, groups = 256 >> a.lanes_log2;
    const int half = a.dim / 2;
    const Lane<V, NV, HALF> L(a, lane, ln);
    const int m0 = blockIdx.x * a.tokens, n = min((int)a.M - m0, a.tokens);
    int k0[2], h0[2];
#pragma unroll
    for (int s = 0; s < 2; ++s) k0[s] = quotient(group, a.magic[s]), h0[s] = group - k0[s] * a.heads[s];
#define WALK(NAME, S, TENSOR) Walk NAME(h0[S], k0[S], a.turn_h[S], a.turn_k[S], a.heads[S], a.t.TENSOR[S].ld, a.t.TENSOR[S].hs)
    WALK(xq, 0, q);
    WALK(xk, 1, q);
    WALK(yq, 0, out);
    WALK(yk, 1, out);
#undef WALK
    const T* xp[2] = {(const T*)a.t.q[0].p + m0 * a.t.q[0].ld, (const T*)a.t.q[1].p + m0 * a.t.q[1].ld};
    T* yp[2] = {(T*)a.t.out[0].p + m0 * a.t.out[0].ld, (T*)a.t.out[1].p + m0 * a.t.out[1].ld};
    int at[2] = {k0[0] * half, k0[1] * half};  // of the token's part of the table
    const int items[2] = {n * a.heads[0], n * a.heads[1]};
    Raw<T, V, HALF> raw[2][NV];
    auto request = [&](int it) {
        if (it < items[0])
#pragma unroll
            for (int v = 0; v < NV; ++v) raw[0][v].fetch(xp[0] + xq.at, L.oa[v], L.ob[v]);
        if (it < items[1])
#pragma unroll
            for (int v = 0; v < NV; ++v) raw[1][v].fetch(xp[1] + xk.at, L.oa[v], L.ob[v]);
        xq.next(a.turn_h[0], a.heads[0]);
        xk.next(a.turn_h[1], a.heads[1]);
    };
    request(group);
    const unsigned first = first_pos(a, m0);
    for (int o = threadIdx.x; o < n * half; o += 256) {
        const int k = quotient(o, a.half_magic), p = o - k * half;
        const float2 e = turn(a, pos_row(a, first, k), p);
        // members of pair p of the head (what is not rotated: as a lane's vectors of it are cut)
        int ia = 2 * p, ib = 2 * p + 1;
        if (HALF) {
            const bool rot = p < a.pairs;
            ia = rot ? p : 2 * (p / V) * V + p % V;
            ib = rot ? a.pairs + p : ia + V;
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const float* w = a.t.w[s];
            const float wa = NORM && w ? w[ia] : 1.0f, wb = NORM && w ? w[ib] : 1.0f;
            table[s * a.tokens * half + o] = v4f{e.x * wa, e.y * wb, e.y * wa, e.x * wb};
        }
    }
    __syncthreads();
    const int most = max(items[0], items[1]);
    for (int it = group; it < most; it += groups) {
        float xa[2][NV][V], xb[2][NV][V];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int v = 0; v < NV; ++v) raw[s][v].get(xa[s][v], xb[s][v]);
        if (it + groups < most) request(it + groups);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (it < items[s]) {
                const v4f* c = table + s * a.tokens * half + at[s];
                T* y = yp[s] + (s ? yk.at : yq.at);
                float rstd = 1.0f;
                if constexpr (NORM) {
                    float ss = 0.0f;
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
                        float t = 0.0f;
#pragma unroll
                        for (int j = 0; j < V; ++j) t = fmaf(xa[s][v][j], xa[s][v][j], fmaf(xb[s][v][j], xb[s][v][j], t));
                        ss += L.has[v] ? t : 0.0f;
                    }
                    rstd = __builtin_amdgcn_rsqf(fmaf(sum_lanes(ss, a.lanes_log2), a.inv_dim, a.eps));
                }
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float ya[V], yb[V];
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const v4f e = c[L.oc[v] + j];
                        ya[j] = fmaf(xa[s][v][j], e[0], -(xb[s][v][j] * e[1]));
                        yb[j] = fmaf(xa[s][v][j], e[2], xb[s][v][j] * e[3]);
                        if (NORM) ya[j] *= rstd, yb[j] *= rstd;
                    }
                    if (L.has[v]) put<T, V, HALF>(y, L.oa[v], L.ob[v], ya, yb);
                }
            }
            at[s] += a.turn_k[s] * half;
            if ((s ? yk.h : yq.h) + a.turn_h[s] >= a.heads[s]) at[s] += half;
        }
        yq.next(a.turn_h[0], a.heads[0]);
        yk.next(a.turn_h[1], a.heads[1]);
    }
}

// Gradient: x is the forward's input (NORM only), g the derivative of its output.  Queries, then keys, one head at a time with the next one already
// requested; dw is summed in registers, then over the wavefront, then over the workgroup's four, into the workgroup's part.
// Bound by the loads two workgroups a compute unit keep in flight (registers): 8192 tokens of 16 + 16 heads of 72, bf16, 33 us traced, 3.4 TB/s; 333 of 12 + 3 fp32 heads of 96 9,
// latency.
template <typename T, int V, int NV, bool HALF, bool NORM>
__global__ void __launch_bounds__(256) qk_bwd_kernel(QkArgs a)
{
    extern __shared__ float2 cs[];  // [token][pair]; with NORM then [wavefront][dim] floats
    const int ln = 1 << a.lanes_log2, lane = threadIdx.x & (ln - 1), group = threadIdx.x >> a.lanes_log2, groups = 256 >> a.lanes_log2;
    const int half = a.dim / 2;
    const Lane<V, NV, HALF> L(a, lane, ln);
    const int m0 = blockIdx.x * a.tokens, n = min((int)a.M - m0, a.tokens);
    float* sums = (float*)(cs + a.tokens * half);
    bool made = false;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const int H = a.heads[s], items = n * H, dh = a.turn_h[s], dk = a.turn_k[s];
        float dw[2 * NV * V], wa[NV][V], wb[NV][V];
#pragma unroll
        for (int v = 0; v < 2 * NV * V; ++v) dw[v] = 0.0f;
        if (H > 0) {
            const int k0 = quotient(group, a.magic[s]), h0 = group - k0 * H;
            Walk wx(h0, k0, dh, dk, H, a.t.q[s].ld, a.t.q[s].hs), wg(h0, k0, dh, dk, H, a.t.grad[s].ld, a.t.grad[s].hs);
            Walk wy(h0, k0, dh, dk, H, a.t.out[s].ld, a.t.out[s].hs), wc(h0, k0, dh, dk, H, half, 0);
            const T* xp = (const T*)a.t.q[s].p + m0 * a.t.q[s].ld;
            const T* gp = (const T*)a.t.grad[s].p + m0 * a.t.grad[s].ld;
            T* yp = (T*)a.t.out[s].p + m0 * a.t.out[s].ld;
            Raw<T, V, HALF> rx[NV], rg[NV];
            auto request = [&](int it) {
                if (it < items)
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
                        if constexpr (NORM) rx[v].fetch(xp + wx.at, L.oa[v], L.ob[v]);
                        rg[v].fetch(gp + wg.at, L.oa[v], L.ob[v]);
                    }
                wx.next(dh, H);
                wg.next(dh, H);
            };
            request(group);
            if constexpr (NORM) {
                const float* w = a.t.w[s];
                if (w) {
#pragma unroll
                    for (int v = 0; v < NV; ++v)
#pragma unroll
                        for (int j = 0; j < V; ++j) wa[v][j] = w[L.oa[v] + L.WS * j], wb[v][j] = w[L.ob[v] + L.WS * j];
                } else {
#pragma unroll
                    for (int v = 0; v < NV; ++v)
#pragma unroll
                        for (int j = 0; j < V; ++j) wa[v][j] = wb[v][j] = 1.0f;
                }
            }
            if (!made) {
                const unsigned first = first_pos(a, m0);
                for (int o = threadIdx.x; o < n * half; o += 256) {
                    const int k = quotient(o, a.half_magic);
                    cs[o] = turn(a, pos_row(a, first, k), o - k * half);
                }
                __syncthreads();
                made = true;
            }
            for (int it = group; it < items; it += groups) {
                float xa[NV][V], xb[NV][V], ga[NV][V], gb[NV][V];
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    if constexpr (NORM) rx[v].get(xa[v], xb[v]);
                    rg[v].get(ga[v], gb[v]);
                }
                request(it + groups);
                const float2* c = cs + wc.at;
                T* y = yp + wy.at;
                float rstd = 1.0f;
                if constexpr (NORM) {
                    float ss = 0.0f;
#pragma unroll
                    for (int v = 0; v < NV; ++v) {
                        float t = 0.0f;
#pragma unroll
                        for (int j = 0; j < V; ++j) t = fmaf(xa[v][j], xa[v][j], fmaf(xb[v][j], xb[v][j], t));
                        ss += L.has[v] ? t : 0.0f;
                    }
                    rstd = __builtin_amdgcn_rsqf(fmaf(sum_lanes(ss, a.lanes_log2), a.inv_dim, a.eps));
                }
                float dot = 0.0f;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float d = 0.0f;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float2 e = c[L.oc[v] + j];
                        const float ra = fmaf(ga[v][j], e.x, gb[v][j] * e.y), rb = fmaf(gb[v][j], e.x, -(ga[v][j] * e.y));
                        ga[v][j] = ra;
                        gb[v][j] = rb;
                        if constexpr (NORM) {
                            xa[v][j] *= rstd;
                            xb[v][j] *= rstd;
                            float &da = dw[(v * V + j) * 2], &db = dw[(v * V + j) * 2 + 1];
                            da = fmaf(ra, xa[v][j], da);
                            db = fmaf(rb, xb[v][j], db);
                            ga[v][j] *= wa[v][j];
                            gb[v][j] *= wb[v][j];
                            d = fmaf(ga[v][j], xa[v][j], fmaf(gb[v][j], xb[v][j], d));
                        }
                    }
                    dot += L.has[v] ? d : 0.0f;
                }
                float mean = 0.0f;
                if constexpr (NORM) mean = sum_lanes(dot, a.lanes_log2) * a.inv_dim;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    if constexpr (NORM)
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            ga[v][j] = rstd * fmaf(-xa[v][j], mean, ga[v][j]);
                            gb[v][j] = rstd * fmaf(-xb[v][j], mean, gb[v][j]);
                        }
                    if (L.has[v]) put<T, V, HALF>(y, L.oa[v], L.ob[v], ga[v], gb[v]);
                }
                wy.next(dh, H);
                wc.next(dh, H);
            }
        }
        if constexpr (NORM) {
            if (a.part) {
                sum_groups(dw, a.lanes_log2);
                float* mine = sums + (threadIdx.x >> 6) * a.dim;
                if ((threadIdx.x & 63) < ln)
#pragma unroll
                    for (int v = 0; v < NV; ++v)
                        if (L.has[v])
#pragma unroll
                            for (int j = 0; j < V; ++j) mine[L.oa[v] + L.WS * j] = dw[(v * V + j) * 2], mine[L.ob[v] + L.WS * j] = dw[(v * V + j) * 2 + 1];
                __syncthreads();
                for (int o = threadIdx.x; o < a.dim; o += 256)
                    a.part[((int64_t)blockIdx.x * 2 + s) * a.dim + o] = (sums[o] + sums[a.dim + o]) + (sums[2 * a.dim + o] + sums[3 * a.dim + o]);
                __syncthreads();
            }
        }
    }
}

// dw: the workgroups' sums in a fixed order; 16 values to a workgroup, 64 shares of the sums each, joined in a tree (one after another their 63 additions were
// most of dw's rounding, and no faster; 512 parts of two heads of 72: 4 us traced, round trips)
__global__ void __launch_bounds__(1024) qk_weight_sum(const float* part, int n, int dim, float* dwq, float* dwk)
{
    __shared__ float sh[16][16];
    const int v = blockIdx.x * 16 + (threadIdx.x & 15), r = threadIdx.x >> 4;
    float t = 0.0f;
    if (v < 2 * dim) {
#pragma unroll 8
        for (int i = r; i < n; i += 64) t += part[(int64_t)i * 2 * dim + v];
    }
    t += __shfl_xor(t, 16);
    t += __shfl_xor(t, 32);
    if ((threadIdx.x & 63) < 16) sh[threadIdx.x >> 6][threadIdx.x & 15] = t;
    __syncthreads();
    if (threadIdx.x < 64) {
        const int c = threadIdx.x & 15;
        t = (sh[r][c] + sh[r + 4][c]) + (sh[r + 8][c] + sh[r + 12][c]);
        t += __shfl_xor(t, 16);
        t += __shfl_xor(t, 32);
        if (r == 0 && v < 2 * dim) (v < dim ? dwq : dwk)[v < dim ? v : v - dim] = t;
    }
}

// ---- host ---------------------------------------------------------------------------------------

// Tokens of a workgroup of the gradient, each of which leaves a part of dw: two workgroups to a compute unit are what its registers allow (us by the number
// of workgroups, 8192 tokens of 16 + 16 heads of 72: 256 37.9, 512 35.9, 1024 39.4, 2048 49.3), one while they have little to do (1000 tokens: 256 13.5,
// 512 14.7).  The table of cosines takes up to 48 KB of the LDS.
static int qk_grad_tokens(const lq_qk_config* c, int64_t M)
{
    const int64_t most = 12288 / c->head_dim, groups = M < 4096 ? 256 : 512, t = (M + groups - 1) / groups;
    return (int)(t < 1 ? 1 : t > most ? most : t);
}

struct QkShape {
    int V, NV, lanes_log2, tokens, lds;
    int64_t grid;
};

// Values per access: the widest at which no vector straddles an axis of members, and every head starts aligned.
static bool fits(const lq_heads& h, int heads, int64_t M, int elem, int bytes)
{
    return ((uintptr_t)h.p % bytes) == 0 && (M < 2 || h.ld * elem % bytes == 0) && (heads < 2 || h.hs * elem % bytes == 0);
}
static QkShape qk_shape(const lq_qk_config* c, const QkTensors* t, int64_t M, bool grad)
{
    const int P = c->pairs[0] + c->pairs[1] + c->pairs[2] + c->pairs[3], elem = c->dtype == LQ_F32 ? 4 : 2;
    const int heads[2] = {c->heads_q, c->heads_k};
    QkShape s;
    // (bf16 halves have vectors of 8, 16 bytes an access, up to heads of 128: us, 8 / 4, 8192 tokens of 18 + 18 heads of 64 21.0 / 23.8, 16380 of 20 + 20 of 112 62.2 /
    // 70.6; of 7 + 7 of 160 23.8 / 22.6, whose 10 vectors leave 6 of 16 lanes idle)
    for (s.V = c->dtype == LQ_BF16 && c->pairing == LQ_PAIR_HALF && c->head_dim <= 128 ? 8 : 4; s.V > 1; s.V /= 2) {
        if (c->head_dim % (2 * s.V) || P % s.V) continue;
        const int bytes = access_align(s.V, c->pairing == LQ_PAIR_HALF, elem);
        bool ok = true;
        for (int k = 0; t && k < 2; ++k)
            if (heads[k])
                ok = ok && (!t->q[k].p || fits(t->q[k], heads[k], M, elem, bytes)) && fits(t->out[k], heads[k], M, elem, bytes) &&
                     (!t->grad[k].p || fits(t->grad[k], heads[k], M, elem, bytes));
        if (ok) break;
    }
    // two or three vectors to a lane (one of the widest), on the fewest lanes: what a turn costs beside its vectors is shared, and three fill 9 of 12 places of a
    // head of 72 where one or two fill 9 of 16
    const int vectors = c->head_dim / (2 * s.V);
    s.lanes_log2 = 0;
    while (((s.V == 8 ? 1 : 3) << s.lanes_log2) < vectors) ++s.lanes_log2;
    s.NV = s.V == 8 ? 1 : vectors <= (2 << s.lanes_log2) ? 2 : 3;
    if (grad) {
        s.tokens = qk_grad_tokens(c, M);
    } else {
        // two heads of each kind to a lane, while there are 1024 workgroups (us by the number of workgroups: 8192 tokens of 16 + 16 heads of 72: 512 25.4, 1024
        // 24.9, 4096 27.6; 16380 of 20 + 20 of 112, two heads with 8192: 1024 62.6, 4096 59.4, 8192 59.2); up to 32 KB of the LDS for the table
        const int groups = 256 >> s.lanes_log2, H = heads[0] > heads[1] ? heads[0] : heads[1];
        const int64_t two = (2 * groups + H - 1) / H, share = M / 1024, most = 2048 / c->head_dim;
        s.tokens = (int)(two < share ? two : share);
        s.tokens = s.tokens > most ? (int)most : s.tokens;
        const int least = M > (1 << 23) ? 2 : 1;  // (a launch stays below 2^32 threads)
        s.tokens = s.tokens < least ? least : s.tokens;
    }
    s.grid = (M + s.tokens - 1) / s.tokens;
    s.lds = s.tokens * c->head_dim / 2 * (grad ? 8 : 32) + (grad ? 4 * c->head_dim * 4 : 0);
    return s;
}

// floor(i / d) = floor(i m / 2^32) for i d < 2^32; 0 stands for d = 1, whose factor does not fit
static unsigned quotient_magic(int d) { return d > 1 ? (unsigned)((((uint64_t)1 << 32) + d - 1) / d) : 0; }

static QkArgs qk_args(const lq_qk_config* c, const QkTensors& t, int64_t M, const QkShape& s)
{
    QkArgs a{};
    a.t = t;
    a.M = M;
    a.heads[0] = c->heads_q;
    a.heads[1] = c->heads_k;
    a.dim = c->head_dim;
    a.axes = c->axes;
    for (int k = 0; k < 4; ++k) a.axis_end[k] = a.pairs += c->pairs[k];
    a.lanes_log2 = s.lanes_log2;
    a.tokens = s.tokens;
    const int groups = 256 >> s.lanes_log2;
    for (int k = 0; k < 2; ++k) {
        a.magic[k] = quotient_magic(a.heads[k]);
        a.turn_k[k] = a.heads[k] ? groups / a.heads[k] : 0;
        a.turn_h[k] = a.heads[k] ? groups % a.heads[k] : 0;
    }
    a.half_magic = quotient_magic(c->head_dim / 2);
    a.eps = c->eps;
    a.inv_dim = 1.0f / (float)c->head_dim;
    return a;
}

template <typename T, int V, int NV, bool HALF, bool GRAD>
static void qk_run(const QkArgs& a, bool norm, const QkShape& s, hipStream_t stream)
{
    const dim3 grid((unsigned)s.grid), block(256);
    if constexpr (GRAD) {
        if (norm) hipLaunchKernelGGL((qk_bwd_kernel<T, V, NV, HALF, true>), grid, block, s.lds, stream, a);
        else hipLaunchKernelGGL((qk_bwd_kernel<T, V, NV, HALF, false>), grid, block, s.lds, stream, a);
    } else {
        if (norm) hipLaunchKernelGGL((qk_fwd_kernel<T, V, NV, HALF, true>), grid, block, s.lds, stream, a);
        else hipLaunchKernelGGL((qk_fwd_kernel<T, V, NV, HALF, false>), grid, block, s.lds, stream, a);
    }
}
template <typename T, int V, bool HALF, bool GRAD>
static void qk_run_nv(const QkArgs& a, bool norm, const QkShape& s, hipStream_t stream)
{
    if (s.NV == 2) qk_run<T, V, 2, HALF, GRAD>(a, norm, s, stream);
    else qk_run<T, V, 3, HALF, GRAD>(a, norm, s, stream);
}
template <typename T, bool HALF, bool GRAD>
static void qk_run_v(const QkArgs& a, bool norm, const QkShape& s, hipStream_t stream)
{
    if constexpr (HALF && sizeof(T) == 2)
        if (s.V == 8) return qk_run<T, 8, 1, HALF, GRAD>(a, norm, s, stream);
    if (s.V == 4) qk_run_nv<T, 4, HALF, GRAD>(a, norm, s, stream);
    else if (s.V == 2) qk_run_nv<T, 2, HALF, GRAD>(a, norm, s, stream);
    else qk_run_nv<T, 1, HALF, GRAD>(a, norm, s, stream);
}
template <bool GRAD>
static hipError_t qk_run_all(const lq_qk_config* c, const QkArgs& a, const QkShape& s, hipStream_t stream)
{
    const bool norm = c->norm == LQ_NORM_RMS, half = c->pairing == LQ_PAIR_HALF;
    if (c->dtype == LQ_F32) {
        if (half) qk_run_v<float, true, GRAD>(a, norm, s, stream);
        else qk_run_v<float, false, GRAD>(a, norm, s, stream);
    } else {
        if (half) qk_run_v<__bf16, true, GRAD>(a, norm, s, stream);
        else qk_run_v<__bf16, false, GRAD>(a, norm, s, stream);
    }
    return hipGetLastError();
}

size_t qk_work_bytes(const lq_qk_config* c, int64_t M)
{
    const int tokens = qk_grad_tokens(c, M);
    return c->norm == LQ_NORM_RMS ? align256((size_t)((M + tokens - 1) / tokens) * 2 * c->head_dim * 4) : 0;
}

hipError_t launch_qk_fwd(const lq_qk_config* c, const QkTensors& t, int64_t M, hipStream_t s)
{
    const QkShape sh = qk_shape(c, &t, M, false);
    return qk_run_all<false>(c, qk_args(c, t, M, sh), sh, s);
}

hipError_t launch_qk_bwd(const lq_qk_config* c, const QkTensors& t, int64_t M, uint8_t* work, hipStream_t s)
{
    const QkShape sh = qk_shape(c, &t, M, true);
    QkArgs a = qk_args(c, t, M, sh);
    const bool dw = c->norm == LQ_NORM_RMS && t.dw[0];
    a.part = dw ? (float*)work : nullptr;
    hipError_t e = hipSuccess;
    if (M > 0) e = qk_run_all<true>(c, a, sh, s);
    if (e != hipSuccess || !dw) return e;
    hipLaunchKernelGGL(qk_weight_sum, dim3((2 * c->head_dim + 15) / 16), dim3(1024), 0, s, (const float*)work, M > 0 ? (int)sh.grid : 0, c->head_dim, t.dw[0], t.dw[1]);
    return hipGetLastError();
}

}  // namespace lq
