// Norm of queries and keys for each head with the rotation by positions of several axes, and its gradient, one pass over the heads each:
//     n = x rsqrt(mean x^2 + eps) w ;  (n_a, n_b) -> (n_a cos t - n_b sin t, n_a sin t + n_b cos t) ,  t = pos[axis] inv_freq
// Bound by memory: two bytes moved per byte of heads, three in the gradient.  A workgroup takes a few tokens; it computes their cosines and
// sines once, into the LDS, for all heads.  A head belongs to a group of 2^k lanes; a lane holds the same V pairs of every head it meets, so that
// its weights, and its sums of dw, stay in registers.
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
    float eps;
    float* part;      // [workgroup][2][dim] sums of dw
};

// N consecutive values at p, as fp32 (N * sizeof(T) bytes of alignment)
template <typename T, int N>
__device__ __forceinline__ void load(const T* p, float (&v)[N])
{
    typedef T vt __attribute__((ext_vector_type(N)));
    if constexpr (N == 1) {
        v[0] = (float)*p;
    } else {
        const vt r = *(const vt*)p;
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = (float)r[j];
    }
}
template <typename T, int N>
__device__ __forceinline__ void store(T* p, const float (&v)[N])
{
    typedef T vt __attribute__((ext_vector_type(N)));
    if constexpr (N == 1) {
        *p = (T)v[0];
    } else {
        vt r;
#pragma unroll
        for (int j = 0; j < N; ++j) r[j] = (T)v[j];
        *(vt*)p = r;
    }
}

// Pair vectors: vector t of a head is the members a, b of V pairs.  Halves: a = x[tV ..], b = x[P + tV ..]; adjacent: 2V consecutive values.
// What is not rotated (values from 2P on) is cut into vectors of 2V consecutive values.
template <typename T, int V, bool HALF>
__device__ __forceinline__ void load_pairs(const T* x, int t, int P, float (&a)[V], float (&b)[V])
{
    if (HALF) {
        const bool rot = t * V < P;
        load<T, V>(x + (rot ? t * V : 2 * t * V), a);
        load<T, V>(x + (rot ? P + t * V : 2 * t * V + V), b);
    } else {
        float v[2 * V];
        load<T, 2 * V>(x + 2 * t * V, v);
#pragma unroll
        for (int j = 0; j < V; ++j) a[j] = v[2 * j], b[j] = v[2 * j + 1];
    }
}
template <typename T, int V, bool HALF>
__device__ __forceinline__ void store_pairs(T* x, int t, int P, const float (&a)[V], const float (&b)[V])
{
    if (HALF) {
        const bool rot = t * V < P;
        store<T, V>(x + (rot ? t * V : 2 * t * V), a);
        store<T, V>(x + (rot ? P + t * V : 2 * t * V + V), b);
    } else {
        float v[2 * V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[2 * j] = a[j], v[2 * j + 1] = b[j];
        store<T, 2 * V>(x + 2 * t * V, v);
    }
}

// cos and sin of the angles of `n` tokens from m0 on: cs[token][pair of the head], ones and zeros for the values that are not rotated.  The
// product of two fp32 numbers is exact in 64 bits; whole turns are taken off there, what is left fits 32.
__device__ __forceinline__ void turn_table(const QkArgs& a, int64_t m0, int n, float2* cs)
{
    const int H = a.dim / 2;
    for (int o = threadIdx.x; o < n * H; o += blockDim.x) {
        const int k = o / H, p = o - k * H;
        float2 v = make_float2(1.0f, 0.0f);
        if (p < a.pairs) {
            const int axis = (p >= a.axis_end[0]) + (p >= a.axis_end[1]) + (p >= a.axis_end[2]);
            const double turns = (double)a.t.pos[((m0 + k) % a.t.pos_rows) * a.axes + axis] * (double)a.t.inv_freq[p] * 0.15915494309189533577;
            const float r = (float)(turns - rint(turns));
            sincospif(2.0f * r, &v.y, &v.x);
        }
        cs[o] = v;
    }
}

__device__ __forceinline__ float sum_lanes(float v, int lanes_log2)
{
    for (int k = 0; k < lanes_log2; ++k) v += __shfl_xor(v, 1 << k);
    return v;
}

// GRAD: x is the forward's input (NORM only), g the derivative of its output.
template <typename T, int V, int NV, bool HALF, bool NORM, bool GRAD>
__global__ void __launch_bounds__(256) qk_kernel(QkArgs a)
{
    extern __shared__ float2 cs[];
    const int ln = 1 << a.lanes_log2, lane = threadIdx.x & (ln - 1), group = threadIdx.x >> a.lanes_log2, groups = 256 >> a.lanes_log2;
    const int vectors = a.dim / (2 * V), H = a.heads[0] + a.heads[1];
    float wa[2][NV][V], wb[2][NV][V], da[2][NV][V], db[2][NV][V];
    bool has[NV];
#pragma unroll
    for (int u = 0; u < NV; ++u) {
        const int t = lane + u * ln;
        has[u] = t < vectors;
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int j = 0; j < V; ++j) wa[s][u][j] = wb[s][u][j] = 1.0f, da[s][u][j] = db[s][u][j] = 0.0f;
        if (NORM && has[u])
#pragma unroll
            for (int s = 0; s < 2; ++s)
                if (a.t.w[s]) {
                    const float* w = a.t.w[s];
                    const bool rot = HALF && t * V < a.pairs;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        wa[s][u][j] = w[HALF ? (rot ? t * V + j : 2 * t * V + j) : 2 * (t * V + j)];
                        wb[s][u][j] = w[HALF ? (rot ? a.pairs + t * V + j : 2 * t * V + V + j) : 2 * (t * V + j) + 1];
                    }
                }
    }
    for (int64_t m0 = (int64_t)blockIdx.x * a.tokens; m0 < a.M; m0 += (int64_t)gridDim.x * a.tokens) {
        const int n = (int)(a.M - m0 < a.tokens ? a.M - m0 : a.tokens);
        __syncthreads();
        turn_table(a, m0, n, cs);
        __syncthreads();
        for (int it = group; it < n * H; it += groups) {
            const int k = it / H, h = it - k * H;
            const int s = h >= a.heads[0];
            const int64_t m = m0 + k;
            const int hh = s ? h - a.heads[0] : h;
            float xa[NV][V], xb[NV][V], ga[NV][V], gb[NV][V];
            float ss = 0.0f;
            if (NORM || !GRAD) {
                const T* x = (const T*)a.t.q[s].p + m * a.t.q[s].ld + hh * a.t.q[s].hs;
#pragma unroll
                for (int u = 0; u < NV; ++u)
                    if (has[u]) {
                        load_pairs<T, V, HALF>(x, lane + u * ln, a.pairs, xa[u], xb[u]);
#pragma unroll
                        for (int j = 0; j < V; ++j) ss += xa[u][j] * xa[u][j] + xb[u][j] * xb[u][j];
                    }
            }
            if (GRAD) {
                const T* g = (const T*)a.t.grad[s].p + m * a.t.grad[s].ld + hh * a.t.grad[s].hs;
#pragma unroll
                for (int u = 0; u < NV; ++u)
                    if (has[u]) load_pairs<T, V, HALF>(g, lane + u * ln, a.pairs, ga[u], gb[u]);
            }
            float rstd = 1.0f;
            if (NORM) rstd = 1.0f / sqrtf(sum_lanes(ss, a.lanes_log2) / (float)a.dim + a.eps);
            T* out = (T*)a.t.out[s].p + m * a.t.out[s].ld + hh * a.t.out[s].hs;
            const float2* c = cs + k * (a.dim / 2);
            if (!GRAD) {
#pragma unroll
                for (int u = 0; u < NV; ++u)
                    if (has[u]) {
                        float ya[V], yb[V];
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            const float2 e = c[(lane + u * ln) * V + j];
                            const float na = NORM ? xa[u][j] * rstd * (s ? wa[1][u][j] : wa[0][u][j]) : xa[u][j];
                            const float nb = NORM ? xb[u][j] * rstd * (s ? wb[1][u][j] : wb[0][u][j]) : xb[u][j];
                            ya[j] = na * e.x - nb * e.y;
                            yb[j] = na * e.y + nb * e.x;
                        }
                        store_pairs<T, V, HALF>(out, lane + u * ln, a.pairs, ya, yb);
                    }
            } else {
                float dot = 0.0f;
#pragma unroll
                for (int u = 0; u < NV; ++u)
                    if (has[u])
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            const float2 e = c[(lane + u * ln) * V + j];
                            const float ra = ga[u][j] * e.x + gb[u][j] * e.y, rb = gb[u][j] * e.x - ga[u][j] * e.y;
                            if (NORM) {
                                xa[u][j] *= rstd;
                                xb[u][j] *= rstd;
                                const float pa = ra * xa[u][j], pb = rb * xb[u][j];
                                da[0][u][j] += s ? 0.0f : pa, db[0][u][j] += s ? 0.0f : pb;
                                da[1][u][j] += s ? pa : 0.0f, db[1][u][j] += s ? pb : 0.0f;
                                const float w0 = s ? wa[1][u][j] : wa[0][u][j], w1 = s ? wb[1][u][j] : wb[0][u][j];
                                dot += pa * w0 + pb * w1;
                                ga[u][j] = ra * w0;
                                gb[u][j] = rb * w1;
                            } else {
                                ga[u][j] = ra;
                                gb[u][j] = rb;
                            }
                        }
                const float mean = NORM ? sum_lanes(dot, a.lanes_log2) / (float)a.dim : 0.0f;
#pragma unroll
                for (int u = 0; u < NV; ++u)
                    if (has[u]) {
                        float ya[V], yb[V];
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            ya[j] = NORM ? rstd * (ga[u][j] - xa[u][j] * mean) : ga[u][j];
                            yb[j] = NORM ? rstd * (gb[u][j] - xb[u][j] * mean) : gb[u][j];
                        }
                        store_pairs<T, V, HALF>(out, lane + u * ln, a.pairs, ya, yb);
                    }
            }
        }
    }
    if constexpr (GRAD && NORM) {  // the groups' sums, one group after another
        if (!a.part) return;
        float* acc = (float*)cs;  // [2][dim]
        for (int o = 0; o < groups; ++o) {
            __syncthreads();
            if (group == o)
#pragma unroll
                for (int u = 0; u < NV; ++u)
                    if (has[u]) {
                        const int t = lane + u * ln;
                        const bool rot = HALF && t * V < a.pairs;
#pragma unroll
                        for (int s = 0; s < 2; ++s)
#pragma unroll
                            for (int j = 0; j < V; ++j) {
                                const int ia = s * a.dim + (HALF ? (rot ? t * V + j : 2 * t * V + j) : 2 * (t * V + j));
                                const int ib = s * a.dim + (HALF ? (rot ? a.pairs + t * V + j : 2 * t * V + V + j) : 2 * (t * V + j) + 1);
                                acc[ia] = o ? acc[ia] + da[s][u][j] : da[s][u][j];
                                acc[ib] = o ? acc[ib] + db[s][u][j] : db[s][u][j];
                            }
                    }
        }
        __syncthreads();
        for (int o = threadIdx.x; o < 2 * a.dim; o += 256) a.part[(int64_t)blockIdx.x * 2 * a.dim + o] = acc[o];
    }
}

// dw: the workgroups' sums in their order; 16 values to a workgroup, 16 shares of the sums each
__global__ void __launch_bounds__(256) qk_weight_sum(const float* part, int n, int dim, float* dwq, float* dwk)
{
    __shared__ float sh[16][17];
    const int v = blockIdx.x * 16 + (threadIdx.x & 15), r = threadIdx.x >> 4;
    float t = 0.0f;
    if (v < 2 * dim)
        for (int i = r; i < n; i += 16) t += part[(int64_t)i * 2 * dim + v];
    sh[r][threadIdx.x & 15] = t;
    __syncthreads();
    if (r == 0 && v < 2 * dim) {
        for (int k = 1; k < 16; ++k) t += sh[k][threadIdx.x];
        (v < dim ? dwq : dwk)[v < dim ? v : v - dim] = t;
    }
}

// ---- host ---------------------------------------------------------------------------------------

constexpr int QK_MAX_GROUPS = 1024;  // workgroups of the gradient, each of which leaves a part of dw

struct QkShape {
    int V, NV, lanes_log2, tokens, lds;
    int64_t grid;
};

// Values per access: the widest at which no vector straddles an axis of members, and every head starts aligned.
static bool fits(const lq_heads& h, int heads, int64_t M, int elem, int bytes)
{
    return ((uintptr_t)h.p % bytes) == 0 && (M < 2 || h.ld * elem % bytes == 0) && (heads < 2 || h.hs * elem % bytes == 0);
}
static QkShape qk_shape(const lq_qk_config* c, const QkTensors* t, int64_t M, int64_t max_grid)
{
    const int P = c->pairs[0] + c->pairs[1] + c->pairs[2] + c->pairs[3], elem = c->dtype == LQ_F32 ? 4 : 2;
    const int heads[2] = {c->heads_q, c->heads_k};
    QkShape s;
    for (s.V = 4; s.V > 1; s.V /= 2) {
        if (c->head_dim % (2 * s.V) || P % s.V) continue;
        int bytes = c->pairing == LQ_PAIR_HALF ? s.V * elem : 2 * s.V * elem;
        bytes = bytes > 16 ? 16 : bytes;
        bool ok = true;
        for (int k = 0; t && k < 2; ++k)
            if (heads[k])
                ok = ok && (!t->q[k].p || fits(t->q[k], heads[k], M, elem, bytes)) && fits(t->out[k], heads[k], M, elem, bytes) &&
                     (!t->grad[k].p || fits(t->grad[k], heads[k], M, elem, bytes));
        if (ok) break;
    }
    const int vectors = c->head_dim / (2 * s.V);
    s.lanes_log2 = 0;
    while ((1 << s.lanes_log2) < vectors && s.lanes_log2 < 6) ++s.lanes_log2;
    s.NV = (vectors + (1 << s.lanes_log2) - 1) >> s.lanes_log2;
    const int H = heads[0] + heads[1], groups = 256 >> s.lanes_log2;
    s.tokens = (2 * groups + H - 1) / H;
    s.tokens = s.tokens < 1 ? 1 : s.tokens > 16 ? 16 : s.tokens;
    s.grid = (M + s.tokens - 1) / s.tokens;
    s.grid = s.grid > max_grid ? max_grid : s.grid;
    const int table = s.tokens * c->head_dim / 2 * 8, sums = 2 * c->head_dim * 4;
    s.lds = table > sums ? table : sums;
    return s;
}

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
    a.eps = c->eps;
    return a;
}

template <typename T, int V, int NV, bool HALF, bool GRAD>
static void qk_run(const QkArgs& a, bool norm, const QkShape& s, hipStream_t stream)
{
    if (norm) hipLaunchKernelGGL((qk_kernel<T, V, NV, HALF, true, GRAD>), dim3((unsigned)s.grid), dim3(256), s.lds, stream, a);
    else hipLaunchKernelGGL((qk_kernel<T, V, NV, HALF, false, GRAD>), dim3((unsigned)s.grid), dim3(256), s.lds, stream, a);
}
template <typename T, bool HALF, bool GRAD>
static void qk_run_v(const QkArgs& a, bool norm, const QkShape& s, hipStream_t stream)
{
    if (s.V == 4) qk_run<T, 4, 1, HALF, GRAD>(a, norm, s, stream);
    else if (s.V == 2) qk_run<T, 2, 1, HALF, GRAD>(a, norm, s, stream);
    else if (s.NV == 1) qk_run<T, 1, 1, HALF, GRAD>(a, norm, s, stream);
    else qk_run<T, 1, 2, HALF, GRAD>(a, norm, s, stream);
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
    const int64_t groups = M < QK_MAX_GROUPS ? M : QK_MAX_GROUPS;
    return c->norm == LQ_NORM_RMS ? align256((size_t)groups * 2 * c->head_dim * 4) : 0;
}

hipError_t launch_qk_fwd(const lq_qk_config* c, const QkTensors& t, int64_t M, hipStream_t s)
{
    const QkShape sh = qk_shape(c, &t, M, 1 << 20);
    return qk_run_all<false>(c, qk_args(c, t, M, sh), sh, s);
}

hipError_t launch_qk_bwd(const lq_qk_config* c, const QkTensors& t, int64_t M, uint8_t* work, hipStream_t s)
{
    const QkShape sh = qk_shape(c, &t, M, QK_MAX_GROUPS);
    QkArgs a = qk_args(c, t, M, sh);
    const bool dw = c->norm == LQ_NORM_RMS && t.dw[0];
    a.part = dw ? (float*)work : nullptr;
    hipError_t e = hipSuccess;
    if (M > 0) e = qk_run_all<true>(c, a, sh, s);
    if (e != hipSuccess || !dw) return e;
    hipLaunchKernelGGL(qk_weight_sum, dim3((2 * c->head_dim + 15) / 16), dim3(256), 0, s, (const float*)work, M > 0 ? (int)sh.grid : 0, c->head_dim, t.dw[0], t.dw[1]);
    return hipGetLastError();
}

}  // namespace lq
