// Norms before and after a block (lq_block.h): forward.
#include <algorithm>

#include "lq_block.h"

namespace lq {

// Forward.  A group of W wavefronts takes `chunk` rows one after another, the next row already requested.  MULTI: the group is the workgroup; otherwise a workgroup
// has four of one wavefront.  8192 rows of 1152, bf16: 15.3 us, 4.9 TB/s; 16384 of 2240, fp32 stream and both norms: 92 us, 4.8 TB/s.
template <typename TH, typename TY, int VEC, int NV, bool ANY, bool POST, bool MULTI, int THREADS>
__global__ void __launch_bounds__(THREADS) block_fwd_kernel(BlockArgs a)
{
    __shared__ float slots[MULTI ? 64 : 1];
    const BlockTensors& t = a.t;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const Columns<VEC, NV, ANY> c(a.dim, MULTI ? threadIdx.x : lane, MULTI ? blockDim.x : 64);
    const int group = MULTI ? blockIdx.x : blockIdx.x * 4 + wave;
    RowSum<MULTI> sum{slots, waves, 0, wave, waves};
    int row = group * a.chunk;
    const int limit = min(row + a.chunk, (int)a.M);
    if (row >= limit) return;
    const Sequences sequences(t);
    Raw<TH, VEC, ANY> rh[NV];
    Raw<TY, VEC, ANY> ry[NV];
    auto request = [&](int m) {
        c.fetch((const TH*)t.h + m * t.ldh, rh);
        if (t.y) c.fetch((const TY*)t.y + m * t.ldy, ry);
    };
    request(row);
    while (row < limit) {
        int end;
        const int s = sequences.find(row, limit, end);
        if (s < 0) {
            row = end;
            if (row < limit) request(row);
            continue;
        }
        float fa[NV][VEC], fb[NV][VEC], fs[NV][VEC];
#pragma unroll
        for (int v = 0; v < NV; ++v) {
            const int at = c.at + v * c.step;
            factor_a<VEC, ANY>(t, at, a.dim, s, fa[v], v < NV - 1);
            factor_b<VEC, ANY>(t, at, a.dim, s, fb[v], v < NV - 1);
#pragma unroll
            for (int i = 0; i < VEC; ++i) fs[v][i] = 0.0f;
            if (t.shift.p) read<VEC, ANY>(t.shift.p + s * t.shift.ld, at, a.dim, fs[v], v < NV - 1);
        }
        for (; row < end; ++row) {
            float h[NV][VEC], y[NV][VEC];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                rh[v].get(h[v]);
                if (t.y) ry[v].get(y[v]);
            }
            if (row + 1 < limit) request(row + 1);
            if (t.y) {
                if (POST) normalise<VEC, NV, ANY, MULTI>(a.post, y, c, sum, a);
                TH* o = (TH*)t.ho + row * t.ldho;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) h[v][i] = fmaf(a.alpha, h[v][i], fb[v][i] * y[v][i]);
                    c.put(o, v, h[v]);
                }
            }
            if (t.x) {
                if (a.pre != LQ_NORM_NONE) normalise<VEC, NV, ANY, MULTI>(a.pre, h, c, sum, a);
                TY* o = (TY*)t.x + row * t.ldx;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
#pragma unroll
                    for (int i = 0; i < VEC; ++i) h[v][i] = fmaf(h[v][i], fa[v][i], fs[v][i]);
                    c.put(o, v, h[v]);
                }
            }
        }
    }
}

// ---- host ---------------------------------------------------------------------------------------

// Rows of a group, one after another: so many that all groups are on the card at once; where that is more than eight, four for rows of several wavefronts, whose factors come again for every group
// but which wait for each other (us: 4000 rows of 4608 by 8, 500 groups 40.0, by 4 42.6, by 2 51.4, by 1 65.0; 2000 of 2240, fp32 and both norms, by 2 16.1, by 1 19.6, by 4 17.1; 16384 of them by 4 91.6,
// by 6 93.6, by 16 97.7), sixteen at most for others (8192 of 1152 by 8 16.8, by 4 15.5, by 2 18.2).
static int block_fwd_chunk(int64_t M, int W, int waves)  // waves: that a compute unit holds
{
    const int64_t groups = 256 * (int64_t)std::max(waves / W, 1), all = (M + groups - 1) / groups;
    return (int)(all <= 8 ? all : W > 1 && M <= (1 << 20) ? 4 : std::min<int64_t>(all, 16));  // (a launch stays below 2^32 threads)
}
template <typename TH, typename TY, int NV, bool ANY, bool POST, bool MULTI, int THREADS>
static void block_fwd_launch(BlockArgs a, int W, hipStream_t s)
{
    constexpr auto kernel = block_fwd_kernel<TH, TY, 4, NV, ANY, POST, MULTI, THREADS>;
    static const int waves = [] {
        int n = 0;
        constexpr int threads = THREADS == 1024 ? 1024 : 256;
        if (hipOccupancyMaxActiveBlocksPerMultiprocessor(&n, kernel, threads, 0) == hipSuccess && n > 0) return n * threads / 64;
        (void)hipGetLastError();  // (not the launch's)
        return 8;
    }();
    a.chunk = block_fwd_chunk(a.M, W, waves);
    const int64_t groups = (a.M + a.chunk - 1) / a.chunk;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(MULTI ? groups : (groups + 3) / 4)), dim3(MULTI ? 64 * W : 256), 0, s, a);
}
template <typename TH, typename TY, int NV, bool ANY, bool POST>
static void block_fwd_run(const BlockArgs& a, int W, hipStream_t s)
{
    if constexpr (NV == 3 || NV == 4)
        if (W > 8) return block_fwd_launch<TH, TY, NV, ANY, POST, true, 1024>(a, W, s);
    if constexpr (NV >= 3)
        if (W > 1) return block_fwd_launch<TH, TY, NV, ANY, POST, true, 512>(a, W, s);
    block_fwd_launch<TH, TY, NV, ANY, POST, false, 256>(a, W, s);
}
template <typename TH, typename TY, bool ANY, bool POST>
static void block_fwd_vectors(const BlockArgs& a, const BlockShape& sh, hipStream_t s)
{
    switch (sh.NV) {
        case 1: return block_fwd_run<TH, TY, 1, ANY, POST>(a, sh.W, s);
        case 2: return block_fwd_run<TH, TY, 2, ANY, POST>(a, sh.W, s);
        case 3: return block_fwd_run<TH, TY, 3, ANY, POST>(a, sh.W, s);
        case 4: return block_fwd_run<TH, TY, 4, ANY, POST>(a, sh.W, s);
        default: return block_fwd_run<TH, TY, 5, ANY, POST>(a, sh.W, s);
    }
}
template <typename TH, typename TY>
static void block_fwd_types(const BlockArgs& a, const BlockShape& sh, hipStream_t s)
{
    const bool post = a.t.y && a.post != LQ_NORM_NONE;
    if (sh.any) post ? block_fwd_vectors<TH, TY, true, true>(a, sh, s) : block_fwd_vectors<TH, TY, true, false>(a, sh, s);
    else post ? block_fwd_vectors<TH, TY, false, true>(a, sh, s) : block_fwd_vectors<TH, TY, false, false>(a, sh, s);
}
hipError_t launch_block_fwd(const lq_block_config* c, const BlockTensors& t, int64_t M, hipStream_t s)
{
    const BlockShape sh = block_shape(c->dim, !block_fours(c, t, M), true);
    const BlockArgs a = block_args(c, t, M);
    if (c->h_dtype == LQ_BF16) block_fwd_types<__bf16, __bf16>(a, sh, s);
    else if (c->y_dtype == LQ_BF16) block_fwd_types<float, __bf16>(a, sh, s);
    else block_fwd_types<float, float>(a, sh, s);
    return hipGetLastError();
}

}  // namespace lq
