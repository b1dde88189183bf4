// Norms before and after a block (lq_block.h): gradient.
#include <algorithm>

#include "lq_block.h"

namespace lq {

// Gradient.  With n = pre(h'), p = post(y) before their weights, r the reciprocal deviations:
//     G = dh' + r (dx a - mean(dx a) - n mean(dx a n)) ;  dh = alpha G ;  dy = r_y (G b - mean(G b) - p mean(G b p))       (the plain means with LQ_NORM_LAYER only)
// and the sums over the rows of a sequence of dx, dx n and G p, from which block_sums makes the gradients of modulation and weights.  A workgroup takes a chunk of rows,
// its groups of W wavefronts in turn; a and b are in the LDS.  At the end of a sequence or of the chunk the groups' sums are joined in the LDS and written to place chunk + s
// of the parts, which no other pair of chunk and sequence has (both rise from one pair to the next).
// 8192 rows of 1152, bf16: 26.5 us (4.3 TB/s) and 4.1 for block_sums; the registers allow two wavefronts a SIMD, which wait 38 % of their cycles.  The next row asked for ahead fits into them in bf16
// without spills and is slower: 32.0 us for 31.1 in all.
// TENSORS.  ALL: all inputs and results of rows are there, and read VEC values at a time.  SOME may be missing (the branches cost registers: 8192 rows of 1152, layer norm, 23.2 us where
// ALL takes 22.7).  LOOSE: any may be missing, and of any alignment.  SOME and LOOSE of one wavefront with four or five vectors, a bf16 branch and POST have 133 to 345 registers in scratch (8192 rows of
// 1152: without dh' 124 us, rows of 1153 136, ALL 32).
enum { ALL, SOME, LOOSE };
template <typename TH, typename TY, int VEC, int NV, int TENSORS, bool POST, bool MULTI, int THREADS>
__global__ void __launch_bounds__(THREADS) block_bwd_kernel(BlockArgs a)
{
    extern __shared__ v4f shared[];
    __shared__ float slots[64];
    constexpr bool ANY = TENSORS == LOOSE;
    const BlockTensors& t = a.t;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, W = MULTI ? a.waves : 1, group = wave / W, groups = waves / W;
    const int padded = (a.dim + VEC - 1) / VEC * VEC;
    float *la = (float*)shared, *lb = la + padded, *joined = lb + padded;  // a, b; [3][groups][padded] sums
    const Columns<VEC, NV, ANY> c(a.dim, threadIdx.x - group * W * 64, W * 64);
    RowSum<MULTI> sum{slots, waves, group * W, wave, W};
    int first = blockIdx.x * a.chunk;
    const int limit = min(first + a.chunk, (int)a.M);
    const bool has_dx = TENSORS == ALL || t.dx, has_y = TENSORS == ALL || t.y, has_dho = TENSORS == ALL || t.dho, want_dh = TENSORS == ALL || t.dh, want_dy = TENSORS == ALL || t.dy;
    const Sequences sequences(t);
    Raw<TH, VEC, ANY> rh[NV], rg[NV];
    Raw<TY, VEC, ANY> ry[NV], rx[NV];
    auto request = [&](int m) {
        if (has_dx) {
            c.fetch((const TH*)t.h + m * t.ldh, rh);
            c.fetch((const TY*)t.dx + m * t.lddx, rx);
        }
        if (has_y) c.fetch((const TY*)t.y + m * t.ldy, ry);
        if (has_dho) c.fetch((const TH*)t.dho + m * t.lddho, rg);
    };
    auto read_factor = [&](const float* l, int v, float (&f)[VEC]) {  // (past the row's end: the first)
        Raw<float, VEC, false> r;
        r.fetch(l + (c.have(v) > 0 ? c.at + v * c.step : 0));
        r.get(f);
    };
    while (first < limit) {
        int end;
        const int s = sequences.find(first, limit, end);
        if (s < 0) {
            first = end;
            continue;
        }
        for (int o = threadIdx.x * VEC; o < padded; o += blockDim.x * VEC) {
            float f[VEC];
            factor_a<VEC, ANY>(t, o, a.dim, s, f, o + VEC <= a.dim);
            Raw<float, VEC, false>::put(la + o, f);
            factor_b<VEC, ANY>(t, o, a.dim, s, f, o + VEC <= a.dim);
#pragma unroll
            for (int i = 0; i < VEC; ++i) f[i] = ANY && i >= a.dim - o ? 0.0f : f[i];
            Raw<float, VEC, false>::put(lb + o, f);
        }
        float s1[NV][VEC], s2[NV][VEC], s3[NV][VEC];
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int i = 0; i < VEC; ++i) s1[v][i] = s2[v][i] = s3[v][i] = 0.0f;
        __syncthreads();
#pragma unroll 1
        for (int base = first; base < end; base += groups) {
            const int row = base + group;
            const bool on = row < end;  // (of a row: all its wavefronts.  The others take part in the barriers with the last row's values, of which nothing is kept)
            if (!MULTI && !on) break;
            asm volatile("" ::: "memory");  // (a and b are read again for every row: kept in registers they would cost a wavefront's)
            request(min(row, end - 1));
            float n[NV][VEC], dx[NV][VEC], g[NV][VEC];
#pragma unroll
            for (int v = 0; v < NV; ++v) {
                if (has_dx) {
                    rh[v].get(n[v]);
                    rx[v].get(dx[v]);
                }
                if (has_dho) rg[v].get(g[v]);
                else
#pragma unroll
                    for (int i = 0; i < VEC; ++i) g[v][i] = 0.0f;
            }
            if (has_dx) {
                float r = 1.0f, u = 0.0f, w = 0.0f;
                if (a.pre != LQ_NORM_NONE) r = normalise<VEC, NV, ANY, MULTI>(a.pre, n, c, sum, a);
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float fa[VEC], tu = 0.0f, tw = 0.0f;
                    read_factor(la, v, fa);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        if (on) {
                            s1[v][i] += dx[v][i];
                            s2[v][i] = fmaf(dx[v][i], n[v][i], s2[v][i]);
                        }
                        dx[v][i] *= fa[i];
                        tu = fmaf(dx[v][i], n[v][i], tu);
                        tw += dx[v][i];
                    }
                    u += c.counted(v, tu);
                    w += c.counted(v, tw);
                }
                if (a.pre != LQ_NORM_NONE) {
                    sum(u, w);
                    u *= a.inv_dim * r;
                    w = a.pre == LQ_NORM_LAYER ? w * a.inv_dim * r : 0.0f;
                } else {
                    u = w = 0.0f;
                }
#pragma unroll
                for (int v = 0; v < NV; ++v)
#pragma unroll
                    for (int i = 0; i < VEC; ++i) g[v][i] += fmaf(r, dx[v][i], fmaf(-n[v][i], u, -w));
            }
            if (want_dh && on) {
                TH* o = (TH*)t.dh + row * t.lddh;
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float d[VEC];
#pragma unroll
                    for (int i = 0; i < VEC; ++i) d[i] = a.alpha * g[v][i];
                    c.put(o, v, d);
                }
            }
            if (has_y) {
                float p[NV][VEC], r = 1.0f, u = 0.0f, w = 0.0f;
#pragma unroll
                for (int v = 0; v < NV; ++v) ry[v].get(p[v]);
                if (POST) r = normalise<VEC, NV, ANY, MULTI>(a.post, p, c, sum, a);
#pragma unroll
                for (int v = 0; v < NV; ++v) {
                    float fb[VEC], tu = 0.0f, tw = 0.0f;
                    read_factor(lb, v, fb);
#pragma unroll
                    for (int i = 0; i < VEC; ++i) {
                        if (on) s3[v][i] = fmaf(g[v][i], p[v][i], s3[v][i]);
                        g[v][i] *= fb[i];
                        if (POST) {
                            tu = fmaf(g[v][i], p[v][i], tu);
                            tw += g[v][i];
                        }
                    }
                    u += c.counted(v, tu);
                    w += c.counted(v, tw);
                }
                if (POST) {
                    sum(u, w);
                    u *= a.inv_dim * r;
                    w = a.post == LQ_NORM_LAYER ? w * a.inv_dim * r : 0.0f;
#pragma unroll
                    for (int v = 0; v < NV; ++v)
#pragma unroll
                        for (int i = 0; i < VEC; ++i) g[v][i] = fmaf(r, g[v][i], fmaf(-p[v][i], u, -w));
                }
                if (want_dy && on) {
                    TY* o = (TY*)t.dy + row * t.lddy;
#pragma unroll
                    for (int v = 0; v < NV; ++v) c.put(o, v, g[v]);
                }
            }
        }
        if (a.part) {
            float* out = a.part + (size_t)(blockIdx.x + s) * 3 * a.dim;
            if (groups == 1) {
#pragma unroll
                for (int k = 0; k < 3; ++k)
#pragma unroll
                    for (int v = 0; v < NV; ++v)
                        Raw<float, VEC, true>::put_end(out + k * a.dim, c.at + v * c.step, a.dim, k == 0 ? s1[v] : k == 1 ? s2[v] : s3[v]);
            } else {
#pragma unroll
                for (int k = 0; k < 3; ++k)
#pragma unroll
                    for (int v = 0; v < NV; ++v)
                        if (c.have(v) > 0) Raw<float, VEC, false>::put(joined + (k * groups + group) * padded + c.at + v * c.step, k == 0 ? s1[v] : k == 1 ? s2[v] : s3[v]);
                __syncthreads();
                for (int o = threadIdx.x * VEC; o < 3 * padded; o += blockDim.x * VEC) {
                    const int k = o >= 2 * padded ? 2 : o >= padded ? 1 : 0, col = o - k * padded;
                    float y[VEC], z[VEC];
                    read<VEC, false>(joined + k * groups * padded, col, padded, y);
                    for (int w = 1; w < groups; ++w) {
                        read<VEC, false>(joined + (k * groups + w) * padded, col, padded, z);
#pragma unroll
                        for (int i = 0; i < VEC; ++i) y[i] += z[i];
                    }
                    Raw<float, VEC, true>::put_end(out + k * a.dim, col, a.dim, y);
                }
            }
        }
        if (end < limit) __syncthreads();  // (a, b and the sums have been read)
        first = end;
    }
}

// Where a sequence's parts begin and end
__device__ __forceinline__ void parts_of(const BlockArgs& a, int s, int& c0, int& c1)
{
    int begin = 0, end = (int)a.M;
    if (a.t.offsets) {
        begin = max(a.t.offsets[s], 0);
        end = min(a.t.offsets[s + 1], (int)a.M);
    }
    c0 = begin / a.chunk;
    c1 = begin < end ? (end - 1) / a.chunk + 1 : c0;
}
// Sums over a sequence's parts in a fixed order, COLS columns of one of the three sums to a workgroup, 64 / COLS parts at a time to a wavefront:
//     dshift = sum dx ;  dscale = w_pre sum dx n ;  dgate = w_post sum G p
// `team` wavefronts share the parts of a sequence out and are joined in a tree; the workgroup's teams take the sequences from blockIdx.z on in turn.  FUSED (one workgroup sees all sequences): also
//     dw_pre = sum over sequences of (1 + scale) sum dx n ;  dw_post = sum of gate sum G p
// Otherwise raw: the last two sums without the weights, for block_weight_sums.  The modulation of a sequence without rows, and the weights beside it, are not used: whatever they hold, it adds nothing
// (times a sum of zero, an infinity would be no number).
// In raw such a sequence has a zero with a sign, which no sum that begins with one without is: block_weight_sums need not look at the offsets (us with them / without, gradient of
// 1000 rows of 1152 in 100 sequences 27.6 / 25.7, of 8192 in 1000 98.1 / 78.3).
constexpr uint32_t NO_ROWS = 0x80000000u;
template <bool FUSED, int COLS>
__global__ void __launch_bounds__(1024) block_sums(BlockArgs a, int team, float* raw)
{
    __shared__ float sh[16][64];
    const BlockTensors& t = a.t;
    const int k = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, col = blockIdx.x * COLS + lane % COLS;
    const int member = wave % team, teams = waves / team;
    const lq_mod_out& o = k == 0 ? t.dshift : k == 1 ? t.dscale : t.dgate;
    const lq_mod& f = k == 1 ? t.scale : t.gate;
    const float* w = k == 0 ? nullptr : k == 1 ? t.w_pre : t.w_post;
    float* dw = k == 0 ? nullptr : k == 1 ? t.dw_pre : t.dw_post;
    float total = 0.0f;
    for (int base = blockIdx.z * teams; base < t.S; base += gridDim.z * teams) {
        const int s = base + wave / team;
        float y = 0.0f;
        bool rows = false;
        if (s < t.S && col < a.dim) {
            int c0, c1;
            parts_of(a, s, c0, c1);
            rows = c0 < c1;
            const float* p = a.part + (size_t)s * 3 * a.dim + k * a.dim + col;
#pragma unroll 8
            for (int i = c0 + member * (64 / COLS) + lane / COLS; i < c1; i += team * (64 / COLS)) y += p[(size_t)i * 3 * a.dim];
        }
#pragma unroll
        for (int half = 32; half >= COLS; half /= 2) y += __shfl_xor(y, half);
        if (team > 1) {
            sh[wave][lane] = y;
            __syncthreads();
            for (int half = team / 2; half > 0; half /= 2) {
                if (member < half) sh[wave][lane] += sh[wave + half][lane];
                __syncthreads();
            }
            y = sh[wave][lane];
        }
        if (member == 0 && lane < COLS && s < t.S && col < a.dim) {
            if (o.p) o.p[s * o.ld + col] = rows && w ? y * w[col] : y;
            if (FUSED) {
                const float g = rows && f.p ? f.p[s * f.ld + col] : k == 1 ? 0.0f : 1.0f;
                total = fmaf(k == 1 ? 1.0f + g : g, y, total);
            } else if (raw && k) {
                raw[((size_t)s * 2 + k - 1) * a.dim + col] = rows ? y : __uint_as_float(NO_ROWS);
            }
        }
        if (team > 1) __syncthreads();
    }
    if (!FUSED || !dw) return;
    __syncthreads();
    sh[wave][lane] = total;  // (zero but in the teams' first wavefronts)
    __syncthreads();
    for (int half = waves / 2; half > 0; half /= 2) {
        if (wave < half) sh[wave][lane] += sh[wave + half][lane];
        __syncthreads();
    }
    if (wave == 0 && lane < COLS && col < a.dim) dw[col] = sh[0][lane];
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
            const float u = raw[((size_t)s * 2 + k) * a.dim + col], g = f.p ? f.p[s * f.ld + col] : k == 0 ? 0.0f : 1.0f;
            y += __float_as_uint(u) == NO_ROWS ? 0.0f : u * (k == 0 ? 1.0f + g : g);
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

// Rows of a workgroup, of which each leaves parts of the sums, and its groups of W wavefronts.  One row up to 512 of them (us: 18 rows of 1528 11.5, four at a time 21.3; 64 of 1152 11.2 / 16.5; 500 of
// 2240, both norms, 21.8 / 25.2; but 1000 of 1152 20.9 / 19.7).  Above, eight wavefronts to a compute unit are what the registers allow (by the number of workgroups of eight, 8192 rows of 1152, bf16:
// 256 31.7, 512 36.9, 768 42.5), with four rows at least or one to each group.
constexpr int FEW_ROWS = 512;
static int block_bwd_groups(int W, int chunk) { return std::min(W > 3 ? 1 : 8 / W, chunk); }
static int block_bwd_chunk(const lq_block_config* c, int64_t M)
{
    if (M <= FEW_ROWS) return 1;
    const int W = block_shape(c->dim, false, false).W, groups = block_bwd_groups(W, 8), workgroups = 256 * (W * groups > 4 ? 1 : 2);
    return std::max((int)((M + workgroups - 1) / workgroups), std::min(groups, 4));
}
// (no chunk leaves more than FEW_ROWS parts and one for each sequence: a workspace serves smaller batches, too)
static size_t block_parts(const lq_block_config* c, int64_t M, int64_t S) { return (size_t)(std::min<int64_t>(M, FEW_ROWS) + S) * 3 * c->dim; }
size_t block_work_bytes(const lq_block_config* c, int64_t M, int64_t S)
{
    return align256(block_parts(c, M, S) * 4) + align256((size_t)S * 2 * c->dim * 4);
}

template <typename TH, typename TY, int NV, int TENSORS, bool POST, bool MULTI, int THREADS>
static hipError_t block_bwd_launch(const BlockArgs& a, hipStream_t s)
{
    const int groups = block_bwd_groups(a.waves, a.chunk);
    const dim3 grid((unsigned)((a.M + a.chunk - 1) / a.chunk)), block(64 * a.waves * groups);
    const size_t lds = (size_t)(groups > 1 ? 3 * groups + 2 : 2) * ((a.dim + 3) / 4 * 4) * 4;  // (up to 140 KB)
    if (lds > 65280) {
        const hipError_t e = allow_lds<block_bwd_kernel<TH, TY, 4, NV, TENSORS, POST, MULTI, THREADS>>(143360);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL((block_bwd_kernel<TH, TY, 4, NV, TENSORS, POST, MULTI, THREADS>), grid, block, lds, s, a);
    return hipGetLastError();
}
template <typename TH, typename TY, int NV, int TENSORS, bool POST>
static hipError_t block_bwd_run(const BlockArgs& a, hipStream_t s)
{
    if constexpr (NV == 3 || NV == 4)
        if (a.waves > 8) return block_bwd_launch<TH, TY, NV, TENSORS, POST, true, 1024>(a, s);
    if constexpr (NV >= 3)
        if (a.waves > 1) return block_bwd_launch<TH, TY, NV, TENSORS, POST, true, 512>(a, s);
    return block_bwd_launch<TH, TY, NV, TENSORS, POST, false, 512>(a, s);
}
template <typename TH, typename TY, int TENSORS, bool POST>
static hipError_t block_bwd_vectors(const BlockArgs& a, const BlockShape& sh, hipStream_t s)
{
    switch (sh.NV) {
        case 1: return block_bwd_run<TH, TY, 1, TENSORS == ALL ? SOME : TENSORS, POST>(a, s);  // (short rows have registers to spare)
        case 2: return block_bwd_run<TH, TY, 2, TENSORS == ALL ? SOME : TENSORS, POST>(a, s);
        case 3: return block_bwd_run<TH, TY, 3, TENSORS, POST>(a, s);
        case 4: return block_bwd_run<TH, TY, 4, TENSORS, POST>(a, s);
        default: return block_bwd_run<TH, TY, 5, TENSORS, POST>(a, s);
    }
}
template <typename TH, typename TY>
static hipError_t block_bwd_types(const BlockArgs& a, const BlockShape& sh, hipStream_t s)
{
    const bool post = a.t.y && a.post != LQ_NORM_NONE;
    const BlockTensors& t = a.t;
    if (sh.any) return post ? block_bwd_vectors<TH, TY, LOOSE, true>(a, sh, s) : block_bwd_vectors<TH, TY, LOOSE, false>(a, sh, s);
    if (!t.dx || !t.dho || !t.y || !t.dh || !t.dy) return post ? block_bwd_vectors<TH, TY, SOME, true>(a, sh, s) : block_bwd_vectors<TH, TY, SOME, false>(a, sh, s);
    return post ? block_bwd_vectors<TH, TY, ALL, true>(a, sh, s) : block_bwd_vectors<TH, TY, ALL, false>(a, sh, s);
}
hipError_t launch_block_bwd(const lq_block_config* c, const BlockTensors& t, int64_t M, uint8_t* work, hipStream_t s)
{
    const bool sums = t.dgate.p || t.dscale.p || t.dshift.p || t.dw_pre || t.dw_post, weights = t.dw_pre || t.dw_post;
    BlockArgs a = block_args(c, t, M);
    a.chunk = block_bwd_chunk(c, M);
    a.part = sums ? (float*)work : nullptr;
    hipError_t e = hipSuccess;
    if (M > 0) {
        const BlockShape sh = block_shape(c->dim, !block_fours(c, t, M), M <= FEW_ROWS);
        a.waves = sh.W;
        e = c->h_dtype == LQ_BF16   ? block_bwd_types<__bf16, __bf16>(a, sh, s)
            : c->y_dtype == LQ_BF16 ? block_bwd_types<float, __bf16>(a, sh, s)
                                    : block_bwd_types<float, float>(a, sh, s);
    }
    if (e != hipSuccess || !sums) return e;
    const int64_t each = (M + a.chunk - 1) / a.chunk / t.S;  // parts of a sequence
    // eight parts to a lane, as far as sixteen wavefronts go; from eight parts on pieces of 16 columns, where a wavefront takes four parts at a time (us with the gradient: 300 fp32 rows in 7 sequences
    // 18.5, by 64 columns 19.0; 64 rows of 1152 11.1 / 11.9)
    const bool narrow = each >= 8;
    int team = 1;
    while (team < 16 && team * (narrow ? 32 : 8) < each) team *= 2;
    const unsigned cols = (unsigned)((c->dim + 63) / 64), pieces = narrow ? (unsigned)((c->dim + 15) / 16) : cols;
    // a launch of its own for the weights' sums costs 4 us; without it the workgroups of all sequences are one
    if (weights && t.S * team <= 64) {
        while (team > 1 && t.S * team > 16) team /= 2;
        if (narrow) hipLaunchKernelGGL((block_sums<true, 16>), dim3(pieces, 3), dim3(1024), 0, s, a, team, nullptr);
        else hipLaunchKernelGGL((block_sums<true, 64>), dim3(pieces, 3), dim3(1024), 0, s, a, team, nullptr);
        return hipGetLastError();
    }
    float* raw = weights ? (float*)(work + align256(block_parts(c, M, t.S) * 4)) : nullptr;
    int waves = team;
    while (waves < 16 && waves < team * t.S) waves *= 2;
    const int64_t teams = waves / team, turns = (t.S + teams - 1) / teams;
    const dim3 grid(pieces, 3, (unsigned)(turns < 4096 ? turns : 4096));
    if (narrow) hipLaunchKernelGGL((block_sums<false, 16>), grid, dim3(64 * waves), 0, s, a, team, raw);
    else hipLaunchKernelGGL((block_sums<false, 64>), grid, dim3(64 * waves), 0, s, a, team, raw);
    e = hipGetLastError();
    if (e != hipSuccess || !weights) return e;
    hipLaunchKernelGGL(block_weight_sums, dim3(cols, 2), dim3(1024), 0, s, a, (const float*)raw);
    return hipGetLastError();
}

}  // namespace lq
