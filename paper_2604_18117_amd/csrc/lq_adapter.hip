// Low-rank adapters of many requests beside a shared projection:
//     Y[m] = Yin[m] + s_a (X[m] A_a^T) B_a^T ,  a = ids[m]
// and its gradients.  A grouping of the batch (the plan) lists the rows adapter by adapter in tiles of up to 64 rows; T = X A^T is held in
// fp32 in the order of the plan ("inter").
//   adapter_shrink   T = X A^T        a workgroup per half tile, its wavefronts share out K and add up in the LDS
//   adapter_expand   Y = Yin + s T B^T  a wavefront per tile and 64 columns
//   adapter_wgrad    dB = s dY^T T, dA = (s dY B)^T X   contraction over the rows of an adapter, in groups of tiles
// The backward runs the first two on the transposed factors (dT = dY B, dX = dXin + s dT A).  No atomics: every sum has a fixed order.
#include "lq_internal.h"

namespace lq {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

constexpr int TILE = 64;          // rows of a tile
constexpr int PLAN_CHUNK = 1024;  // rows that a workgroup of the plan's kernels sorts

// ---- plan ---------------------------------------------------------------------------------

AdapterPlanLayout adapter_plan_layout(int64_t M, int slots)
{
    AdapterPlanLayout l;
    l.chunks = (int)((M + PLAN_CHUNK - 1) / PLAN_CHUNK);
    l.tiles = (int)(M / TILE) + slots + 1;  // every adapter, and the rows without one, may leave one tile that is not full
    size_t o = 0;
    l.off_base = o, o += align256((size_t)(slots + 2) * 4);
    l.off_tbase = o, o += align256((size_t)(slots + 2) * 4);
    l.off_tiles = o, o += align256((size_t)l.tiles * 16);
    l.off_rows = o, o += align256((size_t)M * 4);
    l.off_total = o, o += align256((size_t)(slots + 1) * 4);
    l.off_hist = o, o += align256((size_t)(slots + 1) * l.chunks * 4);
    l.total = o;
    return l;
}

struct PlanPtrs {
    int *base, *tbase, *rows, *total, *hist;
    int4* tiles;
};
static PlanPtrs plan_ptrs(const AdapterPlanLayout& l, uint8_t* p)
{
    return {(int*)(p + l.off_base), (int*)(p + l.off_tbase), (int*)(p + l.off_rows), (int*)(p + l.off_total), (int*)(p + l.off_hist),
            (int4*)(p + l.off_tiles)};
}

__device__ __forceinline__ int slot_of(int id, int slots) { return (unsigned)id < (unsigned)slots ? id : slots; }

// rows of each adapter in each chunk of the batch; hist is [adapter][chunk]
__global__ void __launch_bounds__(256) adapter_plan_count(const int* ids, int M, int slots, int chunks, PlanPtrs p)
{
    __shared__ int h[1025];
    for (int s = threadIdx.x; s <= slots; s += 256) h[s] = 0;
    __syncthreads();
    const int m0 = blockIdx.x * PLAN_CHUNK;
    for (int i = threadIdx.x; i < PLAN_CHUNK && m0 + i < M; i += 256) atomicAdd(&h[slot_of(ids[m0 + i], slots)], 1);
    __syncthreads();
    for (int s = threadIdx.x; s <= slots; s += 256) p.hist[(size_t)s * chunks + blockIdx.x] = h[s];
}

// exclusive sum of v over the workgroup's threads (n of them, a multiple of 64, up to 1024), and the total
__device__ __forceinline__ int block_scan(int v, int* lds, int* total)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, nw = blockDim.x >> 6;
    int x = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 63) lds[w] = x;
    __syncthreads();
    int before = 0, sum = 0;
    for (int i = 0; i < nw; ++i) {
        const int t = lds[i];
        if (i < w) before += t;
        sum += t;
    }
    *total = sum;
    return before + x - v;
}

// hist becomes the number of an adapter's rows in earlier chunks; a workgroup per adapter
__global__ void __launch_bounds__(256) adapter_plan_scan(int chunks, PlanPtrs p)
{
    __shared__ int lds[16];
    int* h = p.hist + (size_t)blockIdx.x * chunks;
    int run = 0;
    for (int c0 = 0; c0 < chunks; c0 += 256) {
        const int c = c0 + (int)threadIdx.x, v = c < chunks ? h[c] : 0;
        int sum;
        const int e = block_scan(v, lds, &sum);
        if (c < chunks) h[c] = run + e;
        run += sum;
    }
    if (threadIdx.x == 0) p.total[blockIdx.x] = run;
}

// first row and first tile of every adapter, and the tiles {first row, rows, adapter, 0} (rows 0: none); one workgroup
__global__ void __launch_bounds__(1024) adapter_plan_tiles(int slots, int cap, PlanPtrs p)
{
    __shared__ int lds[16], tb[1026], bs[1026];
    int row = 0, tile = 0;
    for (int s0 = 0; s0 <= slots; s0 += 1024) {
        const int s = s0 + (int)threadIdx.x, n = s <= slots ? p.total[s] : 0;
        int sn, st;
        const int b = row + block_scan(n, lds, &sn), t = tile + block_scan((n + TILE - 1) / TILE, lds, &st);
        if (s <= slots) bs[s] = p.base[s] = b, tb[s] = p.tbase[s] = t;
        row += sn;
        tile += st;
    }
    if (threadIdx.x == 0) bs[slots + 1] = p.base[slots + 1] = row, tb[slots + 1] = p.tbase[slots + 1] = tile;
    __syncthreads();
    for (int t = threadIdx.x; t < cap; t += 1024) {
        int4 v = make_int4(0, 0, slots, 0);
        if (t < tile) {
            int lo = 0, hi = slots;  // the last adapter whose first tile is at or before t has it: later ones with the same first tile have rows, earlier have none
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (tb[mid] <= t) lo = mid;
                else hi = mid - 1;
            }
            const int r0 = bs[lo] + (t - tb[lo]) * TILE;
            v = make_int4(r0, min(TILE, bs[lo + 1] - r0), lo, 0);
        }
        p.tiles[t] = v;
    }
}

// rows in the order of their adapters, in their own order within one: the wavefronts take turns, and a lane's place among the 64 rows of a
// turn is the number of lower lanes with the same adapter (a ballot per bit of its number)
__global__ void __launch_bounds__(256) adapter_plan_rows(const int* ids, int M, int slots, int chunks, PlanPtrs p)
{
    __shared__ int next[1025];
    for (int s = threadIdx.x; s <= slots; s += 256) next[s] = p.base[s] + p.hist[(size_t)s * chunks + blockIdx.x];
    __syncthreads();
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int g = 0; g < PLAN_CHUNK / 64; ++g) {
        if ((g & 3) == w) {
            const int m = blockIdx.x * PLAN_CHUNK + g * 64 + lane;
            const bool ok = m < M;
            const int s = ok ? slot_of(ids[m], slots) : 0;
            unsigned long long same = __ballot(ok);
            for (int b = 0; b < 11; ++b) {
                const unsigned long long one = __ballot(s >> b & 1);
                same &= s >> b & 1 ? one : ~one;
            }
            const int at = next[s];
            if (ok) p.rows[at + __popcll(same & ((1ull << lane) - 1))] = m;
            // every lane has read before one writes
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
            if (ok && (same >> lane) == 1) next[s] = at + __popcll(same);  // the last lane of each adapter
        }
        __syncthreads();
    }
}

hipError_t launch_adapter_plan(int slots, const int32_t* ids, int64_t M, uint8_t* plan, hipStream_t s)
{
    const AdapterPlanLayout l = adapter_plan_layout(M, slots);
    const PlanPtrs p = plan_ptrs(l, plan);
    hipError_t e;
    if (l.chunks) {
        hipLaunchKernelGGL(adapter_plan_count, dim3(l.chunks), dim3(256), 0, s, ids, (int)M, slots, l.chunks, p);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    hipLaunchKernelGGL(adapter_plan_scan, dim3(slots + 1), dim3(256), 0, s, l.chunks, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(adapter_plan_tiles, dim3(1), dim3(1024), 0, s, slots, l.tiles, p);
    if ((e = hipGetLastError()) != hipSuccess || !l.chunks) return e;
    hipLaunchKernelGGL(adapter_plan_rows, dim3(l.chunks), dim3(256), 0, s, ids, (int)M, slots, l.chunks, p);
    return hipGetLastError();
}

// ---- terms --------------------------------------------------------------------------------

// An fp32 number as bf16 terms, each the leading bits of what the ones before leave (cut off, so that every difference is exact): two
// carry 16 bits of it, three all 24.
__device__ __forceinline__ uint32_t cut(float v) { return __float_as_uint(v) & 0xFFFF0000u; }
template <int TERMS>
__device__ __forceinline__ void split8(const float (&v)[8], v4i (&t)[TERMS])
{
    float r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = v[j];
#pragma unroll
    for (int k = 0; k < TERMS; ++k) {
        uint32_t c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // the last of two terms is rounded: 2^-17 of the value is left instead of 2^-16
            c[j] = cut(TERMS == 2 && k == 1 ? __uint_as_float(__float_as_uint(r[j]) + 0x8000u) : r[j]);
            r[j] -= __uint_as_float(c[j]);
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) t[k][d] = (int)__builtin_amdgcn_perm(c[2 * d + 1], c[2 * d], 0x07060302u);
    }
}
__device__ __forceinline__ v4f mfma(v4i a, v4i b, v4f c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

struct AdapterView {  // of the plan, and the pool's per-adapter numbers
    const int *rows, *tbase;
    const int4* tiles;
    const int32_t* ranks;
    const float* scales;
    int slots, rank, rp;  // rank of the arrays, and rounded up to 16
    int M;
};
__device__ __forceinline__ int rank_of(const AdapterView& v, int slot) { return slot < v.slots ? min(max(v.ranks[slot], 0), v.rank) : 0; }

// ---- T = X W^T ----------------------------------------------------------------------------

struct ShrinkArgs {
    AdapterView v;
    const void* X;  // rows of `depth` values
    const uint16_t* W;  // [adapter][rank][depth]
    float* T;       // [row of the plan][rp]
    int64_t ldx;
    int depth;
};

// A workgroup of 8 wavefronts: 32 rows of a tile, 16 * RT of the rank, the wavefronts' 64-deep pieces of K in turn.  A lane of the 16 x 16
// x 32 product holds 8 values of K; it reads 16 consecutive ones, the first and second half for two products, so that four lanes
// read 128 bytes of a row.
template <bool F32, int RT>
__global__ void __launch_bounds__(512) adapter_shrink(ShrinkArgs a)
{
    __shared__ float red[8][32][RT * 16];
    const int4 tile = a.v.tiles[blockIdx.x >> 1];
    const int h = (blockIdx.x & 1) * 32, n = min(tile.y - h, 32), rank = rank_of(a.v, tile.z), r0 = blockIdx.y * (RT * 16);
    if (n <= 0 || rank == 0) return;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    constexpr int XV = F32 ? 4 : 2, ES = F32 ? 4 : 2;
    const uint8_t* x[2];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt) {
        const int row = a.v.rows[tile.x + h + min(mt * 16 + i, n - 1)];
        x[mt] = (const uint8_t*)a.X + ((int64_t)row * a.ldx + q * 16) * ES;
    }
    const uint8_t* wt[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
        wt[rt] = (const uint8_t*)(a.W + ((int64_t)tile.z * a.v.rank + min(r0 + rt * 16 + i, a.v.rank - 1)) * a.depth + q * 16);
    v4f acc[2][RT];
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[mt][rt] = v4f{0, 0, 0, 0};
    for (int c = w; c < a.depth / 64; c += 8) {
        v4i xv[2][XV], wv[RT][2];
#pragma unroll
        for (int mt = 0; mt < 2; ++mt)
#pragma unroll
            for (int u = 0; u < XV; ++u) xv[mt][u] = ((const v4i*)(x[mt] + (int64_t)c * 64 * ES))[u];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int u = 0; u < 2; ++u) wv[rt][u] = ((const v4i*)(wt[rt] + (int64_t)c * 128))[u];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int mt = 0; mt < 2; ++mt) {
                if constexpr (F32) {
                    float v[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) v[j] = __int_as_float(xv[mt][2 * u + j / 4][j % 4]);
                    v4i t[3];
                    split8<3>(v, t);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int k = 2; k >= 0; --k) acc[mt][rt] = mfma(t[k], wv[rt][u], acc[mt][rt]);
                } else {
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) acc[mt][rt] = mfma(xv[mt][u], wv[rt][u], acc[mt][rt]);
                }
            }
    }
#pragma unroll
    for (int mt = 0; mt < 2; ++mt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int e = 0; e < 4; ++e) red[w][mt * 16 + q * 4 + e][rt * 16 + i] = acc[mt][rt][e];
    __syncthreads();
    for (int o = threadIdx.x; o < 32 * RT * 16; o += 512) {
        const int m = o / (RT * 16), r = o % (RT * 16);
        float t = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) t += red[k][m][r];
        if (m < n && r0 + r < a.v.rp) a.T[(int64_t)(tile.x + h + m) * a.v.rp + r0 + r] = r0 + r < rank ? t : 0.0f;
    }
}

// ---- Y = Yin + s T W^T ----------------------------------------------------------------------

struct ExpandArgs {
    AdapterView v;
    const float* T;
    const uint16_t* W;  // [adapter][width][rank]
    const void* Yin;    // or NULL: zeros
    void* Y;
    int64_t ldyin, ldy;
    int width;
    int in_place;
};

// 16 consecutive values of a row, as fp32
template <bool F32>
__device__ __forceinline__ void load16(const void* p, int64_t at, float (&v)[16])
{
    if constexpr (F32) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const v4f t = ((const v4f*)((const float*)p + at))[u];
#pragma unroll
            for (int e = 0; e < 4; ++e) v[4 * u + e] = t[e];
        }
    } else {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const v4i t = ((const v4i*)((const uint16_t*)p + at))[u];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[8 * u + 2 * e] = __uint_as_float((uint32_t)t[e] << 16);
                v[8 * u + 2 * e + 1] = __uint_as_float((uint32_t)t[e] & 0xFFFF0000u);
            }
        }
    }
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)  // round to nearest even
{
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    const v2bf v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
template <bool F32>
__device__ __forceinline__ void store16(void* p, int64_t at, const float (&v)[16])
{
    if constexpr (F32) {
#pragma unroll
        for (int u = 0; u < 4; ++u) ((v4f*)((float*)p + at))[u] = v4f{v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]};
    } else {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            v4i t;
#pragma unroll
            for (int e = 0; e < 4; ++e) t[e] = (int)pack_bf16(v[8 * u + 2 * e], v[8 * u + 2 * e + 1]);
            ((v4i*)((uint16_t*)p + at))[u] = t;
        }
    }
}

// A workgroup of 4 wavefronts: a tile, 64 columns each.  T's rows are the second operand, so that a lane's four sums are four columns of one
// row; the factor's rows are dealt to the four products so that these are 16 consecutive columns.
template <bool F32, int KS>
__global__ void __launch_bounds__(256) adapter_expand(ExpandArgs a)
{
    constexpr int TERMS = F32 ? 3 : 2;
    __shared__ v4i top[4][KS][TERMS][64];
    const int4 tile = a.v.tiles[blockIdx.x];
    const int n = tile.y, rank = rank_of(a.v, tile.z);
    if (n <= 0 || (rank == 0 && a.in_place)) return;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const int col = (blockIdx.y * 4 + w) * 64;
    const int subs = (n + 15) >> 4;
    if (rank > 0) {
        if (w < subs) {
            const float s = a.v.scales[tile.z];
            const float* T = a.T + (int64_t)(tile.x + min(w * 16 + i, n - 1)) * a.v.rp;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int k = ks * 32 + q * 8;
                float v[8];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const v4f t = *(const v4f*)(T + min(k, a.v.rp - 8) + 4 * u);
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[4 * u + e] = k < rank ? t[e] * s : 0.0f;
                }
                v4i t[TERMS];
                split8<TERMS>(v, t);
#pragma unroll
                for (int k2 = 0; k2 < TERMS; ++k2) top[w][ks][k2][lane] = t[k2];
            }
        }
        __syncthreads();
    }
    if (col >= a.width) return;
    // a lane's part of the factor: rows (i / 4) * 16 + 4 j + i % 4 of the 64, 8 values of the rank from 32 ks + 8 q on
    v4i wv[4][KS];
    if (rank > 0) {
        const uint16_t* W = a.W + ((int64_t)tile.z * a.width + col + (i >> 2) * 16 + (i & 3)) * a.v.rank;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int k = ks * 32 + q * 8, left = rank - k;  // values that the adapter has; the others are cleared whatever they hold
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                v4i t = *(const v4i*)(W + (int64_t)(4 * j) * a.v.rank + min(k, a.v.rank - 8));
#pragma unroll
                for (int d = 0; d < 4; ++d) t[d] = left >= 2 * d + 2 ? t[d] : left == 2 * d + 1 ? t[d] & 0xFFFF : 0;
                wv[j][ks] = t;
            }
        }
    }
#pragma unroll
    for (int sub = 0; sub < 4; ++sub) {
        if (sub >= subs) break;
        const int m = sub * 16 + i;
        const bool ok = m < n;
        const int64_t row = a.v.rows[tile.x + min(m, n - 1)];
        float y[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) y[e] = 0.0f;
        if (ok && a.Yin) load16<F32>(a.Yin, row * a.ldyin + col + q * 16, y);
        if (rank > 0) {
            v4f acc[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = v4f{0, 0, 0, 0};
#pragma unroll
            for (int ks = 0; ks < KS; ++ks)
#pragma unroll
                for (int k = TERMS - 1; k >= 0; --k) {
                    const v4i t = top[sub][ks][k][lane];
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] = mfma(wv[j][ks], t, acc[j]);
                }
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) y[4 * j + e] += acc[j][e];
        }
        if (ok) store16<F32>(a.Y, row * a.ldy + col + q * 16, y);
    }
}

// ---- gradients of the factors -----------------------------------------------------------------

// The factors transposed, zeros in the ranks that an adapter does not have: At [adapter][K][rank], Bt [adapter][rank][N].  64 x 64 squares
// through the LDS; adapters without rows are skipped.
__global__ void __launch_bounds__(256) adapter_transpose(AdapterView v, const uint16_t* A, const uint16_t* B, uint16_t* At, uint16_t* Bt, int N, int K)
{
    __shared__ uint16_t sq[64][65];
    const int slot = blockIdx.z;
    if (v.tbase[slot] == v.tbase[slot + 1]) return;
    const int rank = rank_of(v, slot), r0 = blockIdx.y * 64, kb = K / 64, tx = threadIdx.x & 63, ty = threadIdx.x >> 6;
    const bool isA = (int)blockIdx.x < kb;
    const int c0 = (isA ? (int)blockIdx.x : (int)blockIdx.x - kb) * 64;
    if (isA) {
        for (int y = ty; y < 64; y += 4)
            if (r0 + y < v.rank) sq[y][tx] = r0 + y < rank ? A[((int64_t)slot * v.rank + r0 + y) * K + c0 + tx] : 0;
        __syncthreads();
        for (int y = ty; y < 64; y += 4)
            if (r0 + tx < v.rank) At[((int64_t)slot * K + c0 + y) * v.rank + r0 + tx] = sq[tx][y];
    } else {
        for (int y = ty; y < 64; y += 4)
            if (r0 + tx < v.rank) sq[tx][y] = r0 + tx < rank ? B[((int64_t)slot * N + c0 + y) * v.rank + r0 + tx] : 0;
        __syncthreads();
        for (int y = ty; y < 64; y += 4)
            if (r0 + y < v.rank) Bt[((int64_t)slot * v.rank + r0 + y) * N + c0 + tx] = sq[y][tx];
    }
}

struct WgradArgs {
    AdapterView v;
    const float* T;  // [row of the plan][rp]
    const void* Q;   // rows of `width` values
    float* out;      // [adapter][rank * width]
    float* part;     // [2 * group + (0 | 1)][part_stride]
    int64_t ldq, part_stride;
    int width, per;  // per: tiles of a group
};

// out = s T^T Q over the rows of an adapter, for 128 columns of Q and 16 * RT of the rank.  The tiles of the plan are dealt to groups of `per`;
// an adapter that lies within a group is finished there, one that does not leaves a part in each (2 g where it has the group's first tile, 2 g + 1
// where it starts within), which adapter_wgrad_sum adds up.  The four wavefronts of a workgroup take tiles in turn.
// Both operands need 8 rows of one column in a lane: a lane loads 8 columns of 8 rows and pairs up the halves of the dwords, which gives
// the operands of 8 products, the c-th with columns 8 i + c.
// COLS_FIRST: the columns are the first operand (out is [rank][width], a lane's sums are consecutive columns), else the second ([width][rank]).
template <bool F32, int RT, bool COLS_FIRST>
__global__ void __launch_bounds__(256) adapter_wgrad(WgradArgs a)
{
    constexpr int QT = F32 ? 3 : 1;
    __shared__ v4f red[2][8 * RT][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const int c0 = blockIdx.x * 128, r0 = blockIdx.z * (RT * 16), g = blockIdx.y;
    const int col = c0 + 8 * i < a.width ? c0 + 8 * i : c0;  // (lanes past the width repeat the first columns and store nothing)
    const int last = min((g + 1) * a.per, a.v.tbase[a.v.slots]);
    for (int t0 = g * a.per; t0 < last;) {
        const int slot = a.v.tiles[t0].z, s0 = a.v.tbase[slot], s1 = a.v.tbase[slot + 1], t1 = min(s1, last);
        v4f acc[8][RT];
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) acc[c][rt] = v4f{0, 0, 0, 0};
        for (int t = t0 + w; t < t1; t += 4) {
            const int4 tile = a.v.tiles[t];
            for (int h = 0; h < tile.y; h += 32) {
                const int left = tile.y - h - q * 8;  // rows that this lane's 8 have
                v4i qr[8][F32 ? 2 : 1];
                float tv[RT][8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int pos = tile.x + (j < left ? h + q * 8 + j : tile.y - 1);
                    const int64_t row = a.v.rows[pos];
                    if constexpr (F32) {
#pragma unroll
                        for (int u = 0; u < 2; ++u) qr[j][u] = ((const v4i*)((const float*)a.Q + row * a.ldq + col))[u];
                    } else {
                        qr[j][0] = *(const v4i*)((const uint16_t*)a.Q + row * a.ldq + col);
                    }
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) {
                        const int r = min(r0 + rt * 16 + i, a.v.rp - 1);
                        const float t1v = a.T[(int64_t)pos * a.v.rp + r];
                        tv[rt][j] = j < left ? t1v : 0.0f;
                    }
                }
                v4i tt[RT][3];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) split8<3>(tv[rt], tt[rt]);
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    v4i qt[QT];
                    if constexpr (F32) {
                        float v[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) v[j] = __int_as_float(qr[j][c / 4][c % 4]);
                        split8<3>(v, qt);
                    } else {
#pragma unroll
                        for (int d = 0; d < 4; ++d)
                            qt[0][d] = (int)__builtin_amdgcn_perm((uint32_t)qr[2 * d + 1][0][c / 2], (uint32_t)qr[2 * d][0][c / 2],
                                                                   c & 1 ? 0x07060302u : 0x05040100u);
                    }
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int k = 2; k >= 0; --k)
#pragma unroll
                            for (int u = QT - 1; u >= 0; --u)
                                if (k + u < 3)  // (what is left out is below 2^-24 of the product)
                                    acc[c][rt] = COLS_FIRST ? mfma(qt[u], tt[rt][k], acc[c][rt]) : mfma(tt[rt][k], qt[u], acc[c][rt]);
                }
            }
        }
        // wavefronts 2 and 3 to 0 and 1, then 1 to 0
        __syncthreads();
#pragma unroll
        for (int d = 2; d >= 1; d >>= 1) {
            if (w >= d && w < 2 * d)
#pragma unroll
                for (int c = 0; c < 8; ++c)
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) red[w - d][c * RT + rt][lane] = acc[c][rt];
            __syncthreads();
            if (w < d)
#pragma unroll
                for (int c = 0; c < 8; ++c)
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) acc[c][rt] += red[w][c * RT + rt][lane];
            __syncthreads();
        }
        if (w == 0) {
            const int rank = rank_of(a.v, slot);
            const float s = a.v.scales[slot];
            const bool whole = s0 >= g * a.per && s1 <= (g + 1) * a.per;
            float* out = whole ? a.out + (int64_t)slot * a.v.rank * a.width : a.part + (int64_t)(2 * g + (s0 > g * a.per)) * a.part_stride;
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                if constexpr (COLS_FIRST) {
                    const int r = r0 + rt * 16 + i;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int k = c0 + 8 * (q * 4 + e);
                        if (r < a.v.rank && k < a.width)
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                v4f o;
#pragma unroll
                                for (int c = 0; c < 4; ++c) o[c] = r < rank ? acc[4 * u + c][rt][e] * s : 0.0f;
                                *(v4f*)(out + (int64_t)r * a.width + k + 4 * u) = o;
                            }
                    }
                } else {
                    const int r = r0 + rt * 16 + q * 4;
                    if (r < a.v.rank && c0 + 8 * i < a.width)
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            v4f o;
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[e] = r + e < rank ? acc[c][rt][e] * s : 0.0f;
                            *(v4f*)(out + (int64_t)(c0 + 8 * i + c) * a.v.rank + r) = o;
                        }
                }
            }
        }
        t0 = t1;
    }
}

// Adapters without rows: zeros.  Adapters of more than one group: their parts in the order of the groups.  nb, na: quads of dB and dA.
__global__ void __launch_bounds__(256) adapter_wgrad_sum(AdapterView v, const float* part, int64_t part_stride, int per, v4f* dB, v4f* dA, int64_t nb, int64_t na)
{
    const int slot = blockIdx.y, s0 = v.tbase[slot], s1 = v.tbase[slot + 1];
    const int g0 = s0 / per, g1 = (s1 - 1) / per;
    if (s0 < s1 && g0 == g1) return;
    for (int64_t o = (int64_t)blockIdx.x * 256 + threadIdx.x; o < nb + na; o += (int64_t)gridDim.x * 256) {
        v4f t = {0, 0, 0, 0};
        if (s0 < s1)
            for (int g = g0; g <= g1; ++g) t += ((const v4f*)(part + (int64_t)(2 * g + (s0 > g * per)) * part_stride))[o];
        if (o < nb) dB[(int64_t)slot * nb + o] = t;
        else dA[(int64_t)slot * na + o - nb] = t;
    }
}

__global__ void __launch_bounds__(256) adapter_zero(v4f* p, int64_t n)
{
    for (int64_t o = (int64_t)blockIdx.x * 256 + threadIdx.x; o < n; o += (int64_t)gridDim.x * 256) p[o] = v4f{0, 0, 0, 0};
}

// ---- host ---------------------------------------------------------------------------------------

// Ranks are dealt to workgroups in groups of up to 64.
struct RankSplit {
    int groups, rt;
};
static RankSplit rank_split(int rank)
{
    const int tiles = (rank + 15) / 16, groups = (tiles + 3) / 4;
    return {groups, (tiles + groups - 1) / groups};
}

AdapterWorkLayout adapter_work_layout(const lq_adapter_config* c, int64_t M)
{
    AdapterWorkLayout l;
    const int64_t rp = (c->rank + 15) / 16 * 16;
    const int tiles = (int)(M / TILE) + c->slots + 1;
    // groups of tiles: about 1024 workgroups over all column blocks, so that the card is full and there are few parts
    const int64_t units = ((c->N + 127) / 128 + (c->K + 127) / 128) * rank_split(c->rank).groups;
    int64_t groups = 1024 / units;
    groups = groups < 1 ? 1 : groups;
    l.per = (int)((tiles + groups - 1) / groups);
    l.per = l.per < 4 ? 4 : l.per;
    l.groups = (tiles + l.per - 1) / l.per;
    l.part_stride = (int64_t)c->rank * (c->N + c->K);
    size_t o = 0;
    l.off_dT = o, o += align256((size_t)M * rp * 4);
    l.off_At = o, o += align256((size_t)c->slots * c->rank * c->K * 2);
    l.off_Bt = o, o += align256((size_t)c->slots * c->rank * c->N * 2);
    l.off_part = o, o += l.groups > 1 ? align256((size_t)(2 * l.groups) * l.part_stride * 4) : 0;
    l.total = o;
    return l;
}

static AdapterView view_of(const lq_adapter_config* c, const lq_adapter_pool* pool, const uint8_t* plan, int64_t M)
{
    const AdapterPlanLayout l = adapter_plan_layout(M, c->slots);
    return {(const int*)(plan + l.off_rows), (const int*)(plan + l.off_tbase), (const int4*)(plan + l.off_tiles), pool->ranks, pool->scales,
            c->slots, c->rank, (c->rank + 15) / 16 * 16, (int)M};
}

static hipError_t run_shrink(const ShrinkArgs& a, bool f32, int tiles, hipStream_t s)
{
    const RankSplit rs = rank_split(a.v.rank);
    const dim3 grid(2 * tiles, rs.groups), block(512);
#define SHRINK(RT) \
    if (f32) hipLaunchKernelGGL((adapter_shrink<true, RT>), grid, block, 0, s, a); \
    else hipLaunchKernelGGL((adapter_shrink<false, RT>), grid, block, 0, s, a)
    switch (rs.rt) {
        case 1: SHRINK(1); break;
        case 2: SHRINK(2); break;
        case 3: SHRINK(3); break;
        default: SHRINK(4); break;
    }
#undef SHRINK
    return hipGetLastError();
}

static hipError_t run_expand(const ExpandArgs& a, bool f32, int tiles, hipStream_t s)
{
    const dim3 grid(tiles, (a.width + 255) / 256), block(256);
#define EXPAND(KS) \
    if (f32) hipLaunchKernelGGL((adapter_expand<true, KS>), grid, block, 0, s, a); \
    else hipLaunchKernelGGL((adapter_expand<false, KS>), grid, block, 0, s, a)
    switch ((a.v.rank + 31) / 32) {
        case 1: EXPAND(1); break;
        case 2: EXPAND(2); break;
        case 3: EXPAND(3); break;
        default: EXPAND(4); break;
    }
#undef EXPAND
    return hipGetLastError();
}

template <bool COLS_FIRST>
static hipError_t run_wgrad(const WgradArgs& a, bool f32, int groups, hipStream_t s)
{
    const RankSplit rs = rank_split(a.v.rank);
    const dim3 grid((a.width + 127) / 128, groups, rs.groups), block(256);
    if constexpr (COLS_FIRST) {
        if (f32) {
            switch (rs.rt) {
                case 1: hipLaunchKernelGGL((adapter_wgrad<true, 1, true>), grid, block, 0, s, a); break;
                case 2: hipLaunchKernelGGL((adapter_wgrad<true, 2, true>), grid, block, 0, s, a); break;
                case 3: hipLaunchKernelGGL((adapter_wgrad<true, 3, true>), grid, block, 0, s, a); break;
                default: hipLaunchKernelGGL((adapter_wgrad<true, 4, true>), grid, block, 0, s, a); break;
            }
            return hipGetLastError();
        }
    }
    switch (rs.rt) {
        case 1: hipLaunchKernelGGL((adapter_wgrad<false, 1, COLS_FIRST>), grid, block, 0, s, a); break;
        case 2: hipLaunchKernelGGL((adapter_wgrad<false, 2, COLS_FIRST>), grid, block, 0, s, a); break;
        case 3: hipLaunchKernelGGL((adapter_wgrad<false, 3, COLS_FIRST>), grid, block, 0, s, a); break;
        default: hipLaunchKernelGGL((adapter_wgrad<false, 4, COLS_FIRST>), grid, block, 0, s, a); break;
    }
    return hipGetLastError();
}

hipError_t launch_adapter_fwd(const lq_adapter_config* c, const uint8_t* plan, const lq_adapter_pool* pool, const void* X, int64_t ldx,
                              const void* Yin, int64_t ldyin, void* Y, int64_t ldy, int64_t M, uint8_t* inter, hipStream_t s)
{
    const AdapterView v = view_of(c, pool, plan, M);
    const int tiles = adapter_plan_layout(M, c->slots).tiles;
    hipError_t e = run_shrink({v, X, (const uint16_t*)pool->A, (float*)inter, ldx, (int)c->K}, c->x_dtype == LQ_F32, tiles, s);
    if (e != hipSuccess) return e;
    return run_expand({v, (const float*)inter, (const uint16_t*)pool->B, Yin, Y, ldyin, ldy, (int)c->N, Yin == Y && ldyin == ldy}, false, tiles, s);
}

hipError_t launch_adapter_bwd(const lq_adapter_config* c, const uint8_t* plan, const lq_adapter_pool* pool, const void* X, int64_t ldx,
                              const uint8_t* inter, const void* dY, int64_t lddy, const void* dXin, int64_t lddxin, void* dX, int64_t lddx,
                              float* dA, float* dB, int64_t M, uint8_t* work, hipStream_t s)
{
    const AdapterView v = view_of(c, pool, plan, M);
    const AdapterWorkLayout l = adapter_work_layout(c, M);
    const int tiles = adapter_plan_layout(M, c->slots).tiles;
    const bool f32 = c->x_dtype == LQ_F32;
    float* dT = (float*)(work + l.off_dT);
    uint16_t *At = (uint16_t*)(work + l.off_At), *Bt = (uint16_t*)(work + l.off_Bt);
    float* part = (float*)(work + l.off_part);
    hipError_t e;
    hipLaunchKernelGGL(adapter_transpose, dim3((unsigned)((c->K + c->N) / 64), (c->rank + 63) / 64, c->slots), dim3(256), 0, s, v,
                       (const uint16_t*)pool->A, (const uint16_t*)pool->B, At, Bt, (int)c->N, (int)c->K);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    if ((e = run_shrink({v, dY, Bt, dT, lddy, (int)c->N}, false, tiles, s)) != hipSuccess) return e;
    // dA before dX: X may be read before a caller's dX, which may be its own buffer for dXin only, is written
    if ((e = run_wgrad<false>({v, (const float*)inter, dY, dB, part, lddy, l.part_stride, (int)c->N, l.per}, false, l.groups, s)) != hipSuccess) return e;
    if ((e = run_wgrad<true>({v, dT, X, dA, part + (int64_t)c->rank * c->N, ldx, l.part_stride, (int)c->K, l.per}, f32, l.groups, s)) != hipSuccess) return e;
    const int64_t nb = (int64_t)c->rank * c->N / 4, na = (int64_t)c->rank * c->K / 4;
    int64_t blocks = (nb + na + 1023) / 1024;
    blocks = blocks > 1024 ? 1024 : blocks;
    hipLaunchKernelGGL(adapter_wgrad_sum, dim3((unsigned)blocks, c->slots), dim3(256), 0, s, v, part, l.part_stride, l.per, (v4f*)dB, (v4f*)dA, nb, na);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    return run_expand({v, dT, At, dXin, dX, lddxin, lddx, (int)c->K, dXin == dX && lddxin == lddx}, f32, tiles, s);
}

hipError_t launch_adapter_zero(const lq_adapter_config* c, float* dA, float* dB, hipStream_t s)
{
    const int64_t na = (int64_t)c->slots * c->rank * c->K / 4, nb = (int64_t)c->slots * c->rank * c->N / 4;
    hipLaunchKernelGGL(adapter_zero, dim3((unsigned)((na + 255) / 256 < 4096 ? (na + 255) / 256 : 4096)), dim3(256), 0, s, (v4f*)dA, na);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(adapter_zero, dim3((unsigned)((nb + 255) / 256 < 4096 ? (nb + 255) / 256 : 4096)), dim3(256), 0, s, (v4f*)dB, nb);
    return hipGetLastError();
}

}  // namespace lq
