// Low-rank adapters of many requests beside a shared projection:
//     Y[m] = Yin[m] + s_a (X[m] A_a^T) B_a^T ,  a = ids[m]
// and its gradients.  A grouping of the batch (the plan) lists the rows adapter by adapter in tiles of up to 64 rows; T = X A^T is held in
// fp32 in the order of the plan ("inter").
//   forward    adapter_shrink    T = X A^T             a workgroup per 16 or 32 rows of a tile; its wavefronts share out K and add up in the LDS
//              adapter_expand    Y = Yin + s T B^T     a workgroup per tile and a few times 128 columns (single tokens: adapter_expand_few)
//   backward   adapter_shrink    dT = dY B
//              adapter_wgrad     dB = s dY^T T, dA = (s dT)^T X    contraction over the rows of an adapter, in groups of tiles
//              adapter_bwd_last  dX = dXin + s dT A as adapter_expand does it, and what is left of the sums of dA and dB
// The products are far below the matrix unit's rate: all of it is bound by memory and latency.  The backward has the factors in the other order than
// its products want them; they are turned in registers, 8 x 8 at a time (transposed copies beforehand cost 8 us of a step of 8192 x 1152 -> 3456).
// No atomics on memory: every sum has a fixed order, and T and Y of a row do not depend on the other rows.
#include "lq_internal.h"

#include <type_traits>

namespace lq {

typedef float v4f __attribute__((ext_vector_type(4)));
typedef int v4i __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));

constexpr int TILE = 64;          // rows of a tile
constexpr int PLAN_CHUNK = 1024;  // rows that a workgroup of the plan's kernels sorts

// ---- plan ---------------------------------------------------------------------------------

// The batch sorted by adapter, stably: counts, a scan over adapters and chunks, every row to its place.  Bound by the round trips of a few launches or of one.
// The rows of tile t are at 64 t of `rows`, not behind those of the tile before, so that a kernel asks for a tile and for its rows at once (what lies
// past a tile's last row is never used).

AdapterPlanLayout adapter_plan_layout(int64_t M, int slots)
{
    AdapterPlanLayout l;
    l.chunks = (int)((M + PLAN_CHUNK - 1) / PLAN_CHUNK);
    l.tiles = (int)(M / TILE) + slots + 1;  // every adapter, and the rows without one, may leave one tile that is not full
    size_t o = BLOB_HEADER;
    l.off_base = o, o += align256((size_t)(slots + 2) * 4);
    l.off_tbase = o, o += align256((size_t)(slots + 2) * 4);
    l.off_tiles = o, o += align256((size_t)l.tiles * 16);
    l.off_rows = o, o += align256((size_t)l.tiles * TILE * 4);
    l.off_total = o, o += align256((size_t)(slots + 1) * 4);
    l.off_hist = o, o += align256((size_t)(slots + 1) * l.chunks * 4);
    l.total = o;
    return l;
}

struct PlanPtrs {
    uint32_t* head;
    int *base, *tbase, *rows, *total, *hist;
    int4* tiles;
};
static PlanPtrs plan_ptrs(const AdapterPlanLayout& l, uint8_t* p)
{
    return {(uint32_t*)p, (int*)(p + l.off_base), (int*)(p + l.off_tbase), (int*)(p + l.off_rows), (int*)(p + l.off_total), (int*)(p + l.off_hist),
            (int4*)(p + l.off_tiles)};
}

__device__ __forceinline__ int slot_of(int id, int slots) { return (unsigned)id < (unsigned)slots ? id : slots; }

// rows of each adapter in each chunk of the batch; hist is [adapter][chunk].  The plan is nobody's until the last of its kernels has run.
__global__ void __launch_bounds__(256) adapter_plan_count(const int* ids, int M, int slots, int chunks, PlanPtrs p)
{
    __shared__ int h[1025];
    write_tag(p.head, BlobTag{});
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

// The tiles {first row, rows, adapter, 0} (rows 0: none), from first rows and first tiles in the LDS, by 1024 threads.
__device__ __forceinline__ void write_tiles(int slots, int cap, int tiles, const int* bs, const int* tb, int4* out)
{
    for (int t = threadIdx.x; t < cap; t += 1024) {
        int4 v = make_int4(0, 0, slots, 0);
        if (t < tiles) {
            int lo = 0, hi = slots;  // the last adapter whose first tile is at or before t has it: later ones with the same first tile have rows, earlier have none
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (tb[mid] <= t) lo = mid;
                else hi = mid - 1;
            }
            const int r0 = bs[lo] + (t - tb[lo]) * TILE;
            v = make_int4(r0, min(TILE, bs[lo + 1] - r0), lo, 0);
        }
        out[t] = v;
    }
}

// first row and first tile of every adapter, and the tiles; one workgroup
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
    write_tiles(slots, cap, tile, bs, tb, p.tiles);
}

// The lanes of a wavefront (of those in `ok`) with the same adapter s < 2048: a ballot per bit of its number.
__device__ __forceinline__ unsigned long long same_lanes(int s, bool ok, int bits)
{
    unsigned long long same = __ballot(ok);
    for (int b = 0; b < bits; ++b) {
        const unsigned long long one = __ballot(s >> b & 1);
        same &= s >> b & 1 ? one : ~one;
    }
    return same;
}

// rows in the order of their adapters, in their own order within one: the wavefronts take turns, and a lane's place among the 64 rows of a
// turn is the number of lower lanes with the same adapter (a ballot per bit of its number)
__global__ void __launch_bounds__(256) adapter_plan_rows(const int* ids, int M, int slots, int chunks, PlanPtrs p, BlobTag tag)
{
    __shared__ int next[1025];
    write_tag(p.head, tag);
    for (int s = threadIdx.x; s <= slots; s += 256) next[s] = p.tbase[s] * TILE + p.hist[(size_t)s * chunks + blockIdx.x];
    __syncthreads();
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int g = 0; g < PLAN_CHUNK / 64; ++g) {
        if ((g & 3) == w) {
            const int m = blockIdx.x * PLAN_CHUNK + g * 64 + lane;
            const bool ok = m < M;
            const int s = ok ? slot_of(ids[m], slots) : 0;
            const unsigned long long same = same_lanes(s, ok, 11);
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

// The whole plan in one workgroup: its 16 wavefronts take consecutive sixteenths of the batch, count their rows of each adapter (twice: for the adapters'
// first rows, then on the way to every row's place).
constexpr int PLAN_ONE = 8192;  // rows up to which it is taken (us, 32 adapters: 64 rows 5.1, 8192 13.7, 16384 23.3; four launches 17.3)
__global__ void __launch_bounds__(1024) adapter_plan_one(const int* ids, int M, int slots, int bits, int cap, PlanPtrs p, BlobTag tag)
{
    write_tag(p.head, tag);
    extern __shared__ int mem[];  // first rows, first tiles (slots + 2 each), then [wavefront][adapter] counts of 16 bits
    __shared__ int lds[16];
    int *bs = mem, *tb = mem + slots + 2;
    uint16_t* count = (uint16_t*)(mem + 2 * (slots + 2));
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, per = ((M + 1023) >> 10) << 6, m0 = w * per, m1 = min(M, m0 + per);
    for (int o = threadIdx.x; o < 16 * (slots + 1); o += 1024) count[o] = 0;
    __syncthreads();
    uint16_t* mine = count + w * (slots + 1);
    for (int m = m0; m < m1; m += 64) {
        const bool ok = m + lane < m1;
        const int s = ok ? slot_of(ids[m + lane], slots) : 0;
        const unsigned long long same = same_lanes(s, ok, bits);
        if (ok && (same >> lane) == 1) mine[s] += (uint16_t)__popcll(same);  // the last lane of each adapter
    }
    __syncthreads();
    int row = 0, tile = 0;
    for (int s0 = 0; s0 <= slots; s0 += 1024) {
        const int s = s0 + (int)threadIdx.x;
        int n = 0;
        if (s <= slots)
            for (int k = 0; k < 16; ++k) {  // counts become the rows of earlier wavefronts
                const int c = count[k * (slots + 1) + s];
                count[k * (slots + 1) + s] = (uint16_t)n;
                n += c;
            }
        int sn, st;
        const int b = row + block_scan(n, lds, &sn), t = tile + block_scan((n + TILE - 1) / TILE, lds, &st);
        if (s <= slots) bs[s] = p.base[s] = b, tb[s] = p.tbase[s] = t;
        row += sn;
        tile += st;
    }
    if (threadIdx.x == 0) bs[slots + 1] = p.base[slots + 1] = row, tb[slots + 1] = p.tbase[slots + 1] = tile;
    __syncthreads();
    write_tiles(slots, cap, tile, bs, tb, p.tiles);
    for (int m = m0; m < m1; m += 64) {
        const bool ok = m + lane < m1;
        const int s = ok ? slot_of(ids[m + lane], slots) : 0;
        const unsigned long long same = same_lanes(s, ok, bits);
        const int at = mine[s];
        if (ok) p.rows[tb[s] * TILE + at + __popcll(same & ((1ull << lane) - 1))] = m + lane;
        // every lane has read before one writes
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (ok && (same >> lane) == 1) mine[s] = (uint16_t)(at + __popcll(same));
    }
}

hipError_t launch_adapter_plan(int slots, const int32_t* ids, int64_t M, uint8_t* plan, hipStream_t s)
{
    const AdapterPlanLayout l = adapter_plan_layout(M, slots);
    const PlanPtrs p = plan_ptrs(l, plan);
    if (M <= PLAN_ONE) {
        int bits = 1;
        while (slots >> bits) ++bits;
        hipLaunchKernelGGL(adapter_plan_one, dim3(1), dim3(1024), (2 * (slots + 2)) * 4 + 16 * (slots + 1) * 2, s, ids, (int)M, slots, bits, l.tiles, p,
                           plan_tag(M, slots));
        return hipGetLastError();
    }
    hipError_t e;
    hipLaunchKernelGGL(adapter_plan_count, dim3(l.chunks), dim3(256), 0, s, ids, (int)M, slots, l.chunks, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(adapter_plan_scan, dim3(slots + 1), dim3(256), 0, s, l.chunks, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(adapter_plan_tiles, dim3(1), dim3(1024), 0, s, slots, l.tiles, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(adapter_plan_rows, dim3(l.chunks), dim3(256), 0, s, ids, (int)M, slots, l.chunks, p, plan_tag(M, slots));
    return hipGetLastError();
}

// ---- terms --------------------------------------------------------------------------------

// An fp32 number as three bf16 terms, each the leading bits of what the ones before leave (cut off, so that every difference is exact): they
// carry all 24 bits of it.  (Two, enough for the rounding of a bf16 output, lose the sum where adapter and projection cancel.)  INF: of an infinity the
// first term is one and nothing is left (without, what is left is not a number, and so is every sum that it enters).
__device__ __forceinline__ float cut(uint32_t bits) { return __uint_as_float(bits & 0xFFFF0000u); }
template <bool INF>
__device__ __forceinline__ void split8(const float (&v)[8], v4i (&t)[3])
{
    float r[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = v[j];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
        uint32_t c[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            c[j] = __float_as_uint(r[j]);
            if (k < 2) r[j] = INF && k == 0 && __builtin_isinf(r[j]) ? 0.0f : r[j] - cut(c[j]);
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) t[k][d] = (int)__builtin_amdgcn_perm(c[2 * d + 1], c[2 * d], 0x07060302u);
    }
}
// Where such terms meet an infinity, a later term of zero would make it not a number: it becomes the least number with the first one's sign (2^-126; of
// a zero it stays zero).
__device__ __forceinline__ void fill8(v4i (&t)[3])
{
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int h = 0; h < 32; h += 16) {
            const uint32_t first = (uint32_t)t[0][d] >> h & 0xFFFFu;
#pragma unroll
            for (int k = 1; k < 3; ++k)
                if ((first & 0x7FFFu) && !((uint32_t)t[k][d] >> h & 0x7FFFu)) t[k][d] = (int)(((uint32_t)t[k][d] & ~(0xFFFFu << h)) | ((first & 0x8000u) | 0x80u) << h);
        }
}
// Whether a wavefront's sums hold something that is not a number.
template <int A, int B>
__device__ __forceinline__ bool not_numbers(const v4f (&acc)[A][B])
{
    bool nan = false;
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
        for (int b = 0; b < B; ++b)
#pragma unroll
            for (int e = 0; e < 4; e += 2) nan |= __builtin_isunordered(acc[a][b][e], acc[a][b][e + 1]);
    return __any(nan);
}
__device__ __forceinline__ v4f mfma(v4i a, v4i b, v4f c)
{
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, a), __builtin_bit_cast(v8bf, b), c, 0, 0, 0);
}

// Column e of a block of 8 rows of 8 bf16 values, as the 8 consecutive values that a product takes.
__device__ __forceinline__ v4i column(const v4i* rows, int e)
{
    v4i t;
#pragma unroll
    for (int d = 0; d < 4; ++d)
        t[d] = (int)__builtin_amdgcn_perm((uint32_t)rows[2 * d + 1][e / 2], (uint32_t)rows[2 * d][e / 2], e & 1 ? 0x07060302u : 0x05040100u);
    return t;
}

struct AdapterView {  // of the plan, and the pool's per-adapter numbers
    const uint32_t* head;  // its two words for the kernels
    const int *rows, *tbase;
    const int4* tiles;
    const int32_t* ranks;
    const float* scales;
    int slots, rank, rp;  // rank of the arrays, and rounded up to 16
    int M, cap;           // rows; entries of `tiles`
};
// Whether the plan is one for these M rows and slots (of another one, or of memory that holds none, the rows would be numbers past the batch's).  Asked
// where a tile comes in anyway, in the same round trip: ask_together keeps the comparison behind both loads.
__device__ __forceinline__ uint2 plan_words(const AdapterView& v) { return *(const uint2*)v.head; }
__device__ __forceinline__ void ask_together() { __builtin_amdgcn_sched_barrier(0); }
__device__ __forceinline__ bool planned(const AdapterView& v, const uint2& is)
{
    return ((is.x ^ (uint32_t)v.M) | (is.y ^ (PLAN_SLOTS + (uint32_t)v.slots))) == 0;
}
__device__ __forceinline__ int rank_of(const AdapterView& v, int slot) { return slot < v.slots ? min(max(v.ranks[slot], 0), v.rank) : 0; }

// ---- T = X W^T ----------------------------------------------------------------------------

struct ShrinkArgs {
    AdapterView v;
    const void* X;  // rows of `depth` values
    const uint16_t* W;  // [adapter][rank][depth], or [adapter][depth][rank]
    float* T;       // [row of the plan][rp]
    int64_t ldx;
    int depth;
};

// The rows of a tile have to be there now: keeps their loads before what depends on the tile itself, so that one round trip brings both.
#define TOGETHER(ROWS) \
    _Pragma("unroll") for (int& row : ROWS) asm("" : "+v"(row))

// Orders the LDS accesses of one wavefront on memory of its own (they complete in order; the compiler must not move them either).
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A wavefront's piece of a product: 64 values of K of 16 * MT rows of X and 16 * RT of the factor.  The 16 x 16 x 32 product wants 16 rows in 16
// consecutive lanes; read like that from memory, every 16 bytes are a cache line of their own (40 us for 8191 x 2240, rank 128, whatever was
// in flight).  So 8 (fp32: 16) lanes read a row's 128 (256) consecutive bytes, and the rows go through the wavefront's part of the LDS: unit p of 16
// bytes of row r stands at r * units + (p ^ r % 16), free of bank conflicts both ways (the turned
// form's writes, two ways, and the stores of the sums at the end, four, are not: 19 % of the LDS's cycles, turned 27 %).
// TW: the factor is given as [depth][rank]; a lane reads blocks of 8 x 8 and turns them on the way to the LDS.
template <bool F32, bool TW, int MT, int RT>
struct ShrinkPiece {
    static constexpr int XU = F32 ? 16 : 8;            // units of a row of X
    static constexpr int BLOCKS = (RT + 3) / 4;        // TW: blocks of 8 x 8 of a lane
    static constexpr int XL = MT * 16 * XU / 64, WL = TW ? 8 * BLOCKS : RT * 16 * 8 / 64, WP = TW ? BLOCKS : WL;
    static constexpr int UNITS = MT * 16 * XU + RT * 16 * 8;
    v4i x[XL], w[WL];
    static __device__ __forceinline__ int place(int r, int p) { return MT * 16 * XU + r * 8 + (p ^ ((r + (r >> 3)) & 7)); }
    __device__ __forceinline__ void fetch(const uint8_t* const (&xp)[XL], const uint8_t* const (&wp)[WP], int64_t c, int rank)
    {
#pragma unroll
        for (int u = 0; u < XL; ++u) x[u] = *(const v4i*)(xp[u] + c * (XU * 16));
#pragma unroll
        for (int u = 0; u < WL; ++u) w[u] = TW ? *(const v4i*)(wp[u / 8] + (c * 64 + u % 8) * (rank * 2)) : *(const v4i*)(wp[TW ? 0 : u] + c * 128);
    }
    __device__ __forceinline__ void put(v4i* lds, int lane) const
    {
#pragma unroll
        for (int u = 0; u < XL; ++u) {
            const int r = u * (64 / XU) + lane / XU, p = lane % XU;
            lds[r * XU + (p ^ (r & (XU - 1)))] = x[u];
        }
        if constexpr (TW) {
#pragma unroll
            for (int k = 0; k < BLOCKS; ++k) {
                const int b = lane + 64 * k;
                if (b < 16 * RT)
#pragma unroll
                    for (int e = 0; e < 8; ++e) lds[place(b % (2 * RT) * 8 + e, b / (2 * RT))] = column(w + 8 * k, e);
            }
        } else {
#pragma unroll
            for (int u = 0; u < WL; ++u) lds[place(u * 8 + lane / 8, lane % 8)] = w[u];
        }
    }
    template <bool INF>
    static __device__ __forceinline__ void multiply(const v4i* lds, int i, int q, v4f (&acc)[MT][RT])
    {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            v4i wv[RT];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) wv[rt] = lds[place(rt * 16 + i, u * 4 + q)];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const v4i* row = lds + (mt * 16 + i) * XU;
                if constexpr (F32) {
                    float v[8];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const v4i r = row[(2 * (u * 4 + q) + h) ^ i];
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[4 * h + j] = __int_as_float(r[j]);
                    }
                    v4i t[3];
                    split8<INF>(v, t);
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                        for (int k = 2; k >= 0; --k) acc[mt][rt] = mfma(t[k], wv[rt], acc[mt][rt]);
                } else {
                    const v4i x = row[(u * 4 + q) ^ (i & 7)];
#pragma unroll
                    for (int rt = 0; rt < RT; ++rt) acc[mt][rt] = mfma(x, wv[rt], acc[mt][rt]);
                }
            }
        }
    }
};

// A workgroup of 8 wavefronts: 16 * MT rows of a tile, 16 * RT of the rank; the wavefronts take the pieces of K in turn, the next ones (up to four, as
// the registers allow) requested before the present one is multiplied, and add up in the LDS.  T's bits depend on the row, the factor and K alone.
// Bound by a wavefront's chain of round trips and by what a compute unit's loads bring in, rows and factor alike: us and TB/s of X, traced, 8192 x 1152 rank 32
// 7.8 and 2.4, dY 8192 x 3456 rank 32 26-27 and 2.2, 8191 x 2240 rank 128 30-35 and 1.1 (92 MB past the L2s for 39); of the 26, X alone takes 20 and the factor
// alone 16 (each with the other's loads left out).  64 rows to a workgroup halve the factor's part and the workgroups: 9.8 for 8.5.
template <bool F32, bool TW, int MT, int RT>
__global__ void __launch_bounds__(512) adapter_shrink(ShrinkArgs a)
{
    typedef ShrinkPiece<F32, TW, MT, RT> Piece;
    constexpr int PARTS = TILE / (16 * MT);  // workgroups of a tile
    constexpr int UNITS = Piece::XL + Piece::WL, AHEAD = UNITS <= 6 ? 4 : UNITS <= 14 && !(TW && MT == 2 && RT == 4) ? 2 : 1;
    extern __shared__ v4i lds[];             // a piece per wavefront; then [wavefront][row][rank] sums
    const int4 tile = a.v.tiles[blockIdx.x / PARTS];
    const uint2 is = plan_words(a.v);
    const int h = (blockIdx.x % PARTS) * (16 * MT), r0 = blockIdx.y * (RT * 16);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const uint8_t *xp[Piece::XL], *wp[Piece::WP];
    int rows[Piece::XL];
#pragma unroll
    for (int u = 0; u < Piece::XL; ++u) rows[u] = a.v.rows[(int)(blockIdx.x / PARTS) * TILE + h + u * (64 / Piece::XU) + lane / Piece::XU];
    ask_together();
    TOGETHER(rows);
    const int n = min(tile.y - h, 16 * MT);
    if ((n <= 0) | (tile.z >= a.v.slots) | !planned(a.v, is)) return;
    auto point = [&](const int (&rows)[Piece::XL], int slot) {
        const int first = __builtin_amdgcn_readfirstlane(rows[0]);
#pragma unroll
        for (int u = 0; u < Piece::XL; ++u) {
            const int row = u * (64 / Piece::XU) + lane / Piece::XU < n ? rows[u] : first;
            xp[u] = (const uint8_t*)a.X + (int64_t)row * a.ldx * (F32 ? 4 : 2) + lane % Piece::XU * 16;
        }
        // (ranks past the pool's are read from its last and not stored)
        if constexpr (TW) {
#pragma unroll
            for (int k = 0; k < Piece::BLOCKS; ++k) {
                const int b = lane + 64 * k, block = min(b / (2 * RT), 7), r = min(r0 + b % (2 * RT) * 8, a.v.rank - 8);
                wp[k] = (const uint8_t*)(a.W + ((int64_t)slot * a.depth + block * 8) * a.v.rank + r);
            }
        } else {
#pragma unroll
            for (int u = 0; u < Piece::WL; ++u)
                wp[u] = (const uint8_t*)(a.W + ((int64_t)slot * a.v.rank + min(r0 + u * 8 + lane / 8, a.v.rank - 1)) * a.depth) + lane % 8 * 16;
        }
    };
    point(rows, tile.z);
    v4f acc[MT][RT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) acc[mt][rt] = v4f{0, 0, 0, 0};
    const int pieces = a.depth / 64;
    v4i* mine = lds + w * Piece::UNITS;
    Piece p[AHEAD];
#pragma unroll
    for (int d = 0; d < AHEAD; ++d)
        if (w + 8 * d < pieces) p[d].fetch(xp, wp, w + 8 * d, a.v.rank);
    const int rank = rank_of(a.v, tile.z);
    if (rank == 0) return;
    for (int c0 = w; c0 < pieces; c0 += 8 * AHEAD) {
#pragma unroll
        for (int d = 0; d < AHEAD; ++d) {
            const int c = c0 + 8 * d;
            if (c >= pieces) break;
            wave_sync();
            p[d].put(mine, lane);
            wave_sync();
            if (c + 8 * AHEAD < pieces) p[d].fetch(xp, wp, c + 8 * AHEAD, a.v.rank);
            Piece::template multiply<false>(mine, i, q, acc);
        }
    }
    // Sums that are not a number: once more, for an X with infinities.  Nothing is ahead here, and nothing is kept for it: its rows are looked up again.
    if constexpr (F32)
        if (not_numbers(acc)) {
            int at = blockIdx.x / PARTS, slot = tile.z;
            asm volatile("" : "+s"(at), "+s"(slot));
#pragma unroll
            for (int u = 0; u < Piece::XL; ++u) rows[u] = a.v.rows[at * TILE + h + u * (64 / Piece::XU) + lane / Piece::XU];
            point(rows, slot);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) acc[mt][rt] = v4f{0, 0, 0, 0};
            for (int c = w; c < pieces; c += 8) {
                Piece again;
                again.fetch(xp, wp, c, a.v.rank);
                wave_sync();
                again.put(mine, lane);
                wave_sync();
                Piece::template multiply<true>(mine, i, q, acc);
            }
        }
    constexpr int ROW = RT * 16, ALL = MT * 16 * ROW;
    float* red = (float*)lds;
    __syncthreads();
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int e = 0; e < 4; ++e) red[w * ALL + (mt * 16 + q * 4 + e) * ROW + rt * 16 + i] = acc[mt][rt][e];
    __syncthreads();
    for (int o = threadIdx.x; o < ALL; o += 512) {
        const int m = o / ROW, r = r0 + o % ROW;
        float t = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) t += red[k * ALL + o];
        if (m < n && r < a.v.rp) a.T[(int64_t)(tile.x + h + m) * a.v.rp + r] = r < rank ? t : 0.0f;
    }
}

// ---- Y = Yin + s T W^T ----------------------------------------------------------------------

struct ExpandArgs {
    AdapterView v;
    const float* T;
    const uint16_t* W;  // [adapter][width][rank], or [adapter][rank][width]
    const void* Yin;    // or NULL: zeros
    void* Y;
    int64_t ldyin, ldy;
    int width;
    int in_place;
    int per;              // pieces of 128 columns of a workgroup
    unsigned runs;        // workgroups of a tile
    unsigned unit_magic;  // 2^32 / (rank / 8), rounded up; 0 for rank 8
};

// 8 consecutive values of a row as they lie in memory, at a uniform base and a lane's offset of OFF bytes: with 32 bits an access needs one register
// for its address.
template <bool F32, typename OFF>
struct Row8 {
    v4i v[F32 ? 2 : 1];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int u = 0; u < (F32 ? 2 : 1); ++u) v[u] = v4i{0, 0, 0, 0};
    }
    __device__ __forceinline__ void fetch(const uint8_t* base, OFF off)
    {
#pragma unroll
        for (int u = 0; u < (F32 ? 2 : 1); ++u) v[u] = ((const v4i*)(base + off))[u];
    }
    __device__ __forceinline__ float get(int j) const
    {
        if constexpr (F32) return __int_as_float(v[j / 4][j % 4]);
        else return __uint_as_float(j & 1 ? (uint32_t)v[0][j / 2] & 0xFFFF0000u : (uint32_t)v[0][j / 2] << 16);
    }
    __device__ __forceinline__ void store(uint8_t* base, OFF off) const
    {
#pragma unroll
        for (int u = 0; u < (F32 ? 2 : 1); ++u) ((v4i*)(base + off))[u] = v[u];
    }
};
__device__ __forceinline__ uint32_t pack_bf16(float a, float b)  // round to nearest even
{
    typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
    const v2bf v = {(__bf16)a, (__bf16)b};
    return __builtin_bit_cast(uint32_t, v);
}
// Clears what lies beyond an adapter's rank in 8 values of it, `left` of which it has.
__device__ __forceinline__ v4i keep(v4i t, int left)
{
#pragma unroll
    for (int d = 0; d < 4; ++d) t[d] = left >= 2 * d + 2 ? t[d] : left == 2 * d + 1 ? t[d] & 0xFFFF : 0;
    return t;
}

// A lane's part of a row of s T as terms: ranks 32 ks + 8 q ..  Once more for infinities where there are any (one test for all of them).
template <int KS>
__device__ __forceinline__ void load_terms(const ExpandArgs& a, const float* T, int slot, int rank, int q, v4i (&tt)[KS][3])
{
    const float s = a.v.scales[slot];
    float most = 0.0f;
    auto load = [&](auto infinite) {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            float t[8];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const v4f x = *(const v4f*)(T + min(ks * 32 + q * 8, a.v.rp - 8) + 4 * u);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    t[4 * u + e] = ks * 32 + q * 8 < rank ? x[e] * s : 0.0f;
                    if (!infinite()) most = fmaxf(most, fabsf(t[4 * u + e]));
                }
            }
            split8<infinite()>(t, tt[ks]);
        }
    };
    load(std::false_type());
    if (__any(__builtin_isinf(most))) load(std::true_type());
}

// A workgroup of 4 wavefronts: a tile, 16 rows each, and `per` pieces of 128 columns one after another.  Bound by memory, so it is laid out for its
// accesses: product j of 8 has columns 8 i + j in lane i, so that a lane's sums of the 8 products are 8 consecutive columns of a row and 16 lanes
// read and write 256 consecutive bytes (with 16 rows in 16 lanes every 16 bytes are a cache line of their own).  The factor's 128
// rows are read in order, too, by all four wavefronts, and go through the LDS (unit (j, ks, q, i) of 16 bytes in the order of its
// readers, i turned by what the writers differ in).  The next piece's columns are requested before the present one's are worked on.
// us and TB/s of Yin and Y, traced: 8192 x 3456 rank 32 24-26 and 4.4-4.6, 8191 x 11200 rank 128 100-117 and 3.1-3.7 (299 MB read past the L2s for 199: the factor comes to every XCD more than once); copying the same rows by the same pattern takes 23 and 76, a plain
// copy 23 and 70.  Registers are held by launch bounds to what keeps four wavefronts a SIMD (rank up to 32) or three without spilling; left alone, T's third
// terms cost one each (forward of 8192 x 3456 rank 32 36.4 -> 33.9, 8191 x 11200 rank 128 137 -> 130).  Non-temporal stores save 2-3 of the 25, but Y
// has a reader, for whom it is left in the caches.
// TW: the factor is given as [rank][width]; a thread reads blocks of 8 x 8 and turns them on the way to the LDS.
template <bool F32, bool TW, int KS, typename OFF>
__device__ __forceinline__ void expand_tile(const ExpandArgs& a, int run, int t)
{
    constexpr int ES = F32 ? 4 : 2;
    constexpr int WL = TW ? 8 : KS * 2;       // units of 16 bytes that a thread reads of a piece of the factor: 128 * 4 KS / 256
    constexpr int BUFFERS = KS <= 2 ? 2 : 1;  // (two of the larger ones leave room for two workgroups on a compute unit, one for four)
    __shared__ v4i wl[BUFFERS][8 * KS * 64];
    // The last term or two of T wait in the LDS where their registers would spill or cost a wavefront a SIMD (each lane reads what it wrote itself).
    constexpr int LOW = F32 || KS < (TW ? 2 : 4) ? 0 : KS == 3 ? 2 : 1;
    __shared__ v4i low[LOW ? LOW * KS * 256 : 1];
    const int4 tile = a.v.tiles[t];
    const uint2 is = plan_words(a.v);
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    int rows4[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) rows4[e] = a.v.rows[t * TILE + w * 16 + q * 4 + e];
    int zeroth = a.v.rows[t * TILE];
    ask_together();
    TOGETHER(rows4);
    asm("" : "+v"(zeroth));
    const int n = tile.y;
    if ((n <= 0) | !planned(a.v, is)) return;
    const int rank = rank_of(a.v, tile.z);
    if (rank == 0 && a.in_place) return;
    const int c0 = run * a.per, c1 = min(c0 + a.per, (a.width + 127) / 128);
    const int pr = a.v.rank / 8;  // units of a row of the factor
    const uint16_t* W = a.W + (int64_t)tile.z * a.width * a.v.rank;
    v4i wr[WL];
    auto request_w = [&](int c) {
        if constexpr (TW) {  // thread (p, i): ranks 8 p .., columns 8 i ..
            const int r = (int)threadIdx.x / 16 * 8, x = (int)threadIdx.x % 16 * 8;
            const uint16_t* src = W + c * 128 + (x < a.width - c * 128 ? x : 0);
#pragma unroll
            for (int u = 0; u < 8; ++u) wr[u] = *(const v4i*)(src + (int64_t)min(r + u, a.v.rank - 1) * a.width);
        } else {
            const int units = min(128, a.width - c * 128) * pr;
            const uint8_t* src = (const uint8_t*)(W + (int64_t)c * 128 * a.v.rank);
#pragma unroll
            for (int u = 0; u < WL; ++u) wr[u] = *(const v4i*)(src + (uint32_t)min(u * 256 + (int)threadIdx.x, units - 1) * 16u);
        }
    };
    if (rank > 0) request_w(c0);
    // this lane's four rows of the output
    // (rows and columns past the tile's and the matrix's are read from the last or first ones and not stored; so no load has a branch around it)
    OFF yin[4], yout[4];
    const int mine = n - (w * 16 + q * 4);  // how many of them the tile has
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int row = e < mine ? rows4[e] : zeroth;
        yin[e] = ((OFF)row * (OFF)a.ldyin + 8 * i) * ES;
        yout[e] = ((OFF)row * (OFF)a.ldy + 8 * i) * ES;
    }
    Row8<F32, OFF> y[4];
    auto request_y = [&](int c) {
        const OFF wrap = 8 * i < a.width - c * 128 ? 0 : 8 * i * ES;
        if (a.Yin) {
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e].fetch((const uint8_t*)a.Yin + (int64_t)c * 128 * ES, yin[e] - wrap);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e].clear();
        }
    };
    request_y(c0);
    if (rank == 0) {
        for (int c = c0; c < c1; ++c) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (e < mine && 8 * i < a.width - c * 128) y[e].store((uint8_t*)a.Y + (int64_t)c * 128 * ES, yout[e]);
            if (c + 1 < c1) request_y(c + 1);
        }
        return;
    }
    v4i tt[KS][3];
    load_terms<KS>(a, a.T + (int64_t)(tile.x + min(w * 16 + i, n - 1)) * a.v.rp, tile.z, rank, q, tt);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int k = 3 - LOW; k < 3; ++k) low[((k - 3 + LOW) * KS + ks) * 256 + threadIdx.x] = tt[ks][k];
    // the units that no row of the factor fills (ranks that are no multiple of 32)
    if (!TW && pr < KS * 4) {
        for (int o = threadIdx.x; o < BUFFERS * 8 * KS * 64; o += 256) wl[0][o] = v4i{0, 0, 0, 0};
        __syncthreads();
    }
    for (int c = c0; c < c1; ++c) {
        const int rows = min(128, a.width - c * 128);
        v4i* buf = wl[(c - c0) % BUFFERS];
        if (BUFFERS == 1 && c > c0) __syncthreads();  // (the present piece has been read)
        if constexpr (TW) {
            const int p = (int)threadIdx.x / 16, x = (int)threadIdx.x % 16;
            if (p < KS * 4) {
#pragma unroll
                for (int u = 0; u < 8; ++u)  // (ranks that the adapter does not have, whatever the pool holds there)
                    if (8 * p + u >= rank) wr[u] = v4i{0, 0, 0, 0};
#pragma unroll
                for (int j = 0; j < 8; ++j) buf[(j * KS + (p >> 2)) * 64 + (p & 3) * 16 + (x ^ ((p & 3) + 4 * (((p >> 2) + j) & 1)))] = column(wr, j);
            }
        } else {
#pragma unroll
            for (int u = 0; u < WL; ++u) {
                const int f = u * 256 + (int)threadIdx.x, r = a.unit_magic ? (int)__umulhi((unsigned)f, a.unit_magic) : f, p = f - r * pr;
                if (f < rows * pr) {
                    const int j = r & 7, k = p >> 2, qq = p & 3;
                    buf[(j * KS + k) * 64 + qq * 16 + ((r >> 3) ^ (qq + 4 * ((k + j) & 1)))] = rank < a.v.rank ? keep(wr[u], rank - 8 * p) : wr[u];
                }
            }
        }
        __syncthreads();
        if (c + 1 < c1) request_w(c + 1);
        // a bf16 output's sums start from it (rounded to 8 bits in the end); an fp32 one takes them when they are complete
        v4f acc[8];
        Row8<F32, OFF> o[F32 ? 4 : 1];
#pragma unroll
        for (int j = 0; j < 8; ++j) acc[j] = F32 ? v4f{0, 0, 0, 0} : v4f{y[0].get(j), y[1].get(j), y[2].get(j), y[3].get(j)};
        if constexpr (F32)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = y[e];
        if (c + 1 < c1) request_y(c + 1);
        if (w * 16 >= n) continue;
        auto multiply = [&](int j, int ks, const v4i (&t)[3]) {
            const v4i wv = buf[(j * KS + ks) * 64 + q * 16 + (i ^ (q + 4 * ((ks + j) & 1)))];
#pragma unroll
            for (int k = 2; k >= 0; --k) acc[j] = mfma(t[k], wv, acc[j]);
        };
        if constexpr (LOW > 0) {
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                v4i t[3];
#pragma unroll
                for (int k = 0; k < 3; ++k) t[k] = k < 3 - LOW ? tt[ks][k] : low[((k - 3 + LOW) * KS + ks) * 256 + threadIdx.x];
#pragma unroll
                for (int j = 0; j < 8; ++j) multiply(j, ks, t);
            }
        } else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) multiply(j, ks, tt[ks]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            Row8<F32, OFF> z;
            if constexpr (F32) {
#pragma unroll
                for (int j = 0; j < 8; ++j) z.v[j / 4][j % 4] = __float_as_int(o[e].get(j) + acc[j][e]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) z.v[0][j] = (int)pack_bf16(acc[2 * j][e], acc[2 * j + 1][e]);
            }
            if (e < mine && 8 * i < rows) z.store((uint8_t*)a.Y + (int64_t)c * 128 * ES, yout[e]);
        }
    }
}

// ---- gradients of the factors -----------------------------------------------------------------

struct WgradArgs {
    AdapterView v;
    const float *T, *dT;   // [row of the plan][rp]
    const void *dY, *X;    // rows of N, of K values
    float *dA, *dB;        // [adapter][rank][K], [adapter][N][rank]
    float* part;           // [part_of()][part_stride]: N x rank of dB, then rank x K of dA
    int64_t lddy, ldx, part_stride;
    int N, K, per;         // per: tiles of a group
};

// Where group g keeps its part of an adapter's sums: 2 g where the adapter has the group's first tile, 2 g + 1 where it starts within.  With groups of one
// tile only adapters of more than 64 rows have parts; the last tile of one may hold a single row, all before are full, so that a number made of the tile's
// first row and of which of both it is belongs to one tile, and the batch has few (not one for every adapter of the pool).
__device__ __forceinline__ int64_t part_of(int per, int g, bool within, int row, bool last) { return per > 1 ? 2 * g + within : row / TILE * 2 + last; }

// One group's part of out = s T^T Q, for 128 columns of Q and 16 * RT of the rank (see adapter_wgrad).
// COLS_FIRST: the columns are the first operand (out is [rank][width], a lane's sums are consecutive columns), else the second ([width][rank]).
// ALONE: a wavefront makes the sums of its block by itself, all steps; else the workgroup's four share the steps of one block and join their sums in the LDS.
template <bool F32, int RT, bool COLS_FIRST, bool ALONE>
__device__ __forceinline__ void wgrad_group(const AdapterView& v, const float* T, const void* Q, int64_t ldq, float* whole_out, float* part, int64_t part_stride,
                                            int width, int per, int block, v4f (*red)[ALONE ? 1 : 8 * RT * 64])
{
    constexpr int QT = F32 ? 3 : 1, SHARE = ALONE ? 1 : 4;  // SHARE: wavefronts of a block
    const int lane = threadIdx.x & 63, w = ALONE ? 0 : threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const int c0 = block * 128, r0 = blockIdx.z * (RT * 16), g = blockIdx.y;
    const int col = c0 + 8 * i < width ? c0 + 8 * i : c0;  // (lanes past the width repeat the first columns and store nothing)
    // the group's first and last tile and the ones beside it, requested together: mostly they say all (one adapter), and every lookup that waits for
    // another is half a microsecond of a workgroup that lives for ten
    const int g0 = g * per, g1 = min(g0 + per, v.cap);
    const uint2 is = plan_words(v);
    const int before = g0 > 0 ? v.tiles[g0 - 1].z : -1, after = g1 < v.cap ? v.tiles[g1].z : -1, with = v.tbase[v.slots];
    int4 first = v.tiles[g0];
    const int4 end = v.tiles[g1 - 1];
    ask_together();
    const int last = planned(v, is) ? min(g1, with) : 0;
    for (int t0 = g0; t0 < last;) {
        const int slot = first.z;
        const int t1 = end.z == slot ? g1 : min(v.tbase[slot + 1], last);
        v4f acc[8][RT];
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) acc[c][rt] = v4f{0, 0, 0, 0};
        // Steps of 32 rows of the plan, dealt to the wavefronts.  Under the products of one, Q and T of the next are requested, and the rows of the one
        // after are looked up: a step that began with its own lookups took three dependent round trips.
        const int4 final = t1 == g1 ? end : v.tiles[t1 - 1];
        const int p0 = first.x, p1 = final.x + final.y, steps = (p1 - p0 + 31) / 32;
        const int* rows = v.rows + (t0 * TILE - p0);  // (by place in the plan, as T)
        v4i qn[8][F32 ? 2 : 1];
        float tn[RT][8];
        int rows_n[8];
        auto look = [&](int st) {
            typedef int v4u __attribute__((ext_vector_type(4), aligned(4)));
            const int at = p0 + st * 32 + q * 8;
            if (st < steps) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const v4u r = *(const v4u*)(rows + at + 4 * u);
#pragma unroll
                    for (int e = 0; e < 4; ++e) rows_n[4 * u + e] = r[e];
                }
            }
        };
        auto request = [&](int st) {
            const int at = p0 + st * 32 + q * 8;
            const int zeroth = rows[p0];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // (row and stride have up to 24 and 23 bits, so that one multiplication with a product of 64 will do; a place in T's fits 32)
                const uint64_t off = (uint64_t)(uint32_t)(at + j < p1 ? rows_n[j] : zeroth) * (uint32_t)ldq + (uint32_t)col;
                if constexpr (F32) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) qn[j][u] = ((const v4i*)((const float*)Q + off))[u];
                } else {
                    qn[j][0] = *(const v4i*)((const uint16_t*)Q + off);
                }
                const uint32_t place = __umul24(min(at + j, p1 - 1), v.rp);
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) tn[rt][j] = T[place + (uint32_t)min(r0 + rt * 16 + i, v.rp - 1)];
            }
        };
        // rows past the adapter's last: zeros on both sides (what stands in for them must not reach the sums through an infinity of its own)
        auto clear_past = [&](int st) {
            const int left = p1 - (p0 + st * 32 + q * 8);
            if (st == steps - 1) {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (j >= left) {
#pragma unroll
                        for (int u = 0; u < (F32 ? 2 : 1); ++u) qn[j][u] = v4i{0, 0, 0, 0};
#pragma unroll
                        for (int rt = 0; rt < RT; ++rt) tn[rt][j] = 0.0f;
                    }
            }
        };
        auto multiply = [&](const v4i (&qr)[8][F32 ? 2 : 1], const v4i (&tt)[RT][3], auto infinite) {
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                v4i qt[F32 ? 3 : 1];
                if constexpr (F32) {
                    float x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = __int_as_float(qr[j][c / 4][c % 4]);
                    split8<infinite()>(x, qt);
                    if constexpr (infinite()) fill8(qt);
                } else {
                    v4i rows8[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) rows8[j] = qr[j][0];
                    qt[0] = column(rows8, c);
                }
#pragma unroll
                for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                    for (int k = 2; k >= 0; --k)
#pragma unroll
                        for (int u = QT - 1; u >= 0; --u)
                            if (k + u < 4)  // (what is left out is below 2^-30 of the product)
                                acc[c][rt] = COLS_FIRST ? mfma(qt[u], tt[rt][k], acc[c][rt]) : mfma(tt[rt][k], qt[u], acc[c][rt]);
            }
        };
        if (w < steps) {
            look(w);
            request(w);
            look(w + SHARE);
        }
        for (int st = w; st < steps; st += SHARE) {
            clear_past(st);
            v4i qr[8][F32 ? 2 : 1], tt[RT][3];
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int u = 0; u < (F32 ? 2 : 1); ++u) qr[j][u] = qn[j][u];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) split8<false>(tn[rt], tt[rt]);
            if (st + SHARE < steps) {
                request(st + SHARE);
                look(st + 2 * SHARE);
            }
            multiply(qr, tt, std::false_type());
        }
        // sums that are not a number: once more, for products with an infinity (see fill8); nothing is ahead here
        if (not_numbers(acc)) {
#pragma unroll
            for (int c = 0; c < 8; ++c)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) acc[c][rt] = v4f{0, 0, 0, 0};
            for (int st = w; st < steps; st += SHARE) {
                look(st);
                request(st);
                clear_past(st);
                v4i tt[RT][3];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    split8<true>(tn[rt], tt[rt]);
                    fill8(tt[rt]);
                }
                multiply(qn, tt, std::true_type());
            }
        }
        const int rank = rank_of(v, slot);
        const float s = v.scales[slot];
        const bool whole = (t0 > g0 || before != slot) && (t1 < g1 || after != slot);
        float* out = whole ? whole_out + (int64_t)slot * v.rank * width : part + part_of(per, g, t0 > g0, p0, after != slot) * part_stride;
        if constexpr (ALONE) {
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                if constexpr (COLS_FIRST) {  // lane (i, q) has rank i, columns 8 (4 q + e) + c
                    const int r = r0 + rt * 16 + i;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int k = c0 + 8 * (q * 4 + e);
                        if (r < v.rank && k < width)
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                v4f o;
#pragma unroll
                                for (int c = 0; c < 4; ++c) o[c] = r < rank ? acc[4 * u + c][rt][e] * s : 0.0f;
                                *(v4f*)(out + (int64_t)r * width + k + 4 * u) = o;
                            }
                    }
                } else {  // lane (i, q) has columns 8 i + c, ranks 4 q ..
                    const int r = r0 + rt * 16 + q * 4;
                    if (r < v.rank && c0 + 8 * i < width)
#pragma unroll
                        for (int c = 0; c < 8; ++c) {
                            v4f o;
#pragma unroll
                            for (int e = 0; e < 4; ++e) o[e] = r + e < rank ? acc[c][rt][e] * s : 0.0f;
                            *(v4f*)(out + (int64_t)(c0 + 8 * i + c) * v.rank + r) = o;
                        }
                }
            }
            t0 = t1;
            if (t0 < last) first = v.tiles[t0];
            continue;
        }
        // the wavefronts' sums, in their order: each adds up and stores a quarter of the columns (product c: columns 8 i + c)
        const int waves = min(steps, 4);
#pragma unroll
        for (int c = 0; c < 8; ++c)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
                if (w < waves) red[w][(c * RT + rt) * 64 + lane] = acc[c][rt];
        __syncthreads();
        if constexpr (COLS_FIRST) {  // 2 columns and 16 consecutive ranks' rows: lane (i, q) has rank i, columns 8 (4 q + e) + c
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) {
                v4f t[2];
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    t[u] = red[0][((2 * w + u) * RT + rt) * 64 + lane];
                    for (int k = 1; k < waves; ++k) t[u] += red[k][((2 * w + u) * RT + rt) * 64 + lane];
                }
                const int r = r0 + rt * 16 + i;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int k = c0 + 8 * (q * 4 + e) + 2 * w;
                    typedef float v2f __attribute__((ext_vector_type(2)));
                    if (r < v.rank && k < width) *(v2f*)(out + (int64_t)r * width + k) = r < rank ? v2f{t[0][e] * s, t[1][e] * s} : v2f{0, 0};
                }
            }
        } else {  // lane (i, q) has columns 8 i + c, ranks 4 q ..
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) {
                    v4f t = red[0][((2 * w + u) * RT + rt) * 64 + lane];
                    for (int k = 1; k < waves; ++k) t += red[k][((2 * w + u) * RT + rt) * 64 + lane];
                    const int r = r0 + rt * 16 + q * 4;
#pragma unroll
                    for (int e = 0; e < 4; ++e) t[e] = r + e < rank ? t[e] * s : 0.0f;
                    if (r < v.rank && c0 + 8 * i < width) *(v4f*)(out + (int64_t)(c0 + 8 * i + 2 * w + u) * v.rank + r) = t;
                }
        }
        t0 = t1;
        if (t0 < last) {
            first = v.tiles[t0];
            __syncthreads();
        }
    }
}

// dB = s dY^T T and dA = (s dY B)^T X in one launch, 128 columns of dY or X and 16 * RT of the rank to a workgroup.  The tiles of the plan are dealt
// to groups of `per`; an adapter that lies within a group is finished there, one that does not leaves a part in each, which wgrad_sum adds up.  The products run over rows, of which both operands need 8 of one column in
// a lane: a lane loads 8 columns of 8 rows (16 lanes 256 consecutive bytes) and pairs up the halves of the dwords, which gives the operands of 8
// products, the c-th with columns 8 i + c.  T and dT are fp32, so they go in as three bf16 terms.
// Bound by latency: 8 rows of a step are 8 loads in flight for a wavefront, and the sums leave two wavefronts a SIMD: us and TB/s of X and dY, traced, 8192 rows of
// 1152 and 3456, rank 32: 21-25 and 3.1-3.6 (0.9 wavefronts a SIMD on the average); 301 rows of fp32 1152 and bf16 1152, rank 24: 7.3-7.8.
// (Three wavefronts a SIMD for bf16 and 16 of the rank: what it takes without the second round for infinities, which must not cost one.)
template <bool F32, int RT, bool ALONE>
__global__ void __launch_bounds__(256, (!F32 && RT == 1 ? 3 : 1)) adapter_wgrad(WgradArgs a)
{
    __shared__ v4f red[ALONE ? 1 : 4][ALONE ? 1 : 8 * RT * 64];
    const int nb = (a.N + 127) / 128, kb = (a.K + 127) / 128, block = ALONE ? (int)(blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) : (int)blockIdx.x;
    if (block < nb) wgrad_group<false, RT, false, ALONE>(a.v, a.T, a.dY, a.lddy, a.dB, a.part, a.part_stride, a.N, a.per, block, red);
    else if (block < nb + kb) wgrad_group<F32, RT, true, ALONE>(a.v, a.dT, a.X, a.ldx, a.dA, a.part + (int64_t)a.v.rank * a.N, a.part_stride, a.K, a.per, block - nb, red);
}

// What adapter_wgrad leaves to do, a share of 256 quads at a time.  Adapters without rows: zeros.  Adapters of more than one group: their parts in the order
// of the groups.  nb, na: quads of dB and dA.
struct WgradSumArgs {
    const float* part;
    v4f *dB, *dA;
    int64_t part_stride, nb, na;
    int per, shares;  // shares of an adapter
};
__device__ __forceinline__ void wgrad_sum(const AdapterView& v, const WgradSumArgs& a, int slot, int share)
{
    if (slot >= v.slots) return;
    const uint2 is = plan_words(v);
    const int s0 = v.tbase[slot], s1 = v.tbase[slot + 1], g0 = s0 / a.per, g1 = (s1 - 1) / a.per;
    if (!planned(v, is) | (s0 < s1 && g0 == g1)) return;
    for (int64_t o = (int64_t)share * 256 + threadIdx.x; o < a.nb + a.na; o += (int64_t)a.shares * 256) {
        v4f t = {0, 0, 0, 0};
        if (s0 < s1)
#pragma unroll 8
            for (int g = g0; g <= g1; ++g)
                t += ((const v4f*)(a.part + part_of(a.per, g, s0 > g * a.per, a.per > 1 ? 0 : v.tiles[g].x, g == g1) * a.part_stride))[o];
        if (o < a.nb) a.dB[(int64_t)slot * a.nb + o] = t;
        else a.dA[(int64_t)slot * a.na + o - a.nb] = t;
    }
}

template <bool F32, int KS, typename OFF>
__global__ void __launch_bounds__(256, KS == 1 ? 4 : 3) adapter_expand(ExpandArgs a)
{
    const unsigned t = blockIdx.x / a.runs;
    expand_tile<F32, false, KS, OFF>(a, (int)(blockIdx.x - t * a.runs), (int)t);
}
// The forward's second product where adapters have few rows each (single tokens): a wavefront takes a piece of 128 columns by itself and reads its part of
// the factor straight into the products' operands, 16 rows of the tile at a time.  The same bits as adapter_expand.  Bound by latency: two dependent
// round trips, tile to rows to Yin (64 rows over 32 adapters, 1152 -> 3456 rank 32: 4.6-4.8 us traced for the factors' 7 MB).
template <int KS>
__global__ void __launch_bounds__(256) adapter_expand_few(ExpandArgs a)
{
    const unsigned at = blockIdx.x / a.runs;
    const int4 tile = a.v.tiles[at];
    const uint2 is = plan_words(a.v);
    ask_together();
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, i = lane & 15, q = lane >> 4;
    const int n = tile.y;
    if ((n <= 0) | (tile.z >= a.v.slots && a.in_place) | !planned(a.v, is)) return;
    // the rank is another round trip: with one step of it, whose registers allow it, it is waited for behind the first loads (300 rows over 64 adapters 1152 ->
    // 3456 rank 32 11.7 -> 11.4 us); with more the loads ahead of it take a wavefront a SIMD
    constexpr bool LATE = KS == 1;
    int rank = LATE ? 0 : rank_of(a.v, tile.z);
    if (!LATE && rank == 0 && a.in_place) return;
    const int c = (int)(blockIdx.x - at * a.runs) * 4 + w, rows = min(128, a.width - c * 128);
    if (rows <= 0) return;
    const bool in = 8 * i < rows;  // (columns past the width are read from the piece's first and not stored)
    v4i wv[8][KS];
    if (LATE || rank > 0) {
        const uint16_t* W = a.W + ((int64_t)(tile.z < a.v.slots ? tile.z : 0) * a.width + c * 128 + (in ? 8 * i : 0)) * a.v.rank;
#pragma unroll
        for (int j = 0; j < 8; ++j)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) wv[j][ks] = *(const v4i*)(W + (int64_t)j * a.v.rank + min(ks * 32 + q * 8, a.v.rank - 8));
    }
    if (LATE) rank = rank_of(a.v, tile.z);
    if (LATE && rank == 0 && a.in_place) return;
    for (int h = 0; h < n; h += 16) {
        Row8<false, int64_t> y[4];
        int64_t out[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int64_t row = a.v.rows[(int)at * TILE + min(h + q * 4 + e, n - 1)];
            const int col = c * 128 + (in ? 8 * i : 0);
            y[e].fetch((const uint8_t*)a.Yin, (row * a.ldyin + col) * 2);
            out[e] = (row * a.ldy + col) * 2;
        }
        if (rank > 0) {
            v4i tt[KS][3];
            load_terms<KS>(a, a.T + (int64_t)(tile.x + min(h + i, n - 1)) * a.v.rp, tile.z, rank, q, tt);
            v4f acc[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                acc[j] = v4f{y[0].get(j), y[1].get(j), y[2].get(j), y[3].get(j)};
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    const v4i b = rank < a.v.rank ? keep(wv[j][ks], rank - ks * 32 - q * 8) : wv[j][ks];
#pragma unroll
                    for (int k = 2; k >= 0; --k) acc[j] = mfma(tt[ks][k], b, acc[j]);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int j = 0; j < 4; ++j) y[e].v[0][j] = (int)pack_bf16(acc[2 * j][e], acc[2 * j + 1][e]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (h + q * 4 + e < n && in) y[e].store((uint8_t*)a.Y, out[e]);
    }
}
// The backward's last launch: dX = dXin + s dT A, and beside its tiles what is left of dA and dB (a launch less).  Bound by memory: 8192 x 1152 -> 3456 rank 32 over
// two adapters 14 us traced, 38 MB of dXin and dX and about 10 MB of parts (3.4 TB/s).
template <bool F32, int KS, typename OFF>
__global__ void __launch_bounds__(256, (F32 ? 1 : KS == 4 && sizeof(OFF) == 8 ? 2 : 3)) adapter_bwd_last(ExpandArgs a, WgradSumArgs g, int tiles)
{
    const unsigned t = blockIdx.x / a.runs;
    if (t < (unsigned)tiles) {
        expand_tile<F32, true, KS, OFF>(a, (int)(blockIdx.x - t * a.runs), (int)t);
    } else {
        const int o = (int)(blockIdx.x - tiles * a.runs);
        wgrad_sum(a.v, g, o / g.shares, o % g.shares);
    }
}

__global__ void __launch_bounds__(256) adapter_zero(v4f* p, int64_t n)
{
    for (int64_t o = (int64_t)blockIdx.x * 256 + threadIdx.x; o < n; o += (int64_t)gridDim.x * 256) p[o] = v4f{0, 0, 0, 0};
}

// ---- host ---------------------------------------------------------------------------------------

// Ranks are dealt to workgroups in groups of up to 64, in the factors' gradients of up to 32 (their sums are 8 times 4 registers for 16 of them; us of a
// training step by 16, 32, 48 and 64: 3000 x 2240 -> 11200 rank 128 258 / 220 / 279 / 247, 13066 x 512 -> 768 rank 96 104 / 102 / 118 / 118).
constexpr int WGRAD_RANKS = 2;
struct RankSplit {
    int groups, rt;
};
static RankSplit rank_split(int rank, int most = 4)
{
    const int tiles = (rank + 15) / 16, groups = (tiles + most - 1) / most;
    return {groups, (tiles + groups - 1) / groups};
}

// Adapters with a step of 32 rows each, about, as far as the pool's size says (the host does not know which of them a batch has): nothing to share out among the wavefronts, and a group for every tile (us of a training step, shared / alone: 121
// rows over 31 adapters 256 -> 4864 rank 104 148 / 93, 231 over 25 192 -> 2560 rank 48 43 / 37, 5 over 7 3456 -> 704 rank 96 40 / 31, 368 over 21 64 -> 1728 rank 48
// 32 / 30; with more rows, 327 over 12 384 -> 832 rank 48 24.1 / 25.7).
static bool few_rows(int slots, int64_t M) { return M <= 24 * (int64_t)slots; }

AdapterWorkLayout adapter_work_layout(const lq_adapter_config* c, int64_t M)
{
    AdapterWorkLayout l;
    const int64_t rp = (c->rank + 15) / 16 * 16;
    const int tiles = (int)(M / TILE) + c->slots + 1;
    // groups of tiles: about 512 workgroups over all column blocks, two to a compute unit, so that there are few parts (us of a training step of 8192 x 1152 ->
    // 3456 rank 32 by 256, 512, 1024: 113 / 108 / 115)
    const int64_t units = ((c->N + 127) / 128 + (c->K + 127) / 128) * rank_split(c->rank, WGRAD_RANKS).groups;
    int64_t groups = 512 / units;
    groups = groups < 1 ? 1 : groups;
    l.per = (int)((tiles + groups - 1) / groups);
    if (few_rows(c->slots, M)) l.per = 1;
    l.groups = (tiles + l.per - 1) / l.per;
    l.part_stride = (int64_t)c->rank * (c->N + c->K);
    size_t o = 0;
    l.off_dT = o, o += align256((size_t)M * rp * 4);
    const int64_t parts = l.per > 1 ? (l.groups > 1 ? 2 * l.groups : 0) : M > TILE ? 2 * (M / TILE + 1) : 0;  // (see part_of)
    l.off_part = o, o += align256((size_t)parts * l.part_stride * 4);
    l.total = o;
    return l;
}

static AdapterView view_of(const lq_adapter_config* c, const lq_adapter_pool* pool, const uint8_t* plan, int64_t M)
{
    const AdapterPlanLayout l = adapter_plan_layout(M, c->slots);
    return {(const uint32_t*)plan + 6, (const int*)(plan + l.off_rows), (const int*)(plan + l.off_tbase), (const int4*)(plan + l.off_tiles), pool->ranks, pool->scales,
            c->slots, c->rank, (c->rank + 15) / 16 * 16, (int)M, l.tiles};
}

template <bool F32, bool TW, int MT, int RT>
static hipError_t run_shrink_form(const ShrinkArgs& a, int tiles, int groups, hipStream_t s)
{
    constexpr int pieces = 8 * ShrinkPiece<F32, TW, MT, RT>::UNITS * 16, sums = 8 * MT * 16 * RT * 16 * 4, lds = pieces > sums ? pieces : sums;
    const hipError_t e = allow_lds<adapter_shrink<F32, TW, MT, RT>>(lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((adapter_shrink<F32, TW, MT, RT>), dim3(tiles * (TILE / (16 * MT)), groups), dim3(512), lds, s, a);
    return hipGetLastError();
}
template <bool F32, bool TW, int MT>
static hipError_t run_shrink_ranks(const ShrinkArgs& a, int tiles, hipStream_t s)
{
    if constexpr (!F32 && MT == 2) {
        // (us in one group and in two: rank 80 of 5000 x 3456 23.2 / 28.7, 96 of 8191 x 3456 42.7 / 45.3, 128 of 8191 x 2240 34.6 / 31.1)
        if (a.v.rank > 64 && a.v.rank <= 80) return run_shrink_form<F32, TW, MT, 5>(a, tiles, 1, s);
        if (a.v.rank > 80 && a.v.rank <= 96) return run_shrink_form<F32, TW, MT, 6>(a, tiles, 1, s);
    }
    const RankSplit rs = rank_split(a.v.rank);
    switch (rs.rt) {
        case 1: return run_shrink_form<F32, TW, MT, 1>(a, tiles, rs.groups, s);
        case 2: return run_shrink_form<F32, TW, MT, 2>(a, tiles, rs.groups, s);
        case 3: return run_shrink_form<F32, TW, MT, 3>(a, tiles, rs.groups, s);
        default: return run_shrink_form<F32, TW, MT, 4>(a, tiles, rs.groups, s);
    }
}
// The three forms: (a) 16 rows and 16 of the rank to a workgroup, (b) 16 rows and up to 64 of the rank, (c) 32 rows.  The first spreads the factor over many compute units, the
// last reads it least.  `launched`: workgroups of 16 rows and all of the rank, of which an adapter's four may have no rows but take a place (the larger forms fill a compute
// unit).  (a) with half the compute units or fewer and one for each part with rows; not with the turned factor, of whose rows it would read 32 bytes at a time.  (b) while all
// are there at once.  us of a forward, (a) / (b) / (c): 1 x 4608 -> 1152 rank 128 10.8 / 15.2 / 16.7, 16 over 16 adapters 1152 -> 4608 rank 128 12.5 / 13.2 / 13.9, 300 x 1152 -> 2304 rank 64 8.4 /
// 10.1 / 10.8, 1024 x 1152 -> 3456 rank 32 10.4 / 10.9 / 11.5; 64 over 32 of it 8.7 / 8.4 / 8.9, 2048 of it 14.0 / 13.2 / 13.9, 3000 16.4 / 15.7 / 16.2; 4096 21.4 / 22.0 / 20.5, 300 over 64 11.5 / 11.4 / 10.8,
// 100 over 100 2240 -> 2240 rank 64 25.5 / 25.2 / 18.3.  Of a training step: 128 over 16 1152 -> 1152 rank 128 37.6 / 35.1 / 35.8, 40 over 20 4608 -> 1152 rank 64 47.4 / 45.0 / 47.3, 100 over 100
// 153 / 117 / 103.
template <bool F32, bool TW>
static hipError_t run_shrink(const ShrinkArgs& a, int tiles, hipStream_t s)
{
    const int64_t parts = a.v.M / 16 + a.v.slots + 1, launched = (int64_t)tiles * (TILE / 16), cus = compute_units();  // parts: with rows, at most
    if constexpr (!TW) {
        const int ranks = (a.v.rank + 15) / 16;
        if (2 * launched <= cus && parts * ranks <= cus) return run_shrink_form<F32, TW, 1, 1>(a, tiles, ranks, s);
    }
    return launched * rank_split(a.v.rank).groups <= cus ? run_shrink_ranks<F32, TW, 1>(a, tiles, s) : run_shrink_ranks<F32, TW, 2>(a, tiles, s);
}

// sum: in the backward; NULL in the forward
template <bool F32, bool TW, int KS, typename OFF>
static void run_expand_form(const ExpandArgs& a, int tiles, const WgradSumArgs* sum, hipStream_t s)
{
    if constexpr (TW) hipLaunchKernelGGL((adapter_bwd_last<F32, KS, OFF>), dim3(tiles * a.runs + a.v.slots * sum->shares), dim3(256), 0, s, a, *sum, tiles);
    else hipLaunchKernelGGL((adapter_expand<F32, KS, OFF>), dim3(tiles * a.runs), dim3(256), 0, s, a);
}
template <bool F32, bool TW, typename OFF>
static void run_expand_ranks(const ExpandArgs& a, int tiles, const WgradSumArgs* sum, hipStream_t s)
{
    switch ((a.v.rank + 31) / 32) {
        case 1: run_expand_form<F32, TW, 1, OFF>(a, tiles, sum, s); break;
        case 2: run_expand_form<F32, TW, 2, OFF>(a, tiles, sum, s); break;
        case 3: run_expand_form<F32, TW, 3, OFF>(a, tiles, sum, s); break;
        default: run_expand_form<F32, TW, 4, OFF>(a, tiles, sum, s); break;
    }
}
template <bool F32, bool TW>
static hipError_t run_expand(ExpandArgs a, int tiles, const WgradSumArgs* sum, hipStream_t s)
{
    // pieces of a workgroup: 2048 workgroups, or three pieces each where the factor's part of the work is large and 768 workgroups are left
    const int pieces = (a.width + 127) / 128;
    const int64_t all = (int64_t)tiles * pieces, want = all / 2048;
    a.per = (int)(want < 1 ? 1 : want);
    if (a.per < 3 && a.v.rank > 64 && all >= 3 * 768) a.per = 3;
    a.per = a.per > pieces ? pieces : a.per;
    a.unit_magic = a.v.rank > 8 ? (unsigned)((((uint64_t)1 << 32) + a.v.rank / 8 - 1) / (a.v.rank / 8)) : 0;
    a.runs = (unsigned)((pieces + a.per - 1) / a.per);
    // offsets of 32 bits where the last row's fit
    const int64_t ld = a.ldyin > a.ldy ? a.ldyin : a.ldy;
    if (((int64_t)a.v.M * ld + a.width) * (F32 ? 4 : 2) < ((int64_t)1 << 32)) run_expand_ranks<F32, TW, uint32_t>(a, tiles, sum, s);
    else run_expand_ranks<F32, TW, int64_t>(a, tiles, sum, s);
    return hipGetLastError();
}

static hipError_t run_expand_few(ExpandArgs a, int tiles, hipStream_t s)
{
    a.runs = (unsigned)((a.width + 511) / 512);
    const dim3 grid(tiles * a.runs), block(256);
    switch ((a.v.rank + 31) / 32) {
        case 1: hipLaunchKernelGGL(adapter_expand_few<1>, grid, block, 0, s, a); break;
        case 2: hipLaunchKernelGGL(adapter_expand_few<2>, grid, block, 0, s, a); break;
        case 3: hipLaunchKernelGGL(adapter_expand_few<3>, grid, block, 0, s, a); break;
        default: hipLaunchKernelGGL(adapter_expand_few<4>, grid, block, 0, s, a); break;
    }
    return hipGetLastError();
}

static hipError_t run_wgrad(const WgradArgs& a, bool f32, int groups, hipStream_t s)
{
    const RankSplit rs = rank_split(a.v.rank, WGRAD_RANKS);
    const unsigned blocks = (a.N + 127) / 128 + (a.K + 127) / 128;
    const bool alone = few_rows(a.v.slots, a.v.M);
    const dim3 grid(alone ? (blocks + 3) / 4 : blocks, groups, rs.groups), block(256);
#define WGRAD(RT) \
    if (f32 && alone) hipLaunchKernelGGL((adapter_wgrad<true, RT, true>), grid, block, 0, s, a); \
    else if (f32) hipLaunchKernelGGL((adapter_wgrad<true, RT, false>), grid, block, 0, s, a); \
    else if (alone) hipLaunchKernelGGL((adapter_wgrad<false, RT, true>), grid, block, 0, s, a); \
    else hipLaunchKernelGGL((adapter_wgrad<false, RT, false>), grid, block, 0, s, a)
    if (rs.rt == 1) WGRAD(1);
    else WGRAD(2);
#undef WGRAD
    return hipGetLastError();
}

hipError_t launch_adapter_fwd(const lq_adapter_config* c, const uint8_t* plan, const lq_adapter_pool* pool, const void* X, int64_t ldx,
                              const void* Yin, int64_t ldyin, void* Y, int64_t ldy, int64_t M, uint8_t* inter, hipStream_t s)
{
    const AdapterView v = view_of(c, pool, plan, M);
    const int tiles = adapter_plan_layout(M, c->slots).tiles;
    const ShrinkArgs a{v, X, (const uint16_t*)pool->A, (float*)inter, ldx, (int)c->K};
    const ExpandArgs x{v, (const float*)inter, (const uint16_t*)pool->B, Yin, Y, ldyin, ldy, (int)c->N, Yin == Y && ldyin == ldy};
    const hipError_t e = c->x_dtype == LQ_F32 ? run_shrink<true, false>(a, tiles, s) : run_shrink<false, false>(a, tiles, s);
    if (e != hipSuccess) return e;
    // (us of a forward, few / other form: 64 rows over 32 adapters 1152 -> 3456 rank 32 8.6 / 9.2, 300 over 64 10.9 / 12.9, 1000 over 64 rank 64 18.6 / 19.9, 16 over 16
    // 1152 -> 4608 rank 128 13.0 / 15.0; where the other form's workgroups all fit at once it is ahead: 64 over 4 8.1 / 6.4, 1 x 4608 -> 1152 rank 128 12.9 / 11.3.  The pool
    // stands for the adapters of the batch, which the host does not know: a single token of a pool of 64 takes it, too, 18.8 / 17.3, and 8192 rows of one adapter of 1024
    // 64.7 / 63.2)
    if (M <= 16 * (int64_t)c->slots && (int64_t)tiles * ((c->N + 127) / 128) >= 512) return run_expand_few(x, tiles, s);
    return run_expand<false, false>(x, tiles, nullptr, s);
}

hipError_t launch_adapter_bwd(const lq_adapter_config* c, const uint8_t* plan, const lq_adapter_pool* pool, const void* X, int64_t ldx,
                              const uint8_t* inter, const void* dY, int64_t lddy, const void* dXin, int64_t lddxin, void* dX, int64_t lddx,
                              float* dA, float* dB, int64_t M, uint8_t* work, hipStream_t s)
{
    const AdapterView v = view_of(c, pool, plan, M);
    const AdapterWorkLayout l = adapter_work_layout(c, M);
    const int tiles = adapter_plan_layout(M, c->slots).tiles;
    const bool f32 = c->x_dtype == LQ_F32;
    float *dT = (float*)(work + l.off_dT), *part = (float*)(work + l.off_part);
    hipError_t e = run_shrink<false, true>({v, dY, (const uint16_t*)pool->B, dT, lddy, (int)c->N}, tiles, s);
    if (e != hipSuccess) return e;
    if ((e = run_wgrad({v, (const float*)inter, dT, dY, X, dA, dB, part, lddy, ldx, l.part_stride, (int)c->N, (int)c->K, l.per}, f32, l.groups, s)) != hipSuccess)
        return e;
    const int64_t nb = (int64_t)c->rank * c->N / 4, na = (int64_t)c->rank * c->K / 4, shares = (nb + na + 255) / 256;
    const WgradSumArgs sum{part, (v4f*)dB, (v4f*)dA, l.part_stride, nb, na, l.per, (int)(shares > 2048 ? 2048 : shares)};
    const ExpandArgs x{v, dT, (const uint16_t*)pool->A, dXin, dX, lddxin, lddx, (int)c->K, dXin == dX && lddxin == lddx};
    return f32 ? run_expand<true, true>(x, tiles, &sum, s) : run_expand<false, true>(x, tiles, &sum, s);
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
