// Host side of the C ABI: argument validation, layout arithmetic, dispatch.  Every error is
// detected here, before any launch, so that all error paths can be exercised without a GPU.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <new>
#include <utility>
#include <vector>

#include "lq_internal.h"

namespace lq {

static int int_qmax(int fmt)
{
    switch (fmt) {
        case LQ_INT4: return 7;
        case LQ_INT6: return 31;
        case LQ_INT8: return 127;
        default: return 0;
    }
}

lq_status make_dims(const lq_config* cfg, Dims* d)
{
    if (!cfg) return LQ_ERR_NULL;
    if (cfg->flags & ~LQ_FLAG_SMOOTH) return LQ_ERR_UNSUPPORTED;
    if (cfg->N <= 0 || cfg->K <= 0 || cfg->N > (1 << 24) || cfg->K > (1 << 24)) return LQ_ERR_SHAPE;
    if (cfg->K % 64 != 0 || cfg->N % 64 != 0) return LQ_ERR_SHAPE;
    const int r = cfg->rank;
    if (!(r == 0 || r == 16 || r == 32 || r == 64 || r == 96 || r == 128)) return LQ_ERR_SHAPE;
    if (cfg->x_dtype != LQ_F32 && cfg->x_dtype != LQ_BF16) return LQ_ERR_UNSUPPORTED;
    if (cfg->residual_from_quantized != 0 && cfg->residual_from_quantized != 1) return LQ_ERR_UNSUPPORTED;
    d->N = cfg->N;
    d->K = d->Ks = cfg->K;
    d->r = r;
    d->rp = (r + 31) / 32 * 32;
    d->C64 = (int)(cfg->K / 64);
    d->smooth = (cfg->flags & LQ_FLAG_SMOOTH) != 0;
    d->mx = d->mxb = d->mxi = d->ga = false;
    d->bw_bits = d->mxb_elem = 0;
    if (cfg->main_w == LQ_INT4) {
        if (cfg->main_a != LQ_INT4) return LQ_ERR_UNSUPPORTED;
        if (cfg->main_w_group != 64 && cfg->main_w_group != 128) return LQ_ERR_SHAPE;
        if (cfg->K % cfg->main_w_group != 0) return LQ_ERR_SHAPE;
        if (cfg->main_a_group != 0 && cfg->main_a_group != 64) return LQ_ERR_UNSUPPORTED;
        if (cfg->main_a_group == 64 && cfg->main_w_group != 64) return LQ_ERR_UNSUPPORTED;  // one block size for both operands
        d->ga = cfg->main_a_group == 64;
        if (d->ga && cfg->K > 5632) return LQ_ERR_UNSUPPORTED;  // the forward keeps a tile's token block scales in LDS
        // the forward addresses the channel group scales with 32-bit byte offsets
        if (cfg->N * (cfg->K / cfg->main_w_group) * 4 >= ((int64_t)1 << 31)) return LQ_ERR_UNSUPPORTED;
        const int qw = int_qmax(cfg->br_w), qa = int_qmax(cfg->br_a);
        if (qw == 0 || qa == 0 || cfg->br_a == LQ_INT4) return LQ_ERR_UNSUPPORTED;
        d->mx = false;
        d->g = cfg->main_w_group;
        d->qmax_bw = qw;
        d->qmax_ba = qa;
    } else if (cfg->main_w == LQ_MXFP4_E2M1) {
        if (cfg->main_a != LQ_MXFP4_E2M1) return LQ_ERR_UNSUPPORTED;
        if (cfg->main_w_group != 32 || cfg->main_a_group != 32) return LQ_ERR_SHAPE;
        if (cfg->br_w != cfg->br_a ||
            (cfg->br_w != LQ_FP8_E4M3 && cfg->br_w != LQ_MXFP8_E4M3 && cfg->br_w != LQ_MXFP6_E2M3))
            return LQ_ERR_UNSUPPORTED;
        // the MX forward stages K in steps of 128: an odd number of 64-chunks is padded inside the blobs with one chunk
        // of zero codes (pack and activation kernels write it; sources and views keep the caller's K)
        d->K = (cfg->K + 127) / 128 * 128;
        d->C64 = (int)(d->K / 64);
        d->mxb = cfg->br_w != LQ_FP8_E4M3;
        if (!d->mxb && r == 96) return LQ_ERR_SHAPE;
        d->mxb_elem = cfg->br_w == LQ_MXFP8_E4M3 ? 8 : cfg->br_w == LQ_MXFP6_E2M3 ? 6 : 0;
        if (d->mxb && r % 32 != 0) return LQ_ERR_SHAPE;  // whole blocks of 32 along the rank
        d->mx = true;
        d->g = 32;
        d->qmax_bw = d->qmax_ba = 0;
        d->rp = (r + 63) / 64 * 64;                  // FP8 expansion runs 64 deep
    } else if (cfg->main_w == LQ_MXINT4) {
        if (cfg->main_a != LQ_MXINT4) return LQ_ERR_UNSUPPORTED;
        if (cfg->main_w_group != 32 || cfg->main_a_group != 32) return LQ_ERR_SHAPE;
        if (cfg->br_a != LQ_MXINT8 || (cfg->br_w != LQ_MXINT8 && cfg->br_w != LQ_MXINT4)) return LQ_ERR_UNSUPPORTED;
        if (r % 32 != 0) return LQ_ERR_SHAPE;  // whole blocks of 32 along the rank
        d->mxi = true;
        d->bw_bits = cfg->br_w == LQ_MXINT8 ? 8 : 4;
        d->g = 32;
        d->qmax_bw = d->qmax_ba = 0;
    } else {
        return LQ_ERR_UNSUPPORTED;
    }
    d->G = (int)(cfg->K / d->g);
    {   // FNV-1a over the configuration's fields, in declaration order
        const int64_t f[12] = {cfg->N, cfg->K, cfg->rank, cfg->main_w, cfg->main_a, cfg->main_w_group, cfg->main_a_group,
                               cfg->br_w, cfg->br_a, cfg->residual_from_quantized, cfg->x_dtype, cfg->flags};
        uint64_t h = 1469598103934665603ull;
        for (int i = 0; i < 12; ++i)
            for (int b = 0; b < 8; ++b) {
                h ^= (uint64_t)((f[i] >> (8 * b)) & 0xFF);
                h *= 1099511628211ull;
            }
        d->cfg_hash = h;
    }
    return LQ_OK;
}

PackedLayout packed_layout(const Dims& d)
{
    PackedLayout pl;
    size_t o = BLOB_HEADER;
    pl.off_pq = o;
    o = align256(o + ((d.mx || d.mxi) ? (size_t)d.N * d.K / 2 : (size_t)d.N * d.K / 4 * 3));  // INT family: 6-bit fields
    pl.off_sw = o;
    o = align256(o + ((d.mx || d.mxi) ? (size_t)(d.N / 32) * ((d.C64 + 3) / 4) * 256 : (size_t)d.N * d.G * 4));
    pl.off_lq = o;
    o = align256(o + (size_t)d.N * d.rp * (d.mxi ? 2 : 1));  // MXI: dequantised elements as bf16
    pl.off_sl = o;
    // fp32 per channel; MXFP8e4: a scale dword per (channel, rank half); MXI: a byte per (channel, rank block)
    o = align256(o + (d.mxi ? (size_t)d.N * (d.r / 32) + 4 : (size_t)d.N * (d.mxb ? 8 : 4)));
    pl.off_rq = o;
    o = align256(o + (size_t)d.r * d.K * (d.mxi ? 2 : 1));
    pl.off_sr = o;
    o = align256(o + (d.mxi   ? (size_t)d.r * (d.K / 32) + 4
                      : d.mxb ? (size_t)(d.K / 128) * (d.r / 16) * 256 + 4
                              : (size_t)(d.r > 0 ? d.r : 1) * 4));
    pl.off_rg = o;
    if (d.smooth) o = align256(o + (size_t)d.K * 4);
    pl.total = o;
    return pl;
}

ActLayout act_layout(const Dims& d, int64_t M)
{
    ActLayout al;
    al.Mp = (M + 31) / 32 * 32;
    size_t o = BLOB_HEADER;
    al.off_xq = o;
    o = align256(o + ((d.mx || d.mxi) ? (size_t)al.Mp * d.K / 2 : (size_t)al.Mp * d.K / 4 * 3));
    al.off_sx = o;
    o = align256(o + ((d.mx || d.mxi) ? (size_t)(al.Mp / 32) * ((d.C64 + 3) / 4) * 256
                      : d.ga          ? (size_t)d.G * ((al.Mp + 127) / 128) * 512
                                      : (size_t)al.Mp * 4));
    al.off_tq = o;
    o = align256(o + (size_t)al.Mp * d.rp * (d.mxi ? 2 : 1));
    al.off_st = o;
    o = align256(o + (d.mxi ? (size_t)al.Mp * (d.r / 32) + 4 : (size_t)al.Mp * (d.mxb ? 8 : 4)));
    al.total = o;
    return al;
}

int compute_units()
{
    static std::atomic<int> cached[64];
    int dev = 0, cus = 0;
    if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return 256;
    cus = cached[dev].load(std::memory_order_relaxed);
    if (cus == 0) {
        if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) != hipSuccess || cus <= 0) return 256;
        cached[dev].store(cus, std::memory_order_relaxed);
    }
    return cus;
}

}  // namespace lq

using namespace lq;

// A vector for each of S sequences, or none
template <typename MOD>
static lq_status mod_check(const MOD* m, const lq_block_config* c, int64_t S, MOD* out)
{
    *out = {nullptr, 0};
    if (!m || !m->p) return LQ_OK;
    if (S > 1 && (m->ld < c->dim || m->ld >= ((int64_t)1 << 40))) return LQ_ERR_SHAPE;
    if ((uintptr_t)m->p % 4 != 0) return LQ_ERR_ALIGN;
    *out = *m;
    return LQ_OK;
}

extern "C" {

const char* lq_status_string(lq_status s)
{
    switch (s) {
        case LQ_OK: return "ok";
        case LQ_ERR_NULL: return "null pointer";
        case LQ_ERR_SHAPE: return "shape violates the contract";
        case LQ_ERR_UNSUPPORTED: return "unsupported format combination";
        case LQ_ERR_ALIGN: return "misaligned pointer or stride";
        case LQ_ERR_BUFFER_TOO_SMALL: return "buffer too small";
        case LQ_ERR_DEVICE: return "HIP launch failed";
        case LQ_ERR_STALE_BLOB: return "blob header does not match the configuration";
    }
    return "unknown status";
}

lq_status lq_packed_sizes(const lq_config* cfg, size_t* packed_bytes)
{
    if (!cfg || !packed_bytes) return LQ_ERR_NULL;
    Dims d;
    lq_status st = make_dims(cfg, &d);
    if (st != LQ_OK) return st;
    *packed_bytes = packed_layout(d).total;
    return LQ_OK;
}

lq_status lq_act_sizes(const lq_config* cfg, int64_t M, size_t* act_bytes)
{
    if (!cfg || !act_bytes) return LQ_ERR_NULL;
    Dims d;
    lq_status st = make_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (M < 0 || M > (1 << 24)) return LQ_ERR_SHAPE;
    *act_bytes = M == 0 ? 0 : act_layout(d, M).total;  // (an empty batch needs no blob, not even the header)
    return LQ_OK;
}

static bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

lq_status lq_pack_weights(const lq_config* cfg, const float* W, const float* L, const float* R, void* packed,
                          size_t packed_bytes, void* stream)
{
    Dims d;
    lq_status st = make_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (!W || !packed) return LQ_ERR_NULL;
    if (d.r > 0 && (!L || !R)) return LQ_ERR_NULL;
    if (!aligned(packed, 256) || !aligned(W, 4)) return LQ_ERR_ALIGN;
    if (packed_bytes < packed_layout(d).total) return LQ_ERR_BUFFER_TOO_SMALL;
    hipError_t e = d.mxi ? launch_pack_mxi(d, cfg->residual_from_quantized, W, L, R, (uint8_t*)packed, (hipStream_t)stream)
                   : d.mx ? launch_pack_mx(d, cfg->residual_from_quantized, W, L, R, (uint8_t*)packed, (hipStream_t)stream)
                        : launch_pack_int(d, cfg->residual_from_quantized, W, L, R, (uint8_t*)packed, (hipStream_t)stream);
    return e == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_verify_blob(const lq_config* cfg, int32_t kind, const void* blob, size_t blob_bytes, int64_t M, void* stream)
{
    Dims d;
    lq_status st = make_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (!blob) return LQ_ERR_NULL;
    if (kind != LQ_BLOB_PACKED && kind != LQ_BLOB_ACT) return LQ_ERR_UNSUPPORTED;
    if (kind == LQ_BLOB_ACT && (M < 1 || M > (1 << 24))) return LQ_ERR_SHAPE;
    if (!aligned(blob, 256)) return LQ_ERR_ALIGN;
    const size_t need = kind == LQ_BLOB_PACKED ? packed_layout(d).total : act_layout(d, M).total;
    if (blob_bytes < need) return LQ_ERR_BUFFER_TOO_SMALL;
    BlobTag got;
    if (hipMemcpyAsync(&got, blob, sizeof(got), hipMemcpyDeviceToHost, (hipStream_t)stream) != hipSuccess) return LQ_ERR_DEVICE;
    if (hipStreamSynchronize((hipStream_t)stream) != hipSuccess) return LQ_ERR_DEVICE;
    const BlobTag want = make_tag(d, kind, kind == LQ_BLOB_ACT ? M : 0);
    for (int i = 0; i < 8; ++i)
        if (got.w[i] != want.w[i]) return LQ_ERR_STALE_BLOB;
    return LQ_OK;
}

lq_status lq_set_smoothing(const lq_config* cfg, const float* gamma, void* packed, size_t packed_bytes, void* stream)
{
    Dims d;
    lq_status st = make_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (!d.smooth) return LQ_ERR_UNSUPPORTED;
    if (!gamma || !packed) return LQ_ERR_NULL;
    if (!aligned(packed, 256) || !aligned(gamma, 4)) return LQ_ERR_ALIGN;
    if (packed_bytes < packed_layout(d).total) return LQ_ERR_BUFFER_TOO_SMALL;
    return launch_set_smoothing(d, gamma, (uint8_t*)packed, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_quantize_act(const lq_config* cfg, const void* packed, size_t packed_bytes, const void* X, int64_t M,
                          int64_t ldx, void* act, size_t act_bytes, const lq_act_debug* dbg, void* stream)
{
    Dims d;
    lq_status st = make_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (M == 0) return LQ_OK;  // an empty batch: nothing to do, no launch, the pointers are not looked at
    if (!X || !act) return LQ_ERR_NULL;
    if ((d.r > 0 || d.smooth) && !packed) return LQ_ERR_NULL;
    if (M < 1 || M > (1 << 24) || ldx < d.Ks) return LQ_ERR_SHAPE;
    const size_t es = cfg->x_dtype == LQ_BF16 ? 2 : 4;
    if (!aligned(X, 16) || (ldx * es) % 16 != 0 || !aligned(act, 256) || (packed && !aligned(packed, 256)))
        return LQ_ERR_ALIGN;
    if (act_bytes < act_layout(d, M).total || (packed && packed_bytes < packed_layout(d).total)) return LQ_ERR_BUFFER_TOO_SMALL;
    hipError_t e = d.mxi ? launch_quantize_act_mxi(d, cfg->x_dtype, (const uint8_t*)packed, X, M, ldx, (uint8_t*)act, dbg,
                                                   (hipStream_t)stream)
                   : d.mx ? launch_quantize_act_mx(d, cfg->x_dtype, (const uint8_t*)packed, X, M, ldx, (uint8_t*)act, dbg,
                                                 (hipStream_t)stream)
                        : launch_quantize_act_int(d, cfg->x_dtype, (const uint8_t*)packed, X, M, ldx, (uint8_t*)act, dbg,
                                                  (hipStream_t)stream);
    return e == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_linear_lowrank_fwd(const lq_config* cfg, const void* packed, size_t packed_bytes, const void* act,
                                size_t act_bytes, int64_t M, void* Y, int64_t ldy, const lq_fwd_debug* dbg, void* stream)
{
    Dims d;
    lq_status st = make_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (M == 0) return LQ_OK;  // an empty batch
    if (!packed || !act || !Y) return LQ_ERR_NULL;
    if (M < 1 || M > (1 << 24) || ldy < d.N || ldy > (1 << 22)) return LQ_ERR_SHAPE;
    if (!aligned(packed, 256) || !aligned(act, 256) || !aligned(Y, 16) || (ldy & 7)) return LQ_ERR_ALIGN;
    if (packed_bytes < packed_layout(d).total || act_bytes < act_layout(d, M).total) return LQ_ERR_BUFFER_TOO_SMALL;
    hipError_t e = d.mxi ? launch_fwd_mxi(d, (const uint8_t*)packed, (const uint8_t*)act, M, (uint16_t*)Y, ldy, dbg,
                                          (hipStream_t)stream)
                   : d.mx ? launch_fwd_mx(d, (const uint8_t*)packed, (const uint8_t*)act, M, (uint16_t*)Y, ldy, dbg,
                                        (hipStream_t)stream)
                        : launch_fwd_int(d, (const uint8_t*)packed, (const uint8_t*)act, M, (uint16_t*)Y, ldy, dbg,
                                         (hipStream_t)stream);
    return e == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

static lq_status handoff_dims(const lq_config* next_cfg, Dims* dn)
{
    lq_status st = make_dims(next_cfg, dn);
    if (st != LQ_OK) return st;
    if (!dn->mxi || dn->smooth) return LQ_ERR_UNSUPPORTED;  // integer MX family; smoothing has no place in a hand-off
    return LQ_OK;
}

lq_status lq_handoff_sizes(const lq_config* next_cfg, int64_t M, size_t* codes_bytes)
{
    if (!next_cfg || !codes_bytes) return LQ_ERR_NULL;
    Dims dn;
    lq_status st = handoff_dims(next_cfg, &dn);
    if (st != LQ_OK) return st;
    if (M < 0 || M > (1 << 24)) return LQ_ERR_SHAPE;
    *codes_bytes = handoff_total_bytes(dn, M);
    return LQ_OK;
}

lq_status lq_linear_lowrank_fwd_handoff(const lq_config* cfg, const void* packed, size_t packed_bytes, const void* act,
                                        size_t act_bytes, int64_t M, void* Y, int64_t ldy, const lq_config* next_cfg,
                                        void* act_next, size_t act_next_bytes, void* codes, size_t codes_bytes, void* stream)
{
    Dims d, dn;
    lq_status st = make_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (!next_cfg) return LQ_ERR_NULL;
    st = handoff_dims(next_cfg, &dn);
    if (st != LQ_OK) return st;
    if (!d.mxi) return LQ_ERR_UNSUPPORTED;
    if (dn.K != d.N) return LQ_ERR_SHAPE;
    if (M == 0) return LQ_OK;  // an empty batch
    if (!packed || !act || !act_next || !codes) return LQ_ERR_NULL;
    if (M < 1 || M > (1 << 24) || (Y && (ldy < d.N || ldy > (1 << 22)))) return LQ_ERR_SHAPE;
    if (!aligned(packed, 256) || !aligned(act, 256) || !aligned(act_next, 256) || !aligned(codes, 256) ||
        (Y && (!aligned(Y, 16) || (ldy & 7))))
        return LQ_ERR_ALIGN;
    if (act_next_bytes < act_layout(dn, M).total || codes_bytes < handoff_total_bytes(dn, M) ||
        packed_bytes < packed_layout(d).total || act_bytes < act_layout(d, M).total)
        return LQ_ERR_BUFFER_TOO_SMALL;
    return launch_fwd_handoff_mxi(d, (const uint8_t*)packed, (const uint8_t*)act, M, (uint16_t*)Y, Y ? ldy : d.N, dn,
                                  (uint8_t*)act_next, (uint8_t*)codes, (hipStream_t)stream) == hipSuccess
               ? LQ_OK
               : LQ_ERR_DEVICE;
}

lq_status lq_branch_from_codes(const lq_config* next_cfg, const void* packed_next, size_t packed_next_bytes,
                               const void* codes, size_t codes_bytes, int64_t M, void* act_next, size_t act_next_bytes,
                               void* stream)
{
    Dims dn;
    if (!next_cfg) return LQ_ERR_NULL;
    lq_status st = handoff_dims(next_cfg, &dn);
    if (st != LQ_OK) return st;
    if (M == 0) return LQ_OK;
    if (!codes || !act_next || (dn.r > 0 && !packed_next)) return LQ_ERR_NULL;
    if (M < 1 || M > (1 << 24)) return LQ_ERR_SHAPE;
    if (!aligned(codes, 256) || !aligned(act_next, 256) || (packed_next && !aligned(packed_next, 256))) return LQ_ERR_ALIGN;
    if (act_next_bytes < act_layout(dn, M).total || codes_bytes < handoff_total_bytes(dn, M) ||
        (packed_next && packed_next_bytes < packed_layout(dn).total))
        return LQ_ERR_BUFFER_TOO_SMALL;
    if (dn.r == 0) return LQ_OK;
    return launch_branch_from_codes_mxi(dn, (const uint8_t*)packed_next, (const uint8_t*)codes, M, (uint8_t*)act_next,
                                        (hipStream_t)stream) == hipSuccess
               ? LQ_OK
               : LQ_ERR_DEVICE;
}

lq_status lq_unpack_weights(const lq_config* cfg, const void* packed, const lq_weights_view* out, void* stream)
{
    Dims d;
    lq_status st = make_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (!packed || !out) return LQ_ERR_NULL;
    if (!aligned(packed, 256)) return LQ_ERR_ALIGN;
    hipError_t e = d.mxi ? launch_unpack_weights_mxi(d, (const uint8_t*)packed, out, (hipStream_t)stream)
                   : d.mx ? launch_unpack_weights_mx(d, (const uint8_t*)packed, out, (hipStream_t)stream)
                        : launch_unpack_weights_int(d, (const uint8_t*)packed, out, (hipStream_t)stream);
    return e == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_unpack_act(const lq_config* cfg, const void* act, int64_t M, const lq_act_view* out, void* stream)
{
    Dims d;
    lq_status st = make_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (M == 0) return LQ_OK;  // an empty batch
    if (!act || !out) return LQ_ERR_NULL;
    if (M < 1 || M > (1 << 24)) return LQ_ERR_SHAPE;
    if (!aligned(act, 256)) return LQ_ERR_ALIGN;
    hipError_t e = d.mxi ? launch_unpack_act_mxi(d, (const uint8_t*)act, M, out, (hipStream_t)stream)
                   : d.mx ? launch_unpack_act_mx(d, (const uint8_t*)act, M, out, (hipStream_t)stream)
                        : launch_unpack_act_int(d, (const uint8_t*)act, M, out, (hipStream_t)stream);
    return e == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

static lq_status calib_dims(const lq_config* cfg, Dims* d)
{
    lq_status st = make_dims(cfg, d);
    if (st != LQ_OK) return st;
    if (d->r < 16) return LQ_ERR_SHAPE;
    // the calibration works on the caller's W (N x K), not on packed layouts
    d->K = d->Ks;
    d->C64 = (int)(d->K / 64);
    d->G = (int)(d->K / d->g);
    return LQ_OK;
}

lq_status lq_calib_sizes(const lq_config* cfg, size_t* state_bytes)
{
    if (!cfg || !state_bytes) return LQ_ERR_NULL;
    Dims d;
    lq_status st = calib_dims(cfg, &d);
    if (st != LQ_OK) return st;
    *state_bytes = calib_layout(d).total;
    return LQ_OK;
}

lq_status lq_calib_init(const lq_config* cfg, const float* L, const float* R, void* state, size_t state_bytes, void* stream)
{
    Dims d;
    lq_status st = calib_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (!L || !R || !state) return LQ_ERR_NULL;
    if (!aligned(state, 256) || !aligned(L, 16) || !aligned(R, 16)) return LQ_ERR_ALIGN;
    if (state_bytes < calib_layout(d).total) return LQ_ERR_BUFFER_TOO_SMALL;
    return launch_calib_init(d, L, R, (uint8_t*)state, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_calib_step(const lq_config* cfg, const float* W, void* state, size_t state_bytes, int32_t step,
                        const lq_adam* adam, float* loss, void* stream)
{
    Dims d;
    lq_status st = calib_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (!W || !state || !adam) return LQ_ERR_NULL;
    if (step < 1) return LQ_ERR_SHAPE;
    if (!(adam->lr > 0.f) || !(adam->beta1 >= 0.f && adam->beta1 < 1.f) || !(adam->beta2 >= 0.f && adam->beta2 < 1.f) ||
        !(adam->eps > 0.f))
        return LQ_ERR_UNSUPPORTED;
    if (!aligned(state, 256) || !aligned(W, 16) || (loss && !aligned(loss, 4))) return LQ_ERR_ALIGN;
    if (state_bytes < calib_layout(d).total) return LQ_ERR_BUFFER_TOO_SMALL;
    return launch_calib_step(d, W, (uint8_t*)state, step, adam, loss, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_calib_unpack(const lq_config* cfg, const void* state, const lq_calib_view* out, void* stream)
{
    Dims d;
    lq_status st = calib_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (!state || !out) return LQ_ERR_NULL;
    if (!aligned(state, 256)) return LQ_ERR_ALIGN;
    return launch_calib_unpack(d, (const uint8_t*)state, out, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

static lq_status rot_dims(const lq_config* cfg, Dims* d)
{
    lq_status st = make_dims(cfg, d);
    if (st != LQ_OK) return st;
    if (d->r < 16) return LQ_ERR_SHAPE;
    // the search works on the caller's factors (N x r, r x K), not on packed layouts
    d->K = d->Ks;
    d->C64 = (int)(d->K / 64);
    d->G = (int)(d->K / d->g);
    if ((int64_t)d->r * d->K * 4 >= ((int64_t)1 << 31)) return LQ_ERR_UNSUPPORTED;  // R is read with 32-bit byte offsets
    return LQ_OK;
}

lq_status lq_rot_sizes(const lq_config* cfg, size_t* state_bytes)
{
    if (!cfg || !state_bytes) return LQ_ERR_NULL;
    Dims d;
    lq_status st = rot_dims(cfg, &d);
    if (st != LQ_OK) return st;
    *state_bytes = rot_layout(d).total;
    return LQ_OK;
}

lq_status lq_rot_init(const lq_config* cfg, const float* Omega0, const float* Mom0, void* state, size_t state_bytes,
                      void* stream)
{
    Dims d;
    lq_status st = rot_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (!state) return LQ_ERR_NULL;
    if (!aligned(state, 256) || !aligned(Omega0, 4) || !aligned(Mom0, 4)) return LQ_ERR_ALIGN;
    if (state_bytes < rot_layout(d).total) return LQ_ERR_BUFFER_TOO_SMALL;
    return launch_rot_init(d, Omega0, Mom0, (uint8_t*)state, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_rot_step(const lq_config* cfg, const float* L, const float* R, void* state, size_t state_bytes,
                      const lq_cayley* opt, float* loss, void* stream)
{
    Dims d;
    lq_status st = rot_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (!L || !R || !state || !opt) return LQ_ERR_NULL;
    if (!(opt->lr > 0.f) || !(opt->beta >= 0.f && opt->beta < 1.f) || !(opt->eps > 0.f) || !(opt->q > 0.f && opt->q < 1.f) ||
        opt->s < 0 || opt->s > 16 || !(opt->grad_scale > 0.f))
        return LQ_ERR_UNSUPPORTED;
    if (!aligned(state, 256) || !aligned(L, 16) || !aligned(R, 16) || (loss && !aligned(loss, 4))) return LQ_ERR_ALIGN;
    if (state_bytes < rot_layout(d).total) return LQ_ERR_BUFFER_TOO_SMALL;
    return launch_rot_step(d, L, R, (uint8_t*)state, opt, loss, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_rot_step_static(const lq_config* cfg, const float* L, const float* R, void* state, size_t state_bytes,
                             const lq_cayley* opt, float* loss, void* stream)
{
    Dims d;
    lq_status st = rot_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (!L || !R || !state || !opt) return LQ_ERR_NULL;
    if (!(opt->lr > 0.f) || !(opt->beta >= 0.f && opt->beta < 1.f) || !(opt->eps > 0.f) || !(opt->q > 0.f && opt->q < 1.f) ||
        opt->s < 0 || opt->s > 16 || !(opt->grad_scale > 0.f))
        return LQ_ERR_UNSUPPORTED;
    if (d.r > 64 || rot_static_scratch_needed(d) > LQ_ROT_STATIC_SCRATCH_BYTES) return LQ_ERR_UNSUPPORTED;  // beyond the library's array
    if (!aligned(state, 256) || !aligned(L, 16) || !aligned(R, 16) || (loss && !aligned(loss, 4))) return LQ_ERR_ALIGN;
    if (state_bytes < rot_layout(d).off_ax) return LQ_ERR_BUFFER_TOO_SMALL;  // Omega, momentum, gradient, E1, E2
    return launch_rot_step_static(d, L, R, (uint8_t*)state, opt, loss, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_rot_apply(const lq_config* cfg, const float* L, const float* R, const void* state, float* Lr, float* Rr,
                       void* stream)
{
    Dims d;
    lq_status st = rot_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (!L || !R || !state || !Lr || !Rr) return LQ_ERR_NULL;
    if (!aligned(state, 256) || !aligned(L, 16) || !aligned(R, 16) || !aligned(Lr, 16) || !aligned(Rr, 16)) return LQ_ERR_ALIGN;
    return launch_rot_apply(d, L, R, (const uint8_t*)state, Lr, Rr, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_rot_unpack(const lq_config* cfg, const void* state, const lq_rot_view* out, void* stream)
{
    Dims d;
    lq_status st = rot_dims(cfg, &d);
    if (st != LQ_OK) return st;
    if (!state || !out) return LQ_ERR_NULL;
    if (!aligned(state, 256)) return LQ_ERR_ALIGN;
    return launch_rot_unpack(d, (const uint8_t*)state, out, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

static lq_status adapter_check(const lq_adapter_config* c)
{
    if (!c) return LQ_ERR_NULL;
    if (c->flags != 0 || (c->x_dtype != LQ_F32 && c->x_dtype != LQ_BF16)) return LQ_ERR_UNSUPPORTED;
    if (c->N <= 0 || c->K <= 0 || c->N > (1 << 22) || c->K > (1 << 22) || c->N % 64 != 0 || c->K % 64 != 0) return LQ_ERR_SHAPE;
    if (c->rank < 8 || c->rank > 128 || c->rank % 8 != 0 || c->slots < 1 || c->slots > 1024) return LQ_ERR_SHAPE;
    if ((int64_t)c->slots * c->rank * (c->N + c->K) >= ((int64_t)1 << 32)) return LQ_ERR_UNSUPPORTED;  // (launches stay below 2^32 threads)
    return LQ_OK;
}
static lq_status adapter_batch_check(int64_t M)
{
    return M < 0 || M > (1 << 24) ? LQ_ERR_SHAPE : LQ_OK;
}
// rows of `len` values of `elem` bytes
static lq_status rows_check(const void* p, int64_t ld, int64_t len, int elem)
{
    if (ld < len || ld > (1 << 22)) return LQ_ERR_SHAPE;
    return aligned(p, 16) && ld * elem % 16 == 0 ? LQ_OK : LQ_ERR_ALIGN;
}
static lq_status pool_check(const lq_adapter_pool* p)
{
    if (!p || !p->A || !p->B || !p->ranks || !p->scales) return LQ_ERR_NULL;
    return aligned(p->A, 16) && aligned(p->B, 16) && aligned(p->ranks, 4) && aligned(p->scales, 4) ? LQ_OK : LQ_ERR_ALIGN;
}
static size_t adapter_inter_bytes(const lq_adapter_config* c, int64_t M) { return align256((size_t)M * ((c->rank + 15) / 16 * 16) * 4); }

lq_status lq_adapter_plan_sizes(int64_t M, int32_t slots, size_t* plan_bytes)
{
    if (!plan_bytes) return LQ_ERR_NULL;
    if (M < 0 || M > (1 << 24) || slots < 1 || slots > 1024) return LQ_ERR_SHAPE;
    *plan_bytes = adapter_plan_layout(M, slots).total;
    return LQ_OK;
}

lq_status lq_adapter_plan(int32_t slots, const int32_t* ids, int64_t M, void* plan, size_t plan_bytes, void* stream)
{
    size_t need;
    lq_status st = lq_adapter_plan_sizes(M, slots, &need);
    if (st != LQ_OK) return st;
    if (!plan || (M > 0 && !ids)) return LQ_ERR_NULL;
    if (!aligned(plan, 256) || !aligned(ids, 4)) return LQ_ERR_ALIGN;
    if (plan_bytes < need) return LQ_ERR_BUFFER_TOO_SMALL;
    return launch_adapter_plan(slots, ids, M, (uint8_t*)plan, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_adapter_verify_plan(int32_t slots, int64_t M, const void* plan, size_t plan_bytes, void* stream)
{
    size_t need;
    lq_status st = lq_adapter_plan_sizes(M, slots, &need);
    if (st != LQ_OK) return st;
    if (!plan) return LQ_ERR_NULL;
    if (!aligned(plan, 256)) return LQ_ERR_ALIGN;
    if (plan_bytes < need) return LQ_ERR_BUFFER_TOO_SMALL;
    BlobTag got;
    if (hipMemcpyAsync(&got, plan, sizeof(got), hipMemcpyDeviceToHost, (hipStream_t)stream) != hipSuccess) return LQ_ERR_DEVICE;
    if (hipStreamSynchronize((hipStream_t)stream) != hipSuccess) return LQ_ERR_DEVICE;
    const BlobTag want = plan_tag(M, slots);
    for (int i = 0; i < 8; ++i)
        if (got.w[i] != want.w[i]) return LQ_ERR_STALE_BLOB;
    return LQ_OK;
}

lq_status lq_adapter_sizes(const lq_adapter_config* cfg, int64_t M, size_t* inter_bytes, size_t* work_bytes)
{
    lq_status st = adapter_check(cfg);
    if (st != LQ_OK) return st;
    if ((st = adapter_batch_check(M)) != LQ_OK) return st;
    if (inter_bytes) *inter_bytes = adapter_inter_bytes(cfg, M);
    if (work_bytes) *work_bytes = adapter_work_layout(cfg, M).total;
    return LQ_OK;
}

lq_status lq_adapter_fwd(const lq_adapter_config* cfg, const void* plan, size_t plan_bytes, const lq_adapter_pool* pool, const void* X,
                         int64_t ldx, const void* Yin, int64_t ldyin, void* Y, int64_t ldy, int64_t M, void* inter, size_t inter_bytes,
                         void* stream)
{
    lq_status st = adapter_check(cfg);
    if (st != LQ_OK) return st;
    if ((st = adapter_batch_check(M)) != LQ_OK) return st;
    if (M == 0) return LQ_OK;  // an empty batch
    if (!plan || !X || !Yin || !Y || !inter) return LQ_ERR_NULL;
    if ((st = pool_check(pool)) != LQ_OK) return st;
    if ((st = rows_check(X, ldx, cfg->K, cfg->x_dtype == LQ_F32 ? 4 : 2)) != LQ_OK || (st = rows_check(Yin, ldyin, cfg->N, 2)) != LQ_OK ||
        (st = rows_check(Y, ldy, cfg->N, 2)) != LQ_OK)
        return st;
    if (!aligned(plan, 256) || !aligned(inter, 256)) return LQ_ERR_ALIGN;
    if (plan_bytes < adapter_plan_layout(M, cfg->slots).total || inter_bytes < adapter_inter_bytes(cfg, M)) return LQ_ERR_BUFFER_TOO_SMALL;
    return launch_adapter_fwd(cfg, (const uint8_t*)plan, pool, X, ldx, Yin, ldyin, Y, ldy, M, (uint8_t*)inter, (hipStream_t)stream) == hipSuccess
               ? LQ_OK
               : LQ_ERR_DEVICE;
}

lq_status lq_adapter_bwd(const lq_adapter_config* cfg, const void* plan, size_t plan_bytes, const lq_adapter_pool* pool, const void* X,
                         int64_t ldx, const void* inter, size_t inter_bytes, const void* dY, int64_t lddy, const void* dXin,
                         int64_t lddxin, void* dX, int64_t lddx, float* dA, float* dB, int64_t M, void* work, size_t work_bytes,
                         void* stream)
{
    lq_status st = adapter_check(cfg);
    if (st != LQ_OK) return st;
    if ((st = adapter_batch_check(M)) != LQ_OK) return st;
    if (!dA || !dB) return LQ_ERR_NULL;
    if (!aligned(dA, 16) || !aligned(dB, 16)) return LQ_ERR_ALIGN;
    if (M == 0) return launch_adapter_zero(cfg, dA, dB, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
    if (!plan || !X || !inter || !dY || !dX || !work) return LQ_ERR_NULL;
    if ((st = pool_check(pool)) != LQ_OK) return st;
    const int elem = cfg->x_dtype == LQ_F32 ? 4 : 2;
    if ((st = rows_check(X, ldx, cfg->K, elem)) != LQ_OK || (st = rows_check(dY, lddy, cfg->N, 2)) != LQ_OK ||
        (st = rows_check(dX, lddx, cfg->K, elem)) != LQ_OK || (dXin && (st = rows_check(dXin, lddxin, cfg->K, elem)) != LQ_OK))
        return st;
    if (!aligned(plan, 256) || !aligned(inter, 256) || !aligned(work, 256)) return LQ_ERR_ALIGN;
    if (plan_bytes < adapter_plan_layout(M, cfg->slots).total || inter_bytes < adapter_inter_bytes(cfg, M) ||
        work_bytes < adapter_work_layout(cfg, M).total)
        return LQ_ERR_BUFFER_TOO_SMALL;
    return launch_adapter_bwd(cfg, (const uint8_t*)plan, pool, X, ldx, (const uint8_t*)inter, dY, lddy, dXin, lddxin, dX, lddx, dA, dB, M,
                              (uint8_t*)work, (hipStream_t)stream) == hipSuccess
               ? LQ_OK
               : LQ_ERR_DEVICE;
}

static lq_status qk_check(const lq_qk_config* c, int64_t M)
{
    if (!c) return LQ_ERR_NULL;
    if (c->flags != 0 || (c->dtype != LQ_F32 && c->dtype != LQ_BF16) || (c->pairing != LQ_PAIR_HALF && c->pairing != LQ_PAIR_ADJACENT) ||
        (c->norm != LQ_NORM_NONE && c->norm != LQ_NORM_RMS) || (c->norm == LQ_NORM_RMS && !(c->eps > 0.f)))
        return LQ_ERR_UNSUPPORTED;
    if (c->heads_q < 0 || c->heads_k < 0 || c->heads_q > 4096 || c->heads_k > 4096 || c->heads_q + c->heads_k < 1 ||
        c->heads_q + c->heads_k > 4096 || c->head_dim < 2 || c->head_dim > 256 || c->head_dim % 2 != 0 || c->axes < 0 || c->axes > 4)
        return LQ_ERR_SHAPE;
    int sum = 0;
    for (int k = 0; k < 4; ++k) {
        if (c->pairs[k] < 0 || c->pairs[k] > 128 || (k >= c->axes && c->pairs[k] != 0)) return LQ_ERR_SHAPE;
        sum += c->pairs[k];
    }
    if (2 * sum > c->head_dim || M < 0 || M > (1 << 24)) return LQ_ERR_SHAPE;
    return LQ_OK;
}
static lq_status heads_check(const lq_qk_config* c, const lq_heads* h, int heads, lq_heads* out)
{
    if (heads == 0) return LQ_OK;  // not looked at
    if (!h || !h->p) return LQ_ERR_NULL;
    if (h->ld < 0 || h->hs < 0 || h->ld >= ((int64_t)1 << 40) || h->hs >= ((int64_t)1 << 40)) return LQ_ERR_SHAPE;
    if (!aligned(h->p, c->dtype == LQ_F32 ? 4 : 2)) return LQ_ERR_ALIGN;
    *out = *h;
    return LQ_OK;
}
// Whether the heads of an output lie apart: no two of them have a value in common.
static bool heads_apart(const lq_heads& h, int64_t heads, int64_t dim, int64_t M)
{
    if ((heads > 1 && h.hs < dim) || (M > 1 && h.ld < dim)) return false;
    if (heads < 2 || M < 2 || h.ld - dim >= (heads - 1) * h.hs || (h.hs - dim) / h.ld >= M - 1) return true;  // head by head in a token, or token by token in a head
    for (int64_t b = 1; b < heads; ++b) {  // heads b apart, of tokens so far apart that their offsets are the nearest
        const int64_t at = b * h.hs, a = at / h.ld;
        if ((a >= 1 && a < M && at - a * h.ld < dim) || (a + 1 < M && (a + 1) * h.ld - at < dim)) return false;
    }
    return true;
}
// outputs of queries and keys
static lq_status outputs_check(const lq_qk_config* c, const lq_heads* q, const lq_heads* k, int64_t M, lq_heads* out)
{
    const lq_heads* in[2] = {q, k};
    const int heads[2] = {c->heads_q, c->heads_k};
    for (int s = 0; s < 2; ++s) {
        const lq_status st = heads_check(c, in[s], heads[s], &out[s]);
        if (st != LQ_OK) return st;
        if (heads[s] && !heads_apart(out[s], heads[s], c->head_dim, M)) return LQ_ERR_SHAPE;
    }
    return LQ_OK;
}
static lq_status positions_check(const lq_qk_config* c, const float* pos, int64_t pos_rows, const float* inv_freq)
{
    if (c->pairs[0] + c->pairs[1] + c->pairs[2] + c->pairs[3] == 0) return LQ_OK;
    if (!pos || !inv_freq) return LQ_ERR_NULL;
    if (pos_rows < 1 || pos_rows > (1 << 24)) return LQ_ERR_SHAPE;
    return aligned(pos, 4) && aligned(inv_freq, 4) ? LQ_OK : LQ_ERR_ALIGN;
}

lq_status lq_qk_norm_rope_fwd(const lq_qk_config* cfg, const lq_heads* q, const lq_heads* k, const float* wq, const float* wk,
                              const float* pos, int64_t pos_rows, const float* inv_freq, const lq_heads* qo, const lq_heads* ko, int64_t M,
                              void* stream)
{
    lq_status st = qk_check(cfg, M);
    if (st != LQ_OK) return st;
    if (M == 0) return LQ_OK;  // an empty batch
    QkTensors t{};
    if ((st = heads_check(cfg, q, cfg->heads_q, &t.q[0])) != LQ_OK || (st = heads_check(cfg, k, cfg->heads_k, &t.q[1])) != LQ_OK ||
        (st = outputs_check(cfg, qo, ko, M, t.out)) != LQ_OK ||
        (st = positions_check(cfg, pos, pos_rows, inv_freq)) != LQ_OK)
        return st;
    if (!aligned(wq, 4) || !aligned(wk, 4)) return LQ_ERR_ALIGN;
    t.w[0] = wq;
    t.w[1] = wk;
    t.pos = pos;
    t.pos_rows = pos_rows;
    t.inv_freq = inv_freq;
    return launch_qk_fwd(cfg, t, M, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_qk_work_sizes(const lq_qk_config* cfg, int64_t M, size_t* work_bytes)
{
    if (!cfg || !work_bytes) return LQ_ERR_NULL;
    lq_status st = qk_check(cfg, M);
    if (st != LQ_OK) return st;
    *work_bytes = qk_work_bytes(cfg, M);
    return LQ_OK;
}

lq_status lq_qk_norm_rope_bwd(const lq_qk_config* cfg, const lq_heads* q, const lq_heads* k, const float* wq, const float* wk,
                              const float* pos, int64_t pos_rows, const float* inv_freq, const lq_heads* dqo, const lq_heads* dko,
                              const lq_heads* dq, const lq_heads* dk, float* dwq, float* dwk, int64_t M, void* work, size_t work_bytes,
                              void* stream)
{
    lq_status st = qk_check(cfg, M);
    if (st != LQ_OK) return st;
    const bool norm = cfg->norm == LQ_NORM_RMS;
    if (norm && (!dwq) != (!dwk)) return LQ_ERR_NULL;
    QkTensors t{};
    if (M > 0) {
        if ((norm && ((st = heads_check(cfg, q, cfg->heads_q, &t.q[0])) != LQ_OK || (st = heads_check(cfg, k, cfg->heads_k, &t.q[1])) != LQ_OK)) ||
            (st = heads_check(cfg, dqo, cfg->heads_q, &t.grad[0])) != LQ_OK || (st = heads_check(cfg, dko, cfg->heads_k, &t.grad[1])) != LQ_OK ||
            (st = outputs_check(cfg, dq, dk, M, t.out)) != LQ_OK ||
            (st = positions_check(cfg, pos, pos_rows, inv_freq)) != LQ_OK)
            return st;
        if (norm && dwq && !work) return LQ_ERR_NULL;
        if (norm && dwq && work_bytes < qk_work_bytes(cfg, M)) return LQ_ERR_BUFFER_TOO_SMALL;
    }
    if (!aligned(wq, 4) || !aligned(wk, 4) || (norm && (!aligned(dwq, 4) || !aligned(dwk, 4) || !aligned(work, 256)))) return LQ_ERR_ALIGN;
    t.w[0] = wq;
    t.w[1] = wk;
    t.pos = pos;
    t.pos_rows = pos_rows;
    t.inv_freq = inv_freq;
    t.dw[0] = dwq;
    t.dw[1] = dwk;
    return launch_qk_bwd(cfg, t, M, (uint8_t*)work, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

static lq_status w4_check(const lq_w4_config* c)
{
    if (!c) return LQ_ERR_NULL;
    if (c->flags != 0 || (c->x_dtype != LQ_F32 && c->x_dtype != LQ_BF16) || (c->y_dtype != LQ_F32 && c->y_dtype != LQ_BF16)) return LQ_ERR_UNSUPPORTED;
    if (c->N < 1 || c->K < 1 || c->N > (1 << 18) || c->K > (1 << 16) || (c->group != 32 && c->group != 64 && c->group != 128)) return LQ_ERR_SHAPE;
    return LQ_OK;
}
static lq_status w4_packed_check(const lq_w4_config* c, const void* packed, size_t packed_bytes)
{
    if (!packed) return LQ_ERR_NULL;
    if (!aligned(packed, 256)) return LQ_ERR_ALIGN;
    return packed_bytes < w4_packed_bytes(c) ? LQ_ERR_BUFFER_TOO_SMALL : LQ_OK;
}
// M rows of `len` values that may start anywhere; the stride of a single row says nothing
static lq_status any_rows_check(const void* p, int64_t ld, int64_t len, int64_t M, int elem, int64_t most = ((int64_t)1 << 40) - 1)
{
    if (!p) return LQ_ERR_NULL;
    if (M > 1 && (ld < len || ld > most)) return LQ_ERR_SHAPE;
    return aligned(p, elem) ? LQ_OK : LQ_ERR_ALIGN;
}
static int dtype_bytes(int32_t dtype) { return dtype == LQ_F32 ? 4 : 2; }

lq_status lq_w4_sizes(const lq_w4_config* cfg, size_t* packed_bytes)
{
    lq_status st = w4_check(cfg);
    if (st != LQ_OK) return st;
    if (!packed_bytes) return LQ_ERR_NULL;
    *packed_bytes = w4_packed_bytes(cfg);
    return LQ_OK;
}

lq_status lq_w4_pack(const lq_w4_config* cfg, const float* W, void* packed, size_t packed_bytes, void* stream)
{
    lq_status st = w4_check(cfg);
    if (st != LQ_OK || (st = w4_packed_check(cfg, packed, packed_bytes)) != LQ_OK) return st;
    if (!W) return LQ_ERR_NULL;
    if (!aligned(W, 4)) return LQ_ERR_ALIGN;
    return launch_w4_pack(cfg, W, nullptr, nullptr, (uint8_t*)packed, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_w4_pack_codes(const lq_w4_config* cfg, const int8_t* codes, const float* scales, void* packed, size_t packed_bytes, void* stream)
{
    lq_status st = w4_check(cfg);
    if (st != LQ_OK || (st = w4_packed_check(cfg, packed, packed_bytes)) != LQ_OK) return st;
    if (!codes || !scales) return LQ_ERR_NULL;
    if (!aligned(scales, 4)) return LQ_ERR_ALIGN;
    return launch_w4_pack(cfg, nullptr, codes, scales, (uint8_t*)packed, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_w4_unpack(const lq_w4_config* cfg, const void* packed, size_t packed_bytes, int8_t* codes, float* scales, void* stream)
{
    lq_status st = w4_check(cfg);
    if (st != LQ_OK || (st = w4_packed_check(cfg, packed, packed_bytes)) != LQ_OK) return st;
    if (!aligned(scales, 4)) return LQ_ERR_ALIGN;
    if (!codes && !scales) return LQ_OK;
    return launch_w4_unpack(cfg, (const uint8_t*)packed, codes, scales, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_w4_verify(const lq_w4_config* cfg, const void* packed, size_t packed_bytes, void* stream)
{
    lq_status st = w4_check(cfg);
    if (st != LQ_OK || (st = w4_packed_check(cfg, packed, packed_bytes)) != LQ_OK) return st;
    BlobTag got;
    if (hipMemcpyAsync(&got, packed, sizeof(got), hipMemcpyDeviceToHost, (hipStream_t)stream) != hipSuccess) return LQ_ERR_DEVICE;
    if (hipStreamSynchronize((hipStream_t)stream) != hipSuccess) return LQ_ERR_DEVICE;
    const BlobTag want = w4_tag(cfg);
    for (int i = 0; i < 8; ++i)
        if (got.w[i] != want.w[i]) return LQ_ERR_STALE_BLOB;
    return LQ_OK;
}

static lq_status w4_batch_check(int64_t M) { return M < 0 || M > (1 << 14) ? LQ_ERR_SHAPE : LQ_OK; }

lq_status lq_w4_fwd(const lq_w4_config* cfg, const void* packed, size_t packed_bytes, const void* X, int64_t ldx, const float* bias, void* Y, int64_t ldy,
                    int64_t M, void* stream)
{
    lq_status st = w4_check(cfg);
    if (st != LQ_OK || (st = w4_batch_check(M)) != LQ_OK) return st;
    if (M == 0) return LQ_OK;  // an empty batch
    if ((st = w4_packed_check(cfg, packed, packed_bytes)) != LQ_OK || (st = any_rows_check(X, ldx, cfg->K, M, dtype_bytes(cfg->x_dtype), 1 << 22)) != LQ_OK ||
        (st = any_rows_check(Y, ldy, cfg->N, M, dtype_bytes(cfg->y_dtype), 1 << 22)) != LQ_OK)
        return st;
    if (!aligned(bias, 4)) return LQ_ERR_ALIGN;
    return launch_w4_fwd(cfg, (const uint8_t*)packed, X, ldx, bias, Y, ldy, M, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_w4_work_sizes(const lq_w4_config* cfg, int64_t M, size_t* work_bytes)
{
    lq_status st = w4_check(cfg);
    if (st != LQ_OK || (st = w4_batch_check(M)) != LQ_OK) return st;
    if (!work_bytes) return LQ_ERR_NULL;
    *work_bytes = w4_work_bytes(cfg, M);
    return LQ_OK;
}

lq_status lq_w4_bwd(const lq_w4_config* cfg, const void* packed, size_t packed_bytes, const void* dY, int64_t lddy, void* dX, int64_t lddx, int64_t M, void* work,
                    size_t work_bytes, void* stream)
{
    lq_status st = w4_check(cfg);
    if (st != LQ_OK || (st = w4_batch_check(M)) != LQ_OK) return st;
    if (M == 0) return LQ_OK;  // an empty batch
    if ((st = w4_packed_check(cfg, packed, packed_bytes)) != LQ_OK || (st = any_rows_check(dY, lddy, cfg->N, M, dtype_bytes(cfg->y_dtype), 1 << 22)) != LQ_OK ||
        (st = any_rows_check(dX, lddx, cfg->K, M, dtype_bytes(cfg->x_dtype), 1 << 22)) != LQ_OK)
        return st;
    const size_t need = w4_work_bytes(cfg, M);
    if (need && !work) return LQ_ERR_NULL;
    if (need && !aligned(work, 256)) return LQ_ERR_ALIGN;
    if (work_bytes < need) return LQ_ERR_BUFFER_TOO_SMALL;
    return launch_w4_bwd(cfg, (const uint8_t*)packed, dY, lddy, dX, lddx, M, (uint8_t*)work, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

static bool norm_known(int32_t n) { return n == LQ_NORM_NONE || n == LQ_NORM_RMS || n == LQ_NORM_LAYER; }
static lq_status block_check(const lq_block_config* c, int64_t M, int64_t S, bool offsets)
{
    if (!c) return LQ_ERR_NULL;
    if (c->flags != 0 || !norm_known(c->post) || !norm_known(c->pre) || (c->h_dtype != LQ_F32 && c->h_dtype != LQ_BF16) ||
        (c->y_dtype != LQ_F32 && c->y_dtype != LQ_BF16) || (c->h_dtype == LQ_BF16 && c->y_dtype == LQ_F32))
        return LQ_ERR_UNSUPPORTED;
    if ((c->post != LQ_NORM_NONE || c->pre != LQ_NORM_NONE) && !(c->eps > 0.f)) return LQ_ERR_UNSUPPORTED;
    if (!(c->res_scale - c->res_scale == 0.f)) return LQ_ERR_UNSUPPORTED;  // not finite
    if (c->dim < 1 || c->dim > 16384 || M < 0 || M > (1 << 24) || S < 1 || S > (1 << 20) || (!offsets && S != 1)) return LQ_ERR_SHAPE;
    return LQ_OK;
}
lq_status lq_block_norm_fwd(const lq_block_config* cfg, const void* h, int64_t ldh, const void* y, int64_t ldy, const int32_t* offsets, int32_t S,
                            const lq_mod* gate, const lq_mod* scale, const lq_mod* shift, const float* w_post, const float* w_pre, void* ho,
                            int64_t ldho, void* x, int64_t ldx, int64_t M, void* stream)
{
    lq_status st = block_check(cfg, M, S, offsets != nullptr);
    if (st != LQ_OK) return st;
    BlockTensors t{};
    if ((st = mod_check(gate, cfg, S, &t.gate)) != LQ_OK || (st = mod_check(scale, cfg, S, &t.scale)) != LQ_OK || (st = mod_check(shift, cfg, S, &t.shift)) != LQ_OK) return st;
    if (!aligned(offsets, 4) || !aligned(w_post, 4) || !aligned(w_pre, 4)) return LQ_ERR_ALIGN;
    if (M == 0) return LQ_OK;  // an empty batch
    const int he = dtype_bytes(cfg->h_dtype), ye = dtype_bytes(cfg->y_dtype);
    if ((!y) != (!ho) || (!y && !x)) return LQ_ERR_NULL;
    if ((st = any_rows_check(h, ldh, cfg->dim, M, he)) != LQ_OK || (y && (st = any_rows_check(y, ldy, cfg->dim, M, ye)) != LQ_OK) ||
        (ho && (st = any_rows_check(ho, ldho, cfg->dim, M, he)) != LQ_OK) || (x && (st = any_rows_check(x, ldx, cfg->dim, M, ye)) != LQ_OK))
        return st;
    t.h = h;
    t.ldh = ldh;
    t.y = y;
    t.ldy = ldy;
    t.offsets = offsets;
    t.S = S;
    t.w_post = w_post;
    t.w_pre = w_pre;
    t.ho = ho;
    t.ldho = ldho;
    t.x = x;
    t.ldx = ldx;
    return launch_block_fwd(cfg, t, M, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

lq_status lq_block_work_sizes(const lq_block_config* cfg, int64_t M, int32_t S, size_t* work_bytes)
{
    lq_status st = block_check(cfg, M, S, true);
    if (st != LQ_OK) return st;
    if (!work_bytes) return LQ_ERR_NULL;
    *work_bytes = block_work_bytes(cfg, M, S);
    return LQ_OK;
}

lq_status lq_block_norm_bwd(const lq_block_config* cfg, const void* ho, int64_t ldho, const void* y, int64_t ldy, const int32_t* offsets, int32_t S,
                            const lq_mod* gate, const lq_mod* scale, const float* w_post, const float* w_pre, const void* dho, int64_t lddho,
                            const void* dx, int64_t lddx, const lq_block_grads* out, int64_t M, void* work, size_t work_bytes, void* stream)
{
    lq_status st = block_check(cfg, M, S, offsets != nullptr);
    if (st != LQ_OK) return st;
    if (!out) return LQ_ERR_NULL;
    BlockTensors t{};
    if ((st = mod_check(gate, cfg, S, &t.gate)) != LQ_OK || (st = mod_check(scale, cfg, S, &t.scale)) != LQ_OK ||
        (st = mod_check(&out->dgate, cfg, S, &t.dgate)) != LQ_OK || (st = mod_check(&out->dscale, cfg, S, &t.dscale)) != LQ_OK ||
        (st = mod_check(&out->dshift, cfg, S, &t.dshift)) != LQ_OK)
        return st;
    if (!aligned(offsets, 4) || !aligned(w_post, 4) || !aligned(w_pre, 4) || !aligned(out->dw_post, 4) || !aligned(out->dw_pre, 4)) return LQ_ERR_ALIGN;
    const int he = dtype_bytes(cfg->h_dtype), ye = dtype_bytes(cfg->y_dtype);
    if (M > 0) {
        if (!dho && !dx) return LQ_ERR_NULL;
        if (!y && (out->dy || t.dgate.p || out->dw_post)) return LQ_ERR_NULL;
        if ((dx && ((st = any_rows_check(dx, lddx, cfg->dim, M, ye)) != LQ_OK || (st = any_rows_check(ho, ldho, cfg->dim, M, he)) != LQ_OK)) ||
            (dho && (st = any_rows_check(dho, lddho, cfg->dim, M, he)) != LQ_OK) || (y && (st = any_rows_check(y, ldy, cfg->dim, M, ye)) != LQ_OK) ||
            (out->dh && (st = any_rows_check(out->dh, out->lddh, cfg->dim, M, he)) != LQ_OK) ||
            (out->dy && (st = any_rows_check(out->dy, out->lddy, cfg->dim, M, ye)) != LQ_OK))
            return st;
    }
    if (t.dgate.p || t.dscale.p || t.dshift.p || out->dw_post || out->dw_pre) {
        if (!work) return LQ_ERR_NULL;
        if (!aligned(work, 256)) return LQ_ERR_ALIGN;
        if (work_bytes < block_work_bytes(cfg, M, S)) return LQ_ERR_BUFFER_TOO_SMALL;
    }
    t.h = ho;
    t.ldh = ldho;
    t.y = y;
    t.ldy = ldy;
    t.offsets = offsets;
    t.S = S;
    t.w_post = w_post;
    t.w_pre = w_pre;
    t.dho = dho;
    t.lddho = lddho;
    t.dx = dx;
    t.lddx = lddx;
    t.dh = out->dh;
    t.lddh = out->lddh;
    t.dy = out->dy;
    t.lddy = out->lddy;
    t.dw_post = out->dw_post;
    t.dw_pre = out->dw_pre;
    return launch_block_bwd(cfg, t, M, (uint8_t*)work, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

// Whether the memory that a step writes lies apart.  Tensors of a kind mostly come in the order of their addresses, and kinds often in memory of their own: then a walk shows it.
// (Sorting all of them took longer than the step where many tensors are small.)
struct Spans {
    typedef std::pair<uintptr_t, uintptr_t> Span;
    std::vector<Span> all, hulls;
    std::vector<size_t> kinds;  // where each begins
    bool rising = true;
    void begin()                // the next kind
    {
        hulls.emplace_back(0, 0);
        kinds.push_back(all.size());
    }
    void add(const void* p, int64_t bytes)
    {
        if (!p || bytes == 0) return;
        const Span s((uintptr_t)p, (uintptr_t)p + (uintptr_t)bytes);
        Span& hull = hulls.back();
        if (hull.second == 0) hull.first = s.first;
        else if (s.first < hull.second) rising = false;
        hull.second = s.second;
        all.push_back(s);
    }
    static bool apart(const std::vector<Span>& r)  // in order
    {
        for (size_t i = 1; i < r.size(); ++i)
            if (r[i].first < r[i - 1].second) return false;
        return true;
    }
    bool apart()
    {
        if (!rising) {
            std::sort(all.begin(), all.end());
            return apart(all);
        }
        std::sort(hulls.begin(), hulls.end());
        if (apart(hulls)) return true;
        for (size_t k = 1; k < kinds.size(); ++k)
            std::inplace_merge(all.begin(), all.begin() + kinds[k], k + 1 < kinds.size() ? all.begin() + kinds[k + 1] : all.end());
        return apart(all);
    }
};

lq_status lq_adamw_step(const lq_adamw_config* cfg, const lq_adamw_tensor* tensors, int32_t count, const lq_adamw_args* args, void* stream)
{
    if (!cfg || !args) return LQ_ERR_NULL;
    if (cfg->flags != 0 || cfg->reserved != 0 || (cfg->p_dtype != LQ_F32 && cfg->p_dtype != LQ_BF16) || (cfg->g_dtype != LQ_F32 && cfg->g_dtype != LQ_BF16) ||
        (cfg->state_bits != 32 && cfg->state_bits != 8) || !(cfg->beta1 >= 0.0 && cfg->beta1 < 1.0) || !(cfg->beta2 >= 0.0 && cfg->beta2 < 1.0) || !(cfg->eps >= 1e-30) ||
        !(cfg->weight_decay >= 0.0))
        return LQ_ERR_UNSUPPORTED;
    if (count < 0 || count > 65536 || (!args->step_dev && (args->step < 1 || args->step > 0x7FFFFFFF))) return LQ_ERR_SHAPE;
    if (!args->lr_dev && !(args->lr - args->lr == 0.0)) return LQ_ERR_UNSUPPORTED;  // not finite
    if (!aligned(args->lr_dev, 4) || !aligned(args->step_dev, 4) || !aligned(args->grad_scale, 4)) return LQ_ERR_ALIGN;
    if (count == 0) return LQ_OK;
    if (!tensors) return LQ_ERR_NULL;
    const bool eight = cfg->state_bits == 8;
    const int pe = dtype_bytes(cfg->p_dtype), ge = dtype_bytes(cfg->g_dtype), se = eight ? 1 : 4;
    for (int32_t i = 0; i < count; ++i) {
        const lq_adamw_tensor& t = tensors[i];
        if (t.n < 0 || t.n >= ((int64_t)1 << 32)) return LQ_ERR_SHAPE;
        if (t.n == 0) continue;
        if (!t.p || !t.grad || !t.m || !t.v || (eight && !t.scales)) return LQ_ERR_NULL;
        const uintptr_t odd = ((uintptr_t)t.p & (pe - 1)) | ((uintptr_t)t.grad & (ge - 1)) | (((uintptr_t)t.m | (uintptr_t)t.v) & (se - 1)) |
                              (((uintptr_t)t.master | (uintptr_t)t.scales) & 3);
        if (odd) return LQ_ERR_ALIGN;
    }
    try {
        Spans written;
        written.all.reserve((size_t)count * 5);
        written.begin();
        for (int32_t i = 0; i < count; ++i) written.add(tensors[i].p, tensors[i].n * pe);
        written.begin();
        for (int32_t i = 0; i < count; ++i) written.add(tensors[i].master, tensors[i].n * 4);
        written.begin();
        for (int32_t i = 0; i < count; ++i) written.add(tensors[i].m, tensors[i].n * se);
        written.begin();
        for (int32_t i = 0; i < count; ++i) written.add(tensors[i].v, tensors[i].n * se);
        written.begin();
        for (int32_t i = 0; eight && i < count; ++i) written.add(tensors[i].scales, (tensors[i].n + 255) / 256 * 8);
        if (!written.apart()) return LQ_ERR_SHAPE;
    } catch (const std::bad_alloc&) {
        return LQ_ERR_DEVICE;
    }
    return launch_adamw(cfg, tensors, count, args, (hipStream_t)stream) == hipSuccess ? LQ_OK : LQ_ERR_DEVICE;
}

}  // extern "C"
