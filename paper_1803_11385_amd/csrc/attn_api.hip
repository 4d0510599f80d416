// C entries of attention inside the shapes of a ragged batch.
#include <algorithm>
#include <cmath>

#include "attn_launch.hpp"

namespace {

using hch::attn::Args;

int size_of(hch_dtype t) { return t == HCH_F32 ? 4 : 2; }
size_t round256(size_t x) { return (x + 255) / 256 * 256; }

// How a pass over the keys is cut.
struct Plan {
    bool narrow;           // one row tile of 32 per workgroup, whose wavefronts share the keys
    int64_t slots;
    int splits;
};

// Workgroups of tiles of `size` rows there will be about (offsets are known on the device only).
int64_t tiles_of(int64_t rows, int size, int batch, int heads) { return std::max<int64_t>(batch, (rows + size - 1) / size) * heads; }

// The narrow forms take a quarter of the time for a tile, but hold as much of LDS (in fp32 beyond 32 channels all
// that a compute unit lets two workgroups have) for a quarter of the rows.  They are taken where a single round of them
// takes all tiles: measured at (wide workgroups) bf16 10: 45 -> 22 us, 38: 8.7 -> 7.2, 170: 27 -> 34; fp32 to 32 channels 52: 17 -> 13,
// 192: 20 -> 22; beyond 400: 43 -> 107.
bool narrow_fits(const hch_attn_desc &p, int64_t wide_workgroups)
{
    return wide_workgroups <= (p.dtype == HCH_BF16 || p.head_dim <= 32 ? 128 : 64);
}

Plan plan_keys(const hch_attn_desc &p)
{
    const int group = p.heads_q / p.heads_kv;
    Plan r;
    r.narrow = p.n_q * group <= (int64_t)32 * p.batch || narrow_fits(p, tiles_of(p.n_q * group, 128, p.batch, p.heads_kv));
    const int bq = r.narrow ? 32 : 128;
    r.slots = hch::attn::slots_of(p.n_q, group, bq, p.batch);
    // Where the workgroups do not fill the chip (256 compute units with 4 or 2 of them), the keys are split among
    // several and the parts joined by a second launch.
    const int64_t wgs = tiles_of(p.n_q * group, bq, p.batch, p.heads_kv);
    const int64_t tiles = p.n_k / p.batch / (r.narrow ? 128 : 64), want = r.narrow ? 1024 : 512;
    r.splits = (int)std::max<int64_t>(1, std::min<int64_t>({want / std::max<int64_t>(1, wgs), tiles / (r.narrow ? 2 : 4), 256}));
    return r;
}

bool narrow_queries(const hch_attn_desc &p) { return narrow_fits(p, tiles_of(p.n_k, 128, p.batch, p.heads_kv)); }

size_t part_bytes(const hch_attn_desc &p, int splits) { return splits > 1 ? round256((size_t)splits * p.n_q * p.heads_q * p.head_dim * 4) : 0; }
size_t ml_bytes(const hch_attn_desc &p, int splits) { return splits > 1 ? round256((size_t)splits * p.n_q * p.heads_q * 8) : 0; }
size_t delta_bytes(const hch_attn_desc &p) { return round256((size_t)p.n_q * p.heads_q * 4); }

size_t fwd_bytes(const hch_attn_desc &p)
{
    if (!p.batch || !p.n_q) return 256;
    const Plan r = plan_keys(p);
    return std::max<size_t>(256, part_bytes(p, r.splits) + ml_bytes(p, r.splits));
}
size_t bwd_bytes(const hch_attn_desc &p)
{
    if (!p.batch || !p.n_q) return 256;
    return std::max<size_t>(256, part_bytes(p, plan_keys(p).splits) + delta_bytes(p));
}

// what both calls and the size query ask of the sizes
hch_status check_sizes(const char *who, const hch_attn_desc *p)
{
    const std::string name = who;
    if (!p) return fail(HCH_EINVAL, name + ": null description");
    if (p->dtype != HCH_F32 && p->dtype != HCH_BF16) return fail(HCH_EINVAL, name + ": unknown dtype");
    if (p->batch < 0 || p->n_q < 0 || p->n_k < 0 || p->heads_q <= 0 || p->heads_kv <= 0 || p->head_dim <= 0 || p->heads_q % p->heads_kv)
        return fail(HCH_EINVAL, name + ": bad size, or heads_q not a multiple of heads_kv");
    if (p->head_dim > 128) return fail(HCH_EUNSUPPORTED, name + ": more than 128 channels per head");
    if (p->n_k > 0x7fffffff || p->n_q > 0x7fffffff / p->heads_q) return fail(HCH_EUNSUPPORTED, name + ": more than 2^31 - 1 rows");
    if (p->batch == 0 && (p->n_q || p->n_k)) return fail(HCH_EINVAL, name + ": rows without a shape");
    const int64_t group = p->heads_q / p->heads_kv;
    if (p->batch && (hch::attn::slots_of(p->n_q, (int)group, 32, p->batch) * p->heads_kv * 2 + 1024 > 0x7fffffff ||
                     hch::attn::slots_of(p->n_k, 1, 32, p->batch) * p->heads_kv + 1024 > 0x7fffffff))
        return fail(HCH_EUNSUPPORTED, name + ": too many rows for one launch");
    return HCH_OK;
}

hch_status check_call(const char *who, const hch_attn_desc *p, const void *workspace, size_t ws_bytes, size_t need)
{
    const std::string name = who;
    if (!(p->scale > 0.f) || !std::isfinite(p->scale)) return fail(HCH_EINVAL, name + ": scale must be positive and finite");
    if (p->batch && (!p->q_offsets || !p->k_offsets)) return fail(HCH_EINVAL, name + ": null offsets");
    const int64_t wq = (int64_t)p->heads_q * p->head_dim, wk = (int64_t)p->heads_kv * p->head_dim;
    if (p->ld_q < wq || p->ld_o < wq || p->ld_k < wk || p->ld_v < wk) return fail(HCH_EINVAL, name + ": row stride below a row's length");
    if (std::max({p->ld_q, p->ld_o, p->ld_k, p->ld_v}) >= 1 << 22) return fail(HCH_EUNSUPPORTED, name + ": row stride of 2^22 elements or more");
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255)) return fail(HCH_EINVAL, name + ": workspace null or not 256-byte aligned");
    if (ws_bytes < need) return fail(HCH_EWORKSPACE, name + ": workspace too small");
    return HCH_OK;
}

Args args_of(const hch_attn_desc &p)
{
    Args a = {};
    a.qo = p.q_offsets; a.ko = p.k_offsets; a.mask = p.key_mask;
    a.nq = p.n_q; a.nk = p.n_k;
    a.ld_q = p.ld_q; a.ld_k = p.ld_k; a.ld_v = p.ld_v; a.ld_o = p.ld_o;
    a.ld_do = p.ld_do; a.ld_dq = p.ld_dq; a.ld_dk = p.ld_dk; a.ld_dv = p.ld_dv;
    a.batch = p.batch; a.hq = p.heads_q; a.hkv = p.heads_kv; a.group = p.heads_q / p.heads_kv; a.d = p.head_dim;
    a.scale = p.scale; a.c = p.scale * hch::attn::LOG2E;
    return a;
}

// 16-byte pieces throughout: addresses, strides and head width in whole pieces
bool whole(const hch_attn_desc &p, std::initializer_list<const void *> ptr, std::initializer_list<int64_t> ld)
{
    const int e = 16 / size_of(p.dtype);
    bool ok = p.head_dim % e == 0;
    for (const void *x : ptr) ok = ok && (reinterpret_cast<uintptr_t>(x) & 15) == 0;
    for (int64_t x : ld) ok = ok && x % e == 0;
    return ok;
}

// Query-key pairs if the batch were of equal shapes: for the profile's counts, which know no offsets.
double pairs(const hch_attn_desc &p) { return (double)p.n_q * p.n_k / std::max(1, p.batch) * p.heads_q * p.head_dim; }
double row_bytes(const hch_attn_desc &p, int q, int k) { return (double)size_of(p.dtype) * p.head_dim * ((double)q * p.n_q * p.heads_q + (double)k * p.n_k * p.heads_kv); }

}  // namespace

extern "C" size_t hch_attn_workspace_bytes(const hch_attn_desc *desc, hch_ws_kind kind)
{
    if (check_sizes("hch_attn_workspace_bytes", desc) != HCH_OK) return 0;
    if (kind == HCH_WS_FWD) return fwd_bytes(*desc);
    if (kind == HCH_WS_BWD_DATA) return bwd_bytes(*desc);
    return 0;
}

extern "C" hch_status hch_attn_fwd(const hch_attn_desc *desc, const void *Q, const void *K, const void *V, void *O, float *lse,
                                   void *workspace, size_t ws_bytes, void *stream)
{
    hch_status st = check_sizes("hch_attn_fwd", desc);
    if (st == HCH_OK) st = check_call("hch_attn_fwd", desc, workspace, ws_bytes, fwd_bytes(*desc));
    if (st != HCH_OK) return st;
    const hch_attn_desc &p = *desc;
    if ((p.n_q && (!Q || !O)) || (p.n_k && (!K || !V))) return fail(HCH_EINVAL, "hch_attn_fwd: null pointer");
    if (!p.n_q) return HCH_OK;
    const Plan r = plan_keys(p);
    Args a = args_of(p);
    a.Q = Q; a.K = K; a.V = V; a.Ow = O; a.lse = lse;
    a.vec = whole(p, {Q, K, V, O}, {p.ld_q, p.ld_k, p.ld_v, p.ld_o});
    a.slots = (int)r.slots; a.splits = r.splits; a.total = a.slots * a.splits * a.hkv;
    a.part = (float *)workspace;
    a.ml = (float2 *)((char *)workspace + part_bytes(p, r.splits));
    const double bytes = row_bytes(p, 2, 2), flops = 4 * pairs(p);
    return p.dtype == HCH_F32 ? hch::attn::launch_fwd<float>(a, r.narrow, bytes, flops, (hipStream_t)stream)
                              : hch::attn::launch_fwd<__bf16>(a, r.narrow, bytes, flops, (hipStream_t)stream);
}

extern "C" hch_status hch_attn_bwd(const hch_attn_desc *desc, const void *Q, const void *K, const void *V, const void *O, const float *lse,
                                   const void *dO, void *dQ, void *dK, void *dV, void *workspace, size_t ws_bytes, void *stream)
{
    hch_status st = check_sizes("hch_attn_bwd", desc);
    if (st == HCH_OK) st = check_call("hch_attn_bwd", desc, workspace, ws_bytes, bwd_bytes(*desc));
    if (st != HCH_OK) return st;
    const hch_attn_desc &p = *desc;
    const int64_t wq = (int64_t)p.heads_q * p.head_dim, wk = (int64_t)p.heads_kv * p.head_dim;
    if (p.ld_do < wq || p.ld_dq < wq || p.ld_dk < wk || p.ld_dv < wk) return fail(HCH_EINVAL, "hch_attn_bwd: row stride below a row's length");
    if (std::max({p.ld_do, p.ld_dq, p.ld_dk, p.ld_dv}) >= 1 << 22) return fail(HCH_EUNSUPPORTED, "hch_attn_bwd: row stride of 2^22 elements or more");
    if ((p.n_q && (!Q || !O || !lse || !dO || !dQ)) || (p.n_k && (!K || !V || !dK || !dV))) return fail(HCH_EINVAL, "hch_attn_bwd: null pointer");
    Args a = args_of(p);
    a.Q = Q; a.K = K; a.V = V; a.O = O; a.lse = const_cast<float *>(lse); a.dO = dO; a.dQ = dQ; a.dK = dK; a.dV = dV;
    a.vec = whole(p, {Q, K, V, O, dO, dQ, dK, dV}, {p.ld_q, p.ld_k, p.ld_v, p.ld_o, p.ld_do, p.ld_dq, p.ld_dk, p.ld_dv});
    const hipStream_t s = (hipStream_t)stream;
    if (p.n_q) {
        const Plan r = plan_keys(p);
        a.slots = (int)r.slots; a.splits = r.splits; a.total = a.slots * a.splits * a.hkv;
        a.delta = (float *)workspace;
        a.part = (float *)((char *)workspace + delta_bytes(p));
        const double bytes = row_bytes(p, 4, 2), flops = 6 * pairs(p);
        st = p.dtype == HCH_F32 ? hch::attn::launch_bwd_dq<float>(a, r.narrow, bytes, flops, s)
                                : hch::attn::launch_bwd_dq<__bf16>(a, r.narrow, bytes, flops, s);
        if (st != HCH_OK) return st;
    }
    if (p.n_k) {
        const bool narrow = narrow_queries(p);
        a.slots = (int)hch::attn::slots_of(p.n_k, 1, narrow ? 32 : 128, p.batch); a.splits = 1; a.total = a.slots * a.hkv;
        const double bytes = row_bytes(p, 2, 4), flops = 8 * pairs(p);
        st = p.dtype == HCH_F32 ? hch::attn::launch_bwd_dkv<float>(a, narrow, bytes, flops, s)
                                : hch::attn::launch_bwd_dkv<__bf16>(a, narrow, bytes, flops, s);
    }
    return st;
}
