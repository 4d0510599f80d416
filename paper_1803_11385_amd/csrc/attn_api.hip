// C entries of attention inside the shapes of a ragged batch.
#include <algorithm>
#include <cmath>
#include <exception>
#include <initializer_list>

#include "attn_launch.hpp"

namespace {

using hch::attn::Args;

int size_of(hch_dtype t) { return t == HCH_F32 ? 4 : 2; }
size_t round256(size_t x) { return (x + 255) / 256 * 256; }

// How a pass is cut into workgroups.
struct Plan {
    bool narrow;           // tiles of 32 rows (keys) whose wavefronts share what streams past, not of 128
    int splits;            // parts of what streams past, joined by a second launch
    int64_t slots;
    double us, workgroups; // what it takes by the reckoning below, and about how many have work
};
struct Plans {             // the best one with wide tiles and with narrow ones
    Plan form[2];
    const Plan &best() const { return form[form[1].us < form[0].us]; }
};

// What a pass takes, as a sum of steps (64 streamed rows in bf16, 32 in fp32; narrow 128, and 64 in fp32 beyond 64 channels):
// microseconds of a step of a workgroup that has a compute unit to itself, by head width up to 32, 64, 96, 128, and
// how many workgroups a compute unit takes on before that grows in proportion.  START: before and after the steps; JOIN: the
// launch that joins splits; dQ and the keys' gradients cost so many times as much as the forward pass.  Fitted to
// 1020 timings (14 batches of 1 to 32 shapes of 80 to 6000 rows and 3 with 1 or 3 queries a shape, both types, three passes, both
// forms, 1 to 16 splits; the logarithm is off by 0.15 rms): the choice by it takes 1.02 times as long as the best
// one in the mean, 1.33 at most; always wide tiles without splits 1.9 and 35 times.
struct Step { double us, at_once; };
constexpr Step STEP[2][2][4] = {{{{0.93, 1.59}, {1.62, 1.37}, {2.15, 1.03}, {3.51, 1.21}}, {{1.71, 1.87}, {2.90, 0.99}, {3.28, 0.95}, {4.27, 1.18}}},
                                {{{0.67, 2.61}, {0.84, 1.69}, {1.06, 1.58}, {2.39, 1.96}}, {{0.69, 2.97}, {0.81, 1.72}, {1.21, 1.24}, {3.75, 2.21}}}};
constexpr double START = 5.3, JOIN = 5.7, FWD = 1.0, DQ = 1.33, DKV = 1.45, JOIN_SPLIT = 0.03, BYTES_PER_US = 4e6, MEMORY = 5e6, UNITS = 256, UNEVEN = 1.25;

// rows: of the tiles, over all shapes, `heads` times; stream: rows that one of those tiles sees on average; width: bytes of a
// row's partial sums; moved: bytes of what streams past, all of it once.  Offsets are known on the device only, so
// shapes count as equal, the longest as UNEVEN times the mean.
Plans plan(const hch_attn_desc &p, int64_t rows, int rows_each, int heads, double stream, double cost, double width, double moved)
{
    const int type = p.dtype == HCH_BF16, dc = std::min(3, (p.head_dim - 1) / 32);
    Plans r = {};
    rows *= rows_each;
    for (int narrow = 0; narrow < 2; ++narrow) {
        const Step &st = STEP[type][narrow][dc];
        const int size = narrow ? 32 : 128, step = narrow ? (!type && dc >= 2 ? 64 : 128) : type ? 64 : 32;
        const double wgs = std::max<double>(p.batch, (double)rows / size + 0.5 * p.batch) * heads, steps = std::max(1.0, std::ceil(stream / step));
        // half as many again from time to time, and as many as make whole rounds of workgroups
        constexpr int SPLITS[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, 96, 128, 192, 256}, COUNT = sizeof(SPLITS) / sizeof(int);
        for (int i = 0; i < COUNT + 4; ++i) {
            const int splits = i < COUNT ? SPLITS[i] : (int)std::min(256.0, UNITS * (i - COUNT + 1) / wgs);
            if (splits < 1 || splits > steps || (splits > 1 && wgs * splits > 4 * UNITS)) continue;
            const double each = std::ceil(wgs * splits / UNITS), busy = each <= 1.0 ? 1.0 : std::max(1.0, each / st.at_once);
            double us = (START + std::ceil(UNEVEN * steps / splits) * st.us * cost) * busy;
            // Memory: at its rate if the compute units share evenly.  Shapes of different lengths do not split into equal parts, which
            // several workgroups a unit even out (one query for each of 8 shapes of 609323 keys together, 2 heads of 32, bf16: 256 workgroups 70 us,
            // 512 42, 768 36, 1024 47; 304000 keys, 4 heads of 64: 93, 70, 65, 66).  Against a share of 1 this changes the choice for 243 of 1500
            // drawn batches of 1 to 16 queries a shape; 100 of those take 0.96 of the time in the mean, uneven shapes 0.93 (0.65 to
            // 1.18), equal ones, which are not known here, 1.06 (0.95 to 1.24).  A single shape beyond two rounds: 0.97 of the time in
            // the middle of 40 (mostly 0.95 to 1.02).
            const double share = p.batch == 1 ? (each > 2.0 ? 1.1 : 1.0) : each <= 1.0 ? 1.45 : each <= 2.0 ? 1.12 : each <= 3.0 ? 1.0 : 1.1;
            const double move = moved / MEMORY * each * UNITS / (wgs * splits) * share;
            us = std::max(us, move) + 0.2 * std::min(us, move);         // (they do not overlap altogether)
            if (splits > 1) us += JOIN + JOIN_SPLIT * splits + 2.0 * splits * rows * heads * width / BYTES_PER_US;
            if (i == 0 || us < r.form[narrow].us) r.form[narrow] = {narrow != 0, splits, 0, us, wgs * splits};
        }
        r.form[narrow].slots = hch::attn::slots_of(rows / rows_each, rows_each, size, p.batch);
    }
    return r;
}

double row_bytes(const hch_attn_desc &p, int q, int k) { return (double)size_of(p.dtype) * p.head_dim * ((double)q * p.n_q * p.heads_q + (double)k * p.n_k * p.heads_kv); }

Plans plan_keys(const hch_attn_desc &p, double cost)    // forward and dQ: tiles of query rows, keys stream past
{
    return plan(p, p.n_q, p.heads_q / p.heads_kv, p.heads_kv, (double)p.n_k / p.batch, cost, 4.0 * p.head_dim, row_bytes(p, 0, 2));
}

Plans plan_queries(const hch_attn_desc &p)              // dK and dV: tiles of keys, the queries of a head's group stream past
{
    return plan(p, p.n_k, 1, p.heads_kv, (double)p.n_q / p.batch * (p.heads_q / p.heads_kv), DKV, 8.0 * p.head_dim, row_bytes(p, 2, 0));
}

// The backward pass: dQ, then dK and dV, each with the tiles that are best for it; or, in whole pieces, both in one launch where all their
// workgroups find room on the compute units at once, after a launch that takes START for D.  ROOM: workgroups of a compute unit by type,
// form and head width, from the kernels' registers.  (Of 70 batches the 39 within that room took 0.74 of the two
// launches' time in the mean, 0.61 to 1.01; most of those beyond it would take as long either way.)
constexpr int ROOM[2][2][4] = {{{2, 1, 1, 1}, {2, 1, 1, 1}}, {{4, 2, 2, 1}, {3, 2, 1, 1}}};
struct Backward {
    Plan dq, dkv;          // two launches
    Plan dq1, dkv1;        // one
    bool together;
};
Backward plan_backward(const hch_attn_desc &p)
{
    const Plans q = plan_keys(p, DQ), k = plan_queries(p);
    Backward r = {q.best(), k.best(), {}, {}, false};
    double least = r.dq.us + r.dkv.us;
    for (int narrow = 0; narrow < 2; ++narrow) {
        const int room = ROOM[p.dtype == HCH_BF16][narrow][std::min(3, (p.head_dim - 1) / 32)];
        const double us = START + std::max(q.form[narrow].us, k.form[narrow].us);
        if (q.form[narrow].workgroups + k.form[narrow].workgroups > room * UNITS || us >= least) continue;
        least = us;
        r.dq1 = q.form[narrow]; r.dkv1 = k.form[narrow];
        r.together = true;
    }
    return r;
}

size_t part_bytes(const hch_attn_desc &p, int splits) { return splits > 1 ? round256((size_t)splits * p.n_q * p.heads_q * p.head_dim * 4) : 0; }
size_t ml_bytes(const hch_attn_desc &p, int splits) { return splits > 1 ? round256((size_t)splits * p.n_q * p.heads_q * 8) : 0; }
size_t key_part_bytes(const hch_attn_desc &p, int splits) { return splits > 1 ? round256((size_t)splits * p.n_k * p.heads_kv * p.head_dim * 8) : 0; }
size_t delta_bytes(const hch_attn_desc &p) { return round256((size_t)p.n_q * p.heads_q * 4); }

size_t fwd_bytes(const hch_attn_desc &p, const Plan &r) { return std::max<size_t>(256, part_bytes(p, r.splits) + ml_bytes(p, r.splits)); }
size_t bwd_bytes(const hch_attn_desc &p, const Backward &r)         // whichever it will be
{
    const auto bytes = [&](const Plan &dq, const Plan &dkv) { return part_bytes(p, dq.splits) + key_part_bytes(p, dkv.splits); };
    return std::max<size_t>(256, delta_bytes(p) + std::max(bytes(r.dq, r.dkv), r.together ? bytes(r.dq1, r.dkv1) : 0));
}

constexpr int64_t ROWS = 0x7fffffff - 256;              // the last tile's end is an int too

// what both calls and the size query ask of the sizes
hch_status check_sizes(const char *who, const hch_attn_desc *p)
{
    const auto no = [&](hch_status st, const char *what) { return fail(st, std::string(who) + what); };
    if (!p) return no(HCH_EINVAL, ": null description");
    if (p->dtype != HCH_F32 && p->dtype != HCH_BF16) return no(HCH_EINVAL, ": unknown dtype");
    if (p->batch < 0 || p->n_q < 0 || p->n_k < 0 || p->heads_q <= 0 || p->heads_kv <= 0 || p->head_dim <= 0 || p->heads_q % p->heads_kv)
        return no(HCH_EINVAL, ": bad size, or heads_q not a multiple of heads_kv");
    if (p->head_dim > 128) return no(HCH_EUNSUPPORTED, ": more than 128 channels per head");
    if (p->n_k > ROWS || p->n_q > ROWS / p->heads_q || p->heads_q > 0x7fff) return no(HCH_EUNSUPPORTED, ": 2^31 - 256 rows or more, or 2^15 heads or more");
    if (p->batch == 0 && (p->n_q || p->n_k)) return no(HCH_EINVAL, ": rows without a shape");
    return HCH_OK;
}
bool launchable(const hch_attn_desc &p, const Plan &r) { return hch::attn::work_shape(r.slots, r.splits, p.heads_kv).grid <= hch::attn::MAX_GRID; }

hch_status check_call(const char *who, const hch_attn_desc *p, const void *workspace, size_t ws_bytes, size_t need)
{
    const auto no = [&](hch_status st, const char *what) { return fail(st, std::string(who) + what); };
    if (!(p->scale > 0.f) || !std::isfinite(p->scale)) return no(HCH_EINVAL, ": scale must be positive and finite");
    if (p->batch && (!p->q_offsets || !p->k_offsets)) return no(HCH_EINVAL, ": null offsets");
    const int64_t wq = (int64_t)p->heads_q * p->head_dim, wk = (int64_t)p->heads_kv * p->head_dim;
    if (p->ld_q < wq || p->ld_o < wq || p->ld_k < wk || p->ld_v < wk) return no(HCH_EINVAL, ": row stride below a row's length");
    if (std::max({p->ld_q, p->ld_o, p->ld_k, p->ld_v}) >= 1 << 22) return no(HCH_EUNSUPPORTED, ": row stride of 2^22 elements or more");
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255)) return no(HCH_EINVAL, ": workspace null or not 256-byte aligned");
    if (ws_bytes < need) return no(HCH_EWORKSPACE, ": workspace too small");
    return HCH_OK;
}

// Rows of a shape that stream past, from which on units go by their number: keys, or in the pass over the keys the queries of a head's
// group (1 query for each of 32 shapes of about 5000 keys, fp32: dK and dV 58 us in that order, 44 without; 32 shapes
// of 4000 queries and 200 keys, 8 heads of 64: 831 with it, 1077 without).
constexpr int64_t SORT_FROM = 1024;

Args args_of(const hch_attn_desc &p)
{
    Args a = {};
    a.sorted = p.batch > 1 && p.n_k / std::max(1, p.batch) >= SORT_FROM;
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

}  // namespace

extern "C" size_t hch_attn_workspace_bytes(const hch_attn_desc *desc, hch_ws_kind kind)
try {
    if (check_sizes("hch_attn_workspace_bytes", desc) != HCH_OK || (kind != HCH_WS_FWD && kind != HCH_WS_BWD_DATA)) return 0;
    if (!desc->n_q) return 256;
    return kind == HCH_WS_FWD ? fwd_bytes(*desc, plan_keys(*desc, FWD).best()) : bwd_bytes(*desc, plan_backward(*desc));
} catch (const std::exception &) {
    return 0;
}

extern "C" hch_status hch_attn_fwd(const hch_attn_desc *desc, const void *Q, const void *K, const void *V, void *O, float *lse,
                                   void *workspace, size_t ws_bytes, void *stream)
try {
    hch_status st = check_sizes("hch_attn_fwd", desc);
    if (st != HCH_OK) return st;
    const hch_attn_desc &p = *desc;
    const Plan r = p.n_q ? plan_keys(p, FWD).best() : Plan{false, 1, 0, 0.0, 0.0};
    st = check_call("hch_attn_fwd", desc, workspace, ws_bytes, fwd_bytes(p, r));
    if (st != HCH_OK) return st;
    if ((p.n_q && (!Q || !O)) || (p.n_k && (!K || !V))) return fail(HCH_EINVAL, "hch_attn_fwd: null pointer");
    if (!launchable(p, r)) return fail(HCH_EUNSUPPORTED, "hch_attn_fwd: more than 2^24 - 1 workgroups in a launch");
    if (!p.n_q) return HCH_OK;
    Args a = args_of(p);
    a.Q = Q; a.K = K; a.V = V; a.Ow = O; a.lse = lse;
    a.vec = whole(p, {Q, K, V, O}, {p.ld_q, p.ld_k, p.ld_v, p.ld_o});
    a.slots = (int)r.slots; a.splits = r.splits; hch::attn::set_work(a);
    a.part = (float *)workspace;
    a.ml = (float2 *)((char *)workspace + part_bytes(p, r.splits));
    const double bytes = row_bytes(p, 2, 2), flops = 4 * pairs(p);
    return p.dtype == HCH_F32 ? hch::attn::launch_fwd<float>(a, r.narrow, bytes, flops, (hipStream_t)stream)
                              : hch::attn::launch_fwd<__bf16>(a, r.narrow, bytes, flops, (hipStream_t)stream);
} catch (const std::exception &) {
    return HCH_ENOMEM;
}

extern "C" hch_status hch_attn_bwd(const hch_attn_desc *desc, const void *Q, const void *K, const void *V, const void *O, const float *lse,
                                   const void *dO, void *dQ, void *dK, void *dV, void *workspace, size_t ws_bytes, void *stream)
try {
    hch_status st = check_sizes("hch_attn_bwd", desc);
    if (st != HCH_OK) return st;
    const hch_attn_desc &p = *desc;
    const Plan none = {false, 1, p.batch ? hch::attn::slots_of(p.n_k, 1, 128, p.batch) : 0, 0.0, 0.0};       // without queries: zeros
    const Backward r = p.n_q ? plan_backward(p) : Backward{none, none, {}, {}, false};
    st = check_call("hch_attn_bwd", desc, workspace, ws_bytes, p.n_q ? bwd_bytes(p, r) : 256);
    if (st != HCH_OK) return st;
    const int64_t wq = (int64_t)p.heads_q * p.head_dim, wk = (int64_t)p.heads_kv * p.head_dim;
    if (p.ld_do < wq || p.ld_dq < wq || p.ld_dk < wk || p.ld_dv < wk) return fail(HCH_EINVAL, "hch_attn_bwd: row stride below a row's length");
    if (std::max({p.ld_do, p.ld_dq, p.ld_dk, p.ld_dv}) >= 1 << 22) return fail(HCH_EUNSUPPORTED, "hch_attn_bwd: row stride of 2^22 elements or more");
    if ((p.n_q && (!Q || !O || !lse || !dO || !dQ)) || (p.n_k && (!K || !V || !dK || !dV))) return fail(HCH_EINVAL, "hch_attn_bwd: null pointer");
    if (!launchable(p, r.dq) || !launchable(p, r.dkv)) return fail(HCH_EUNSUPPORTED, "hch_attn_bwd: more than 2^24 - 1 workgroups in a launch");
    Args a = args_of(p);
    a.Q = Q; a.K = K; a.V = V; a.O = O; a.lse = const_cast<float *>(lse); a.dO = dO; a.dQ = dQ; a.dK = dK; a.dV = dV;
    a.vec = whole(p, {Q, K, V, O, dO, dQ, dK, dV}, {p.ld_q, p.ld_k, p.ld_v, p.ld_o, p.ld_do, p.ld_dq, p.ld_dk, p.ld_dv});
    a.delta = (float *)workspace;
    const bool together = r.together && a.vec && p.n_k;
    const Plan &rq = together ? r.dq1 : r.dq, &rk = together ? r.dkv1 : r.dkv;
    float *const q_part = (float *)((char *)workspace + delta_bytes(p));
    a.part = q_part;
    const hipStream_t s = (hipStream_t)stream;
    Args b = a;
    b.sorted = p.batch > 1 && p.n_q / std::max(1, p.batch) * (p.heads_q / p.heads_kv) >= SORT_FROM;     // queries stream past
    b.part = (float *)((char *)q_part + part_bytes(p, rq.splits));
    a.slots = (int)rq.slots; a.splits = rq.splits; hch::attn::set_work(a);
    b.slots = (int)rk.slots; b.splits = rk.splits; hch::attn::set_work(b);
    if (together) {
        a.delta = nullptr;                              // D is there already
        const double bytes = row_bytes(p, 5, 6), flops = 14 * pairs(p);
        st = p.dtype == HCH_F32 ? hch::attn::launch_bwd_both<float>(a, b, rq.narrow, bytes, flops, s)
                                : hch::attn::launch_bwd_both<__bf16>(a, b, rq.narrow, bytes, flops, s);
        if (st != HCH_OK) return st;
    } else {
        if (p.n_q) {
            const double bytes = row_bytes(p, 4, 2), flops = 6 * pairs(p);
            st = p.dtype == HCH_F32 ? hch::attn::launch_bwd_dq<float>(a, rq.narrow, bytes, flops, s)
                                    : hch::attn::launch_bwd_dq<__bf16>(a, rq.narrow, bytes, flops, s);
            if (st != HCH_OK) return st;
        }
        if (p.n_k) {
            const double bytes = row_bytes(p, 2, 4), flops = 8 * pairs(p);
            st = p.dtype == HCH_F32 ? hch::attn::launch_bwd_dkv<float>(b, rk.narrow, bytes, flops, s)
                                    : hch::attn::launch_bwd_dkv<__bf16>(b, rk.narrow, bytes, flops, s);
            if (st != HCH_OK) return st;
        }
    }
    if (rq.splits > 1 || (p.n_k && rk.splits > 1))
        st = p.dtype == HCH_F32 ? hch::attn::launch_bwd_join<float>(b, q_part, rq.splits, s) : hch::attn::launch_bwd_join<__bf16>(b, q_part, rq.splits, s);
    return st;
} catch (const std::exception &) {
    return HCH_ENOMEM;
}
