// C entries of the norms of queries and keys by head with rotary positions in the same pass.
#include "rows.hpp"

#include "qknorm.hip.hpp"

namespace {

// Workgroups of the backward pass at most, each with sums of its own: five on a compute unit, as many as registers allow (46514 rows of 16 heads of 128, bf16:
// four 105 us, five 107, six, of which the last wait for the first, 128; 9533 of 24 of 64: 23.8, 24.3 and 26.8).
constexpr int PARTS = 1280;

struct HeadTensor { const void *p; int64_t ld; int bytes; };
bool whole(std::initializer_list<HeadTensor> tensors, int head_dim, int w)
{
    if (head_dim % w) return false;
    for (const HeadTensor &t : tensors) if (t.ld * t.bytes % std::min(16, w * t.bytes) || !aligned(t.p, std::min(16, w * t.bytes))) return false;
    return true;
}

// lanes of a head (4 .. 64), channels of a lane, and how many of them are read at a time: all, two or one, as width, strides and addresses
// allow (46514 rows of 16 heads, one by one and by pairs: of 34, bf16, 56 and 48 us forward, 90 and 84 back; of 66 92 and 83, but 136 and 152 back; of 250 266 and
// 192, 360 and 336; of 66, fp32, 130 and 99, 186 and 136).  8 channels where one of the types
// is bf16, so that its pieces are 16 bytes (46514 rows of 16 heads of 128, bf16: by 4 84 us forward and 122 back, by 8 74 and 107), unless half of
// the lanes would have none (300000 rows of 4 heads of 16, bf16, forward: by 4 21 us, by 8 24).
template <typename F> void with_head_shape(int head_dim, int run, F &&f)
{
#define HCH_HEAD(L, W, R) if (head_dim <= L * W) return f(Int<L>{}, Int<W>{}, Int<R>{});
#define HCH_HEADS(R) HCH_HEAD(4, 4, R) HCH_HEAD(8, 4, R) HCH_HEAD(16, 4, R) HCH_HEAD(32, 4, R) HCH_HEAD(64, 4, R)
    if (run == 8) { HCH_HEAD(4, 8, 8) HCH_HEAD(8, 8, 8) HCH_HEAD(16, 8, 8) HCH_HEAD(32, 8, 8) }
    if (run == 4) { HCH_HEADS(4) }
    if (run == 2) { HCH_HEADS(2) }
    HCH_HEADS(1)
#undef HCH_HEADS
#undef HCH_HEAD
}
int run_of(std::initializer_list<HeadTensor> tensors, int head_dim, bool eight)
{
    int run = eight && head_dim > 16 ? 8 : 4;
    while (run > 1 && !whole(tensors, head_dim, run)) run /= 2;
    return run;
}

// Rows of a workgroup, as many as LDS has turns for at most.  Forward: eight heads for each group of lanes where there are many (46514 rows of 16 heads of
// 128, bf16: 2 heads 77 us, 4 76, 8 74, 16 81).
int fwd_rows(int64_t n, int heads, int groups, int pairs)
{
    int64_t rows = std::max(1, groups * 8 / heads);
    rows = std::min<int64_t>(rows, std::max<int64_t>((groups + heads - 1) / heads, n / 1024));
    rows = std::min<int64_t>(rows, hch::qknorm::ROWS);
    if (pairs) rows = std::min<int64_t>(rows, hch::qknorm::ENTRIES / pairs);
    return (int)std::max<int64_t>(rows, 1);
}
// Backward: the fewest that give every group a head of each kind, so that workgroups that run at once lie close together in memory (46514 rows of 16 heads of
// 128, bf16: 4 rows 107 us, 8 rows 112, 16 rows 130), but 1024 workgroups where there are rows for them.
int bwd_rows(int64_t n, int heads_q, int heads_k, int others, int groups, int pairs)
{
    int least = 1 << 30;
    for (int h : {heads_q, heads_k, others}) if (h) least = std::min(least, h);
    int64_t rows = std::max(2, (groups - 1) / least + 1);
    rows = std::min<int64_t>(rows, (n - 1) / 1024 + 1);
    if (n * (heads_q + heads_k + others) <= 2 * groups) rows = n;              // one workgroup, and no launch to join sums behind it (4 rows of 8 heads of 64: 13 -> 10 us)
    rows = std::min<int64_t>(rows, hch::qknorm::ROWS);
    if (pairs) rows = std::min<int64_t>(rows, hch::qknorm::ENTRIES / pairs);
    return (int)rows;
}

struct Heads { int64_t n; int32_t heads, heads_q, heads_k, head_dim; };

hch_status positions_of(const std::string &name, double sign, int head_dim, const int32_t *sections, float base, float scale, hch::qknorm::Positions &P)
{
    if (!(base > 0.f) || !std::isfinite(base) || !std::isfinite(scale)) return fail(HCH_EINVAL, name + ": base must be positive, base and scale finite");
    P = {};
    P.unit = sign * scale / M_PI;
    P.log2_base = std::log2((double)base);
    for (int a = 0; a < 3; ++a) {
        if (sections[a] < 0 || sections[a] > head_dim / 2 - P.pairs) return fail(HCH_EINVAL, name + ": sections exceed the pairs of a head");
        P.sections[a] = sections[a];
        P.pairs += sections[a];
    }
    return HCH_OK;
}

hch_status check(const std::string &name, const Heads &h, float eps)
{
    if (h.n < 0 || h.heads <= 0 || h.heads_q < 0 || h.heads_k < 0 || h.heads_q > h.heads || h.heads_k > h.heads - h.heads_q || h.head_dim <= 0 || h.head_dim % 2)
        return fail(HCH_EINVAL, name + ": bad size");
    if (!(eps >= 0.f) || !std::isfinite(eps)) return fail(HCH_EINVAL, name + ": eps must be finite and not negative");
    if (h.head_dim > 2 * hch::rope::MAX_PAIRS) return fail(HCH_EUNSUPPORTED, name + ": more than 256 channels per head");
    if ((int64_t)h.heads * h.head_dim > (1 << 22)) return fail(HCH_EUNSUPPORTED, name + ": more than 2^22 elements in a row");
    return HCH_OK;
}

}  // namespace

extern "C" hch_status hch_qknorm_rope_fwd(hch_dtype x_dtype, const void *X, int64_t ld_x, hch_dtype y_dtype, void *Y, int64_t ld_y,
                                          const float *gamma_q, const float *gamma_k, const int32_t *coords, int64_t n, int32_t heads,
                                          int32_t heads_q, int32_t heads_k, int32_t head_dim, const int32_t *sections, float base, float scale,
                                          float eps, void *stream)
try {
    const std::string name = "hch_qknorm_rope_fwd";
    const Heads hs = {n, heads, heads_q, heads_k, head_dim};
    if (!known(x_dtype) || !known(y_dtype)) return fail(HCH_EINVAL, name + ": unknown dtype");
    if ((n && (!X || !Y)) || !sections) return fail(HCH_EINVAL, name + ": null pointer");
    if (const hch_status st = check(name, hs, eps)) return st;
    const int64_t width = (int64_t)heads * head_dim;
    if (ld_x < width || ld_y < width) return fail(HCH_EINVAL, name + ": row stride below heads * head_dim");
    hch::qknorm::Positions positions;
    if (const hch_status st = positions_of(name, 1.0, head_dim, sections, base, scale, positions)) return st;
    const int normed = heads_q + heads_k;
    if (!normed) positions.pairs = 0;
    const int pairs = positions.pairs;
    if (n && !coords && pairs) return fail(HCH_EINVAL, name + ": coords is null");
    if (n && X == Y && (x_dtype != y_dtype || ld_x != ld_y)) return fail(HCH_EINVAL, name + ": in place needs one type and one row stride");
    const int walked = X == Y ? normed : heads;              // in place, the other heads are where they belong
    if (n == 0 || walked == 0) return HCH_OK;
    const int sx = size_of(x_dtype), sy = size_of(y_dtype);
    const int run = run_of({{X, ld_x, sx}, {Y, ld_y, sy}}, head_dim, sx + sy < 8);
    hch_status st = HCH_OK;
    with_types(x_dtype, y_dtype, [&](auto tx, auto ty) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        with_head_shape(head_dim, run, [&](auto l, auto w, auto r) {
            constexpr int L = decltype(l)::value, W = decltype(w)::value, RUN = decltype(r)::value;
            if constexpr (W == 4 || sizeof(TX) + sizeof(TY) < 8) {
                const int rows = fwd_rows(n, walked, hch::qknorm::THREADS / L, pairs);
                const int64_t blocks = (n - 1) / rows + 1;
                if (blocks > 0xffffffffll / hch::qknorm::THREADS) { st = fail(HCH_EUNSUPPORTED, name + ": more than 2^24 - 1 workgroups in a launch"); return; }
                static const int id = instance_id<TX, TY>("qknorm::qknorm_rope_fwd_kernel", {L, W, RUN});
                hch::LaunchTimer lt(id, (hipStream_t)stream, (double)n * walked * head_dim * (sx + sy) + 12.0 * n, 7.0 * n * normed * head_dim);
                constexpr auto kernel = hch::qknorm::qknorm_rope_fwd_kernel<TX, TY, L, W, RUN>;
                HCH_LAUNCH(kernel, dim3((unsigned)blocks), dim3(hch::qknorm::THREADS), 0, (hipStream_t)stream, (const TX *)X, ld_x, (TY *)Y, ld_y,
                           gamma_q, gamma_k, coords, n, walked, heads_q, normed, head_dim, rows, eps, positions);
            }
        });
    });
    if (st) return st;
    HCH_LAUNCH_CHECK("qknorm_rope_fwd_kernel");
    return HCH_OK;
} catch (const std::exception &) {
    return HCH_ENOMEM;
}

extern "C" size_t hch_qknorm_rope_workspace_bytes(int64_t n, int32_t heads_q, int32_t heads_k, int32_t head_dim)
{
    if (n < 0 || heads_q < 0 || heads_k < 0 || head_dim <= 0 || head_dim > 2 * hch::rope::MAX_PAIRS || head_dim % 2) return 0;
    const int64_t parts = std::min<int64_t>(PARTS, n);
    return std::max<size_t>(256, ((size_t)parts * 2 * head_dim * sizeof(float) + 255) / 256 * 256);
}

extern "C" hch_status hch_qknorm_rope_bwd(hch_dtype x_dtype, const void *X, int64_t ld_x, hch_dtype dy_dtype, const void *dY, int64_t ld_dy,
                                          hch_dtype dx_dtype, void *dX, int64_t ld_dx, const float *gamma_q, const float *gamma_k, float *dgamma_q,
                                          float *dgamma_k, const int32_t *coords, int64_t n, int32_t heads, int32_t heads_q, int32_t heads_k,
                                          int32_t head_dim, const int32_t *sections, float base, float scale, float eps, void *workspace,
                                          size_t ws_bytes, void *stream)
try {
    const std::string name = "hch_qknorm_rope_bwd";
    const Heads hs = {n, heads, heads_q, heads_k, head_dim};
    if (!known(x_dtype) || !known(dy_dtype) || !known(dx_dtype)) return fail(HCH_EINVAL, name + ": unknown dtype");
    if ((n && (!X || !dY || !dX)) || !sections || (dgamma_q != nullptr) != (dgamma_k != nullptr))
        return fail(HCH_EINVAL, name + ": null pointer, or only one of dgamma_q and dgamma_k");
    if (const hch_status st = check(name, hs, eps)) return st;
    const int64_t width = (int64_t)heads * head_dim;
    if (ld_x < width || ld_dy < width || ld_dx < width) return fail(HCH_EINVAL, name + ": row stride below heads * head_dim");
    hch::qknorm::Positions positions;
    if (const hch_status st = positions_of(name, -1.0, head_dim, sections, base, scale, positions)) return st;
    const int normed = heads_q + heads_k;
    if (!normed) positions.pairs = 0;
    const int pairs = positions.pairs;
    if (n && !coords && pairs) return fail(HCH_EINVAL, name + ": coords is null");
    if (n && dY == dX && (dy_dtype != dx_dtype || ld_dy != ld_dx)) return fail(HCH_EINVAL, name + ": in place needs one type and one row stride");
    if (n && X == dX && (x_dtype != dx_dtype || ld_x != ld_dx)) return fail(HCH_EINVAL, name + ": in place needs one type and one row stride");
    if (dgamma_q) {
        if (!workspace || !aligned(workspace, 256)) return fail(HCH_EINVAL, name + ": workspace null or not 256-byte aligned");
        if (ws_bytes < hch_qknorm_rope_workspace_bytes(n, heads_q, heads_k, head_dim)) return fail(HCH_EWORKSPACE, name + ": workspace too small");
    }
    float *part = dgamma_q ? (float *)workspace : nullptr;
    const int walked = dY == dX ? normed : heads;
    int64_t blocks = 0;
    if (n && walked) {
        const int sx = size_of(x_dtype), sy = size_of(dy_dtype), sd = size_of(dx_dtype);
        const int run = run_of({{X, ld_x, sx}, {dY, ld_dy, sy}, {dX, ld_dx, sd}}, head_dim, sx + sy < 8);
        with_types(x_dtype, dy_dtype, [&](auto tx, auto ty) {
            using TX = decltype(tx);
            using TY = decltype(ty);
            with_head_shape(head_dim, run, [&](auto l, auto w, auto r) {
                constexpr int L = decltype(l)::value, W = decltype(w)::value, RUN = decltype(r)::value;
                if constexpr (W == 4 || sizeof(TX) + sizeof(TY) < 8) {
                    const int rows = bwd_rows(n, heads_q, heads_k, walked - normed, hch::qknorm::THREADS / L, pairs);
                    blocks = std::min<int64_t>(PARTS, (n - 1) / rows + 1);
                    static const int id = instance_id<TX, TY>("qknorm::qknorm_rope_bwd_kernel", {L, W, RUN});
                    hch::LaunchTimer lt(id, (hipStream_t)stream, (double)n * head_dim * ((double)normed * sx + (double)walked * (sy + sd)) + 12.0 * n, 14.0 * n * normed * head_dim);
                    constexpr auto kernel = hch::qknorm::qknorm_rope_bwd_kernel<TX, TY, L, W, RUN>;
                    HCH_LAUNCH(kernel, dim3((unsigned)blocks), dim3(hch::qknorm::THREADS), 0, (hipStream_t)stream, (const TX *)X, ld_x, (const TY *)dY, ld_dy,
                               dX, ld_dx, dx_dtype == HCH_BF16, gamma_q, gamma_k, part, dgamma_q, dgamma_k, coords, n, walked, heads_q, normed, head_dim, rows, eps, positions);
                }
            });
        });
        HCH_LAUNCH_CHECK("qknorm_rope_bwd_kernel");
    }
    return dgamma_q && blocks != 1 ? join_sums(part, dgamma_q, dgamma_k, (int)blocks, head_dim, stream) : HCH_OK;
} catch (const std::exception &) {
    return HCH_ENOMEM;
}
