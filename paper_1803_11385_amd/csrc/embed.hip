// C entries of the embedding and of the gradient of its table.
#include "rows.hpp"

#include "embed.hip.hpp"

namespace {

constexpr int64_t MAX_ROWS = (int64_t(1) << 31) - 4096;

// Rows of a tile of the sort for each of its threads: few, so that many workgroups share the work, and so many that a workgroup can add up all
// tiles' counts (up to TILES) by itself; beyond, where a thread has 8, a launch of its own does (609323 rows of 64, bf16, 32768 labels: 75 tiles 69 us, 149 56, 298,
// counted by a launch, 66).  What the lines cost, the last call before each and the first behind it: 163840 rows 33.8 and 35.5 us, 327680 40.7 and 45.4,
// 655360 58.0 and 70.2 (with 4 rows a thread, and a launch that counts 161 tiles, 58.1; 900000 rows 82.5, so 72.7).  8192 rows are one tile,
// sorted in one launch (32.1 us; 8193 rows by several 26.1).
constexpr int TILES = 160;
int items_of(int64_t n)
{
    if (n <= hch::embed::SORT * 8) return n <= hch::embed::SORT ? 1 : n <= hch::embed::SORT * 2 ? 2 : n <= hch::embed::SORT * 4 ? 4 : 8;
    for (int items = 1; items < 8; items *= 2) if (n <= (int64_t)hch::embed::SORT * items * TILES) return items;
    return 8;
}

// lanes of a row in the sums, and channels of a lane
int lanes_of(int c, int w)
{
    int l = 1;
    while (l < 64 && c > l * w) l *= 2;
    return l;
}

// a workspace's parts, in words of 4 bytes from its start
struct Plan {
    int items;
    int64_t tiles, pairs[2], count, total, left, start, ends, part, words;
};
Plan plan_of(int64_t n, int c, int vocab)
{
    using namespace hch::embed;
    Plan p = {};
    auto take = [&](int64_t words) { const int64_t at = p.words; p.words += (words + 63) / 64 * 64; return at; };
    if (!n) return p;
    p.items = items_of(n);
    p.tiles = (n - 1) / (SORT * p.items) + 1;
    for (int64_t &pairs : p.pairs) pairs = take(2 * (n + 2 * SORT));          // a tile of the sums reads up to 1280 behind the last
    p.count = take((int64_t)p.tiles << MOST);
    p.total = take(1 << MOST);
    p.left = take(1);
    p.start = take(vocab);
    const int64_t tiles = (n - 1) / (THREADS / lanes_of(c, 4) * sub(lanes_of(c, 4))) + 1;         // of the sums: the most there may be
    p.ends = take(tiles);
    p.part = take(tiles * 2 * c);
    return p;
}

hch_status check(const std::string &name, int64_t n, int32_t c, int32_t vocab, float scale)
{
    if (n < 0 || c <= 0 || vocab <= 0) return fail(HCH_EINVAL, name + ": bad size");
    if (!std::isfinite(scale)) return fail(HCH_EINVAL, name + ": scale must be finite");
    if (n > MAX_ROWS) return fail(HCH_EUNSUPPORTED, name + ": more than 2^31 - 4096 rows");
    if (c > (1 << 22)) return fail(HCH_EUNSUPPORTED, name + ": more than 2^22 channels");
    return HCH_OK;
}

}  // namespace

extern "C" hch_status hch_embed_fwd(hch_dtype table_dtype, const void *table, const int32_t *ids, hch_dtype y_dtype, void *Y, int64_t ld_y,
                                    int64_t n, int32_t c, int32_t vocab, float scale, void *stream)
try {
    const std::string name = "hch_embed_fwd";
    if (!known(table_dtype) || !known(y_dtype)) return fail(HCH_EINVAL, name + ": unknown dtype");
    if (n && (!table || !ids || !Y)) return fail(HCH_EINVAL, name + ": null pointer");
    if (const hch_status st = check(name, n, c, vocab, scale)) return st;
    if (ld_y < c) return fail(HCH_EINVAL, name + ": row stride below c");
    if (n == 0) return HCH_OK;
    const int st = size_of(table_dtype), sy = size_of(y_dtype);
    int run = st + sy < 8 ? 8 : 4;         // 16 bytes of the shorter type
    while (run > 1 && (c % run || ld_y % run || !aligned(table, std::min(16, run * st)) || !aligned(Y, std::min(16, run * sy)))) run /= 2;
    // where a thread would write less than 8 bytes, rows that lie one behind the other are written 16 bytes at a time (609323 rows, from 4096 labels of fp32 to
    // bf16, of 50: 24 -> 19 us, of 63: 48 -> 43, from bf16 48 -> 37)
    const bool flat = run * sy < 8 && c >= 8 && ld_y == c && aligned(Y, 16);
    const int64_t units = n * (c / run), each = hch::embed::THREADS * hch::embed::AT_ONCE;
    const unsigned grid = (unsigned)std::min<int64_t>((units - 1) / each + 1, 1 << 16);
    with_types(table_dtype, y_dtype, [&](auto tt, auto ty) {
        using TT = decltype(tt);
        using TY = decltype(ty);
        auto launch = [&](auto w) {
            constexpr int W = decltype(w)::value;
            if constexpr (W < 8 || sizeof(TT) + sizeof(TY) < 8) {
                static const int id = instance_id<TT, TY>("embed::embed_fwd_kernel", {W});
                hch::LaunchTimer lt(id, (hipStream_t)stream, (double)n * c * sy + (double)std::min<int64_t>(n, vocab) * c * st + 4.0 * n, (double)n * c);
                constexpr auto kernel = hch::embed::embed_fwd_kernel<TT, TY, W>;
                HCH_LAUNCH(kernel, dim3(grid), dim3(hch::embed::THREADS), 0, (hipStream_t)stream, (const TT *)table, ids, (TY *)Y, ld_y, n, c, vocab, scale);
            }
        };
        auto launch_flat = [&](auto r) {
            constexpr int RUN = decltype(r)::value;
            static const int id = instance_id<TT, TY>("embed::embed_fwd_flat_kernel", {RUN});
            hch::LaunchTimer lt(id, (hipStream_t)stream, (double)n * c * sy + (double)std::min<int64_t>(n, vocab) * c * st + 4.0 * n, (double)n * c);
            constexpr auto kernel = hch::embed::embed_fwd_flat_kernel<TT, TY, RUN>;
            HCH_LAUNCH(kernel, dim3((unsigned)std::min<int64_t>((n * c - 1) / (hch::embed::THREADS * 16) + 1, 1 << 16)), dim3(hch::embed::THREADS), 0, (hipStream_t)stream,
                       (const TT *)table, ids, (TY *)Y, n, c, vocab, scale);
        };
        const bool twos = c % 2 == 0 && aligned(table, 2 * st);
        if (flat && twos) launch_flat(Int<2>{});
        else if (flat) launch_flat(Int<1>{});
        else if (run == 8) launch(Int<8>{});
        else if (run == 4) launch(Int<4>{});
        else if (run == 2) launch(Int<2>{});
        else launch(Int<1>{});
    });
    HCH_LAUNCH_CHECK("embed_fwd_kernel");
    return HCH_OK;
} catch (const std::exception &) {
    return HCH_ENOMEM;
}

extern "C" size_t hch_embed_workspace_bytes(int64_t n, int32_t c, int32_t vocab)
{
    if (n < 0 || c <= 0 || vocab <= 0 || n > MAX_ROWS || c > (1 << 22)) return 0;
    return std::max<size_t>(256, (size_t)plan_of(n, c, vocab).words * 4);
}

namespace {

template <typename TY> void sum_runs(const hch::embed::Runs &R, const void *dY, int64_t ld_dy, float *dtable, int64_t n, int64_t tiles, int lanes, int c,
                                     float scale, int run, void *stream)
{
    auto launch = [&](auto l, auto w, auto r) {
        constexpr int L = decltype(l)::value, W = decltype(w)::value, RUN = decltype(r)::value;
        if constexpr (W == 8 && sizeof(TY) == 4) return;
        else {
            static const int id = instance_id<TY, TY>("embed::embed_sum_kernel", {L, W, RUN});
            hch::LaunchTimer lt(id, (hipStream_t)stream, (double)n * ((double)c * sizeof(TY) + 8.0), (double)n * c);
            constexpr auto kernel = hch::embed::embed_sum_kernel<TY, L, W, RUN>;
            HCH_LAUNCH(kernel, dim3((unsigned)tiles, (unsigned)((c - 1) / (L * W) + 1)), dim3(hch::embed::THREADS), 0, (hipStream_t)stream, R, (const TY *)dY,
                       ld_dy, dtable, c, scale);
        }
    };
    auto by_run = [&](auto l) {
        if (run == 8) launch(l, Int<8>{}, Int<8>{});
        else if (run == 4) launch(l, Int<4>{}, Int<4>{});
        else if (run == 2) launch(l, Int<4>{}, Int<2>{});
        else launch(l, Int<4>{}, Int<1>{});
    };
    if (lanes == 1) by_run(Int<1>{});
    else if (lanes == 2) by_run(Int<2>{});
    else if (lanes == 4) by_run(Int<4>{});
    else if (lanes == 8) by_run(Int<8>{});
    else if (lanes == 16) by_run(Int<16>{});
    else if (lanes == 32) by_run(Int<32>{});
    else by_run(Int<64>{});
}

template <typename F> void with_digits(int items, int bits, F &&f)
{
    auto with_items = [&](auto b) {
        if (items == 1) f(Int<1>{}, b);
        else if (items == 2) f(Int<2>{}, b);
        else if (items == 4) f(Int<4>{}, b);
        else f(Int<8>{}, b);
    };
    if (bits <= 6) with_items(Int<6>{});
    else if (bits == 7) with_items(Int<7>{});
    else if (bits == 8) with_items(Int<8>{});
    else with_items(Int<9>{});
}

// (label, row) by label; returns where they are
const int2 *sort_rows(const int32_t *ids, const Plan &plan, int32_t *words, float *dtable, int64_t n, int c, int vocab, hipStream_t s)
{
    using namespace hch::embed;
    int bits = 1;
    while (bits < 31 && vocab > (1 << bits)) ++bits;
    // digits of 9 bits where 8 would take a pass more (558080 rows of 16, 74218 labels: 60 -> 53 us)
    const int passes = (bits + MOST - 1) / MOST, width = std::max(LEAST, (bits + passes - 1) / passes);
    const int64_t all = (int64_t)vocab * c;
    int2 *const pairs[2] = {(int2 *)(words + plan.pairs[0]), (int2 *)(words + plan.pairs[1])};
    Pass P = {};
    P.count = words + plan.count;
    P.total = plan.tiles > TILES ? words + plan.total : nullptr;
    P.left = words + plan.left;
    P.n = n;
    P.vocab = vocab;
    P.tiles = (int)plan.tiles;
    for (int i = 0; i < passes; ++i) {
        P.ids = i ? nullptr : ids;
        P.in = pairs[(i + 1) & 1];
        P.out = pairs[i & 1];
        P.shift = i * width;
        with_digits(plan.items, width, [&](auto k, auto b) {
            constexpr int ITEMS = decltype(k)::value, BITS = decltype(b)::value;
            static const int count_id = hch::Profiler::get().id_for("embed::embed_count_kernel<" + std::to_string(ITEMS) + ", " + std::to_string(BITS) + ">");
            static const int scatter_id = hch::Profiler::get().id_for("embed::embed_scatter_kernel<" + std::to_string(ITEMS) + ", " + std::to_string(BITS) + ">");
            // the first launch has workgroups that clear the gradient
            const unsigned tiles = (unsigned)plan.tiles, grid = tiles + (i ? 0 : (unsigned)std::min<int64_t>((all - 1) / (4 * SORT) + 1, 512));
            if (tiles > 1) {
                {
                    hch::LaunchTimer lt(count_id, s, (i ? 8.0 : 4.0) * n + (i ? 0.0 : 4.0 * all), 0.0);
                    constexpr auto kernel = embed_count_kernel<ITEMS, BITS>;
                    HCH_LAUNCH(kernel, dim3(grid), dim3(SORT), 0, s, P, dtable, all);
                }
                if (P.total) {
                    static const int id = hch::Profiler::get().id_for("embed::embed_scan_kernel<" + std::to_string(BITS) + ">");
                    hch::LaunchTimer lt(id, s, 8.0 * plan.tiles * (1 << BITS), 0.0);
                    HCH_LAUNCH(embed_scan_kernel<BITS>, dim3((1u << BITS) / 16), dim3(SORT), 0, s, P);
                }
            }
            hch::LaunchTimer lt(scatter_id, s, (i ? 16.0 : 12.0) * n, 0.0);
            constexpr auto kernel = embed_scatter_kernel<ITEMS, BITS>;
            HCH_LAUNCH(kernel, dim3(tiles > 1 ? tiles : grid), dim3(SORT), 0, s, P, tiles > 1 ? 1 : passes, pairs[1], dtable, all);
        });
        if (plan.tiles == 1) return pairs[(passes - 1) & 1];
    }
    return P.out;
}

}  // namespace

extern "C" hch_status hch_embed_bwd(const int32_t *ids, hch_dtype dy_dtype, const void *dY, int64_t ld_dy, float *dtable, int64_t n, int32_t c,
                                    int32_t vocab, float scale, void *workspace, size_t ws_bytes, void *stream)
try {
    using namespace hch::embed;
    const std::string name = "hch_embed_bwd";
    if (!known(dy_dtype)) return fail(HCH_EINVAL, name + ": unknown dtype");
    if ((n && (!ids || !dY)) || !dtable) return fail(HCH_EINVAL, name + ": null pointer");
    if (const hch_status st = check(name, n, c, vocab, scale)) return st;
    if (ld_dy < c) return fail(HCH_EINVAL, name + ": row stride below c");
    if (!workspace || !aligned(workspace, 256)) return fail(HCH_EINVAL, name + ": workspace null or not 256-byte aligned");
    if (ws_bytes < hch_embed_workspace_bytes(n, c, vocab)) return fail(HCH_EWORKSPACE, name + ": workspace too small");
    const hipStream_t s = (hipStream_t)stream;
    if (n == 0) {
        const int64_t all = (int64_t)vocab * c;
        {
            hch::LaunchTimer lt(HCH_KERNEL_ID("embed::embed_clear_kernel"), s, 4.0 * all, 0.0);
            HCH_LAUNCH(embed_clear_kernel, dim3((unsigned)std::min<int64_t>((all - 1) / THREADS + 1, 4096)), dim3(THREADS), 0, s, dtable, all);
        }
        HCH_LAUNCH_CHECK("embed_clear_kernel");
        return HCH_OK;
    }
    const int sy = size_of(dy_dtype);
    int run = sy == 2 ? 8 : 4;             // neighbours that a lane reads at once
    while (run > 1 && (c % run || ld_dy % run || !aligned(dY, std::min(16, run * sy)) || !aligned(dtable, std::min(16, run * 4)))) run /= 2;
    const int lanes = lanes_of(c, run == 8 ? 8 : 4), rows = THREADS / lanes * sub(lanes);
    const int64_t tiles = (n - 1) / rows + 1;
    if (tiles > 0xffffffffll / JOIN) return fail(HCH_EUNSUPPORTED, name + ": more than 2^24 - 1 workgroups in a launch");
    const Plan plan = plan_of(n, c, vocab);
    int32_t *const words = (int32_t *)workspace;
    Runs R = {};
    R.pairs = sort_rows(ids, plan, words, dtable, n, c, vocab, s);
    HCH_LAUNCH_CHECK("embed_scatter_kernel");
    R.left = words + plan.left;
    R.start = words + plan.start;
    R.ends = words + plan.ends;
    R.part = (float *)(words + plan.part);
    if (dy_dtype == HCH_F32) sum_runs<float>(R, dY, ld_dy, dtable, n, tiles, lanes, c, scale, run, stream);
    else sum_runs<__bf16>(R, dY, ld_dy, dtable, n, tiles, lanes, c, scale, run, stream);
    HCH_LAUNCH_CHECK("embed_sum_kernel");
    if (tiles > 1) {
        const int wide = c % 4 == 0 && aligned(dtable, 16) ? 4 : c % 2 == 0 && aligned(dtable, 8) ? 2 : 1, pieces = c / wide;
        int across = 1;
        while (across < pieces && across < JOIN) across *= 2;
        {
            static const int ids_of[] = {HCH_KERNEL_ID("embed::embed_join_kernel<1>"), HCH_KERNEL_ID("embed::embed_join_kernel<2>"), HCH_KERNEL_ID("embed::embed_join_kernel<4>")};
            hch::LaunchTimer lt(ids_of[wide / 2], s, 8.0 * tiles * c, 0.0);
            if (wide == 4) HCH_LAUNCH(embed_join_kernel<4>, dim3((unsigned)tiles), dim3(JOIN), 0, s, R, dtable, c, rows, scale, across);
            else if (wide == 2) HCH_LAUNCH(embed_join_kernel<2>, dim3((unsigned)tiles), dim3(JOIN), 0, s, R, dtable, c, rows, scale, across);
            else HCH_LAUNCH(embed_join_kernel<1>, dim3((unsigned)tiles), dim3(JOIN), 0, s, R, dtable, c, rows, scale, across);
        }
        HCH_LAUNCH_CHECK("embed_join_kernel");
    }
    return HCH_OK;
} catch (const std::exception &) {
    return HCH_ENOMEM;
}
