// C entries of the row-wise operators of an attention block: layer norm and rotary positions.
#include "api_common.hpp"

#include <algorithm>
#include <cmath>
#include <exception>
#include <initializer_list>
#include <type_traits>

#include "norm.hip.hpp"
#include "rope.hip.hpp"

namespace {

bool known(hch_dtype t) { return t == HCH_F32 || t == HCH_BF16; }
int size_of(hch_dtype t) { return t == HCH_F32 ? 4 : 2; }
bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int MAX_CHANNELS = 8192;        // a workgroup of 256 holds 8 vectors of 4 per thread

// Lanes per row: the fewest that hold it at 4 channels each; a wavefront up to 1024 channels, a workgroup beyond.  With 8
// channels each where memory holds bf16: 16 bytes a lane.
struct RowShape { int lpr, nv; };
RowShape row_shape(int c, int w)
{
    for (int l = 4; l <= 64; l *= 2) if (c <= w * l) return {l, 1};
    if (c <= 128 * w) return {64, 2};
    if (c <= 1024) return {64, 4};
    return {256, c <= 2048 ? 2 : c <= 4096 ? 4 : 8};
}

// workgroups of the backward pass, and with them the parts of its sums: by the sizes alone
int bwd_blocks(int64_t n, int c)
{
    const int groups = hch::norm::THREADS / row_shape(c, 4).lpr;
    return (int)std::min<int64_t>(1024, std::max<int64_t>(1, (n + 4 * groups - 1) / (4 * groups)));
}

template <int N> using Int = std::integral_constant<int, N>;
// run: neighbours that a lane reads at once: 8 (16 bytes of bf16), 4, 2 or 1
template <typename F> void with_row_shape(int c, int run, F &&f)
{
    const RowShape s = row_shape(c, run == 8 ? 8 : 4);
#define HCH_SHAPE(L, V) if (s.lpr == L && s.nv == V) return run == 4 ? f(Int<L>{}, Int<4>{}, Int<V>{}, Int<4>{}) : run == 2 ? f(Int<L>{}, Int<4>{}, Int<V>{}, Int<2>{}) : f(Int<L>{}, Int<4>{}, Int<V>{}, Int<1>{});
#define HCH_WIDE(L, V) if (s.lpr == L && s.nv == V) return f(Int<L>{}, Int<8>{}, Int<V>{}, Int<8>{});
    if (run == 8) { HCH_WIDE(4, 1) HCH_WIDE(8, 1) HCH_WIDE(16, 1) HCH_WIDE(32, 1) HCH_WIDE(64, 1) HCH_WIDE(64, 2) }
    HCH_SHAPE(4, 1) HCH_SHAPE(8, 1) HCH_SHAPE(16, 1) HCH_SHAPE(32, 1) HCH_SHAPE(64, 1) HCH_SHAPE(64, 2) HCH_SHAPE(64, 4)
    HCH_SHAPE(256, 2) HCH_SHAPE(256, 4) HCH_SHAPE(256, 8)
#undef HCH_WIDE
#undef HCH_SHAPE
}
struct Tensor { const void *p; int bytes; };            // of an element
int run_of(int c, bool wide, std::initializer_list<Tensor> tensors)
{
    for (int run = wide && c <= 1024 ? 8 : 4; run > 1; run /= 2) {
        bool whole = c % run == 0;
        for (const Tensor &t : tensors) whole = whole && aligned(t.p, std::min(16, run * t.bytes));
        if (whole) return run;
    }
    return 1;
}

// id of an instance's name, as a profiler prints it: types, numbers, and what is behind them
template <typename TX, typename TY> int instance_id(const char *kernel, std::initializer_list<int> numbers, const char *end = ">")
{
    std::string name = std::string(kernel) + "<" + (sizeof(TX) == 4 ? "float" : "__bf16") + ", " + (sizeof(TY) == 4 ? "float" : "__bf16");
    for (int i : numbers) name += ", " + std::to_string(i);
    return hch::Profiler::get().id_for(name + end);
}

template <typename F> void with_types(hch_dtype a, hch_dtype b, F &&f)
{
    if (a == HCH_F32 && b == HCH_F32) f(float{}, float{});
    else if (a == HCH_F32) f(float{}, __bf16{});
    else if (b == HCH_F32) f(__bf16{}, float{});
    else f(__bf16{}, __bf16{});
}

}  // namespace

extern "C" hch_status hch_layernorm_fwd(hch_dtype x_dtype, const void *X, const void *R, void *S, const float *gamma, const float *beta,
                                        hch_dtype y_dtype, void *Y, float *stats, int64_t n, int32_t c, float eps, void *stream)
try {
    if (!known(x_dtype) || !known(y_dtype)) return fail(HCH_EINVAL, "hch_layernorm_fwd: unknown dtype");
    if ((n && (!X || !Y)) || (R != nullptr) != (S != nullptr)) return fail(HCH_EINVAL, "hch_layernorm_fwd: null pointer, or only one of R and S");
    if (n < 0 || c <= 0 || !(eps >= 0.f)) return fail(HCH_EINVAL, "hch_layernorm_fwd: bad size or eps");
    if (c > MAX_CHANNELS) return fail(HCH_EUNSUPPORTED, "hch_layernorm_fwd: more than 8192 channels");
    if (n == 0) return HCH_OK;
    const int sx = size_of(x_dtype), run = run_of(c, x_dtype == HCH_BF16 || y_dtype == HCH_BF16, {{X, sx}, {R, sx}, {S, sx}, {Y, size_of(y_dtype)}, {gamma, 4}, {beta, 4}});
    const int groups = hch::norm::THREADS / row_shape(c, run == 8 ? 8 : 4).lpr;
    const unsigned grid = (unsigned)std::min<int64_t>((n + groups - 1) / groups, 4096);
    {
        with_types(x_dtype, y_dtype, [&](auto tx, auto ty) {
            using TX = decltype(tx);
            using TY = decltype(ty);
            with_row_shape(c, run, [&](auto l, auto w, auto v, auto b) {
                static const int id = instance_id<TX, TY>("norm::layernorm_fwd_kernel", {decltype(l)::value, decltype(w)::value, decltype(v)::value, decltype(b)::value});
                hch::LaunchTimer lt(id, (hipStream_t)stream, (double)n * c * (size_of(x_dtype) * (R ? 3 : 1) + size_of(y_dtype)), 8.0 * n * c);
                constexpr auto kernel = hch::norm::layernorm_fwd_kernel<TX, TY, decltype(l)::value, decltype(w)::value, decltype(v)::value, decltype(b)::value>;
                HCH_LAUNCH(kernel, dim3(grid), dim3(hch::norm::THREADS), 0, (hipStream_t)stream, (const TX *)X, (const TX *)R, (TX *)S,
                           gamma, beta, (TY *)Y, stats, n, c, eps);
            });
        });
    }
    HCH_LAUNCH_CHECK("layernorm_fwd_kernel");
    return HCH_OK;
} catch (const std::exception &) {
    return HCH_ENOMEM;
}

extern "C" size_t hch_layernorm_workspace_bytes(int64_t n, int32_t c)
{
    if (n < 0 || c <= 0 || c > MAX_CHANNELS) return 0;
    return std::max<size_t>(256, ((size_t)bwd_blocks(n, c) * 2 * c * sizeof(float) + 255) / 256 * 256);
}

extern "C" hch_status hch_layernorm_bwd(hch_dtype x_dtype, const void *X, const float *stats, const float *gamma, hch_dtype dy_dtype,
                                        const void *dY, const void *dS, void *dX, float *dgamma, float *dbeta, int64_t n, int32_t c,
                                        void *workspace, size_t ws_bytes, void *stream)
try {
    if (!known(x_dtype) || !known(dy_dtype)) return fail(HCH_EINVAL, "hch_layernorm_bwd: unknown dtype");
    if ((n && (!X || !stats || !dY || !dX)) || (dgamma != nullptr) != (dbeta != nullptr))
        return fail(HCH_EINVAL, "hch_layernorm_bwd: null pointer, or only one of dgamma and dbeta");
    if (n < 0 || c <= 0) return fail(HCH_EINVAL, "hch_layernorm_bwd: bad size");
    if (c > MAX_CHANNELS) return fail(HCH_EUNSUPPORTED, "hch_layernorm_bwd: more than 8192 channels");
    const int blocks = n ? bwd_blocks(n, c) : 0;
    if (dgamma) {
        if (!workspace || !aligned(workspace, 256)) return fail(HCH_EINVAL, "hch_layernorm_bwd: workspace null or not 256-byte aligned");
        if (ws_bytes < hch_layernorm_workspace_bytes(n, c)) return fail(HCH_EWORKSPACE, "hch_layernorm_bwd: workspace too small");
    }
    float *part = dgamma ? (float *)workspace : nullptr;
    if (n) {
        // (fp32 rows with a bf16 gradient are faster by 4 channels: 47 against 50 us at 100000 rows of 256)
        const int sx = size_of(x_dtype), run = run_of(c, x_dtype == HCH_BF16, {{X, sx}, {dS, sx}, {dX, sx}, {dY, size_of(dy_dtype)}, {gamma, 4}});
        {
            with_types(x_dtype, dy_dtype, [&](auto tx, auto ty) {
                using TX = decltype(tx);
                using TY = decltype(ty);
                with_row_shape(c, run, [&](auto l, auto w, auto v, auto b) {
                    static const int id = instance_id<TX, TY>("norm::layernorm_bwd_kernel", {decltype(l)::value, decltype(w)::value, decltype(v)::value, decltype(b)::value});
                    hch::LaunchTimer lt(id, (hipStream_t)stream, (double)n * c * (size_of(x_dtype) * (dS ? 3 : 2) + size_of(dy_dtype)) + 8.0 * n, 14.0 * n * c);
                    constexpr auto kernel = hch::norm::layernorm_bwd_kernel<TX, TY, decltype(l)::value, decltype(w)::value, decltype(v)::value, decltype(b)::value>;
                    HCH_LAUNCH(kernel, dim3(blocks), dim3(hch::norm::THREADS), 0, (hipStream_t)stream, (const TX *)X, stats, gamma,
                               (const TY *)dY, (const TX *)dS, (TX *)dX, part, n, c);
                });
            });
        }
        HCH_LAUNCH_CHECK("layernorm_bwd_kernel");
    }
    if (dgamma) {
        {
            hch::LaunchTimer lt(2 * c <= 256 ? HCH_KERNEL_ID("norm::layernorm_sum_kernel<4>") : HCH_KERNEL_ID("norm::layernorm_sum_kernel<16>"), (hipStream_t)stream, 8.0 * blocks * c, 2.0 * blocks * c);
            if (2 * c <= 256)
                HCH_LAUNCH(hch::norm::layernorm_sum_kernel<4>, dim3((2 * c + 3) / 4), dim3(hch::norm::THREADS), 0, (hipStream_t)stream, part, dgamma,
                           dbeta, blocks, c);
            else
                HCH_LAUNCH(hch::norm::layernorm_sum_kernel<16>, dim3((2 * c + 15) / 16), dim3(hch::norm::THREADS), 0, (hipStream_t)stream, part,
                           dgamma, dbeta, blocks, c);
        }
        HCH_LAUNCH_CHECK("layernorm_sum_kernel");
    }
    return HCH_OK;
} catch (const std::exception &) {
    return HCH_ENOMEM;
}

namespace {

hch_status rope(const char *who, double sign, hch_dtype x_dtype, const void *X, int64_t ld_x, hch_dtype y_dtype, void *Y, int64_t ld_y,
                const int32_t *coords, int64_t n, int32_t heads, int32_t rot_heads, int32_t head_dim, const int32_t *sections, float base,
                float scale, void *stream)
{
    const std::string name = who;
    if (!known(x_dtype) || !known(y_dtype)) return fail(HCH_EINVAL, name + ": unknown dtype");
    if ((n && (!X || !Y)) || !sections) return fail(HCH_EINVAL, name + ": null pointer");
    if (n < 0 || heads <= 0 || rot_heads < 0 || rot_heads > heads || head_dim <= 0 || head_dim % 2) return fail(HCH_EINVAL, name + ": bad size");
    if (head_dim > 2 * hch::rope::MAX_PAIRS) return fail(HCH_EUNSUPPORTED, name + ": more than 256 channels per head");
    if (ld_x < (int64_t)heads * head_dim || ld_y < (int64_t)heads * head_dim) return fail(HCH_EINVAL, name + ": row stride below heads * head_dim");
    if (!(base > 0.f) || !std::isfinite(base) || !std::isfinite(scale)) return fail(HCH_EINVAL, name + ": base must be positive, base and scale finite");
    int pairs = 0;
    hch::rope::Table table = {};
    for (int a = 0; a < 3; ++a) {
        if (sections[a] < 0 || sections[a] > head_dim / 2 - pairs) return fail(HCH_EINVAL, name + ": sections exceed the pairs of a head");
        for (int j = 0; j < sections[a]; ++j, ++pairs) {
            table.turns[pairs] = sign * scale * std::pow((double)base, -(double)j / sections[a]) / M_PI;
            table.axis[pairs] = (uint8_t)a;
        }
    }
    if (n && !coords && rot_heads && pairs) return fail(HCH_EINVAL, name + ": coords is null");
    if (n && X == Y && (x_dtype != y_dtype || ld_x != ld_y)) return fail(HCH_EINVAL, name + ": in place needs one type and one row stride");
    if (n == 0) return HCH_OK;
    if ((int64_t)heads * head_dim > (1 << 22)) return fail(HCH_EUNSUPPORTED, name + ": more than 2^22 elements in a row");
    const int sx = size_of(x_dtype), sy = size_of(y_dtype);
    const bool vec = head_dim % 4 == 0 && ld_x % 4 == 0 && ld_y % 4 == 0 && aligned(X, 4 * sx) && aligned(Y, 4 * sy);
    const bool eight = vec && x_dtype == HCH_BF16 && head_dim % 8 == 0 && ld_x % 8 == 0 && ld_y % 8 == 0 && aligned(X, 16) && aligned(Y, 16);
    const int w = eight ? 8 : vec ? 4 : 2, pieces = heads * head_dim / w, wide = std::min(pieces, hch::rope::THREADS);
    // rows of a workgroup: what its threads have on the way at once, twice where there are many; as many as LDS has room for
    const int step = hch::rope::THREADS / wide * hch::rope::AT_ONCE;
    const int turned = rot_heads ? pairs : 0;
    int rows = n >= (int64_t)16384 * step / 8 ? 2 * step : step;
    if (turned) rows = std::min(rows, hch::rope::ENTRIES / turned);
    const int64_t blocks = (n - 1) / rows + 1;
    if (blocks > 0xffffffffll / hch::rope::THREADS) return fail(HCH_EUNSUPPORTED, name + ": more than 2^24 - 1 workgroups in a launch");
    {
        with_types(x_dtype, y_dtype, [&](auto tx, auto ty) {
            using TX = decltype(tx);
            using TY = decltype(ty);
            auto launch = [&](auto k, auto v) {
                static const int id = instance_id<TX, TY>("rope::rope_kernel", {decltype(k)::value}, decltype(v)::value ? ", true>" : ", false>");
                hch::LaunchTimer lt(id, (hipStream_t)stream, (double)n * heads * head_dim * (sx + sy) + 12.0 * n, 6.0 * n * rot_heads * pairs);
                constexpr auto kernel = hch::rope::rope_kernel<TX, TY, decltype(k)::value, decltype(v)::value>;
                HCH_LAUNCH(kernel, dim3((unsigned)blocks, (unsigned)((pieces + hch::rope::THREADS - 1) / hch::rope::THREADS)), dim3(hch::rope::THREADS),
                           0, (hipStream_t)stream, (const TX *)X, ld_x, (TY *)Y, ld_y, coords, n, pieces, wide, rows, rot_heads, head_dim, turned, table);
            };
            if (eight) launch(Int<8>{}, std::true_type{});
            else if (vec) launch(Int<4>{}, std::true_type{});
            else launch(Int<2>{}, std::false_type{});
        });
    }
    HCH_LAUNCH_CHECK("rope_kernel");
    return HCH_OK;
}

}  // namespace

extern "C" hch_status hch_rope_fwd(hch_dtype x_dtype, const void *X, int64_t ld_x, hch_dtype y_dtype, void *Y, int64_t ld_y,
                                   const int32_t *coords, int64_t n, int32_t heads, int32_t rot_heads, int32_t head_dim,
                                   const int32_t *sections, float base, float scale, void *stream)
try {
    return rope("hch_rope_fwd", 1.0, x_dtype, X, ld_x, y_dtype, Y, ld_y, coords, n, heads, rot_heads, head_dim, sections, base, scale, stream);
} catch (const std::exception &) {
    return HCH_ENOMEM;
}

extern "C" hch_status hch_rope_bwd(hch_dtype dy_dtype, const void *dY, int64_t ld_dy, hch_dtype dx_dtype, void *dX, int64_t ld_dx,
                                   const int32_t *coords, int64_t n, int32_t heads, int32_t rot_heads, int32_t head_dim,
                                   const int32_t *sections, float base, float scale, void *stream)
try {
    return rope("hch_rope_bwd", -1.0, dy_dtype, dY, ld_dy, dx_dtype, dX, ld_dx, coords, n, heads, rot_heads, head_dim, sections, base, scale, stream);
} catch (const std::exception &) {
    return HCH_ENOMEM;
}
