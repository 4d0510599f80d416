// C entries of the row-wise operators of an attention block: layer norm and rotary positions.
#include "api_common.hpp"

#include <algorithm>
#include <cmath>

#include "norm.hip.hpp"
#include "rope.hip.hpp"

namespace {

bool known(hch_dtype t) { return t == HCH_F32 || t == HCH_BF16; }
int size_of(hch_dtype t) { return t == HCH_F32 ? 4 : 2; }
bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

constexpr int MAX_CHANNELS = 8192;        // a workgroup of 256 holds 8 vectors of 4 per thread

// Lanes per row: the fewest that hold it at 4 channels each; a wavefront up to 1024 channels, a workgroup beyond.
struct RowShape { int lpr, nv; };
RowShape row_shape(int c)
{
    for (int l = 4; l <= 64; l *= 2) if (c <= 4 * l) return {l, 1};
    if (c <= 512) return {64, 2};
    if (c <= 1024) return {64, 4};
    return {256, c <= 2048 ? 2 : c <= 4096 ? 4 : 8};
}

// workgroups of the backward pass, and with them the parts of its sums: by the sizes alone
int bwd_blocks(int64_t n, int c)
{
    const int groups = hch::norm::THREADS / row_shape(c).lpr;
    return (int)std::min<int64_t>(1024, std::max<int64_t>(1, (n + 4 * groups - 1) / (4 * groups)));
}

template <typename F> void with_row_shape(int c, F &&f)
{
    const RowShape s = row_shape(c);
    auto k = [&](auto l, auto v) { f(l, v); };
#define HCH_SHAPE(L, V) if (s.lpr == L && s.nv == V) return k(std::integral_constant<int, L>{}, std::integral_constant<int, V>{});
    HCH_SHAPE(4, 1) HCH_SHAPE(8, 1) HCH_SHAPE(16, 1) HCH_SHAPE(32, 1) HCH_SHAPE(64, 1) HCH_SHAPE(64, 2) HCH_SHAPE(64, 4)
    HCH_SHAPE(256, 2) HCH_SHAPE(256, 4) HCH_SHAPE(256, 8)
#undef HCH_SHAPE
}

template <typename F> void with_types(hch_dtype a, hch_dtype b, F &&f)
{
    if (a == HCH_F32 && b == HCH_F32) f(float{}, float{});
    else if (a == HCH_F32) f(float{}, __bf16{});
    else if (b == HCH_F32) f(__bf16{}, float{});
    else f(__bf16{}, __bf16{});
}

template <typename F> void with_bool(bool b, F &&f)
{
    if (b) f(std::true_type{});
    else f(std::false_type{});
}

}  // namespace

extern "C" hch_status hch_layernorm_fwd(hch_dtype x_dtype, const void *X, const void *R, void *S, const float *gamma, const float *beta,
                                        hch_dtype y_dtype, void *Y, float *stats, int64_t n, int32_t c, float eps, void *stream)
{
    if (!known(x_dtype) || !known(y_dtype)) return fail(HCH_EINVAL, "hch_layernorm_fwd: unknown dtype");
    if (!X || !Y || (R != nullptr) != (S != nullptr)) return fail(HCH_EINVAL, "hch_layernorm_fwd: null pointer, or only one of R and S");
    if (n < 0 || c <= 0 || !(eps >= 0.f)) return fail(HCH_EINVAL, "hch_layernorm_fwd: bad size or eps");
    if (c > MAX_CHANNELS) return fail(HCH_EUNSUPPORTED, "hch_layernorm_fwd: more than 8192 channels");
    if (n == 0) return HCH_OK;
    const size_t ax = 4 * size_of(x_dtype), ay = 4 * size_of(y_dtype);
    const bool vec = c % 4 == 0 && aligned(X, ax) && aligned(R, ax) && aligned(S, ax) && aligned(Y, ay) && aligned(gamma, 16) && aligned(beta, 16);
    const int groups = hch::norm::THREADS / row_shape(c).lpr;
    const unsigned grid = (unsigned)std::min<int64_t>((n + groups - 1) / groups, 4096);
    {
        hch::LaunchTimer lt(HCH_KERNEL_ID("layernorm_fwd_kernel"), (hipStream_t)stream,
                            (double)n * c * (size_of(x_dtype) * (R ? 3 : 1) + size_of(y_dtype)), 8.0 * n * c);
        with_types(x_dtype, y_dtype, [&](auto tx, auto ty) {
            using TX = decltype(tx);
            using TY = decltype(ty);
            with_row_shape(c, [&](auto l, auto v) {
                with_bool(vec, [&](auto w) {
                    constexpr auto kernel = hch::norm::layernorm_fwd_kernel<TX, TY, decltype(l)::value, decltype(v)::value, decltype(w)::value>;
                    HCH_LAUNCH(kernel, dim3(grid), dim3(hch::norm::THREADS), 0, (hipStream_t)stream, (const TX *)X, (const TX *)R, (TX *)S,
                               gamma, beta, (TY *)Y, stats, n, c, eps);
                });
            });
        });
    }
    HCH_LAUNCH_CHECK("layernorm_fwd_kernel");
    return HCH_OK;
}

extern "C" size_t hch_layernorm_workspace_bytes(int64_t n, int32_t c)
{
    if (n < 0 || c <= 0 || c > MAX_CHANNELS) return 0;
    return std::max<size_t>(256, ((size_t)bwd_blocks(n, c) * 2 * c * sizeof(float) + 255) / 256 * 256);
}

extern "C" hch_status hch_layernorm_bwd(hch_dtype x_dtype, const void *X, const float *stats, const float *gamma, hch_dtype dy_dtype,
                                        const void *dY, const void *dS, void *dX, float *dgamma, float *dbeta, int64_t n, int32_t c,
                                        void *workspace, size_t ws_bytes, void *stream)
{
    if (!known(x_dtype) || !known(dy_dtype)) return fail(HCH_EINVAL, "hch_layernorm_bwd: unknown dtype");
    if (!X || !stats || !dY || !dX || (dgamma != nullptr) != (dbeta != nullptr))
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
        const size_t ax = 4 * size_of(x_dtype), ay = 4 * size_of(dy_dtype);
        const bool vec = c % 4 == 0 && aligned(X, ax) && aligned(dS, ax) && aligned(dX, ax) && aligned(dY, ay) && aligned(gamma, 16);
        {
            hch::LaunchTimer lt(HCH_KERNEL_ID("layernorm_bwd_kernel"), (hipStream_t)stream,
                                (double)n * c * (size_of(x_dtype) * (dS ? 3 : 2) + size_of(dy_dtype)) + 8.0 * n, 14.0 * n * c);
            with_types(x_dtype, dy_dtype, [&](auto tx, auto ty) {
                using TX = decltype(tx);
                using TY = decltype(ty);
                with_row_shape(c, [&](auto l, auto v) {
                    with_bool(vec, [&](auto w) {
                        constexpr auto kernel = hch::norm::layernorm_bwd_kernel<TX, TY, decltype(l)::value, decltype(v)::value, decltype(w)::value>;
                        HCH_LAUNCH(kernel, dim3(blocks), dim3(hch::norm::THREADS), 0, (hipStream_t)stream, (const TX *)X, stats, gamma,
                                   (const TY *)dY, (const TX *)dS, (TX *)dX, part, n, c);
                    });
                });
            });
        }
        HCH_LAUNCH_CHECK("layernorm_bwd_kernel");
    }
    if (dgamma) {
        {
            hch::LaunchTimer lt(HCH_KERNEL_ID("layernorm_sum_kernel"), (hipStream_t)stream, 8.0 * blocks * c, 2.0 * blocks * c);
            HCH_LAUNCH(hch::norm::layernorm_sum_kernel, dim3((2 * c + 15) / 16), dim3(hch::norm::THREADS), 0, (hipStream_t)stream, part, dgamma,
                       dbeta, blocks, c);
        }
        HCH_LAUNCH_CHECK("layernorm_sum_kernel");
    }
    return HCH_OK;
}

namespace {

hch_status rope(const char *who, double sign, hch_dtype x_dtype, const void *X, int64_t ld_x, hch_dtype y_dtype, void *Y, int64_t ld_y,
                const int32_t *coords, int64_t n, int32_t heads, int32_t rot_heads, int32_t head_dim, const int32_t *sections, float base,
                float scale, void *stream)
{
    const std::string name = who;
    if (!known(x_dtype) || !known(y_dtype)) return fail(HCH_EINVAL, name + ": unknown dtype");
    if (!X || !Y || !sections) return fail(HCH_EINVAL, name + ": null pointer");
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
    if (!coords && rot_heads && pairs) return fail(HCH_EINVAL, name + ": coords is null");
    if (X == Y && (x_dtype != y_dtype || ld_x != ld_y)) return fail(HCH_EINVAL, name + ": in place needs one type and one row stride");
    if (n == 0) return HCH_OK;
    const int sx = size_of(x_dtype), sy = size_of(y_dtype);
    const bool vec = head_dim % 4 == 0 && ld_x % 4 == 0 && ld_y % 4 == 0 && aligned(X, 4 * sx) && aligned(Y, 4 * sy);
    const int pieces = head_dim / (vec ? 4 : 2);
    // Heads per thread: all of a row's, which computes an angle once, unless that leaves fewer threads than the chip
    // holds (256 compute units of 2048): then as few as fill it.
    int per = heads;
    while (per > 1 && n * pieces * ((heads + per - 1) / per) < 256 * 2048) per = (per + 1) / 2;
    const int runs = (heads + per - 1) / per;
    const int64_t blocks = (n * pieces * runs + 255) / 256;
    if (blocks > 0x7fffffff) return fail(HCH_EUNSUPPORTED, name + ": too many rows for one launch");
    {
        hch::LaunchTimer lt(HCH_KERNEL_ID("rope_kernel"), (hipStream_t)stream, (double)n * heads * head_dim * (sx + sy) + 12.0 * n,
                            6.0 * n * rot_heads * pairs);
        with_types(x_dtype, y_dtype, [&](auto tx, auto ty) {
            using TX = decltype(tx);
            using TY = decltype(ty);
            with_bool(vec, [&](auto w) {
                constexpr auto kernel = hch::rope::rope_kernel<TX, TY, decltype(w)::value ? 2 : 1>;
                HCH_LAUNCH(kernel, dim3((unsigned)blocks), dim3(256), 0, (hipStream_t)stream, (const TX *)X, ld_x, (TY *)Y, ld_y, coords, n,
                           heads, rot_heads, head_dim, pairs, runs, per, table);
            });
        });
    }
    HCH_LAUNCH_CHECK("rope_kernel");
    return HCH_OK;
}

}  // namespace

extern "C" hch_status hch_rope_fwd(hch_dtype x_dtype, const void *X, int64_t ld_x, hch_dtype y_dtype, void *Y, int64_t ld_y,
                                   const int32_t *coords, int64_t n, int32_t heads, int32_t rot_heads, int32_t head_dim,
                                   const int32_t *sections, float base, float scale, void *stream)
{
    return rope("hch_rope_fwd", 1.0, x_dtype, X, ld_x, y_dtype, Y, ld_y, coords, n, heads, rot_heads, head_dim, sections, base, scale, stream);
}

extern "C" hch_status hch_rope_bwd(hch_dtype dy_dtype, const void *dY, int64_t ld_dy, hch_dtype dx_dtype, void *dX, int64_t ld_dx,
                                   const int32_t *coords, int64_t n, int32_t heads, int32_t rot_heads, int32_t head_dim,
                                   const int32_t *sections, float base, float scale, void *stream)
{
    return rope("hch_rope_bwd", -1.0, dy_dtype, dY, ld_dy, dx_dtype, dX, ld_dx, coords, n, heads, rot_heads, head_dim, sections, base, scale, stream);
}
