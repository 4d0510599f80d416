// C entries of dropout: alone (with a sum), and with the residual sum and the layer norm behind it.
#include "rows.hpp"

#include "dropout.hip.hpp"

namespace {

hch_status drop_of(const std::string &name, float p, uint64_t seed, const int64_t *step, hch::dropout::Drop &d)
{
    if (!(p >= 0.f && p <= 1.f)) return fail(HCH_EINVAL, name + ": p must be between 0 and 1");
    if (!aligned(step, 8)) return fail(HCH_EINVAL, name + ": step is not aligned to 8 bytes");
    d.key0 = (uint32_t)seed;
    d.key1 = (uint32_t)(seed >> 32);
    d.least = (uint32_t)std::floor((double)p * 65536.0 + 0.5);
    d.scale = d.least < 65536 ? (float)(65536.0 / (65536.0 - d.least)) : 0.f;
    d.step = step;
    return HCH_OK;
}

// Backward, rows of bf16 by pairs: 8 channels a lane, so that a block of numbers is a lane's own and half as many lanes repeat what each does for its
// row (300000 rows of 50, bf16: by 4 53 us, by 8 44; 100000 of 250 67 and 58; fp32 rows and the forward pass are up to a fifth slower so).
template <typename TX, typename F> void with_bwd_shape(int c, int run, F &&f)
{
    if constexpr (sizeof(TX) == 2)
        if (run == 2 && c <= 1024) {
            const RowShape s = row_shape(c, 8);
#define HCH_SHAPE(L, V) if (s.lpr == L && s.nv == V) return f(Int<L>{}, Int<8>{}, Int<V>{}, Int<2>{});
            HCH_SHAPE(4, 1) HCH_SHAPE(8, 1) HCH_SHAPE(16, 1) HCH_SHAPE(32, 1) HCH_SHAPE(64, 1) HCH_SHAPE(64, 2)
#undef HCH_SHAPE
        }
    with_row_shape(c, run, f);
}

hch_status dropout(const char *who, hch_dtype x_dtype, const void *X, const void *R, hch_dtype y_dtype, void *Y, int64_t n, int32_t c, float p,
                   uint64_t seed, const int64_t *step, void *stream)
{
    const std::string name = who;
    if (!known(x_dtype) || !known(y_dtype)) return fail(HCH_EINVAL, name + ": unknown dtype");
    if (n && (!X || !Y)) return fail(HCH_EINVAL, name + ": null pointer");
    if (n < 0 || c <= 0) return fail(HCH_EINVAL, name + ": bad size");
    hch::dropout::Drop drop;
    if (const hch_status st = drop_of(name, p, seed, step, drop)) return st;
    if (n && X == Y && x_dtype != y_dtype) return fail(HCH_EINVAL, name + ": in place needs one type");
    if (n > (int64_t(1) << 60) / c) return fail(HCH_EUNSUPPORTED, name + ": more than 2^60 elements");
    if (n == 0) return HCH_OK;
    const int sx = size_of(x_dtype), sy = size_of(y_dtype);
    const bool vec = aligned(X, 16) && aligned(R, 16) && aligned(Y, 16);
    const unsigned grid = (unsigned)std::min<int64_t>((n * c - 1) / 4096 + 1, 4096);
    with_types(x_dtype, y_dtype, [&](auto tx, auto ty) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        auto launch = [&](auto b, auto v) {
            constexpr bool B = decltype(b)::value, V = decltype(v)::value;
            static const int id = instance_id<TX, TY>("dropout::dropout_kernel", {}, B ? V ? ", true, true>" : ", true, false>" : V ? ", false, true>" : ", false, false>");
            hch::LaunchTimer lt(id, (hipStream_t)stream, (double)n * c * (sx + sy * (R ? 2 : 1)), 2.0 * n * c);
            constexpr auto kernel = hch::dropout::dropout_kernel<TX, TY, B, V>;
            HCH_LAUNCH(kernel, dim3(grid), dim3(hch::dropout::THREADS), 0, (hipStream_t)stream, (const TX *)X, (const TY *)R, (TY *)Y, n, c, drop);
        };
        if (c % 8 == 0) vec ? launch(std::true_type{}, std::true_type{}) : launch(std::true_type{}, std::false_type{});
        else vec ? launch(std::false_type{}, std::true_type{}) : launch(std::false_type{}, std::false_type{});
    });
    HCH_LAUNCH_CHECK("dropout_kernel");
    return HCH_OK;
}

}  // namespace

extern "C" hch_status hch_dropout_fwd(hch_dtype x_dtype, const void *X, const void *R, hch_dtype y_dtype, void *Y, int64_t n, int32_t c, float p,
                                      uint64_t seed, const int64_t *step, void *stream)
try {
    return dropout("hch_dropout_fwd", x_dtype, X, R, y_dtype, Y, n, c, p, seed, step, stream);
} catch (const std::exception &) {
    return HCH_ENOMEM;
}

extern "C" hch_status hch_dropout_bwd(hch_dtype dy_dtype, const void *dY, hch_dtype dx_dtype, void *dX, int64_t n, int32_t c, float p,
                                      uint64_t seed, const int64_t *step, void *stream)
try {
    return dropout("hch_dropout_bwd", dy_dtype, dY, nullptr, dx_dtype, dX, n, c, p, seed, step, stream);
} catch (const std::exception &) {
    return HCH_ENOMEM;
}

extern "C" hch_status hch_dropout_layernorm_fwd(hch_dtype x_dtype, const void *X, const void *R, void *S, const float *gamma, const float *beta,
                                                hch_dtype y_dtype, void *Y, float *stats, int64_t n, int32_t c, float eps, float p, uint64_t seed,
                                                const int64_t *step, void *stream)
try {
    const std::string name = "hch_dropout_layernorm_fwd";
    if (!known(x_dtype) || !known(y_dtype)) return fail(HCH_EINVAL, name + ": unknown dtype");
    if (n && (!X || !R || !S || !Y)) return fail(HCH_EINVAL, name + ": null pointer");
    if (n < 0 || c <= 0 || !(eps >= 0.f)) return fail(HCH_EINVAL, name + ": bad size or eps");
    if (n && Y == S) return fail(HCH_EINVAL, name + ": S and Y are one tensor");
    if (n && (Y == X || Y == R) && x_dtype != y_dtype) return fail(HCH_EINVAL, name + ": in place needs one type");
    hch::dropout::Drop drop;
    if (const hch_status st = drop_of(name, p, seed, step, drop)) return st;
    if (c > MAX_CHANNELS) return fail(HCH_EUNSUPPORTED, name + ": more than 8192 channels");
    if (n == 0) return HCH_OK;
    const int sx = size_of(x_dtype), run = run_of(c, x_dtype == HCH_BF16 || y_dtype == HCH_BF16, {{X, sx}, {R, sx}, {S, sx}, {Y, size_of(y_dtype)}, {gamma, 4}, {beta, 4}});
    const int groups = hch::norm::THREADS / row_shape(c, run == 8 ? 8 : 4).lpr;
    const unsigned grid = (unsigned)std::min<int64_t>((n + groups - 1) / groups, 4096);
    with_types(x_dtype, y_dtype, [&](auto tx, auto ty) {
        using TX = decltype(tx);
        using TY = decltype(ty);
        with_row_shape(c, run, [&](auto l, auto w, auto v, auto b) {
            static const int id = instance_id<TX, TY>("dropout::dropout_layernorm_fwd_kernel", {decltype(l)::value, decltype(w)::value, decltype(v)::value, decltype(b)::value});
            hch::LaunchTimer lt(id, (hipStream_t)stream, (double)n * c * (size_of(x_dtype) * 3 + size_of(y_dtype)), 10.0 * n * c);
            constexpr auto kernel = hch::dropout::dropout_layernorm_fwd_kernel<TX, TY, decltype(l)::value, decltype(w)::value, decltype(v)::value, decltype(b)::value>;
            HCH_LAUNCH(kernel, dim3(grid), dim3(hch::dropout::THREADS), 0, (hipStream_t)stream, (const TX *)X, (const TX *)R, (TX *)S, gamma, beta,
                       (TY *)Y, stats, n, c, eps, drop);
        });
    });
    HCH_LAUNCH_CHECK("dropout_layernorm_fwd_kernel");
    return HCH_OK;
} catch (const std::exception &) {
    return HCH_ENOMEM;
}

extern "C" hch_status hch_dropout_layernorm_bwd(hch_dtype x_dtype, const void *S, const float *stats, const float *gamma, hch_dtype dy_dtype,
                                                const void *dY, const void *dS, void *dR, hch_dtype dx_dtype, void *dX, float *dgamma, float *dbeta,
                                                int64_t n, int32_t c, float p, uint64_t seed, const int64_t *step, void *workspace, size_t ws_bytes,
                                                void *stream)
try {
    const std::string name = "hch_dropout_layernorm_bwd";
    if (!known(x_dtype) || !known(dy_dtype) || !known(dx_dtype)) return fail(HCH_EINVAL, name + ": unknown dtype");
    if ((n && (!S || !stats || !dY || !dR || !dX)) || (dgamma != nullptr) != (dbeta != nullptr))
        return fail(HCH_EINVAL, name + ": null pointer, or only one of dgamma and dbeta");
    if (n < 0 || c <= 0) return fail(HCH_EINVAL, name + ": bad size");
    if (n && (dX == dR || dX == S || dX == dY || dX == dS)) return fail(HCH_EINVAL, name + ": dX is another tensor of the call too");
    if (n && dR == dY && x_dtype != dy_dtype) return fail(HCH_EINVAL, name + ": in place needs one type");
    hch::dropout::Drop drop;
    if (const hch_status st = drop_of(name, p, seed, step, drop)) return st;
    if (c > MAX_CHANNELS) return fail(HCH_EUNSUPPORTED, name + ": more than 8192 channels");
    const int blocks = n ? bwd_blocks(n, c) : 0;
    if (dgamma) {
        if (!workspace || !aligned(workspace, 256)) return fail(HCH_EINVAL, name + ": workspace null or not 256-byte aligned");
        if (ws_bytes < hch_layernorm_workspace_bytes(n, c)) return fail(HCH_EWORKSPACE, name + ": workspace too small");
    }
    float *part = dgamma ? (float *)workspace : nullptr;
    if (n) {
        const int sx = size_of(x_dtype), sy = size_of(dy_dtype), sd = size_of(dx_dtype);
        const int run = run_of(c, x_dtype == HCH_BF16, {{S, sx}, {dS, sx}, {dR, sx}, {dX, sd}, {dY, sy}, {gamma, 4}});
        with_types(x_dtype, dy_dtype, [&](auto tx, auto ty) {
            using TX = decltype(tx);
            using TY = decltype(ty);
            with_bwd_shape<TX>(c, run, [&](auto l, auto w, auto v, auto b) {
                static const int id = instance_id<TX, TY>("dropout::dropout_layernorm_bwd_kernel", {decltype(l)::value, decltype(w)::value, decltype(v)::value, decltype(b)::value});
                hch::LaunchTimer lt(id, (hipStream_t)stream, (double)n * c * (sx * (dS ? 3 : 2) + sy + sd) + 8.0 * n, 16.0 * n * c);
                constexpr auto kernel = hch::dropout::dropout_layernorm_bwd_kernel<TX, TY, decltype(l)::value, decltype(w)::value, decltype(v)::value, decltype(b)::value>;
                HCH_LAUNCH(kernel, dim3(blocks), dim3(hch::dropout::THREADS), 0, (hipStream_t)stream, (const TX *)S, stats, gamma, (const TY *)dY,
                           (const TX *)dS, (TX *)dR, dX, dx_dtype == HCH_BF16, part, dgamma, dbeta, n, c, drop);
            });
        });
        HCH_LAUNCH_CHECK("dropout_layernorm_bwd_kernel");
    }
    if (!dgamma || blocks == 1) return HCH_OK;              // one workgroup has joined its sums itself (2 rows of 128: 9 us; two launches take 12.6)
    return join_sums(part, dgamma, dbeta, blocks, c, stream);
} catch (const std::exception &) {
    return HCH_ENOMEM;
}
