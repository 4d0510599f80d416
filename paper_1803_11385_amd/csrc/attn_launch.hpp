// Launches of the attention kernels: the choice of an instance by element type and head width.  The instances of a type
// are compiled in a source of their own (attn_bf16.hip, attn_f32.hip).
#pragma once
#include <cstdio>

#include "api_common.hpp"
#include "attn.hip.hpp"

namespace hch {
namespace attn {

// `narrow`: one tile of 32 rows (keys) per workgroup (Keys<E, D, 1>, Queries<E, D, 1>).  flops: of the whole pass, for the profile.
template <typename T> hch_status launch_fwd(const Args &a, bool narrow, double bytes, double flops, hipStream_t s);
template <typename T> hch_status launch_bwd_dq(const Args &a, bool narrow, double bytes, double flops, hipStream_t s);
template <typename T> hch_status launch_bwd_dkv(const Args &a, bool narrow, double bytes, double flops, hipStream_t s);
// dQ (a) and dK, dV (b) in one launch, after one for D; both `narrow` or not, everything in whole pieces
template <typename T> hch_status launch_bwd_both(const Args &a, const Args &b, bool narrow, double bytes, double flops, hipStream_t s);
// dQ from its splits, and dK and dV from theirs (those of `a`); 1 split: written already
template <typename T> hch_status launch_bwd_join(const Args &a, const float *q_part, int q_splits, hipStream_t s);

#ifdef HCH_ATTN_TYPE
template <typename T> struct EngineOf { typedef Bf16 E; };
template <> struct EngineOf<float> { typedef Split E; };

// The instance for heads of d channels.  fp32's narrow forms share a result's channels between two wavefronts beyond 64: no 96.
template <typename T, typename F> void with_width(int d, bool narrow, bool vec, F &&f)
{
    auto g = [&](auto w) {
        if (vec) f(w, std::true_type{});
        else f(w, std::false_type{});
    };
    if (d <= 32) g(std::integral_constant<int, 32>{});
    else if (d <= 64) g(std::integral_constant<int, 64>{});
    else if (d <= 96 && !(narrow && sizeof(T) == 4)) g(std::integral_constant<int, 96>{});
    else g(std::integral_constant<int, 128>{});
}
// id of an instance's name, as a profiler prints it
inline int instance_id(const char *kernel, const char *engine, int d, int form, bool vec)
{
    char name[96];
    snprintf(name, sizeof name, "%s<%s, %d, %d, %s>", kernel, engine, d, form, vec ? "true" : "false");
    return Profiler::get().id_for(name);
}
inline int both_id(const char *engine, int d, int form)
{
    char name[96];
    snprintf(name, sizeof name, "attn::attn_bwd_both_kernel<%s, %d, %d>", engine, d, form);
    return Profiler::get().id_for(name);
}
template <typename T> constexpr const char *TYPE_NAME = sizeof(T) == 4 ? "float" : "__bf16";
inline int join_id(const char *kernel, const char *type, int groups)
{
    char name[64];
    if (groups) snprintf(name, sizeof name, "%s<%s, %d>", kernel, type, groups);
    else snprintf(name, sizeof name, "%s<%s>", kernel, type);
    return Profiler::get().id_for(name);
}

template <typename T, int D> constexpr bool has_narrow = sizeof(T) == 2 || D != 96;

template <typename T> hch_status launch_fwd(const Args &a, bool narrow, double bytes, double flops, hipStream_t s)
{
    with_width<T>(a.d, narrow, a.vec, [&](auto w, auto v) {
        typedef typename EngineOf<T>::E E;
        constexpr int D = decltype(w)::value;
        constexpr bool V = decltype(v)::value;
        if (!narrow) {
            static const int id = instance_id("attn::attn_fwd_kernel", E::NAME, D, 4, V);
            constexpr auto kernel = attn_fwd_kernel<E, D, 4, V>;
            LaunchTimer lt(id, s, bytes, flops);
            HCH_LAUNCH(kernel, dim3(work_grid(a)), dim3((Keys<E, D, 4, V>::THREADS)), 0, s, a);
        } else if constexpr (has_narrow<T, D>) {
            static const int id = instance_id("attn::attn_fwd_kernel", E::NAME, D, 1, V);
            constexpr auto kernel = attn_fwd_kernel<E, D, 1, V>;
            LaunchTimer lt(id, s, bytes, flops);
            HCH_LAUNCH(kernel, dim3(work_grid(a)), dim3((Keys<E, D, 1, V>::THREADS)), 0, s, a);
        }
    });
    HCH_LAUNCH_CHECK("attn_fwd_kernel");
    if (a.splits > 1) {
        {
            const int64_t rows = a.nq * a.hq;
            static const int id1 = join_id("attn::attn_join_kernel", TYPE_NAME<T>, 1), id8 = join_id("attn::attn_join_kernel", TYPE_NAME<T>, 8);
            LaunchTimer lt(a.splits <= 8 || rows >= 4096 ? id1 : id8, s, (double)a.splits * rows * (4 * a.d + 8), 0.0);
            constexpr auto one = attn_join_kernel<T, 1>;
            constexpr auto eight = attn_join_kernel<T, 8>;
            if (a.splits <= 8 || rows >= 4096) HCH_LAUNCH(one, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, s, a);
            else HCH_LAUNCH(eight, dim3((unsigned)rows), dim3(256), 0, s, a);
        }
        HCH_LAUNCH_CHECK("attn_join_kernel");
    }
    return HCH_OK;
}

template <typename T> hch_status launch_bwd_dq(const Args &a, bool narrow, double bytes, double flops, hipStream_t s)
{
    with_width<T>(a.d, narrow, a.vec, [&](auto w, auto v) {
        typedef typename EngineOf<T>::E E;
        constexpr int D = decltype(w)::value;
        constexpr bool V = decltype(v)::value;
        if (!narrow) {
            static const int id = instance_id("attn::attn_bwd_dq_kernel", E::NAME, D, 4, V);
            constexpr auto kernel = attn_bwd_dq_kernel<E, D, 4, V>;
            LaunchTimer lt(id, s, bytes, flops);
            HCH_LAUNCH(kernel, dim3(work_grid(a)), dim3((Keys<E, D, 4, V>::THREADS)), 0, s, a);
        } else if constexpr (has_narrow<T, D>) {
            static const int id = instance_id("attn::attn_bwd_dq_kernel", E::NAME, D, 1, V);
            constexpr auto kernel = attn_bwd_dq_kernel<E, D, 1, V>;
            LaunchTimer lt(id, s, bytes, flops);
            HCH_LAUNCH(kernel, dim3(work_grid(a)), dim3((Keys<E, D, 1, V>::THREADS)), 0, s, a);
        }
    });
    HCH_LAUNCH_CHECK("attn_bwd_dq_kernel");
    return HCH_OK;
}

template <typename T> hch_status launch_bwd_dkv(const Args &a, bool narrow, double bytes, double flops, hipStream_t s)
{
    with_width<T>(a.d, narrow, a.vec, [&](auto w, auto v) {
        typedef typename EngineOf<T>::E E;
        constexpr int D = decltype(w)::value;
        constexpr bool V = decltype(v)::value;
        if (!narrow) {
            static const int id = instance_id("attn::attn_bwd_dkv_kernel", E::NAME, D, 4, V);
            constexpr auto kernel = attn_bwd_dkv_kernel<E, D, 4, V>;
            LaunchTimer lt(id, s, bytes, flops);
            HCH_LAUNCH(kernel, dim3(work_grid(a)), dim3((Queries<E, D, 4, V>::THREADS)), 0, s, a);
        } else if constexpr (has_narrow<T, D>) {
            static const int id = instance_id("attn::attn_bwd_dkv_kernel", E::NAME, D, 1, V);
            constexpr auto kernel = attn_bwd_dkv_kernel<E, D, 1, V>;
            LaunchTimer lt(id, s, bytes, flops);
            HCH_LAUNCH(kernel, dim3(work_grid(a)), dim3((Queries<E, D, 1, V>::THREADS)), 0, s, a);
        }
    });
    HCH_LAUNCH_CHECK("attn_bwd_dkv_kernel");
    return HCH_OK;
}

template <typename T> hch_status launch_bwd_both(const Args &a, const Args &b, bool narrow, double bytes, double flops, hipStream_t s)
{
    {
        const int64_t rows = a.nq * a.hq;
        int lanes = 1;
        while (lanes * 16 < a.d * (int)sizeof(T)) lanes *= 2;
        static const int id = join_id("attn::attn_delta_kernel", TYPE_NAME<T>, 0);
        LaunchTimer lt(id, s, (double)rows * (2 * a.d * sizeof(T) + 8), 0.0);
        constexpr auto kernel = attn_delta_kernel<T>;
        HCH_LAUNCH(kernel, dim3((unsigned)((rows * lanes + 255) / 256)), dim3(256), 0, s, b, lanes);
    }
    HCH_LAUNCH_CHECK("attn_delta_kernel");
    with_width<T>(a.d, narrow, true, [&](auto w, auto) {
        typedef typename EngineOf<T>::E E;
        constexpr int D = decltype(w)::value;
        if (!narrow) {
            static const int id = both_id(E::NAME, D, 4);
            constexpr auto kernel = attn_bwd_both_kernel<E, D, 4>;
            LaunchTimer lt(id, s, bytes, flops);
            HCH_LAUNCH(kernel, dim3(work_grid(a) + work_grid(b)), dim3((Keys<E, D, 4, true>::THREADS)), 0, s, a, b, (int)work_grid(a));
        } else if constexpr (has_narrow<T, D>) {
            static const int id = both_id(E::NAME, D, 1);
            constexpr auto kernel = attn_bwd_both_kernel<E, D, 1>;
            LaunchTimer lt(id, s, bytes, flops);
            HCH_LAUNCH(kernel, dim3(work_grid(a) + work_grid(b)), dim3((Keys<E, D, 1, true>::THREADS)), 0, s, a, b, (int)work_grid(a));
        }
    });
    HCH_LAUNCH_CHECK("attn_bwd_both_kernel");
    return HCH_OK;
}

template <typename T> hch_status launch_bwd_join(const Args &a, const float *q_part, int q_splits, hipStream_t s)
{
    const int64_t nq = q_splits > 1 ? a.nq * a.hq * a.d : 0, nk = a.splits > 1 ? 2 * a.nk * a.hkv * a.d : 0, blocks = (nq + 255) / 256;
    static const int id = join_id("attn::attn_bwd_join_kernel", TYPE_NAME<T>, 0);
    LaunchTimer lt(id, s, 4.0 * ((double)q_splits * nq + (double)a.splits * nk), 0.0);
    constexpr auto kernel = attn_bwd_join_kernel<T>;
    HCH_LAUNCH(kernel, dim3((unsigned)(blocks + (nk + 255) / 256)), dim3(256), 0, s, a, q_part, q_splits, (int)blocks);
    HCH_LAUNCH_CHECK("attn_bwd_join_kernel");
    return HCH_OK;
}

template hch_status launch_fwd<HCH_ATTN_TYPE>(const Args &, bool, double, double, hipStream_t);
template hch_status launch_bwd_dq<HCH_ATTN_TYPE>(const Args &, bool, double, double, hipStream_t);
template hch_status launch_bwd_dkv<HCH_ATTN_TYPE>(const Args &, bool, double, double, hipStream_t);
template hch_status launch_bwd_both<HCH_ATTN_TYPE>(const Args &, const Args &, bool, double, double, hipStream_t);
template hch_status launch_bwd_join<HCH_ATTN_TYPE>(const Args &, const float *, int, hipStream_t);
#endif

}  // namespace attn
}  // namespace hch
