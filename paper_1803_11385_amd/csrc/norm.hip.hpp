// Layer norm over the channels of a voxel row, with the residual sum in front of it, and its gradients.
//   forward   s = x + r;  mu = mean(s);  v = mean((s - mu)^2);  y = (s - mu) / sqrt(v + eps) * gamma + beta
//   backward  h = (x - mu) rs;  w = dy gamma;  dx = rs (w - mean(w) - h mean(w h)) + ds
//             dgamma = sum over rows of dy h;  dbeta = sum over rows of dy
// A row is held by LPR lanes, NV vectors of W channels each, and read once: mean and variance come from the
// registers (two passes over them, so a row with a large mean loses nothing), all sums in fp32.  LPR is the least number of lanes that holds the row
// in pieces of up to 16 bytes, so that short rows share a wavefront and no lane idles.  Bound by memory: 609323 rows of 64, fp32 with a
// residual sum, to bf16: 101 us, 5.4 TB/s (a copy of 2 GB: 4.9); backward of 279722 rows of 128, bf16, with a residual's gradient: 51 to 58 us, 4.9 to
// 5.6 TB/s; 752 rows of 64 take 3 us, a launch.  Sums over the rows (dgamma, dbeta) are taken by workgroup and added up by a second launch in a
// fixed order, not by atomics, whose order would change the bits from run to run.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace hch {
namespace norm {

constexpr int THREADS = 256;

template <typename T, int W> struct Vec { typedef T type __attribute__((ext_vector_type(W))); };

// the sum over a group of LPR lanes (4 .. 64), in every lane of the group; a fixed order
template <int CTRL> __device__ __forceinline__ float dpp_add(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}
template <int LPR> __device__ __forceinline__ float group_sum(float v)
{
    v = dpp_add<0xB1>(v);                                   // lane ^ 1
    v = dpp_add<0x4E>(v);                                   // lane ^ 2
    if constexpr (LPR >= 8) v = dpp_add<0x141>(v);          // the other 4 of 8
    if constexpr (LPR >= 16) v = dpp_add<0x140>(v);         // the other 8 of 16
    if constexpr (LPR >= 32) {
        const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    if constexpr (LPR >= 64) {
        const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(s[0]) + __uint_as_float(s[1]);
    }
    return v;
}
// the same where a row has a workgroup to itself (LPR = 256); `turn` alternates between calls
template <int LPR> __device__ __forceinline__ float row_sum(float v, float *lds, int &turn)
{
    if constexpr (LPR <= 64) return group_sum<LPR>(v);
    else {
        v = group_sum<64>(v);
        float *p = lds + 4 * turn;
        turn ^= 1;                                          // a wavefront may be one call ahead of another, not two
        if ((threadIdx.x & 63) == 0) p[threadIdx.x >> 6] = v;
        __syncthreads();
        return (p[0] + p[1]) + (p[2] + p[3]);
    }
}

// Channel of element j of vector v of a lane.  A lane has RUN neighbours at a time, W, 2 or 1, as width and alignment allow; the
// lanes' runs lie side by side, so that a wavefront reads runs of memory in any case (300000 rows of 50, bf16 with a residual: one by one
// 53 us forward and 96 backward, by pairs 36 and 43).
template <int LPR, int W, int RUN> __device__ __forceinline__ int channel(int lane, int v, int j)
{
    return ((v * (W / RUN) + j / RUN) * LPR + lane) * RUN + j % RUN;
}
template <typename T, int LPR, int W, int NV, int RUN>
__device__ __forceinline__ void load_row(const T *row, int lane, int c, float (&x)[W * NV])
{
    typedef typename Vec<T, RUN>::type V;
#pragma unroll
    for (int i = 0; i < W * NV; i += RUN) {
        const int e = channel<LPR, W, RUN>(lane, i / W, i % W);
        V t = {};
        if (e < c) t = *(const V *)(row + e);
#pragma unroll
        for (int j = 0; j < RUN; ++j) x[i + j] = (float)t[j];
    }
}
template <typename T, int LPR, int W, int NV, int RUN>
__device__ __forceinline__ void store_row(T *row, int lane, int c, const float (&x)[W * NV])
{
    typedef typename Vec<T, RUN>::type V;
#pragma unroll
    for (int i = 0; i < W * NV; i += RUN) {
        const int e = channel<LPR, W, RUN>(lane, i / W, i % W);
        if (e >= c) continue;
        V t;
#pragma unroll
        for (int j = 0; j < RUN; ++j) t[j] = (T)x[i + j];
        *(V *)(row + e) = t;
    }
}

template <typename TX, typename TY, int LPR, int W, int NV, int RUN>
__global__ __launch_bounds__(THREADS) void layernorm_fwd_kernel(const TX *X, const TX *R, TX *S, const float *gamma,
                                                                const float *beta, TY *Y, float *stats, int64_t n, int c, float eps)
{
    __shared__ float lds[8];
    int turn = 0;
    constexpr int GROUPS = THREADS / LPR;
    const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
    float g[W * NV], b[W * NV];
    if (gamma) load_row<float, LPR, W, NV, RUN>(gamma, lane, c, g);
    if (beta) load_row<float, LPR, W, NV, RUN>(beta, lane, c, b);
#pragma unroll
    for (int i = 0; i < W * NV; ++i) { if (!gamma) g[i] = 1.f; if (!beta) b[i] = 0.f; }
    const float width = (float)c;                           // divided by, not multiplied with 1 / c: the mean of equal channels is exact
    for (int64_t row = (int64_t)blockIdx.x * GROUPS + group; row < n; row += (int64_t)gridDim.x * GROUPS) {
        float x[W * NV];
        load_row<TX, LPR, W, NV, RUN>(X + row * c, lane, c, x);
        if (R) {
            float r[W * NV];
            load_row<TX, LPR, W, NV, RUN>(R + row * c, lane, c, r);
#pragma unroll
            for (int i = 0; i < W * NV; ++i) x[i] += r[i];
            store_row<TX, LPR, W, NV, RUN>(S + row * c, lane, c, x);
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < W * NV; ++i) sum += x[i];       // channels past the row hold 0
        const float mean = row_sum<LPR>(sum, lds, turn) / width;
        float sq = 0.f;
#pragma unroll
        for (int v = 0; v < NV; ++v)
#pragma unroll
            for (int j = 0; j < W; ++j) {
                x[W * v + j] -= mean;
                sq += channel<LPR, W, RUN>(lane, v, j) < c ? x[W * v + j] * x[W * v + j] : 0.f;
            }
        const float rs = 1.f / sqrtf(row_sum<LPR>(sq, lds, turn) / width + eps);
        if (stats && lane == 0) { stats[2 * row] = mean; stats[2 * row + 1] = rs; }
#pragma unroll
        for (int i = 0; i < W * NV; ++i) x[i] = x[i] * rs * g[i] + b[i];
        store_row<TY, LPR, W, NV, RUN>(Y + row * c, lane, c, x);
    }
}

// part: [gridDim.x][2][c], the sums of dy h and of dy over a workgroup's rows; null: not wanted
template <typename TX, typename TY, int LPR, int W, int NV, int RUN>
__global__ __launch_bounds__(THREADS) void layernorm_bwd_kernel(const TX *X, const float *stats, const float *gamma, const TY *dY,
                                                                const TX *dS, TX *dX, float *part, int64_t n, int c)
{
    __shared__ float lds[8];
    __shared__ float sums[2 * THREADS * W * NV];
    int turn = 0;
    constexpr int GROUPS = THREADS / LPR;
    const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR;
    float g[W * NV], dg[W * NV], db[W * NV];
    if (gamma) load_row<float, LPR, W, NV, RUN>(gamma, lane, c, g);
#pragma unroll
    for (int i = 0; i < W * NV; ++i) { if (!gamma) g[i] = 1.f; dg[i] = db[i] = 0.f; }
    const float inv = 1.f / (float)c;
    for (int64_t row = (int64_t)blockIdx.x * GROUPS + group; row < n; row += (int64_t)gridDim.x * GROUPS) {
        float x[W * NV], y[W * NV];
        load_row<TX, LPR, W, NV, RUN>(X + row * c, lane, c, x);
        load_row<TY, LPR, W, NV, RUN>(dY + row * c, lane, c, y);
        const float mean = stats[2 * row], rs = stats[2 * row + 1];
        float sw = 0.f, swh = 0.f;
#pragma unroll
        for (int i = 0; i < W * NV; ++i) {                  // dy is 0 past the row: nothing is added there
            const float h = (x[i] - mean) * rs, w = y[i] * g[i];
            dg[i] += y[i] * h;
            db[i] += y[i];
            sw += w;
            swh += w * h;
            x[i] = h;
            y[i] = w;
        }
        sw = row_sum<LPR>(sw, lds, turn) * inv;
        swh = row_sum<LPR>(swh, lds, turn) * inv;
#pragma unroll
        for (int i = 0; i < W * NV; ++i) x[i] = rs * (y[i] - sw - x[i] * swh);
        if (dS) {
            load_row<TX, LPR, W, NV, RUN>(dS + row * c, lane, c, y);
#pragma unroll
            for (int i = 0; i < W * NV; ++i) x[i] += y[i];
        }
        store_row<TX, LPR, W, NV, RUN>(dX + row * c, lane, c, x);
    }
    if (!part) return;
    constexpr int WIDE = LPR * W * NV;                         // channels of a group, those past the row among them
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const int e = channel<LPR, W, RUN>(lane, v, j);
            sums[group * WIDE + e] = dg[W * v + j];
            sums[(GROUPS + group) * WIDE + e] = db[W * v + j];
        }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * c; i += THREADS) {
        const int k = i / c, e = i - k * c;
        float t = 0.f;
        for (int q = 0; q < GROUPS; ++q) t += sums[(k * GROUPS + q) * WIDE + e];
        part[(int64_t)blockIdx.x * 2 * c + i] = t;
    }
}

// dgamma, dbeta from the workgroups' sums, always in the same order: COLS columns by interleaved chains.  4 columns where there
// are few, or a handful of workgroups adds up everything (50 channels, 990 parts: 6.4 -> 5.0 us).
template <int COLS> __global__ __launch_bounds__(THREADS) void layernorm_sum_kernel(const float *part, float *dgamma, float *dbeta, int blocks, int c)
{
    constexpr int CHAINS = THREADS / COLS;
    __shared__ float lds[CHAINS][COLS + 1];
    const int x = threadIdx.x % COLS, col = blockIdx.x * COLS + x, chain = threadIdx.x / COLS;
    float t = 0.f;
    if (col < 2 * c)
#pragma unroll 8
        for (int b = chain; b < blocks; b += CHAINS) t += part[(int64_t)b * 2 * c + col];
    lds[chain][x] = t;
    __syncthreads();
    if (chain == 0 && col < 2 * c) {
        t = 0.f;
#pragma unroll
        for (int k = 0; k < CHAINS; ++k) t += lds[k][x];
        (col < c ? dgamma : dbeta)[col < c ? col : col - c] = t;
    }
}

}  // namespace norm
}  // namespace hch
