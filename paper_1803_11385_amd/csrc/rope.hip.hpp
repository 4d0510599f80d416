// Rotary positions with three axes.  Channels (2p, 2p+1) of a head are turned by the angle
//     scale * coordinate(axis of p) * base^(-j / pairs of that axis),   j = p's place among its axis' pairs;
// the gradient turns back.  Heads beyond `rot` and pairs beyond the three sections go through unturned
// (converted, where the two types differ).
// Bound by memory: each element is read and written once.  A workgroup has a few rows; its sines and cosines, which do not
// depend on the head, are computed once, into LDS, while the rows' first pieces are on their way.  A thread keeps its
// place in the row and walks down the rows, so rows are read and written in runs (152331 rows of 12 heads of 32, bf16, from
// memory: 63 us with a thread for 4 channels of all heads, whose reads are 64 bytes here and there, 52 so).  The angle is
// formed in units of a half turn and reduced in 64 bits, since coordinates go up to 32768 and beyond: a product in 32
// bits is off by 2e-3 there.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace hch {
namespace rope {

constexpr int MAX_PAIRS = 128, THREADS = 256, AT_ONCE = 4, ENTRIES = 2048;

struct Table {                            // of a head's pairs
    double turns[MAX_PAIRS];              // half turns per unit of the coordinate, sign included
    uint8_t axis[MAX_PAIRS];
};

template <typename T, int N> struct VecN { typedef T type __attribute__((ext_vector_type(N))); };

// blockIdx.x: `rows` rows, blockIdx.y: THREADS pieces of W channels of them; `wide` threads side by side, the others below them
template <typename TX, typename TY, int W, bool VEC>
__global__ __launch_bounds__(THREADS) void rope_kernel(const TX *X, int64_t ld_x, TY *Y, int64_t ld_y, const int32_t *coords, int64_t n,
                                                       int pieces, int wide, int rows, int rot, int head_dim, int pairs, Table table)
{
    typedef typename VecN<TX, W>::type VX;
    typedef typename VecN<TY, W>::type VY;
    __shared__ float2 turn[ENTRIES];      // [rows][pairs] cosine and sine
    const int64_t row0 = (int64_t)blockIdx.x * rows;
    const int count = (int)min((int64_t)rows, n - row0);
    const int below = threadIdx.x / wide, step = THREADS / wide, piece = blockIdx.y * THREADS + threadIdx.x - below * wide;
    const bool some = below < step && piece < pieces;
    const int e = piece * W, head = e / head_dim, p0 = (e - head * head_dim) / 2;
    const TX *x = X + row0 * ld_x + e;
    TY *y = Y + row0 * ld_y + e;

    VX a[AT_ONCE];
    auto load = [&](int first) {
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int r = first + i * step;
            if (!some || r >= count) continue;
            if constexpr (VEC) a[i] = *(const VX *)(x + r * ld_x);
            else
#pragma unroll
                for (int j = 0; j < W; ++j) a[i][j] = x[r * ld_x + j];
        }
    };
    load(below);
    for (int i = threadIdx.x; i < count * pairs; i += THREADS) {
        const int r = i / pairs, p = i - r * pairs;
        const double t = (double)coords[(row0 + r) * 3 + table.axis[p]] * table.turns[p];
        float2 v;
        sincospif((float)(t - 2.0 * rint(0.5 * t)), &v.y, &v.x);
        turn[i] = v;
    }
    __syncthreads();
    for (int first = below; first < count; first += AT_ONCE * step) {
        if (first != below) load(first);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int r = first + i * step;
            if (!some || r >= count) continue;
            VY b;
#pragma unroll
            for (int k = 0; k < W / 2; ++k) {
                const float u = (float)a[i][2 * k], w = (float)a[i][2 * k + 1];
                float v0 = u, v1 = w;                   // unturned elements keep their bits: no 0 * infinity
                if (head < rot && p0 + k < pairs) {
                    const float2 t = turn[r * pairs + p0 + k];
                    v0 = u * t.x - w * t.y;
                    v1 = u * t.y + w * t.x;
                }
                b[2 * k] = (TY)v0;
                b[2 * k + 1] = (TY)v1;
            }
            if constexpr (VEC) *(VY *)(y + r * ld_y) = b;
            else
#pragma unroll
                for (int j = 0; j < W; ++j) y[r * ld_y + j] = b[j];
        }
    }
}

}  // namespace rope
}  // namespace hch
