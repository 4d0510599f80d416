// Rotary positions with three axes.  Channels (2p, 2p+1) of a head are turned by the angle
//     scale * coordinate(axis of p) * base^(-j / pairs of that axis),   j = p's place among its axis' pairs;
// the gradient turns back.  Heads beyond `rot` and pairs beyond the three sections go through unturned
// (converted, where the two types differ).
// One thread holds PAIRS neighbouring pairs of one row for a run of heads: the angle does not depend on the
// head, so its sine and cosine are computed once per run.  The angle is formed in units of a half turn and
// reduced in 64 bits, since coordinates go up to 32768 and beyond: a product in 32 bits is off by 2e-3 there.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace hch {
namespace rope {

constexpr int MAX_PAIRS = 128;

struct Table {                            // of a head's pairs
    double turns[MAX_PAIRS];              // half turns per unit of the coordinate, sign included
    uint8_t axis[MAX_PAIRS];
};

template <typename T, int N> struct VecN { typedef T type __attribute__((ext_vector_type(N))); };

// items = n rows * (head_dim / (2 PAIRS)) pieces * runs of `per` heads, row by row
template <typename TX, typename TY, int PAIRS>
__global__ __launch_bounds__(256) void rope_kernel(const TX *X, int64_t ld_x, TY *Y, int64_t ld_y, const int32_t *coords, int64_t n,
                                                   int heads, int rot, int head_dim, int pairs, int runs, int per, Table table)
{
    typedef typename VecN<TX, 2 * PAIRS>::type VX;
    typedef typename VecN<TY, 2 * PAIRS>::type VY;
    const int pieces = head_dim / (2 * PAIRS), width = pieces * runs;
    const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x, row = item / width;
    if (row >= n) return;
    const int rest = (int)(item - row * width), run = rest / pieces, p0 = (rest - run * pieces) * PAIRS;
    const int first = run * per, last = min(first + per, heads);
    float co[PAIRS], si[PAIRS];
#pragma unroll
    for (int k = 0; k < PAIRS; ++k) {
        co[k] = 1.f;
        si[k] = 0.f;
        if (first < rot && p0 + k < pairs) {
            const double t = (double)coords[row * 3 + table.axis[p0 + k]] * table.turns[p0 + k];
            sincospif((float)(t - 2.0 * rint(0.5 * t)), &si[k], &co[k]);
        }
    }
    const TX *x = X + row * ld_x + 2 * p0;
    TY *y = Y + row * ld_y + 2 * p0;
#pragma unroll 4
    for (int h = first; h < last; ++h) {
        VX a;
        if constexpr (PAIRS > 1) a = *(const VX *)(x + (int64_t)h * head_dim);
        else { a[0] = x[(int64_t)h * head_dim]; a[1] = x[(int64_t)h * head_dim + 1]; }
        VY b;
#pragma unroll
        for (int k = 0; k < PAIRS; ++k) {
            const float u = (float)a[2 * k], w = (float)a[2 * k + 1];
            const float c = h < rot ? co[k] : 1.f, s = h < rot ? si[k] : 0.f;
            // (an unturned element keeps its bits: no 0 * infinity)
            const bool turned = h < rot && p0 + k < pairs;
            b[2 * k] = (TY)(turned ? u * c - w * s : u);
            b[2 * k + 1] = (TY)(turned ? u * s + w * c : w);
        }
        if constexpr (PAIRS > 1) *(VY *)(y + (int64_t)h * head_dim) = b;
        else { y[(int64_t)h * head_dim] = b[0]; y[(int64_t)h * head_dim + 1] = b[1]; }
    }
}

}  // namespace rope
}  // namespace hch
