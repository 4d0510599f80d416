// Embedding of a label per voxel, y_i = scale T[id_i] (0 where id_i is outside [0, vocab)), and the gradient of its table,
// dT[v] = scale times the sum of dy_i over the rows with id_i = v.
// Forward: rows of the table are read where they lie in cache and written in the order of memory; bound by the rows written: 609323
// rows of 64 from 4096 labels, fp32 to bf16: 16 us, 5.1 TB/s.
// Gradient: no atomics on the table, whose order would change the bits from run to run.  Rows are sorted by label (stable, by
// digits of 6 to 9 bits, as many as the table's size needs), a group of lanes adds up to 16 rows of that order, a workgroup joins its
// groups' runs, and a last launch those that go over several workgroups.  So up to there the work is spread by rows, whatever
// labels they have; but the parts of one label's run are added up by one workgroup, which tells where a run has hundreds of them: 609323 rows of 64, bf16,
// of one label 38 us, of 4096 labels 50; 152343 of 256, fp32, 81 and 57; 40000 of 1030, bf16, 147 and 56.  Sums are fp32: of 16 rows, by trees over a
// workgroup's rows, and over workgroups by chains in blocks of 64 and a tree over the chains.
// 609323 rows of 64, bf16, 32768 labels: 56 us: two passes of the sort 33, the rows 24 (18 at a copy's rate: they are read 128 bytes here and
// there, and the table is cleared first), the join 5.  63331 rows of 50, fp32, 50 labels: 17 us, four launches of 3 to 7 us that wait for memory, not for its
// rate (2.6).  Tried and not kept: sums of a small table's labels in LDS, a thread's own by LDS additions, which take 200 cycles a row (609323
// rows of 64, 50 labels 204 us, so 52).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

#include "norm.hip.hpp"
#include "qknorm.hip.hpp"

namespace hch {
namespace embed {

constexpr int THREADS = 256, AT_ONCE = 4;
constexpr int LEAST = 6, MOST = 9;         // bits of a digit
constexpr int SORT = 1024;                 // threads of the sort's kernels
constexpr int JOIN = 256;                  // threads that join a run's parts
using qknorm::Piece;

// W: neighbours that a thread moves; a workgroup has THREADS * AT_ONCE of them at a time, in the order of memory
template <typename TT, typename TY, int W>
__global__ __launch_bounds__(THREADS) void embed_fwd_kernel(const TT *table, const int32_t *ids, TY *Y, int64_t ld_y, int64_t n, int c, int vocab,
                                                            float scale)
{
    const int pieces = c / W;
    const int64_t all = n * pieces;
    for (int64_t u0 = (int64_t)blockIdx.x * (THREADS * AT_ONCE); u0 < all; u0 += (int64_t)gridDim.x * (THREADS * AT_ONCE)) {
        const int64_t row0 = u0 / pieces;
        const uint32_t rest = (uint32_t)(u0 - row0 * pieces);
        const int here = (int)min((int64_t)(THREADS * AT_ONCE), all - u0);
        int64_t row[AT_ONCE];
        int at[AT_ONCE], id[AT_ONCE];
        Piece<TT, W, W> a[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int k = i * THREADS + threadIdx.x;
            const uint32_t down = (rest + k) / (uint32_t)pieces;
            row[i] = row0 + down;
            at[i] = (int)(rest + k - down * pieces) * W;
            id[i] = k < here ? ids[row[i]] : -1;
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) a[i].load(table + (int64_t)id[i] * c + at[i], (uint32_t)id[i] < (uint32_t)vocab ? W : 0);
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            if (i * THREADS + (int)threadIdx.x >= here) continue;
            Piece<TY, W, W> b;
#pragma unroll
            for (int j = 0; j < W; ++j) b.set(j, (uint32_t)id[i] < (uint32_t)vocab ? a[i].get(j) * scale : 0.f);
            b.store(Y + row[i] * ld_y + at[i], W);
        }
    }
}

// The same where a row is not in pieces of 8 bytes but all rows lie one behind the other: a thread has EIGHT elements of that, which may go on in the next
// row (c >= EIGHT), reads the table RUN at a time and writes 16 bytes.
template <typename TT, typename TY, int RUN>
__global__ __launch_bounds__(THREADS) void embed_fwd_flat_kernel(const TT *table, const int32_t *ids, TY *Y, int64_t n, int c, int vocab, float scale)
{
    constexpr int EIGHT = 8, PIECES = 2;
    typedef TT V __attribute__((ext_vector_type(RUN)));
    const int64_t all = n * c;
    constexpr int TILE = THREADS * EIGHT * PIECES;
    for (int64_t t0 = (int64_t)blockIdx.x * TILE; t0 < all; t0 += (int64_t)gridDim.x * TILE) {
        const int64_t row0 = t0 / c;
        const uint32_t rest = (uint32_t)(t0 - row0 * c);
        const int here = (int)min((int64_t)TILE, all - t0);
        V a[PIECES][EIGHT / RUN];
        bool there[PIECES][2];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int k = (i * THREADS + threadIdx.x) * EIGHT;
            const uint32_t down = (rest + k) / (uint32_t)c;
            const int at = (int)(rest + k - down * c);
            const int64_t row = row0 + down;
            const int32_t first = k < here ? ids[row] : -1, second = k < here && row + 1 < n ? ids[row + 1] : -1;
            there[i][0] = (uint32_t)first < (uint32_t)vocab;
            there[i][1] = (uint32_t)second < (uint32_t)vocab;
            const TT *const p = table + (int64_t)first * c + at, *const q = table + (int64_t)second * c + at - c;
#pragma unroll
            for (int j = 0; j < EIGHT / RUN; ++j) {
                const bool next = at + j * RUN >= c;
                a[i][j] = V{};
                if (there[i][next ? 1 : 0]) a[i][j] = *(const V *)((next ? q : p) + j * RUN);
            }
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int k = (i * THREADS + threadIdx.x) * EIGHT;
            if (k >= here) continue;
            Piece<TY, EIGHT, EIGHT> b;
#pragma unroll
            for (int j = 0; j < EIGHT; ++j) b.set(j, (float)a[i][j / RUN][j % RUN] * scale);
            if (here - k >= EIGHT) b.store(Y + t0 + k, EIGHT);
            else
                for (int j = 0; j < EIGHT; ++j) if (j < here - k) Y[t0 + k + j] = b.v[j / Piece<TY, EIGHT, EIGHT>::N][j % Piece<TY, EIGHT, EIGHT>::N];
        }
    }
}

// ---- sort ----

// What a pass of the sort reads and writes.  Rows go with their labels as pairs; the first pass takes the ids themselves and leaves out those
// outside the table.
struct Pass {
    const int32_t *ids;                    // of the first pass; null later
    const int2 *in;                        // (label, row) of the later ones
    int2 *out;
    int32_t *count;                        // [tiles][1 << BITS], of each tile's rows
    int32_t *total;                        // [1 << BITS], null where a tile's workgroup adds up the tiles' counts itself; else those are
    int32_t *left;                         // the counts of the tiles before.  [1] rows in the sort, written by the first pass
    int64_t n;
    int vocab, tiles, shift;
};

__device__ __forceinline__ bool key_of(const Pass &P, int64_t i, int64_t n, int2 &pair)
{
    pair = make_int2(0, (int)i);
    if (i >= n) return false;
    if (!P.ids) {
        pair = P.in[i];
        return true;
    }
    pair.x = P.ids[i];
    return (uint32_t)pair.x < (uint32_t)P.vocab;
}

// the table's gradient: 0 until a run of rows writes a label's
__device__ __forceinline__ void clear(float *dT, int64_t words, int64_t thread, int64_t threads)
{
    for (int64_t i = thread; i < words; i += threads) dT[i] = 0.f;
}
__global__ __launch_bounds__(THREADS) void embed_clear_kernel(float *dT, int64_t words)
{
    clear(dT, words, (int64_t)blockIdx.x * THREADS + threadIdx.x, (int64_t)gridDim.x * THREADS);
}

// how many of a tile's rows have each digit; workgroups behind the tiles clear the gradient
template <int ITEMS, int BITS> __global__ __launch_bounds__(SORT) void embed_count_kernel(Pass P, float *dT, int64_t words)
{
    constexpr int DIGITS = 1 << BITS;
    __shared__ int32_t count[DIGITS];
    if ((int)blockIdx.x >= P.tiles) {
        clear(dT, words, (int64_t)(blockIdx.x - P.tiles) * SORT + threadIdx.x, (int64_t)(gridDim.x - P.tiles) * SORT);
        return;
    }
    const int64_t n = P.ids ? P.n : *P.left, first = (int64_t)blockIdx.x * (SORT * ITEMS);
    if (threadIdx.x < DIGITS) count[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < ITEMS; ++k) {
        int2 pair;
        if (key_of(P, first + k * SORT + threadIdx.x, n, pair)) atomicAdd(&count[pair.x >> P.shift & (DIGITS - 1)], 1);
    }
    __syncthreads();
    if (threadIdx.x < DIGITS) P.count[(int64_t)blockIdx.x * DIGITS + threadIdx.x] = count[threadIdx.x];
}

// counts of the tiles before each, and totals, where tiles are many: 16 digits a workgroup, 64 chains of tiles
template <int BITS> __global__ __launch_bounds__(SORT) void embed_scan_kernel(Pass P)
{
    constexpr int CHAINS = SORT / 16;
    __shared__ int32_t sums[CHAINS][16];
    const int x = threadIdx.x % 16, digit = blockIdx.x * 16 + x, chain = threadIdx.x / 16, each = (P.tiles + CHAINS - 1) / CHAINS;
    const int first = chain * each, last = min(first + each, P.tiles);
    int32_t t = 0;
#pragma unroll 8
    for (int i = first; i < last; ++i) t += P.count[((int64_t)i << BITS) + digit];
    sums[chain][x] = t;
    __syncthreads();
    int32_t before = 0, all = 0;
    for (int k = 0; k < CHAINS; ++k) {
        before += k < chain ? sums[k][x] : 0;
        all += sums[k][x];
    }
    for (int i = first; i < last; ++i) {
        const int32_t here = P.count[((int64_t)i << BITS) + digit];
        P.count[((int64_t)i << BITS) + digit] = before;
        before += here;
    }
    if (chain == 0) P.total[digit] = all;
}

// lanes of the wavefront that have this lane's digit, among those that have one
template <int BITS> __device__ __forceinline__ uint64_t same_digit(bool live, int digit)
{
    const uint64_t all = __ballot(live);
    uint32_t low = (uint32_t)all, high = (uint32_t)(all >> 32);
#pragma unroll
    for (int b = 0; b < BITS; ++b) {
        const uint64_t with = __ballot(digit >> b & 1);
        const uint32_t mine = (uint32_t)__builtin_amdgcn_sbfe(digit, b, 1);           // all ones where this lane has the bit
        low &= ~((uint32_t)with ^ mine);
        high &= ~((uint32_t)(with >> 32) ^ mine);
    }
    return (uint64_t)high << 32 | low;
}

// A tile's rows to their places by a digit, in the order in which they are.  One tile alone (P.tiles = 1): all `passes` in one launch, the
// rows by turns in P.out and `other`, workgroups from 1 on clear the gradient.
template <int ITEMS, int BITS> __global__ __launch_bounds__(SORT) void embed_scatter_kernel(Pass P, int passes, int2 *other, float *dT, int64_t words)
{
    constexpr int WAVES = SORT / 64, DIGITS = 1 << BITS;
    __shared__ int32_t before[WAVES][DIGITS], part[DIGITS / 64];
    // a row of counts is `ACROSS` threads wide, and there are PARTS sums of them: of a wavefront each, or of two
    constexpr int ACROSS = DIGITS / 4, CHAINS = SORT / ACROSS, PARTS = ACROSS > 64 ? CHAINS : WAVES;
    __shared__ int4 ahead_of[PARTS * ACROSS], all_of[PARTS * ACROSS];
    const bool alone = P.tiles == 1;
    if (alone && blockIdx.x > 0) {
        clear(dT, words, (int64_t)(blockIdx.x - 1) * SORT + threadIdx.x, (int64_t)(gridDim.x - 1) * SORT);
        return;
    }
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, tile = blockIdx.x;
    for (int pass = 0; pass < passes; ++pass) {
        const int64_t n = P.ids ? P.n : *P.left, first = (int64_t)tile * (SORT * ITEMS) + wave * (64 * ITEMS) + lane;
        int2 pair[ITEMS];
        int32_t rank[ITEMS];
        bool live[ITEMS];
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) live[k] = key_of(P, first + k * 64, n, pair[k]);
        if (!alone) {                                       // the digits' rows in the tiles before this one, and in all
            const int x = threadIdx.x % ACROSS, chain = threadIdx.x / ACROSS;
            const int4 *count = (const int4 *)P.count + x;
            int4 a = make_int4(0, 0, 0, 0), t = a;
            auto add = [](int4 &to, const int4 &c, bool on) {
                to.x += on ? c.x : 0;
                to.y += on ? c.y : 0;
                to.z += on ? c.z : 0;
                to.w += on ? c.w : 0;
            };
            if (P.total) {
                if (chain == 0) {
                    a = count[(int64_t)tile * ACROSS];
                    t = ((const int4 *)P.total)[x];
                }
            } else {
#pragma unroll 8
                for (int i = chain; i < P.tiles; i += CHAINS) {
                    const int4 c = count[(int64_t)i * ACROSS];
                    add(a, c, i < tile);
                    add(t, c, true);
                }
            }
#pragma unroll
            for (int d = 32; d >= ACROSS; d /= 2) {         // chains of one wavefront
                auto other = [&](const int4 &v) { return make_int4(__shfl_xor(v.x, d), __shfl_xor(v.y, d), __shfl_xor(v.z, d), __shfl_xor(v.w, d)); };
                add(a, other(a), true);
                add(t, other(t), true);
            }
            const int at = ACROSS > 64 ? threadIdx.x : wave * ACROSS + lane;
            if (ACROSS > 64 || lane < ACROSS) {
                ahead_of[at] = a;
                all_of[at] = t;
            }
        }
        #pragma unroll
        for (int i = threadIdx.x; i < WAVES * DIGITS; i += SORT) before[i / DIGITS][i % DIGITS] = 0;
        __syncthreads();
        // rank among the wavefront's rows of the same digit, in their order
#pragma unroll
        for (int k = 0; k < ITEMS; ++k) {
            const int digit = pair[k].x >> P.shift & (DIGITS - 1);
            const uint64_t same = same_digit<BITS>(live[k], digit);
            const int ahead = __builtin_amdgcn_mbcnt_hi((uint32_t)(same >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)same, 0));
            rank[k] = live[k] ? before[wave][digit] + ahead : 0;
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            if (live[k] && ahead == 0) before[wave][digit] = rank[k] + __popcll(same);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        }
        __syncthreads();
        // a digit's first place: of a thread of the first wavefronts each, by a sum over the digits before
        int32_t at = 0, t = 0, s = 0;
        if (threadIdx.x < DIGITS) {
            if (alone)
                for (int w = 0; w < WAVES; ++w) t += before[w][threadIdx.x];
            else
#pragma unroll
                for (int k = 0; k < PARTS; ++k) {
                    at += ((const int32_t *)ahead_of)[k * DIGITS + threadIdx.x];
                    t += ((const int32_t *)all_of)[k * DIGITS + threadIdx.x];
                }
            s = t;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int32_t u = __shfl_up(s, d);
                s += lane >= d ? u : 0;
            }
            if (lane == 63) part[wave] = s;
        }
        __syncthreads();
        if (threadIdx.x < DIGITS) {
            at += s - t;
            for (int w = 0; w < wave; ++w) at += part[w];
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const int32_t here = before[w][threadIdx.x];
                before[w][threadIdx.x] = at;
                at += here;
            }
        }
        if (P.ids && tile == 0 && threadIdx.x == 0) {
            int32_t all = 0;
            for (int w = 0; w < DIGITS / 64; ++w) all += part[w];
            *P.left = all;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < ITEMS; ++k)
            if (live[k]) P.out[before[wave][pair[k].x >> P.shift & (DIGITS - 1)] + rank[k]] = pair[k];
        if (pass + 1 == passes) break;
        __syncthreads();                                    // this workgroup's rows are in P.out
        int2 *const to = other;
        other = P.out;
        P.in = P.out;
        P.out = to;
        P.ids = nullptr;
        P.shift += BITS;
    }
}

// ---- sums over runs of equal labels in the sorted order ----

struct Runs {
    const int2 *pairs;
    const int32_t *left;
    int32_t *start, *ends;                 // [vocab] the tile in which a label's run begins; [tiles] the run of the tile's first row comes from the tile before
    float *part;                           // and ends here.  [tiles][2][c]: the sum of that run's rows in the tile; of the run that goes on in the next tile,
};                                         // where it begins in this one

template <typename T, int W, int RUN> struct Raw {        // a lane's channels as memory holds them
    typedef T type __attribute__((ext_vector_type(RUN)));
    type v[W / RUN];
};

// rows that a group of LPR lanes adds up: 16, fewer where groups are many, so that a workgroup has 1024 at most (98963 rows of 4 channels, 4178 labels, the whole
// gradient: a lane a row, four rows each, 24.4 us; four lanes, of which three have nothing, 16 rows each, 26.5)
constexpr int sub(int lpr) { return lpr >= 4 ? 16 : 4 * lpr; }

// A workgroup has a tile of GROUPS * SUB rows of the sorted order, LPR * W channels of them (blockIdx.y); a group of LPR lanes adds up SUB rows, all
// of them on their way at once.  A run that lies within a group's rows goes to the table.  The others: each group has a
// part of the run that it is handed (0 if there is none), and adds the parts of the groups behind it as far as that run goes on, by a
// scan over the wavefront's groups and over the wavefronts; the group in which a run begins adds that to its own part, and
// writes it to the table, or to R.part if it goes on in another tile.
template <typename TY, int LPR, int W, int RUN>
__global__ __launch_bounds__(THREADS) void embed_sum_kernel(Runs R, const TY *dY, int64_t ld_dy, float *dT, int c, float scale)
{
    constexpr int SUB = sub(LPR), GROUPS = THREADS / LPR, ROWS = GROUPS * SUB, WIDE = LPR * W, WAVES = THREADS / 64;
    __shared__ int2 pairs[ROWS + 2];                        // from the row before the tile to the one behind it
    __shared__ float handed[WAVES][WIDE];                   // what a wavefront's first group is handed and the groups behind it
    __shared__ int through[WAVES];                          // all rows of a wavefront are one run, from before it to behind it
    const int lane = threadIdx.x % LPR, group = threadIdx.x / LPR, wave = threadIdx.x / 64, in_wave = threadIdx.x & 63;
    const int64_t t0 = (int64_t)blockIdx.x * ROWS;
    constexpr int EACH = (ROWS + 1) / THREADS + 1;
    int2 read[EACH];                                        // before it is known how many there are: the workspace goes on behind them
#pragma unroll
    for (int k = 0; k < EACH; ++k) read[k] = R.pairs[max((int64_t)0, t0 + k * THREADS + (int)threadIdx.x - 1)];
    const int64_t m = *R.left;
    if (t0 >= m) return;
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
        const int i = k * THREADS + threadIdx.x;
        const int64_t p = t0 + i - 1;
        if (i < ROWS + 2) pairs[i] = p >= 0 && p < m ? read[k] : make_int2(-1, 0);
    }
    __syncthreads();
    const int2 *const mine = pairs + 1 + group * SUB;
    const int col0 = blockIdx.y * WIDE, width = c - col0;
    const bool notes = lane == 0 && blockIdx.y == 0;
    dY += col0;
    float *const out = dT + col0;
    Raw<TY, W, RUN> x[SUB];
#pragma unroll
    for (int k = 0; k < SUB; ++k) {
        const int2 p = mine[k];
#pragma unroll
        for (int i = 0; i < W / RUN; ++i) {
            const int e = norm::channel<LPR, W, RUN>(lane, 0, i * RUN);
            x[k].v[i] = typename Raw<TY, W, RUN>::type{};
            if (p.x >= 0 && e < width) x[k].v[i] = *(const typename Raw<TY, W, RUN>::type *)(dY + (int64_t)p.y * ld_dy + e);
        }
    }
    float acc[W], first[W];                                 // of the run at hand; of the one that the group is handed
#pragma unroll
    for (int j = 0; j < W; ++j) acc[j] = first[j] = 0.f;
    auto to_table = [&](int32_t label) {
#pragma unroll
        for (int j = 0; j < W; ++j) acc[j] *= scale;
        norm::store_row<float, LPR, W, 1, RUN>(out + (int64_t)label * c, lane, width, acc);
    };
    auto to_part = [&](int which, const float (&v)[W]) { norm::store_row<float, LPR, W, 1, RUN>(R.part + ((int64_t)blockIdx.x * 2 + which) * c + col0, lane, width, v); };
    int32_t label[SUB + 1];
#pragma unroll
    for (int k = 0; k <= SUB; ++k) label[k] = mine[k].x;
    const int32_t head = label[0], last = label[SUB - 1];
    const bool enters = head >= 0 && mine[-1].x == head, leaves = last >= 0 && label[SUB] == last;
    bool brought = enters;
#pragma unroll
    for (int k = 0; k < SUB; ++k) {
        if (label[k] < 0) continue;
#pragma unroll
        for (int j = 0; j < W; ++j) acc[j] += (float)x[k].v[j / RUN][j % RUN];
        if (label[k + 1] == label[k]) continue;               // at k = SUB - 1, what is handed on stays in acc
        if (brought) {
#pragma unroll
            for (int j = 0; j < W; ++j) first[j] = acc[j];
        } else to_table(label[k]);
        brought = false;
#pragma unroll
        for (int j = 0; j < W; ++j) acc[j] = 0.f;
    }
    const bool whole = enters && leaves && head == last;    // one run, handed on as a whole
    if (whole) {
#pragma unroll
        for (int j = 0; j < W; ++j) {
            first[j] = acc[j];
            acc[j] = 0.f;
        }
    }
    // first = its own + those of the groups behind, as far as they are handed on
    int on = whole;
#pragma unroll
    for (int d = LPR; d < 64; d *= 2) {
        const int on_there = __shfl_down(on, d);
        const bool there = in_wave + d < 64;
#pragma unroll
        for (int j = 0; j < W; ++j) {
            const float t = __shfl_down(first[j], d);
            first[j] += on && there ? t : 0.f;
        }
        on = there ? on && on_there : on;
    }
    if (in_wave < LPR) {
#pragma unroll
        for (int j = 0; j < W; ++j) handed[wave][norm::channel<LPR, W, RUN>(lane, 0, j)] = first[j];
        if (lane == 0) through[wave] = on;
    }
    __syncthreads();
    float behind[W];                                        // of the wavefronts behind this one
#pragma unroll
    for (int j = 0; j < W; ++j) behind[j] = 0.f;
#pragma unroll
    for (int w = WAVES - 1; w > 0; --w)
        if (w > wave) {
            const bool goes_on = through[w];
#pragma unroll
            for (int j = 0; j < W; ++j) {
                const float t = handed[w][norm::channel<LPR, W, RUN>(lane, 0, j)];
                behind[j] = goes_on ? t + behind[j] : t;
            }
        }
    const int32_t end = pairs[ROWS].x, next = pairs[ROWS + 1].x;
    // the group behind, with what is behind its wavefront if that is reached
#pragma unroll
    for (int j = 0; j < W; ++j) {
        first[j] += on ? behind[j] : 0.f;                   // `on`: from here to the wavefront's end
        float t = LPR < 64 ? __shfl_down(first[j], LPR) : 0.f;
        if (in_wave + LPR >= 64) t = behind[j];
        acc[j] += t;
    }
    if (group == 0) {
        if (enters) to_part(0, first);
        if (notes) R.ends[blockIdx.x] = enters && !(end == head && next == head);
    }
    if (leaves && !whole) {
        if (end != last || next != last) to_table(last);
        else {
            to_part(1, acc);
            if (notes) R.start[last] = (int32_t)blockIdx.x;
        }
    }
}

// Runs that go over several tiles: the tile in which one ends adds up its parts, in the tiles' order by as many chains as a workgroup has room
// for and a tree over them.  `lanes` threads have a row's pieces of N channels.  A chain's parts are added up by BLOCK, and those sums behind each other:
// what additions round away has one sign where rows are alike, and grows with their number (200001 like rows of 1031, fp32, one label, 3126 parts in a
// chain: off by up to 4.6e-5 part by part, 1.6e-6 so).  AHEAD parts are on their way at once (one label, 40000 rows of 1030, bf16: 148 us, part by part 149;
// 152343 of 256, fp32: 81 and 79).
template <int N> __global__ __launch_bounds__(JOIN) void embed_join_kernel(Runs R, float *dT, int c, int rows, float scale, int lanes)
{
    typedef float V __attribute__((ext_vector_type(N)));
    constexpr int BLOCK = 64, AHEAD = 8;
    __shared__ V lds[JOIN];
    const int64_t tile = blockIdx.x;
    const int32_t label = R.pairs[tile * rows].x, ends = R.ends[tile];        // read at once; they say nothing behind the last row
    if (tile * rows >= *R.left || !ends) return;
    const int64_t first = R.start[label], count = tile - first + 1;
    const int piece0 = threadIdx.x % lanes, group = threadIdx.x / lanes, groups = JOIN / lanes, pieces = c / N;
    for (int piece1 = 0; piece1 < pieces; piece1 += lanes) {
        const int piece = piece1 + piece0;
        V t = {};
        if (piece < pieces) {
            auto part = [&](int64_t i) { return *(const V *)(R.part + ((first + i) * 2 + (i == 0)) * c + piece * N); };
            int64_t i = group;
            while (i + (int64_t)(BLOCK - 1) * groups < count) {
                V b = {};
                for (int k = 0; k < BLOCK; k += AHEAD, i += AHEAD * groups) {
                    V v[AHEAD];
#pragma unroll
                    for (int j = 0; j < AHEAD; ++j) v[j] = part(i + j * groups);
#pragma unroll
                    for (int j = 0; j < AHEAD; ++j) b += v[j];
                }
                t += b;
            }
            V b = {};
#pragma unroll 8
            for (; i < count; i += groups) b += part(i);
            t += b;
        }
        lds[threadIdx.x] = t;
        __syncthreads();
        int half = groups / 2;
        while (half >= count && half > 0) half /= 2;        // chains without a part
        for (; half > 0; half /= 2) {
            if (group < half) lds[threadIdx.x] += lds[threadIdx.x + half * lanes];
            __syncthreads();
        }
        if (group == 0 && piece < pieces) *(V *)(dT + (int64_t)label * c + piece * N) = lds[threadIdx.x] * scale;
        __syncthreads();
    }
}

}  // namespace embed
}  // namespace hch
