// Attention inside the shapes of a ragged batch, forward and backward, on the matrix instructions.
//
//   forward   s_ij = scale q_i.k_j;  o_i = sum_j exp(s_ij - m_i) v_j / l_i with the running maximum m and sum l
//             of the keys seen so far: one pass over the keys, no score goes to memory
//   backward  p_ij = exp(s_ij - lse_i);  D_i = dO_i . o_i;  dS_ij = p_ij (dO_i . v_j - D_i)
//             dV_j = sum_i p_ij dO_i;  dK_j = scale sum_i dS_ij q_i;  dQ_i = scale sum_j dS_ij k_j
//
// All kernels multiply 32 x 32 tiles with the 32x32x16 bf16 instruction.  The scores are always formed so that what stays
// fixed for a wavefront (its queries, or in the pass over keys its keys) is the column, i.e. the lane, and what
// streams past is the row, i.e. the register.  Then
//   * a row's maximum and sum are sums over a lane's own registers and one exchange between the two
//     half-wavefronts, and what scales a query is one number per lane;
//   * the probabilities are already laid out as the right operand of the second product, whose reduction runs
//     over the streamed rows: register r of half h is row 8 (r / 4) + 4 h + r % 4, and the left operand is read
//     in the same order, so nothing is exchanged between the products.
// The streamed tile lies row by row in LDS and serves both: ds_read_b128 for products over the channels (16
// consecutive bytes of a row), for products over the rows the transposing ds_read_b64_tr_b16 (16 lanes give the
// addresses of 4 rows x 16 channels and get 4 rows of one channel each).
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace hch {
namespace attn {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) void lds_void;

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.69314718055994530942f;
constexpr int SRD3 = 0x00020000, OUT = 0x7fffffff;      // raw buffer descriptor; an offset past every buffer

struct Args {
    const void *Q, *K, *V, *O, *dO;
    void *Ow, *dQ, *dK, *dV;               // outputs
    float *lse;                            // [n_q][hq]
    const int32_t *qo, *ko;                // [batch + 1]
    const uint8_t *mask;                   // [n_k] or null
    float *part;                           // [splits][n_q * hq][d] sums of a split over the keys
    float2 *ml;                            // [splits][n_q * hq]    their maximum and sum
    float *delta;                          // [n_q * hq] D
    int64_t nq, nk, ld_q, ld_k, ld_v, ld_o, ld_do, ld_dq, ld_dk, ld_dv;
    int batch, hq, hkv, group, d;
    int slots, splits, run, per_head;      // tiles per head at most, splits over the streamed rows; see work_item
    int vec;                               // everything in 16-byte pieces
    int sorted;                            // units in the order of what streams past them, the longest first; of up to 64 shapes
    float scale, c;                        // c = scale log2(e)
};

// ---------------------------------------------------------------------------------------------
// how operands are multiplied
// ---------------------------------------------------------------------------------------------
// An engine E: T is the type in memory, Part one lane's share of 16 terms of an operand, PLANES the parts a tile has in
// LDS, AHEAD the operands of a product over the channels that are read before the first is multiplied.
//   rows   from a tile: 32 rows, 16 channels
//   cols   from a tile, transposed: 32 channels, 16 rows
//   col    from a product's result: its registers 8 s .. 8 s + 7, 16 streamed rows
//   mul    acc += a b
constexpr int CHUNK = 16;

// A tile's rows lie one after the other, their 16-byte units swapped: unit u of row r at u ^ swap(r), so that neither
// product's reads meet in a bank (LDS has 64 of 4 bytes).  ds_read_b128 of one unit of 32 rows serves 16 lanes a
// clock whose rows differ modulo 16: these have to spread over the 16 units that the banks hold.  The transposing read
// serves 4 rows x 4 neighbouring units a clock: the rows' groups of 4 units have to differ.  (With 16 bytes between the rows
// instead, the second kind took twice (64 channels) to four times (128) as long.)
template <int D> struct Layout {
    static constexpr int STRIDE = 2 * D;
    static __device__ __forceinline__ int swap(int r)
    {
        return (r >> 2 & 3) | (D == 128 ? (r & 3) << 2 : D == 64 ? (r >> 1 & 1) << 2 : 0);
    }
    // offset of this lane's row of 32, unit 16 s + 8 h channels, of a product over the channels: from the s = 0 one
    static __device__ __forceinline__ int row0(int lane) { const int r = lane & 31; return r * STRIDE + (((lane >> 5) ^ swap(r)) << 4); }
    static __device__ __forceinline__ int row(int at, int s)
    {
        constexpr int X = D == 128 ? 7 : D == 64 ? 3 : 1;      // what of s lies within the units that are swapped
        return (at ^ (s & X) << 5) + ((s & ~X) << 5);
    }
    // offset of this lane's address in the transposing read of rows 0 .. 3 and 4 .. 7 (by half), channels 0 .. 31
    static __device__ __forceinline__ int left0(int lane)
    {
        const int r = 4 * (lane >> 5) + ((lane & 15) >> 2), u = 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
        return r * STRIDE + ((u ^ swap(r)) << 4) + 8 * (lane & 1);
    }
    static __device__ __forceinline__ int left(int at, int dt) { return D == 96 ? at + (dt << 6) : at ^ dt << 6; }
};
// 16 streamed rows x 32 channels, transposed: row 4 h + j and 8 + 4 h + j of channel lane % 32
template <int D> __device__ __forceinline__ bf16x8 transposed(const char *rows16, int at)
{
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(s16x4 *)(rows16 + at));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(s16x4 *)(rows16 + 8 * Layout<D>::STRIDE + (at ^ 32)));
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
__device__ __forceinline__ f32x16 mfma16(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }

struct Bf16 {
    typedef __bf16 T;
    static constexpr const char *NAME = "attn::Bf16";
    static constexpr int PLANES = 1, AHEAD = 4;
    typedef bf16x8 Part;
    static __device__ __forceinline__ Part part(const __bf16 (&x)[8]) { return __builtin_bit_cast(bf16x8, x); }
    static __device__ __forceinline__ Part rows(const char *p, int) { return *(const bf16x8 *)p; }
    template <int D> static __device__ __forceinline__ Part cols(const char *rows16, int, int at) { return transposed<D>(rows16, at); }
    static __device__ __forceinline__ Part col(const f32x16 &p, int s)
    {
        Part c;
#pragma unroll
        for (int j = 0; j < 8; ++j) c[j] = (__bf16)p[8 * s + j];
        return c;
    }
    static __device__ __forceinline__ f32x16 mul(const Part &a, const Part &b, f32x16 acc) { return mfma16(a, b, acc); }
    // 16 bytes of memory into a row whose units are swapped by `swap`
    static __device__ __forceinline__ void store(char *row, int, int swap, int piece, u32x4 v) { *(u32x4 *)(row + 16 * (piece ^ swap)) = v; }
};

// fp32 on the bf16 instruction: every number is the sum of three bf16 numbers (8 bits each, so exact), and of the nine
// products of two such sums the six leading ones are taken; what is left out is at most 2^-23 of the
// product.  Six bf16 steps take 6/16 of the time of the fp32 instruction for the same terms.  (Parts of numbers below 2^-110
// are lost one by one as they fall below 2^-133; an infinite operand makes its sums NaN.)
struct Split {
    typedef float T;
    static constexpr const char *NAME = "attn::Split";
    static constexpr int PLANES = 3, AHEAD = 1;
    struct Part { bf16x8 v[3]; };
    static __device__ __forceinline__ uint32_t round2(float a, float b)
    {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
    }
    // two numbers as three packed pairs; both differences are exact
    static __device__ __forceinline__ void cut(float a, float b, uint32_t (&v)[3])
    {
        v[0] = round2(a, b);
        const float ra = a - __uint_as_float(v[0] << 16), rb = b - __uint_as_float(v[0] & 0xffff0000u);
        v[1] = round2(ra, rb);
        v[2] = round2(ra - __uint_as_float(v[1] << 16), rb - __uint_as_float(v[1] & 0xffff0000u));
    }
    static __device__ __forceinline__ Part part(const float (&x)[8])
    {
        u32x4 t[3];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            uint32_t v[3];
            cut(x[2 * j], x[2 * j + 1], v);
#pragma unroll
            for (int k = 0; k < 3; ++k) t[k][j] = v[k];
        }
        Part p;
#pragma unroll
        for (int k = 0; k < 3; ++k) p.v[k] = __builtin_bit_cast(bf16x8, t[k]);
        return p;
    }
    static __device__ __forceinline__ Part rows(const char *p, int plane)
    {
        return Part{{*(const bf16x8 *)p, *(const bf16x8 *)(p + plane), *(const bf16x8 *)(p + 2 * plane)}};
    }
    template <int D> static __device__ __forceinline__ Part cols(const char *rows16, int plane, int at)
    {
        return Part{{transposed<D>(rows16, at), transposed<D>(rows16 + plane, at), transposed<D>(rows16 + 2 * plane, at)}};
    }
    static __device__ __forceinline__ Part col(const f32x16 &p, int s)
    {
        const float x[8] = {p[8 * s], p[8 * s + 1], p[8 * s + 2], p[8 * s + 3], p[8 * s + 4], p[8 * s + 5], p[8 * s + 6], p[8 * s + 7]};
        return part(x);
    }
    static __device__ __forceinline__ f32x16 mul(const Part &a, const Part &b, f32x16 acc)
    {
        constexpr int PA[6] = {2, 0, 1, 1, 0, 0}, PB[6] = {0, 2, 1, 0, 1, 0};      // the smallest first
#pragma unroll
        for (int i = 0; i < 6; ++i) acc = mfma16(a.v[PA[i]], b.v[PB[i]], acc);
        return acc;
    }
    static __device__ __forceinline__ void store(char *row, int plane, int swap, int piece, u32x4 v)
    {
        const f32x4 x = __builtin_bit_cast(f32x4, v);
        uint32_t lo[3], hi[3];
        cut(x[0], x[1], lo);
        cut(x[2], x[3], hi);
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int k = 0; k < 3; ++k) *(u32x2 *)(row + k * plane + 8 * (piece ^ 2 * swap)) = u32x2{lo[k], hi[k]};
    }
};

// the other half-wavefront's value
__device__ __forceinline__ float other_half(float v)
{
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float((threadIdx.x & 32) ? s[0] : s[1]);
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// row of register r of a tile, less the 4 h of the half
__device__ __forceinline__ constexpr int reg_row(int r) { return 8 * (r >> 2) + (r & 3); }

// ---------------------------------------------------------------------------------------------
// work distribution
// ---------------------------------------------------------------------------------------------
// A unit of work is one split of one tile of one key head.  Where what streams past is long, units of a head are ordered by
// shape, the longest first, so that a launch ends with its shortest (46514 voxels in 4 shapes, 4 heads of 128, bf16: 1196 -> 1140
// us; where it is short, finding the order would take longer than it saves); heads alternate.  Workgroups go to the 8 XCDs in turn.  With many units, runs of `run`
// neighbours of a head are kept on one XCD: they read the same keys, from its L2.  With few, one by one (512 of
// dQ, 8 shapes of 2000 rows, 32 channels, fp32: 108 us in runs of 16, 81 so), and all heads of a tile on one XCD, since they share
// lines of memory (8 shapes of 76165 keys, 2 heads of 32, bf16, one query: 47 us apart, 27 together).
struct WorkShape { int run; int64_t per_head, grid; };
inline WorkShape work_shape(int64_t slots, int splits, int heads)
{
    const int64_t each = slots * splits, total = each * heads;
    WorkShape w;
    w.run = total >= 4096 ? 16 : total >= 1024 ? 4 : 1;
    const int whole = w.run == 1 ? 8 : w.run;
    w.per_head = (each + whole - 1) / whole * whole;
    w.grid = (w.per_head * heads + 8 * w.run - 1) / (8 * w.run) * (8 * w.run);
    return w;
}
constexpr int64_t MAX_GRID = 0xffffffffll / 256;         // a launch's work items are counted in 32 bits
inline void set_work(Args &a)
{
    const WorkShape w = work_shape(a.slots, a.splits, a.hkv);
    a.run = w.run;
    a.per_head = (int)w.per_head;
}
inline unsigned work_grid(const Args &a) { return (unsigned)work_shape(a.slots, a.splits, a.hkv).grid; }
struct Work { int head, slot, split; };         // slot beyond the last: nothing to do
__device__ __forceinline__ Work work_of(const Args &a, int id)
{
    int head, unit;
    if (a.run == 1) {
        const int turn = id >> 3;
        head = turn % a.hkv;
        unit = turn / a.hkv * 8 + (id & 7);
    } else {
        const int r = (id >> 3) / a.run * 8 + (id & 7);
        head = r % a.hkv;
        unit = r / a.hkv * a.run + (id >> 3) % a.run;
    }
    const int slot = unit / a.splits;
    return {head, unit < a.per_head ? slot : a.slots, unit - slot * a.splits};
}

// A shape's rows [begin, end) of n, safe whatever the offsets hold.
struct Span { int begin, end; };
__device__ __forceinline__ int clamped(int32_t v, int64_t n) { return (int)max((int64_t)0, min((int64_t)v, n)); }
__device__ __forceinline__ Span span_of(const int32_t *off, int b, int64_t n)
{
    Span s;
    s.begin = __builtin_amdgcn_readfirstlane(clamped(off[b], n));
    s.end = __builtin_amdgcn_readfirstlane(clamped(off[b + 1], n));
    s.end = max(s.end, s.begin);
    return s;
}
// Where a slot's tile lies: its rows are of `own` (rows_each for each of its shape's), what streams past it of `stream`.
struct Place { Span own, stream; int tile; };   // tile < 0: there is none
__device__ __forceinline__ Place place_of(const int32_t *own, int64_t n_own, const int32_t *stream, int64_t n_stream, int batch, bool sorted,
                                          int rows_each, int size, int slot, int lane)
{
    // In the shapes' own order no sum over them is needed: shape b's tiles have the slots from floor(offset_b / size) + b on, which
    // is room enough, as ceil(len / size) <= floor(end / size) - floor(begin / size) + 1.
    auto first = [&](int begin, int b) { return (int)((int64_t)begin * rows_each / size) + b; };
    if (batch <= 64) {                              // a lane per shape
        const int i = min(lane, batch - 1);
        const int o0 = clamped(own[i], n_own), o1 = max(o0, clamped(own[i + 1], n_own));
        const int s0 = clamped(stream[i], n_stream), s1 = max(s0, clamped(stream[i + 1], n_stream));
        const int tiles = lane < batch ? (int)(((int64_t)(o1 - o0) * rows_each + size - 1) / size) : 0, len = s1 - s0;
        int before = first(o0, lane);
        if (sorted) {
            before = 0;
            for (int j = 0; j < batch; ++j) {
                const int tj = __builtin_amdgcn_readlane(tiles, j), lj = __builtin_amdgcn_readlane(len, j);
                if (lj > len || (lj == len && j < lane)) before += tj;
            }
        }
        const uint64_t hit = __ballot(slot >= before && slot - before < tiles);
        if (!hit) return {{0, 0}, {0, 0}, -1};
        const int b = __builtin_ctzll(hit);
        return {{__builtin_amdgcn_readlane(o0, b), __builtin_amdgcn_readlane(o1, b)}, {__builtin_amdgcn_readlane(s0, b), __builtin_amdgcn_readlane(s1, b)},
                slot - __builtin_amdgcn_readlane(before, b)};
    }
    // more: by 64-fold search
    int lo = 0, cnt = batch;
    while (cnt > 1) {
        const int step = (cnt + 63) >> 6, i = lane * step;
        const bool in = i < cnt && first(clamped(own[lo + (i < cnt ? i : 0)], n_own), lo + i) <= slot;
        const int k = max(0, (int)__popcll(__ballot(in)) - 1);
        lo += k * step;
        cnt = min(step, cnt - k * step);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const Span o = span_of(own, lo, n_own);
    const int tile = slot - first(o.begin, lo);
    return {o, span_of(stream, lo, n_stream), tile >= 0 && (int64_t)tile * size < (int64_t)(o.end - o.begin) * rows_each ? tile : -1};
}
inline int64_t slots_of(int64_t n, int rows_each, int size, int batch) { return n * rows_each / size + batch; }

// ---------------------------------------------------------------------------------------------
// tiles
// ---------------------------------------------------------------------------------------------
template <typename E, int D> struct Tile {
    static constexpr int STRIDE = Layout<D>::STRIDE, CHUNKS = D / CHUNK, DT = D / 32;
};

// 16 bytes from element 0 .. of a row, `have` of them there; zeros behind
template <typename T> __device__ __forceinline__ u32x4 load_elements(__amdgpu_buffer_rsrc_t rs, int offset, int have)
{
    u32x4 v;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = __builtin_amdgcn_raw_buffer_load_b32(rs, j < have ? offset + 4 * j : OUT, 0, 0);
    } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, 2 * j < have ? offset + 4 * j : OUT, 0, 0);
            const uint32_t hi = (uint16_t)__builtin_amdgcn_raw_buffer_load_b16(rs, 2 * j + 1 < have ? offset + 4 * j + 2 : OUT, 0, 0);
            v[j] = lo | hi << 16;
        }
    }
    return v;
}

// The part of a tile of ROWS rows that a thread moves from memory to LDS: fixed pieces of 16 bytes.
template <typename E, int D, int ROWS, int THREADS> struct Stage {
    typedef typename E::T T;
    static constexpr int PER_ROW = D * (int)sizeof(T) / 16, PIECES = ROWS * PER_ROW, N = (PIECES + THREADS - 1) / THREADS;
    u32x4 r[N];
    // rows [row0, row0 + ROWS) of a matrix that ends before row `end`; `base`: channel 0 of row 0.  Rows and channels that
    // do not exist come back as zeros, from the bounds of the descriptor.
    __device__ __forceinline__ void load(const T *base, int64_t ld, int row0, int end, int d, bool vec, int tid)
    {
        const int rows = max(0, min(ROWS, end - row0));
        const int bytes = rows ? (int)(((rows - 1) * ld + d) * (int)sizeof(T)) : 0;
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)(base + row0 * ld), 0, bytes, SRD3);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = tid + i * THREADS, row = p / PER_ROW, e = (p - row * PER_ROW) * (16 / (int)sizeof(T));
            const int have = PIECES % THREADS && p >= PIECES ? 0 : d - e;
            const int offset = (int)(row * ld + e) * (int)sizeof(T);
            if (vec) r[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rs, have > 0 ? offset : OUT, 0, 0));
            else r[i] = load_elements<T>(rs, offset, row < rows ? have : 0);
        }
    }
    // rows whose bit of `keep` is clear are written as zeros, unless `all` are to be kept
    template <int W> __device__ __forceinline__ void store(char *tile, int tid, bool all, const uint64_t (&keep)[W])
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int p = tid + i * THREADS, row = p / PER_ROW, col = p - row * PER_ROW;
            if (PIECES % THREADS && p >= PIECES) continue;
            u32x4 v = r[i];
            if (!all && !((W > 1 && row >= 64 ? keep[W - 1] : keep[0]) >> (row & 63) & 1)) v = u32x4{0, 0, 0, 0};
            E::store(tile + row * Tile<E, D>::STRIDE, ROWS * Tile<E, D>::STRIDE, Layout<D>::swap(row), col, v);
        }
    }
    __device__ __forceinline__ void store(char *tile, int tid) { store(tile, tid, true, {0ull}); }
};

// The same without registers, for bf16 in whole pieces: every instruction moves 64 pieces from memory to 1 KB of LDS,
// lane by lane.  As the place in LDS is the lane's, the swap of the units is in the lane's address in memory.
template <int D, int ROWS> struct Direct {
    static constexpr int PER_ROW = D / 8, N = ROWS * PER_ROW / 256;
    static __device__ __forceinline__ void piece(int i, int wave, int lane, int &row, int &e)
    {
        const int p = (wave + 4 * i) * 64 + lane;
        row = p / PER_ROW;
        e = ((p - row * PER_ROW) ^ Layout<D>::swap(row)) * 8;
    }
    static __device__ __forceinline__ void load(const __bf16 *base, int64_t ld, int row0, int end, int d, char *tile, int wave, int lane)
    {
        const int rows = max(0, min(ROWS, end - row0));
        const int bytes = rows ? (int)(((rows - 1) * ld + d) * 2) : 0;
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void *)(base + row0 * ld), 0, bytes, SRD3);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int row, e;
            piece(i, wave, lane, row, e);
            to_lds(rs, e < d ? (int)(row * ld + e) * 2 : OUT, tile + (wave + 4 * i) * 1024);
        }
    }
    // Written out, as the compiler would wait for all of them before the next transposing read of any part of LDS; that
    // they have arrived is waited for in wait().  m0: where in LDS lane 0's piece goes; a reserved register, in which the compiler keeps
    // nothing from one instruction to the next, and which a list of overwritten registers may not name.
    static __device__ __forceinline__ void to_lds(__amdgpu_buffer_rsrc_t rs, int offset, char *to)
    {
        const uint32_t m0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(lds_void *)(void *)to);
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(m0), "v"(offset), "s"(rs) : "memory");
    }
    static __device__ __forceinline__ void clear(char *tile, int wave, int lane, uint64_t keep)
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int row, e;
            piece(i, wave, lane, row, e);
            if (!(keep >> row & 1)) *(u32x4 *)(tile + (wave + 4 * i) * 1024 + 16 * lane) = u32x4{0, 0, 0, 0};
        }
    }
    // this wavefront's loads have arrived
    static __device__ __forceinline__ void wait() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
};

// `count` elements of a row from element e on; zeros where there are none
template <typename T, int N> __device__ __forceinline__ void load_piece(const T *row, int e, bool valid, int d, bool vec, T (&x)[N])
{
    if (valid && vec && e < d) {
#pragma unroll
        for (int i = 0; i < N * (int)sizeof(T) / 16; ++i) __builtin_memcpy((char *)x + 16 * i, (const char *)(row + e) + 16 * i, 16);
    } else
#pragma unroll
        for (int j = 0; j < N; ++j) x[j] = valid && e + j < d ? row[e + j] : (T)0.f;
}

// A wavefront's own 32 rows as an operand of products over the channels: of each chunk the half's share.
template <typename E, int D> struct Own {
    typename E::Part v[Tile<E, D>::CHUNKS];
    __device__ __forceinline__ void load(const typename E::T *row, bool valid, int d, bool vec, int h)
    {
#pragma unroll
        for (int s = 0; s < Tile<E, D>::CHUNKS; ++s) {
            typename E::T x[CHUNK / 2];
            load_piece(row, CHUNK * s + CHUNK / 2 * h, valid, d, vec && d % (CHUNK / 2) == 0, x);
            v[s] = E::part(x);
        }
    }
};

// Nothing but arithmetic other than products moves across: the compiler would read every operand from LDS right before
// the product that takes it, and wait for it.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0x406); }

// out[i] += (rows 32 i .. of the tile) . own, for N runs of 32 rows.  G operands are read before the first product, and as
// many more while those multiply.  full: the last 16 channels are not all zeros; in fp32 their products are left out otherwise
// (8 shapes of 2048, 8 heads of 16 channels: forward 220 -> 207 us, dQ 298 -> 259; of 40: 347 -> 324, 550 -> 517; in bf16 they wait
// for other things.  The pass over the keys leaves none out: 358 -> 336 at 16 channels, but 357 -> 368 at 32 and 718 -> 748 at 64).
template <typename E, int D, int N, int G = E::AHEAD>
__device__ __forceinline__ void products(const char *tile, int plane, const Own<E, D> &own, int lane, bool full, f32x16 (&out)[N])
{
    constexpr int CH = Tile<E, D>::CHUNKS, TOTAL = N * CH;
    const int at = Layout<D>::row0(lane);
    typename E::Part a[2][G];
    auto read = [&](int g) {
#pragma unroll
        for (int i = 0; i < G; ++i)
            if (g * G + i < TOTAL) a[g & 1][i] = E::rows(tile + 32 * ((g * G + i) / CH) * Tile<E, D>::STRIDE + Layout<D>::row(at, (g * G + i) % CH), plane);
    };
    read(0);
#pragma unroll
    for (int g = 0; g * G < TOTAL; ++g) {
        if ((g + 1) * G < TOTAL) read(g + 1);
        keep_order();
#pragma unroll
        for (int i = 0; i < G; ++i)
            if (g * G + i < TOTAL) {
                const int n = (g * G + i) / CH, c = (g * G + i) % CH;
                if (E::PLANES == 3 && c == CH - 1 && !full) continue;
                out[n] = E::mul(a[g & 1][i], own.v[c], out[n]);
            }
        keep_order();
    }
}

// acc[dt] += (rows of a tile, transposed) p, for the channels from `left`'s on, 16 rows at a time.  The first operands are read
// by the constructor, so that they arrive while p is still being made.
template <typename E, int D, int DT, int G = E::PLANES == 1 ? DT : 1> struct Fold {     // G operands read ahead
    typename E::Part a[2][G];
    const char *tile;
    int plane, left;
    __device__ __forceinline__ void read(int g)
    {
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int step = (g * G + i) / DT, dt = (g * G + i) % DT;
            a[g & 1][i] = E::template cols<D>(tile + 16 * step * Tile<E, D>::STRIDE, plane, Layout<D>::left(left, dt));
        }
    }
    __device__ __forceinline__ Fold(const char *t, int pl, int l) : tile(t), plane(pl), left(l)
    {
        read(0);
        keep_order();
    }
    template <int N> __device__ __forceinline__ void run(const f32x16 (&p)[N], f32x16 (&acc)[DT])
    {
        typename E::Part b;
#pragma unroll
        for (int g = 0; g * G < 2 * N * DT; ++g) {
            if ((g + 1) * G < 2 * N * DT) read(g + 1);
            keep_order();
            if (g * G % DT == 0) b = E::col(p[g * G / DT >> 1], g * G / DT & 1);
#pragma unroll
            for (int i = 0; i < G; ++i) acc[(g * G + i) % DT] = E::mul(a[g & 1][i], b, acc[(g * G + i) % DT]);
            keep_order();
        }
    }
};
// this lane's row of a result: channel 32 dt + 8 (r / 4) + 4 h + r % 4
template <typename U, int DT>
__device__ __forceinline__ void store_row(U *row, const f32x16 (&acc)[DT], float f, int d, bool vec, int h)
{
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const int e = 32 * dt + reg_row(r) + 4 * h;
            if (e >= d) continue;
            typedef U U4 __attribute__((ext_vector_type(4)));
            U4 v;
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = (U)(acc[dt][r + j] * f);
            if (vec) *(U4 *)(row + e) = v;
            else
#pragma unroll
                for (int j = 0; j < 4; ++j) if (e + j < d) row[e + j] = v[j];
        }
}

// Whether a key is there and seen: its byte of the mask, 1 without one.
__device__ __forceinline__ int key_byte(const uint8_t *mask, int key, int end) { return key < end ? (mask ? (int)mask[key] : 1) : 0; }

// Sizes of the passes over the keys.  QW wavefronts have rows of their own and KW share a row tile's keys: 4 x 1 (wide)
// where there are rows for every compute unit, 1 x 4 (narrow) where there are few and the keys are most of what there
// is to read or to wait for.  Where four tiles of keys are too much for LDS, two are shared by two wavefronts
// each, DW, which form the same scores and half of the result's channels.
template <typename E, int D, int QW, bool VEC> struct Keys {
    static constexpr int WAVES = 4, THREADS = 64 * WAVES, DW = QW == 1 && E::PLANES == 3 && D > 64 ? 2 : 1, KW = WAVES / QW / DW, BQ = 32 * QW;
    static constexpr int DT = D / 32 / DW;                  // of a wavefront's result
    static constexpr int AHEAD = E::PLANES == 1 && D == 128 ? 2 : E::AHEAD, FOLD = E::PLANES > 1 ? 1 : D == 128 ? 2 : DT;      // of dQ: registers
    static constexpr int BK = QW == 1 ? 32 * KW : E::PLANES == 1 ? 64 : 32, NT = BK / 32 / KW;
    static constexpr int PLANE = BK * Tile<E, D>::STRIDE, TILE = E::PLANES * PLANE;
    static constexpr int BUFFER = 2 * TILE + 4 * BK, BUFFERS = QW == 1 || 2 * BUFFER > 80 * 1024 ? 1 : 2;   // two where two workgroups still share a compute unit
    static constexpr int WORDS = (BK + 63) / 64;
    static constexpr bool DIRECT = VEC && E::PLANES == 1 && QW == 4;   // two buffers, so the loads of the next tile need no registers
    // Workgroups that share a compute unit, i.e. wavefronts a SIMD, i.e. registers: one more where a few registers decide, which
    // then wait in scratch (fp32, 8 shapes of 2048, 8 heads: dQ of 64 channels 588 us with 260 registers, 501 with 256; of
    // 32 333 -> 311; bf16, 16 of 4096, 16 heads of 96, forward 1780 -> 1660).  Where more would have to move it is slower (fp32
    // dQ of 96 channels 870 -> 1725, forward of 128 763 -> 1033).
    static constexpr int AT_ONCE_FWD = !DIRECT ? 1 : D == 96 ? 3 : 2;
    static constexpr int AT_ONCE_DQ = DIRECT ? 2 : E::PLANES == 1 || QW == 1 ? 1 : D == 32 ? 3 : D == 64 ? 2 : 1;
    static constexpr int JOIN = QW == 1 ? WAVES * 32 * (32 * DT + 4) * 4 : 0, LDS = BUFFERS * BUFFER > JOIN ? BUFFERS * BUFFER : JOIN;
};

// ---------------------------------------------------------------------------------------------
// forward
// ---------------------------------------------------------------------------------------------
// Query rows of the heads that share a key head are one list, row = token * group + (head within the group), so that
// a tile of keys serves the whole group.  The weights p (0 to 2^8) are rounded to bf16 where the second product takes them (in three
// parts with fp32); their sum l is of what they were before.
// Bound by the matrix pipes and the softmax between the products: at 64 channels the pipes work 0.45 of the time, at 128 0.56, and the vector
// units most of the rest.  bf16, 16 shapes of 4096, 16 heads of 32 / 64 / 96 / 128 channels: 947 / 1225 / 1630 / 2100 us, 580 / 900 / 1010 /
// 1050 TFLOP/s (a large product of the library: 1080).  fp32, 8 of 2048, 8 heads: 240 / 360 / 510 / 780 us, 143 / 191 / 202 / 176 TFLOP/s (the
// library's fp32 product: 153).  One query a shape is a pass over K and V: 8 shapes of 609323 keys together, 2 heads of 32, bf16: 37 us
// from memory (4.2 TB/s; 28 where the last-level cache still has them) and 5.5 to join the splits.
template <typename E, int D, int QW, bool VEC>
__global__ __launch_bounds__((Keys<E, D, QW, VEC>::THREADS), (Keys<E, D, QW, VEC>::AT_ONCE_FWD)) void attn_fwd_kernel(Args a)
{
    typedef Keys<E, D, QW, VEC> S;
    typedef Tile<E, D> L;
    typedef typename E::T T;
    __shared__ __align__(16) char lds[S::LDS];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int qw = QW == 1 ? 0 : wave, kw = QW == 1 ? wave % S::KW : 0, dw = QW == 1 ? wave / S::KW : 0;
    const Work w = work_of(a, blockIdx.x);
    const int split = w.split, slot = w.slot, kvh = w.head;
    if (slot >= a.slots) return;
    const Place place = place_of(a.qo, a.nq, a.ko, a.nk, a.batch, a.sorted, a.group, S::BQ, slot, lane);
    if (place.tile < 0) return;
    const Span q = place.own, k = place.stream;
    // n_q * heads_q and a tile more are below 2^31
    const int rows = (q.end - q.begin) * a.group, row = place.tile * S::BQ + 32 * qw + (lane & 31);
    const bool valid = row < rows;
    const int token = q.begin + (valid ? row / a.group : 0), head = kvh * a.group + (valid ? row % a.group : 0), at = token * a.hq + head;
    const int tiles = (k.end - k.begin + S::BK - 1) / S::BK;
    const int t0 = (int)((int64_t)tiles * split / a.splits), t1 = (int)((int64_t)tiles * (split + 1) / a.splits);
    const T *kp = (const T *)a.K + k.begin * a.ld_k + (int64_t)kvh * a.d, *vp = (const T *)a.V + k.begin * a.ld_v + (int64_t)kvh * a.d;
    const uint8_t *mask = a.mask ? a.mask + k.begin : nullptr;
    const int len = k.end - k.begin;
    const int left = Layout<D>::left(Layout<D>::left0(lane), S::DT * dw);
    const bool full = a.d > D - CHUNK;                      // the last 16 channels are not all zeros

    f32x16 acc[S::DT];
#pragma unroll
    for (int dt = 0; dt < S::DT; ++dt) acc[dt] = f32x16{};
    float m = -INFINITY, l = 0.f;
    bool some = false;                                      // a key was seen

    // The next tile is on its way while this one is multiplied: in registers, or straight to the other buffer.
    typedef Stage<E, D, S::BK, S::THREADS> Regs;
    typedef Direct<D, S::BK> Dir;
    Regs ks, vs;
    int seen[S::WORDS];
    auto buffer = [&](int t) { return lds + (S::BUFFERS == 2 ? (t & 1) * S::BUFFER : 0); };
    auto load = [&](int t) {
        if constexpr (S::DIRECT) {
            Dir::load(kp, a.ld_k, t * S::BK, len, a.d, buffer(t), wave, lane);
            Dir::load(vp, a.ld_v, t * S::BK, len, a.d, buffer(t) + S::TILE, wave, lane);
        } else {
            ks.load(kp, a.ld_k, t * S::BK, len, a.d, VEC, tid);
            vs.load(vp, a.ld_v, t * S::BK, len, a.d, VEC, tid);
        }
#pragma unroll
        for (int i = 0; i < S::WORDS; ++i) seen[i] = key_byte(mask, t * S::BK + 64 * i + lane, len);
    };
    // Tile t in LDS, keys that are not seen as zeros (they may hold anything, and 0 * NaN is NaN); behind it what the scores of its
    // keys start from: 0, or -inf for a key that is not seen.
    auto arrive = [&](int t) {
        char *kt = buffer(t), *vt = kt + S::TILE;
        uint64_t keep[S::WORDS];
        bool all = true;
#pragma unroll
        for (int i = 0; i < S::WORDS; ++i) {
            keep[i] = __ballot(seen[i] != 0);
            some |= keep[i] != 0;
            all &= S::BK - 64 * i >= 64 ? keep[i] == ~0ull : (uint32_t)keep[i] == ~0u;
        }
        if constexpr (S::DIRECT) {
            Dir::wait();
            if (!all) {
                Dir::clear(vt, wave, lane, keep[0]);
                Dir::clear(kt, wave, lane, keep[0]);
            }
        } else {
            if (S::BUFFERS == 1) __syncthreads();
            ks.store(kt, tid, all, keep);
            vs.store(vt, tid, all, keep);
        }
#pragma unroll
        for (int i = 0; i < S::WORDS; ++i)
            if (wave == i && 64 * i + lane < S::BK) ((float *)(kt + 2 * S::TILE))[64 * i + lane] = seen[i] ? 0.f : -INFINITY;
        __syncthreads();
    };
    auto start = [&](int t, int run) {
        f32x16 s;
        const float *p = (const float *)(buffer(t) + 2 * S::TILE) + 32 * run + 4 * h;
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const f32x4 x = *(const f32x4 *)(p + reg_row(r));
#pragma unroll
            for (int j = 0; j < 4; ++j) s[r + j] = x[j];
        }
        return s;
    };
    if (t0 < t1) load(t0);                              // before the own rows, so that neither waits for the other
    Own<E, D> own;
    own.load((const T *)a.Q + token * a.ld_q + (int64_t)head * a.d, valid, a.d, VEC, h);
    for (int t = t0; t < t1; ++t) {
        char *kt = buffer(t), *vt = kt + S::TILE;
        arrive(t);
        if (t + 1 < t1) load(t + 1);

        const int sub = QW == 1 ? kw : 0;               // the first of this wavefront's runs of 32 keys
        f32x16 s[S::NT];
#pragma unroll
        for (int i = 0; i < S::NT; ++i) s[i] = start(t, sub + i);
        // Products go before another wavefront's softmax, which then fills the time that theirs leave (bf16, 16 shapes of 4096, 16 heads of
        // 64: 1369 -> 1330 us, of 32 1033 -> 1000; the passes of the gradient lose by it, dQ of 64 channels 1690 -> 1815).
        __builtin_amdgcn_s_setprio(1);
        products<E, D, S::NT>(kt + 32 * sub * L::STRIDE, S::PLANE, own, lane, full, s);
        __builtin_amdgcn_s_setprio(0);
        Fold<E, D, S::DT> fold(vt + 32 * sub * L::STRIDE, S::PLANE, left);
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < S::NT; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, s[i][r]);
        top = fmaxf(top, other_half(top)) * a.c;
        // The sums are kept relative to a maximum that is brought up only when a score exceeds it by 2^8: exact in
        // fp32 either way (exponents have room), and nearly every tile is spared the scaling of the sums.
        if (__any(top > m + 8.f)) {
            const bool up = top > m + 8.f;
            const float f = up ? exp2_fast(m - top) : 1.f;
            if (up) m = top;
            l *= f;
#pragma unroll
            for (int dt = 0; dt < S::DT; ++dt)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[dt][r] *= f;
        }
        const float base = m == -INFINITY ? 0.f : m;    // no key yet: exp2(-inf) = 0, not -inf + inf
        // Weights are added up by tiles first: one by one, 300000 equal ones are rounded to the same side each time, 1e-3 of l in all
        // (by tiles 1e-5; the sum with what each addition loses carried along 2e-6, but one register too many for fp32 of 96
        // channels, 485 -> 578 us).
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < S::NT; ++i)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[i][r] = exp2_fast(__builtin_fmaf(s[i][r], a.c, -base));
                sum += s[i][r];
            }
        l += sum;
        __builtin_amdgcn_s_setprio(1);
        fold.run(s, acc);
        __builtin_amdgcn_s_setprio(0);
    }
    l += other_half(l);
    // Rows that saw no key are 0 whatever their queries hold: NaN and infinity have met the zeros of keys that are left out, and
    // made NaN of them.
    if (!some) {
        m = -INFINITY;
        l = 0.f;
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) acc[dt] = f32x16{};
    }

    if constexpr (QW == 1) {                            // the wavefronts' shares of the keys, joined in LDS
        __syncthreads();
        constexpr int W = 32 * S::DT + 4;               // floats of a row: its sums, then maximum and sum of weights
        float *mine = (float *)lds + (wave * 32 + (lane & 31)) * W;
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; r += 4)
                *(f32x4 *)(mine + 32 * dt + reg_row(r) + 4 * h) = f32x4{acc[dt][r], acc[dt][r + 1], acc[dt][r + 2], acc[dt][r + 3]};
        if (h == 0) { mine[32 * S::DT] = m; mine[32 * S::DT + 1] = l; }
        __syncthreads();
        if (kw) return;
        float f[S::KW];
        m = -INFINITY;
#pragma unroll
        for (int i = 0; i < S::KW; ++i) m = fmaxf(m, mine[i * 32 * W + 32 * S::DT]);
        l = 0.f;
#pragma unroll
        for (int i = 0; i < S::KW; ++i) {
            f[i] = m == -INFINITY ? 0.f : exp2_fast(mine[i * 32 * W + 32 * S::DT] - m);
            l += f[i] * mine[i * 32 * W + 32 * S::DT + 1];
        }
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt)
#pragma unroll
            for (int r = 0; r < 16; r += 4) {
                f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < S::KW; ++i) t += f[i] * *(const f32x4 *)(mine + i * 32 * W + 32 * dt + reg_row(r) + 4 * h);
#pragma unroll
                for (int j = 0; j < 4; ++j) acc[dt][r + j] = t[j];
            }
    }
    if (!valid) return;
    const int e0 = 32 * S::DT * dw;
    if (a.splits == 1) {
        store_row<T>((T *)a.Ow + token * a.ld_o + (int64_t)head * a.d + e0, acc, l > 0.f || l != l ? 1.f / l : 0.f, a.d - e0, VEC, h);
        if (a.lse && h == 0 && dw == 0) a.lse[at] = l > 0.f || l != l ? m * LN2 + logf(l) : -INFINITY;
    } else {
        const int64_t p = split * a.nq * a.hq + at;
        if (l > 0.f || l != l) store_row<float>(a.part + p * a.d + e0, acc, 1.f, a.d - e0, a.d % 4 == 0, h);
        if (h == 0 && dw == 0) a.ml[p] = make_float2(m, l);
    }
}

// Joins the splits of a row: G groups of 32 lanes deal the splits among them, a lane has 4 channels.  8 groups for a row
// where there are few rows of many splits; else a group for each (10778 rows x 2 heads of 3 splits: 34 -> 5 us).  A group
// first turns its splits' maxima into weights, 32 at a time, then adds their sums up without waiting for one before the next
// (64 rows of 128 splits: 16 -> 6 us).
template <typename T, int G> __global__ __launch_bounds__(256) void attn_join_kernel(Args a)
{
    __shared__ __align__(16) float sums[8][128];
    __shared__ float weight[8][32];
    __shared__ float2 ml[8];
    const int x = threadIdx.x & 31, group = threadIdx.x >> 5, g = group % G;
    const int64_t rows = a.nq * a.hq, at = (int64_t)blockIdx.x * (8 / G) + group / G;
    const bool there = at < rows, whole = a.d % 4 == 0;
    float m = -INFINITY, l = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    const int mine = there ? (a.splits - g + G - 1) / G : 0;        // splits g, g + G, ...
    for (int first = 0; first < mine; first += 32) {
        const int n = min(32, mine - first);
        float2 v = make_float2(-INFINITY, 0.f);
        if (x < n) v = a.ml[(int64_t)(g + G * (first + x)) * rows + at];
        const bool some = v.y > 0.f || v.y != v.y;      // a split without a key has written no sums
        float top = m;
        {
            float t = some ? v.x : -INFINITY;
#pragma unroll
            for (int i = 16; i; i >>= 1) t = fmaxf(t, __shfl_xor(t, i));
            top = fmaxf(m, t);
        }
        const float w = some ? exp2_fast(v.x - top) : 0.f, old = m == -INFINITY ? 0.f : exp2_fast(m - top);
        float sum = some ? w * v.y : 0.f;
#pragma unroll
        for (int i = 16; i; i >>= 1) sum += __shfl_xor(sum, i);
        l = l * old + sum;
        acc *= old;
        m = top;
        weight[group][x] = w;
        __builtin_amdgcn_wave_barrier();
        const float *p = a.part + ((int64_t)(g + G * first) * rows + at) * a.d + 4 * x;
        const int64_t step = (int64_t)G * rows * a.d;
        if (4 * x < a.d) {
            if (whole) {
#pragma unroll 8
                for (int i = 0; i < n; ++i) {
                    const f32x4 t = *(const f32x4 *)(p + i * step);
                    const float f = weight[group][i];
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[j] += f == 0.f ? 0.f : f * t[j];
                }
            } else
                for (int i = 0; i < n; ++i) {
                    const float f = weight[group][i];
#pragma unroll
                    for (int j = 0; j < 4; ++j) if (4 * x + j < a.d) acc[j] += f == 0.f ? 0.f : f * p[i * step + j];
                }
        }
        __builtin_amdgcn_wave_barrier();
    }
    if constexpr (G > 1) {
        *(f32x4 *)&sums[g][4 * x] = acc;
        if (x == 0) ml[g] = make_float2(m, l);
        __syncthreads();
        if (g) return;
        m = -INFINITY;
#pragma unroll
        for (int i = 0; i < G; ++i) m = fmaxf(m, ml[i].x);
        l = 0.f;
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < G; ++i) {
            if (ml[i].y == 0.f) continue;
            const float f = exp2_fast(ml[i].x - m);
            l += f * ml[i].y;
            acc += f * *(const f32x4 *)&sums[i][4 * x];
        }
    }
    if (!there) return;
    const int64_t token = at / a.hq;
    const bool some = l > 0.f || l != l;
    T *o = (T *)a.Ow + token * a.ld_o + (at - token * a.hq) * a.d;
#pragma unroll
    for (int j = 0; j < 4; ++j) if (4 * x + j < a.d) o[4 * x + j] = (T)(some ? acc[j] / l : 0.f);
    if (a.lse && x == 0) a.lse[at] = some ? m * LN2 + logf(l) : -INFINITY;
}

// ---------------------------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------------------------
// a . b of this lane's row; each half takes every other piece
template <typename T, int D> __device__ __forceinline__ float row_dot(const T *a, const T *b, bool valid, int d, bool vec, int h)
{
    constexpr int N = 16 / (int)sizeof(T);
    float t = 0.f;
#pragma unroll
    for (int s = 0; s < D / N / 2; ++s) {
        T x[N], y[N];
        load_piece(a, (2 * s + h) * N, valid, d, vec, x);
        load_piece(b, (2 * s + h) * N, valid, d, vec, y);
#pragma unroll
        for (int j = 0; j < N; ++j) t += (float)x[j] * (float)y[j];
    }
    return t + other_half(t);
}

// acc of the first wavefront = the sum of those of WAVES neighbours, in their order; every wavefront of the workgroup takes part
template <int DT, int WAVES> __device__ __forceinline__ void join_waves(char *lds, f32x16 (&acc)[DT], int wave, int lane)
{
    constexpr int W = 32 * DT + 4;                      // floats of a row; 16 bytes further on each
    const int h = lane >> 5;
    float *mine = (float *)lds + (wave * 32 + (lane & 31)) * W + 4 * h;
    __syncthreads();
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; r += 4) *(f32x4 *)(mine + 32 * dt + reg_row(r)) = f32x4{acc[dt][r], acc[dt][r + 1], acc[dt][r + 2], acc[dt][r + 3]};
    __syncthreads();
    if (wave % WAVES) return;
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < WAVES; ++i) t += *(const f32x4 *)(mine + i * 32 * W + 32 * dt + reg_row(r));
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[dt][r + j] = t[j];
        }
}

// dQ, and D for the pass over the keys: the walk of the forward kernel.  dS is rounded to bf16 where the product with K takes it,
// which together with dQ's own rounding makes 2.4e-3 of its size in bf16; two parts of dS would take that back to 1.7e-3 for a third more
// products.  D comes from O as it was stored, rounded: 2e-4 of dQ's size where a row's weight is spread over many keys, 2e-3 where a few keys
// have most of it (3.3e-3 in all).  Without that it would be the sum of p dP over the keys, known when they have all gone past, and what is
// then to be taken off, the sum of p k, as many products more again as dS k.
// Bound by the matrix pipes (busy 0.60 of the time at 64 channels): bf16, 16 shapes of 4096, 16 heads of 32 / 64 / 96 / 128: 970 / 1520 / 2240 / 3030
// us, 850 / 1085 / 1100 / 1090 TFLOP/s; fp32, 8 of 2048, 8 heads: 311 / 501 / 830 / 1132 us, 166 / 206 / 187 / 182 TFLOP/s.
template <typename E, int D, int QW, bool VEC> __device__ __forceinline__ void bwd_dq(const Args &a, int id, char *lds)
{
    typedef Keys<E, D, QW, VEC> S;
    typedef Tile<E, D> L;
    typedef typename E::T T;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int qw = QW == 1 ? 0 : wave, kw = QW == 1 ? wave % S::KW : 0, dw = QW == 1 ? wave / S::KW : 0;
    const Work w = work_of(a, id);
    const int split = w.split, slot = w.slot, kvh = w.head;
    if (slot >= a.slots) return;
    const Place place = place_of(a.qo, a.nq, a.ko, a.nk, a.batch, a.sorted, a.group, S::BQ, slot, lane);
    if (place.tile < 0) return;
    const Span q = place.own, k = place.stream;
    // n_q * heads_q and a tile more are below 2^31
    const int rows = (q.end - q.begin) * a.group, row = place.tile * S::BQ + 32 * qw + (lane & 31);
    const bool valid = row < rows;
    const int token = q.begin + (valid ? row / a.group : 0), head = kvh * a.group + (valid ? row % a.group : 0), at = token * a.hq + head;
    const int tiles = (k.end - k.begin + S::BK - 1) / S::BK;
    const int t0 = (int)((int64_t)tiles * split / a.splits), t1 = (int)((int64_t)tiles * (split + 1) / a.splits);
    const T *kp = (const T *)a.K + k.begin * a.ld_k + (int64_t)kvh * a.d, *vp = (const T *)a.V + k.begin * a.ld_v + (int64_t)kvh * a.d;
    const uint8_t *mask = a.mask ? a.mask + k.begin : nullptr;
    const int len = k.end - k.begin;
    const int left = Layout<D>::left(Layout<D>::left0(lane), S::DT * dw);
    const bool full = a.d > D - CHUNK;                      // the last 16 channels are not all zeros

    f32x16 acc[S::DT];
#pragma unroll
    for (int dt = 0; dt < S::DT; ++dt) acc[dt] = f32x16{};
    // The next tile is on its way while this one is multiplied: in registers, or straight to the other buffer.
    typedef Stage<E, D, S::BK, S::THREADS> Regs;
    typedef Direct<D, S::BK> Dir;
    Regs ks, vs;
    int seen[S::WORDS];
    auto buffer = [&](int t) { return lds + (S::BUFFERS == 2 ? (t & 1) * S::BUFFER : 0); };
    auto load = [&](int t) {
        if constexpr (S::DIRECT) {
            Dir::load(kp, a.ld_k, t * S::BK, len, a.d, buffer(t), wave, lane);
            Dir::load(vp, a.ld_v, t * S::BK, len, a.d, buffer(t) + S::TILE, wave, lane);
        } else {
            ks.load(kp, a.ld_k, t * S::BK, len, a.d, VEC, tid);
            vs.load(vp, a.ld_v, t * S::BK, len, a.d, VEC, tid);
        }
#pragma unroll
        for (int i = 0; i < S::WORDS; ++i) seen[i] = key_byte(mask, t * S::BK + 64 * i + lane, len);
    };
    // Tile t in LDS, keys that are not seen as zeros (they may hold anything, and 0 * NaN is NaN); behind it what the scores of its
    // keys start from: 0, or -inf for a key that is not seen.
    auto arrive = [&](int t) {
        char *kt = buffer(t), *vt = kt + S::TILE;
        uint64_t keep[S::WORDS];
        bool all = true;
#pragma unroll
        for (int i = 0; i < S::WORDS; ++i) {
            keep[i] = __ballot(seen[i] != 0);
            all &= S::BK - 64 * i >= 64 ? keep[i] == ~0ull : (uint32_t)keep[i] == ~0u;
        }
        if constexpr (S::DIRECT) {
            Dir::wait();
            if (!all) {
                Dir::clear(vt, wave, lane, keep[0]);
                Dir::clear(kt, wave, lane, keep[0]);
            }
        } else {
            if (S::BUFFERS == 1) __syncthreads();
            ks.store(kt, tid, all, keep);
            vs.store(vt, tid, all, keep);
        }
#pragma unroll
        for (int i = 0; i < S::WORDS; ++i)
            if (wave == i && 64 * i + lane < S::BK) ((float *)(kt + 2 * S::TILE))[64 * i + lane] = seen[i] ? 0.f : -INFINITY;
        __syncthreads();
    };
    auto start = [&](int t, int run) {
        f32x16 s;
        const float *p = (const float *)(buffer(t) + 2 * S::TILE) + 32 * run + 4 * h;
#pragma unroll
        for (int r = 0; r < 16; r += 4) {
            const f32x4 x = *(const f32x4 *)(p + reg_row(r));
#pragma unroll
            for (int j = 0; j < 4; ++j) s[r + j] = x[j];
        }
        return s;
    };
    if (t0 < t1) load(t0);
    const float lse = a.lse[at];
    const bool part = valid && lse != -INFINITY;        // a row that saw no key: its gradient is zero, whatever dO holds
    const float lse2 = part ? lse * LOG2E : INFINITY;
    Own<E, D> own, grad;
    const T *gp = (const T *)a.dO + token * a.ld_do + (int64_t)head * a.d;
    own.load((const T *)a.Q + token * a.ld_q + (int64_t)head * a.d, valid, a.d, VEC, h);
    grad.load(gp, valid, a.d, VEC, h);
    float delta = row_dot<T, D>(gp, (const T *)a.O + token * a.ld_o + (int64_t)head * a.d, valid, a.d, VEC, h);
    if (!part) delta = 0.f;
    if (a.delta && valid && split == 0 && kw == 0 && dw == 0 && h == 0) a.delta[at] = delta;
    for (int t = t0; t < t1; ++t) {
        char *kt = buffer(t), *vt = kt + S::TILE;
        arrive(t);
        if (t + 1 < t1) load(t + 1);
#pragma unroll
        for (int i = 0; i < S::NT; ++i) {
            const int sub = QW == 1 ? kw : i;
            f32x16 s[1] = {start(t, sub)}, g[1];
#pragma unroll
            for (int r = 0; r < 16; ++r) g[0][r] = -delta;
            products<E, D, 1, S::AHEAD>(kt + 32 * sub * L::STRIDE, S::PLANE, own, lane, full, s);
            products<E, D, 1, S::AHEAD>(vt + 32 * sub * L::STRIDE, S::PLANE, grad, lane, full, g);
            Fold<E, D, S::DT, S::FOLD> fold(kt + 32 * sub * L::STRIDE, S::PLANE, left);
#pragma unroll
            for (int r = 0; r < 16; ++r) g[0][r] *= exp2_fast(__builtin_fmaf(s[0][r], a.c, -lse2));
            fold.run(g, acc);
        }
    }
    if constexpr (QW == 1) {
        join_waves<S::DT, S::KW>(lds, acc, wave, lane);
        if (kw) return;
    }
    if (!valid) return;
    if (!part)
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) acc[dt] = f32x16{};
    const int e0 = 32 * S::DT * dw;
    if (a.splits == 1) store_row<T>((T *)a.dQ + token * a.ld_dq + (int64_t)head * a.d + e0, acc, a.scale, a.d - e0, VEC, h);
    else store_row<float>(a.part + (split * a.nq * a.hq + at) * a.d + e0, acc, a.scale, a.d - e0, a.d % 4 == 0, h);
}

template <typename E, int D, int QW, bool VEC>
__global__ __launch_bounds__((Keys<E, D, QW, VEC>::THREADS), (Keys<E, D, QW, VEC>::AT_ONCE_DQ)) void attn_bwd_dq_kernel(Args a)
{
    __shared__ __align__(16) char lds[Keys<E, D, QW, VEC>::LDS];
    bwd_dq<E, D, QW, VEC>(a, blockIdx.x, lds);
}

// dK and dV: a wavefront has 32 keys, the queries of all heads that share their head stream past, one head after
// the other, so the sum over them is taken in registers in a fixed order.  KW wavefronts have keys of their own (4, wide)
// or all share 32 keys and deal the queries of a tile among them (1, narrow).  p and dS are rounded to bf16 for the products, as above.
// Bound by the matrix pipes and, with one or two wavefronts a SIMD (a key's two sums and two operands fill the registers), by the steps' own
// latencies: busy 0.54 of the time at 64 channels.  bf16, 16 shapes of 4096, 16 heads of 32 / 64 / 96 / 128: 1250 / 2320 / 3150 / 5500 us, 880 / 945 / 1045 / 800
// TFLOP/s; fp32, 8 of 2048, 8 heads: 400 / 715 / 1036 / 1370 us, 172 / 192 / 199 / 201 TFLOP/s.
template <typename E, int D, int KW, bool VEC> struct Queries {
    static constexpr int WAVES = 4, THREADS = 64 * WAVES, DW = KW == 1 && E::PLANES == 3 && D > 64 ? 2 : 1, QW = WAVES / KW / DW, BK = 32 * KW;
    static constexpr int DT = D / 32 / DW;
    static constexpr int BR = KW == 1 ? 32 * QW : E::PLANES == 1 ? 64 : 32, NT = BR / 32 / QW;
    static constexpr int PLANE = BR * Tile<E, D>::STRIDE, TILE = E::PLANES * PLANE, BUFFER = 2 * TILE + 2 * BR * 4;
    static constexpr int BUFFERS = KW == 1 || 2 * BUFFER > 80 * 1024 ? 1 : 2;
    static constexpr bool DIRECT = VEC && E::PLANES == 1 && KW == 4;
    // fp32 of 64 channels could have two, with 36 registers in scratch: 752 -> 716 us with workgroups for every compute unit twice over, but
    // 22 -> 35 where each is alone (21 shapes of 4971 rows together, 2 heads of 40)
    static constexpr int AT_ONCE = DIRECT && D < 128 ? 2 : 1;
    static constexpr int JOIN = KW == 1 ? WAVES * 32 * (32 * DT + 4) * 4 : 0, LDS = BUFFERS * BUFFER > JOIN ? BUFFERS * BUFFER : JOIN;
};
template <typename E, int D, int KW, bool VEC> __device__ __forceinline__ void bwd_dkv(const Args &a, int id, char *lds)
{
    typedef Queries<E, D, KW, VEC> S;
    typedef Tile<E, D> L;
    typedef typename E::T T;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), h = lane >> 5;
    const int kw = KW == 1 ? 0 : wave, qw = KW == 1 ? wave % S::QW : 0, dw = KW == 1 ? wave / S::QW : 0;
    const Work w = work_of(a, id);
    const int split = w.split, slot = w.slot, kvh = w.head;
    if (slot >= a.slots) return;
    const Place place = place_of(a.ko, a.nk, a.qo, a.nq, a.batch, a.sorted, 1, S::BK, slot, lane);
    if (place.tile < 0) return;
    const Span q = place.stream, k = place.own;

    const int key = k.begin + place.tile * S::BK + 32 * kw + (lane & 31);
    const bool valid = key < k.end, seen = valid && (!a.mask || a.mask[key]);
    const int len = q.end - q.begin, tiles = (len + S::BR - 1) / S::BR;
    const int s0 = (int)((int64_t)tiles * a.group * split / a.splits), s1 = (int)((int64_t)tiles * a.group * (split + 1) / a.splits);
    const int left = Layout<D>::left(Layout<D>::left0(lane), S::DT * dw);
    f32x16 dk[S::DT], dv[S::DT];
#pragma unroll
    for (int dt = 0; dt < S::DT; ++dt) dk[dt] = dv[dt] = f32x16{};

    typedef Stage<E, D, S::BR, S::THREADS> Regs;
    typedef Direct<D, S::BR> Dir;
    Regs qs, gs;
    float lse = 0.f, delta = 0.f;
    auto buffer = [&](int step) { return lds + (S::BUFFERS == 2 ? (step & 1) * S::BUFFER : 0); };
    auto load = [&](int step, int head, int t) {
        const T *qp = (const T *)a.Q + q.begin * a.ld_q + (int64_t)head * a.d, *gp = (const T *)a.dO + q.begin * a.ld_do + (int64_t)head * a.d;
        if constexpr (S::DIRECT) {
            Dir::load(qp, a.ld_q, t * S::BR, len, a.d, buffer(step), wave, lane);
            Dir::load(gp, a.ld_do, t * S::BR, len, a.d, buffer(step) + S::TILE, wave, lane);
        } else {
            qs.load(qp, a.ld_q, t * S::BR, len, a.d, VEC, tid);
            gs.load(gp, a.ld_do, t * S::BR, len, a.d, VEC, tid);
        }
        if (tid < S::BR) {
            const int row = t * S::BR + tid;
            const int64_t at = (int64_t)(q.begin + row) * a.hq + head;
            lse = row < len ? a.lse[at] : -INFINITY;
            delta = row < len ? a.delta[at] : 0.f;
        }
    };
    int head = kvh * a.group + (s0 < s1 ? s0 / tiles : 0), t = s0 < s1 ? s0 % tiles : 0;
    if (s0 < s1) load(s0, head, t);
    Own<E, D> kk, vv;
    kk.load((const T *)a.K + (valid ? key : 0) * a.ld_k + (int64_t)kvh * a.d, seen, a.d, VEC, h);
    vv.load((const T *)a.V + (valid ? key : 0) * a.ld_v + (int64_t)kvh * a.d, seen, a.d, VEC, h);
    for (int step = s0; step < s1; ++step) {
        char *qt = buffer(step), *gt = qt + S::TILE;
        float *stat = (float *)(gt + S::TILE);
        if constexpr (S::DIRECT) {
            Dir::wait();
        } else {
            if (S::BUFFERS == 1) __syncthreads();
            qs.store(qt, tid);
            gs.store(gt, tid);
        }
        if (tid < S::BR) {
            stat[tid] = lse == -INFINITY ? -INFINITY : -lse * LOG2E;    // no such row, or one that saw no key: p = 0
            stat[S::BR + tid] = -delta;
        }
        __syncthreads();
        if (++t == tiles) { t = 0; ++head; }
        if (step + 1 < s1) load(step + 1, head, t);
#pragma unroll
        for (int i = 0; i < S::NT; ++i) {
            const int sub = KW == 1 ? qw : i;
            f32x16 p[1] = {f32x16{}}, g[1];
            f32x4 x[4];
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                x[r] = *(const f32x4 *)(stat + 32 * sub + 8 * r + 4 * h);
                const f32x4 y = *(const f32x4 *)(stat + S::BR + 32 * sub + 8 * r + 4 * h);
#pragma unroll
                for (int j = 0; j < 4; ++j) g[0][4 * r + j] = y[j];
            }
            products<E, D, 1>(qt + 32 * sub * L::STRIDE, S::PLANE, kk, lane, true, p);
            products<E, D, 1>(gt + 32 * sub * L::STRIDE, S::PLANE, vv, lane, true, g);
            {
                Fold<E, D, S::DT> fold(gt + 32 * sub * L::STRIDE, S::PLANE, left);
#pragma unroll
                for (int r = 0; r < 16; ++r) p[0][r] = exp2_fast(__builtin_fmaf(p[0][r], a.c, x[r >> 2][r & 3]));
                fold.run(p, dv);
            }
            Fold<E, D, S::DT> fold(qt + 32 * sub * L::STRIDE, S::PLANE, left);
#pragma unroll
            for (int r = 0; r < 16; ++r) g[0][r] *= p[0][r];
            fold.run(g, dk);
        }
    }
    if constexpr (KW == 1) {
        join_waves<S::DT, S::QW>(lds, dk, wave, lane);
        join_waves<S::DT, S::QW>(lds, dv, wave, lane);
        if (qw) return;
    }
    if (!valid) return;
    if (!seen)                                          // a key that is left out: zero, whatever its lane added up
#pragma unroll
        for (int dt = 0; dt < S::DT; ++dt) dk[dt] = dv[dt] = f32x16{};
    const int e0 = 32 * S::DT * dw;
    if (a.splits == 1) {
        store_row<T>((T *)a.dK + key * a.ld_dk + (int64_t)kvh * a.d + e0, dk, a.scale, a.d - e0, VEC, h);
        store_row<T>((T *)a.dV + key * a.ld_dv + (int64_t)kvh * a.d + e0, dv, 1.f, a.d - e0, VEC, h);
    } else {
        const int64_t rows = a.nk * a.hkv;
        float *p = a.part + (split * 2 * rows + (int64_t)key * a.hkv + kvh) * a.d + e0;
        store_row<float>(p, dk, a.scale, a.d - e0, a.d % 4 == 0, h);
        store_row<float>(p + rows * a.d, dv, 1.f, a.d - e0, a.d % 4 == 0, h);
    }
}

template <typename E, int D, int KW, bool VEC>
__global__ __launch_bounds__((Queries<E, D, KW, VEC>::THREADS), (Queries<E, D, KW, VEC>::AT_ONCE)) void attn_bwd_dkv_kernel(Args a)
{
    __shared__ __align__(16) char lds[Queries<E, D, KW, VEC>::LDS];
    bwd_dkv<E, D, KW, VEC>(a, blockIdx.x, lds);
}

// Both passes in one launch, for calls neither of which fills the compute units (8 shapes of 2381 rows together, 8 heads of 32, fp32: 48 -> 40 us and 5
// for D; one of 665, 4 of 64, bf16: 26 -> 17 in all): the first `q_grid` workgroups form dQ, the others dK
// and dV, from a D that attn_delta_kernel left.
template <typename E, int D, int W> struct Both {
    typedef Keys<E, D, W, true> K;
    typedef Queries<E, D, W, true> Q;
    static constexpr int AT_ONCE = K::AT_ONCE_DQ < Q::AT_ONCE ? K::AT_ONCE_DQ : Q::AT_ONCE, LDS = K::LDS > Q::LDS ? K::LDS : Q::LDS;
};
template <typename E, int D, int W>
__global__ __launch_bounds__((Keys<E, D, W, true>::THREADS), (Both<E, D, W>::AT_ONCE)) void attn_bwd_both_kernel(Args a, Args b, int q_grid)
{
    __shared__ __align__(16) char lds[Both<E, D, W>::LDS];
    if ((int)blockIdx.x < q_grid) bwd_dq<E, D, W, true>(a, blockIdx.x, lds);
    else bwd_dkv<E, D, W, true>(b, blockIdx.x - q_grid, lds);
}
// D of every row, by `lanes` lanes (a power of two) of 16 bytes a row; 0 where the row saw no key
template <typename T> __global__ __launch_bounds__(256) void attn_delta_kernel(Args a, int lanes)
{
    constexpr int N = 16 / (int)sizeof(T);
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / lanes;
    const int lane = threadIdx.x % lanes, e = lane * N;
    if (at >= a.nq * a.hq) return;                      // (whole groups of lanes)
    const int64_t token = at / a.hq, head = at - token * a.hq;
    T x[N], y[N];
    load_piece((const T *)a.dO + token * a.ld_do + head * a.d, e, true, a.d, true, x);
    load_piece((const T *)a.O + token * a.ld_o + head * a.d, e, true, a.d, true, y);
    float t = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) t += (float)x[j] * (float)y[j];
    for (int i = 1; i < lanes; i <<= 1) t += __shfl_xor(t, i);
    if (lane == 0) a.delta[at] = a.lse[at] == -INFINITY ? 0.f : t;
}

// The gradients whose passes were split = the sums of their splits, in their order; a thread per element.  One launch for all three: the
// first `q_blocks` workgroups have dQ, the others dK and dV (none, where a pass was not split).
template <typename T> __global__ __launch_bounds__(256) void attn_bwd_join_kernel(Args a, const float *q_part, int q_splits, int q_blocks)
{
    const bool query = (int)blockIdx.x < q_blocks;
    const int64_t i = (int64_t)(blockIdx.x - (query ? 0 : q_blocks)) * 256 + threadIdx.x;
    const int heads = query ? a.hq : a.hkv, splits = query ? q_splits : a.splits;
    const int64_t n = (query ? a.nq : a.nk) * heads * a.d, all = query ? n : 2 * n;       // dK, then dV
    if (i >= all) return;
    const float *p = (query ? q_part : a.part) + i;
    float t = 0.f;
    for (int s = 0; s < splits; ++s) t += p[s * all];
    const int64_t e = i < n ? i : i - n, at = e / a.d, row = at / heads, col = (at - row * heads) * a.d + (e - at * a.d);
    if (query) ((T *)a.dQ)[row * a.ld_dq + col] = (T)t;
    else if (i < n) ((T *)a.dK)[row * a.ld_dk + col] = (T)t;
    else ((T *)a.dV)[row * a.ld_dv + col] = (T)t;
}

}  // namespace attn
}  // namespace hch
