// Products of rows with the weights of their experts, and both gradients (definitions: dear_ops.h).
//
//     y[m, n] = sum over k of x[m, k] w[e, n, k];  dx[m, k] = sum over n of dy[m, n] w[e, n, k]
//     dw[e, n, k] = sum over the rows m of e of dy[m, n] x[m, k]
//
// All three are sums of products of two operands that lie in memory either along the summed index (x and w for y, dy for dx) or across
// it (w for dx, both for dw); the former are read from LDS in rows, the latter with the transposing reads.  Rows of an expert start
// anywhere: a workgroup finds the expert of its tile from the ends, on the device, so that nothing waits for the host to know them.
//
// Matrix instructions bound large calls, at the clock that the card's power leaves them (16384 uneven rows, 4096 x 1024 over 8, bf16: 980, 985 and 855
// TFLOP/s for the three products, a library's of 8192 x 8192 x 8192 1394); the weights' way from memory bounds few rows (32: 4.5 TB/s).
#include <type_traits>

#include "experts_cut.h"
#include "ops_common.h"

#pragma clang fp contract(fast)

namespace {

using namespace dear_ops;

struct params {
    const void *a, *b;  // operands of the outputs' rows and columns
    int64_t a_stride, b_stride;
    const int32_t *ends;
    void *out;
    int64_t rows;
    int32_t experts;
    int32_t sum;         // summed index (of a weight gradient, the expert's rows)
    int32_t n_a, n_b;    // outputs' rows (of a weight gradient; otherwise the tile's expert has them) and columns
    int32_t a_tiles, b_tiles;
    int32_t splits, chunk;  // of the summed index: sums of their own, and how much of it each has
    float *parts;           // [splits, outputs], where there are several
};

// ------------------------------------------------------------------------------------ a tile's expert
struct part {
    int32_t expert;        // experts: the rows behind the last one's
    int64_t begin, end;    // its rows
    int64_t first;         // of the tile
    bool none;             // there are fewer tiles
};

// Ends are made to ascend, and to stay within the rows: of 64 experts at a time, one a lane, each wave for itself.
__device__ __forceinline__ int32_t max_before(int32_t x, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int32_t y = __shfl_up(x, d);
        if (lane >= d) x = max(x, y);
    }
    return x;
}
__device__ __forceinline__ int32_t sum_before(int32_t x, int lane) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int32_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

// Tile `id` of all experts' rows in tiles of BM, those behind the last expert's included.
template <int BM> __device__ __forceinline__ part find(const params &p, int32_t id) {
    const int lane = threadIdx.x & 63, rows = (int)p.rows;
    int32_t before = 0, tiles = 0;  // rows and tiles of the experts of earlier steps
    for (int e0 = 0; e0 <= p.experts; e0 += 64) {
        const int e = e0 + lane;
        int32_t end = e < p.experts ? min(max(p.ends[e], 0), rows) : rows;
        end = max(max_before(end, lane), before);
        int32_t begin = __shfl_up(end, 1);
        if (lane == 0) begin = before;
        const int32_t mine = e <= p.experts ? (int32_t)(((uint32_t)(end - begin) + BM - 1) / BM) : 0;
        const int32_t upto = tiles + sum_before(mine, lane);
        const uint64_t found = __ballot(upto > id);
        if (found) {
            const int k = __builtin_ctzll(found);
            part t;
            t.expert = e0 + k;
            t.begin = __builtin_amdgcn_readfirstlane(__shfl(begin, k));
            t.end = __builtin_amdgcn_readfirstlane(__shfl(end, k));
            t.first = t.begin + (int64_t)(id - __builtin_amdgcn_readfirstlane(__shfl(upto - mine, k))) * BM;
            t.none = false;
            return t;
        }
        before = __builtin_amdgcn_readfirstlane(__shfl(end, 63));
        tiles = __builtin_amdgcn_readfirstlane(__shfl(upto, 63));
    }
    return part{0, 0, 0, 0, true};
}

// The rows of an expert.
__device__ __forceinline__ part rows_of(const params &p, int32_t expert) {
    const int lane = threadIdx.x & 63, rows = (int)p.rows;
    int32_t before = 0, end = 0;
    for (int e0 = 0;; e0 += 64) {
        const int e = e0 + lane;
        end = e < p.experts ? min(max(p.ends[e], 0), rows) : rows;
        end = max(max_before(end, lane), before);
        if (expert < e0 + 64) break;
        before = __builtin_amdgcn_readfirstlane(__shfl(end, 63));
    }
    int32_t begin = __shfl_up(end, 1);
    if (lane == 0) begin = before;
    part t;
    t.expert = expert, t.none = false;
    t.begin = t.first = __builtin_amdgcn_readfirstlane(__shfl(begin, expert & 63));
    t.end = __builtin_amdgcn_readfirstlane(__shfl(end, expert & 63));
    return t;
}

// ------------------------------------------------------------------------------------ any type, any size
// An operand's part of a step on its way from memory to LDS, in pieces of 16 bytes: OUT rows of BS values along the summed index or, ACROSS
// it, BS rows of OUT values.  Values beyond the sum are zeros in both operands, so that nothing that stands there counts; rows and columns
// beyond the outputs are whatever is there, and not stored.  No load has a branch of its own, which would wait for the one before: pieces
// beyond an end are read from before it, and pieces that begin before a row's end and end behind it are read as they are, up to the end of the
// matrix; only steps that would pass that go value by value (bf16 333 rows, 1001 x 999 over 5, input gradient, 28 us with branches).
template <typename T, bool VEC, bool ACROSS, int OUT, int BS> struct stage {
    static constexpr int E = 16 / sizeof(T), N = OUT * BS / E / THREADS, W = ACROSS ? OUT : BS, ROWS = THREADS * E / W;
    static_assert(N * E * THREADS == OUT * BS && THREADS * E % W == 0, "whole pieces for every thread, in one column");
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
    typedef vec vec_anywhere __attribute__((aligned(sizeof(T))));  // global memory takes 16-byte loads from any element on
    vec v[N];
    const T *data;
    int64_t at[N];      // this lane's pieces of the next step
    int64_t furthest;   // the last piece of the tile's rows and columns, with the step's first of the summed index
    int64_t stop;       // the matrix's end
    int64_t stride;
    int row, col;       // of the lane's first piece; the others are ROWS rows further on each

    // Where the last of `n` values' piece begins; all pieces of a whole tile lie before its end.
    static __device__ __forceinline__ int begin_of_last(int n, int whole) { return n >= whole ? whole - E : VEC ? (n - 1) / E * E : n - 1; }
    // out0, outs: the tile's first output, and how many there are from it on, one at least; s0: the first of the summed index
    __device__ __forceinline__ void aim(const T *data_, int64_t stride_, int64_t rows, int64_t width, int64_t out0, int64_t outs_left, int64_t s0) {
        data = data_, stride = stride_, row = (int)threadIdx.x / (W / E), col = (int)threadIdx.x % (W / E) * E;
        const int outs = (int)min(outs_left, (int64_t)OUT);
        const int64_t first = ACROSS ? s0 * stride + out0 : out0 * stride + s0;
        stop = (rows - 1) * stride + width;
        furthest = ACROSS ? first + begin_of_last(outs, OUT) : first + (outs - 1) * stride;
#pragma unroll
        for (int i = 0; i < N; ++i)
            at[i] = ACROSS ? first + (row + i * ROWS) * stride + min(col, begin_of_last(outs, OUT)) : first + min(row + i * ROWS, outs - 1) * stride + col;
    }
    // left: of the summed index from the step's first on, one at least
    __device__ __forceinline__ void load(int left) {
        int64_t p[N];
#pragma unroll
        for (int i = 0; i < N; ++i) p[i] = at[i];
        if (left < BS) {
#pragma unroll
            for (int i = 0; i < N; ++i)
                p[i] += ACROSS ? (min(row + i * ROWS, left - 1) - (row + i * ROWS)) * stride : (int64_t)(min(col, begin_of_last(left, BS)) - col);
        }
        const int64_t end = furthest + (ACROSS ? (min(left, BS) - 1) * stride : (int64_t)begin_of_last(left, BS)) + E;
        if (VEC) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = *(const vec *)(data + p[i]);
        } else if (end <= stop) {
#pragma unroll
            for (int i = 0; i < N; ++i) v[i] = *(const vec_anywhere *)(data + p[i]);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int u = 0; u < E; ++u) v[i][u] = data[min(p[i] + u, stop - 1)];
        }
        furthest += ACROSS ? BS * stride : BS;
#pragma unroll
        for (int i = 0; i < N; ++i) at[i] += ACROSS ? BS * stride : BS;
    }
    __device__ __forceinline__ void store(DEAR_LDS T *s, int left) {
        if (left < BS)
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int u = 0; u < E; ++u)
                    if ((ACROSS ? row + i * ROWS : col + u) >= left) v[i][u] = (T)0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) *(DEAR_LDS vec *)(s + (row + i * ROWS) * tile<T, W>::stride + col) = v[i];
    }
};

// Rows row0 .. +31 of a tile along the summed index, in the order of a result's rows, which `transposed` reads in.
template <int W> __device__ __forceinline__ bf16x8 along(const DEAR_LDS bf16 *s, int row0, int kk, int lane) {
    const DEAR_LDS bf16 *p = s + (row0 + (lane & 31)) * tile<bf16, W>::stride + 16 * kk + 4 * (lane >> 5);
    const bf16x4 a = *(const DEAR_LDS bf16x4 *)p, b = *(const DEAR_LDS bf16x4 *)(p + 8);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <int W> __device__ __forceinline__ f32x8 along(const DEAR_LDS float *s, int row0, int kk, int lane) {
    const DEAR_LDS float *p = s + (row0 + (lane & 31)) * tile<float, W>::stride + 16 * kk + 4 * (lane >> 5);
    const f32x4 a = *(const DEAR_LDS f32x4 *)p, b = *(const DEAR_LDS f32x4 *)(p + 8);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// BA x 128 outputs a workgroup: four waves of 64 x 64, of 32 x 64 or, of 32 rows, of 32 x 32.  A step's operands, BS of the summed index, go
// through registers to LDS, the next one's loads beside its products.
template <typename T, bool VEC, int KIND, int BA, int BS> __global__ __launch_bounds__(THREADS, 2) void experts_kernel(params p) {
    constexpr bool A_ACROSS = KIND == WEIGHT_GRAD, B_ACROSS = KIND != LINEAR;
    constexpr int WAVES_A = BA == 32 ? 1 : 2, WAVES_B = 4 / WAVES_A, F = BA / WAVES_A / 32, G = BB / WAVES_B / 32;
    typedef stage<T, VEC, A_ACROSS, BA, BS> stage_a;
    typedef stage<T, VEC, B_ACROSS, BB, BS> stage_b;
    constexpr int BYTES_A = tile<T, stage_a::W>::bytes(A_ACROSS ? BS : BA), BYTES_B = tile<T, stage_b::W>::bytes(B_ACROSS ? BS : BB);
    __shared__ __attribute__((aligned(16))) char lds[BYTES_A + BYTES_B];
    DEAR_LDS T *as = (DEAR_LDS T *)lds, *bs = (DEAR_LDS T *)(lds + BYTES_A);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned per = (unsigned)p.a_tiles * p.b_tiles, id = blockIdx.x % per, block = blockIdx.x / per;
    const unsigned which = KIND == WEIGHT_GRAD ? block / (unsigned)p.experts : block;  // split
    const part t = KIND == WEIGHT_GRAD ? rows_of(p, (int)(block - which * (unsigned)p.experts)) : find<BA>(p, (int)(id / p.b_tiles));
    if (t.none) return;
    const int b0 = (int)(id % p.b_tiles) * BB, a0 = KIND == WEIGHT_GRAD ? (int)(id / p.b_tiles) * BA : 0;
    const bool behind = KIND != WEIGHT_GRAD && t.expert == p.experts;  // rows of no expert
    const int64_t chunk = KIND == WEIGHT_GRAD ? ((t.end - t.begin + p.splits - 1) / p.splits + BS - 1) / BS * BS : p.chunk;
    const int64_t begin = (KIND == WEIGHT_GRAD ? t.begin : 0) + which * chunk;
    const int64_t end = behind ? 0 : min(begin + chunk, KIND == WEIGHT_GRAD ? t.end : (int64_t)p.sum);
    const T *a = (const T *)p.a, *b = (const T *)p.b;
    if (KIND == LINEAR) b += (int64_t)t.expert * p.n_b * p.sum;
    if (KIND == INPUT_GRAD) b += (int64_t)t.expert * p.sum * p.n_b;
    f32x16 acc[F][G] = {};
    stage_a sa;
    stage_b sb;
    const int64_t out0 = KIND == WEIGHT_GRAD ? a0 : t.first, outs = (KIND == WEIGHT_GRAD ? p.n_a : t.end) - out0;
    auto left = [&](int64_t s0) { return (int)min(end - s0, (int64_t)BS); };
    if (begin < end) {
        sa.aim(a, p.a_stride, p.rows, KIND == WEIGHT_GRAD ? p.n_a : p.sum, out0, outs, begin);
        sb.aim(b, p.b_stride, KIND == LINEAR ? p.n_b : KIND == INPUT_GRAD ? p.sum : p.rows, KIND == LINEAR ? p.sum : p.n_b, b0, p.n_b - b0, begin);
        sa.load(left(begin)), sb.load(left(begin));
    }
    for (int64_t s0 = begin; s0 < end; s0 += BS) {
        __syncthreads();
        sa.store(as, left(s0));
        sb.store(bs, left(s0));
        __syncthreads();
        if (s0 + BS < end) sa.load(left(s0 + BS)), sb.load(left(s0 + BS));
#pragma unroll
        for (int s = 0; s < BS / 16; ++s) {
            frag<T> f[F], g[G];
#pragma unroll
            for (int u = 0; u < F; ++u) {
                const int row = (wave / WAVES_B) * F * 32 + 32 * u;
                f[u] = A_ACROSS ? transposed<stage_a::W>(as, 16 * s, row, lane) : along<stage_a::W>(as, row, s, lane);
            }
#pragma unroll
            for (int u = 0; u < G; ++u) {
                const int col = (wave % WAVES_B) * G * 32 + 32 * u;
                g[u] = B_ACROSS ? transposed<stage_b::W>(bs, 16 * s, col, lane) : along<stage_b::W>(bs, col, s, lane);
            }
#pragma unroll
            for (int u = 0; u < F; ++u)
#pragma unroll
                for (int w = 0; w < G; ++w) acc[u][w] = mma(f[u], g[w], acc[u][w]);
        }
    }
    typedef typename std::conditional<KIND == WEIGHT_GRAD, float, T>::type O;
    const int64_t row0 = KIND == WEIGHT_GRAD ? a0 : t.first, row_end = KIND == WEIGHT_GRAD ? p.n_a : t.end;
    auto store = [&](auto *out) {
        typedef typename std::remove_reference<decltype(*out)>::type to;
#pragma unroll
        for (int u = 0; u < F; ++u)
#pragma unroll
            for (int w = 0; w < G; ++w) {
                const int col = b0 + (wave % WAVES_B) * G * 32 + 32 * w + (lane & 31);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int64_t row = row0 + (wave / WAVES_B) * F * 32 + 32 * u + row_of(r, lane >> 5);
                    if (row < row_end && col < p.n_b) out[row * p.n_b + col] = (to)acc[u][w][r];
                }
            }
    };
    const int64_t first = KIND == WEIGHT_GRAD ? (int64_t)t.expert * p.n_a * p.n_b : 0;
    if (p.splits > 1) store(p.parts + which * (KIND == WEIGHT_GRAD ? p.experts * (int64_t)p.n_a : p.rows) * p.n_b + first);
    else store((O *)p.out + first);
}

// Sum of the splits, in their order, eight loads in flight, rounded once.
template <typename T> __global__ __launch_bounds__(256) void parts_sum_kernel(const float *parts, int splits, int64_t n, T *out) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float s = 0.f;
    for (int k = 0; k < splits; k += 8) {
        float x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = parts[min(k + u, splits - 1) * n + i];
#pragma unroll
        for (int u = 0; u < 8; ++u) s += k + u < splits ? x[u] : 0.f;
    }
    out[i] = (T)s;
}

// ------------------------------------------------------------------------------------ bf16, whole vectors
// SIZE x SIZE outputs a workgroup, a quarter of them a wave, 64 of the summed index a step.  In tiles of 256 a wave's sums fill half of a
// SIMD's registers, so that it reads 16 KB from LDS for 64 matrix instructions; it is then alone on its SIMD, and all that is not a matrix
// instruction has to be issued beside them: fragments of a quarter step are read while those of the one before are multiplied, across the
// barrier of a step too, and memory fills one half of LDS by itself while the other is read.  Workgroups stay for several tiles: the first
// step of the next tile is loaded beside the last one of this, and sums are stored beside the loads of the second.
constexpr int TABLE = 1024;     // experts that the table in LDS has places for

// An operand's step in LDS, for SIZE outputs that WAYS groups of waves have a part of each.  Along the summed index: SIZE rows of 64 values,
// read in rows.  Across it: 64 rows of 128 columns, twice in tiles of 256, read with transposing reads so that slots 0 .. 7 of half h are
// rows 8 h .. 8 h + 7 of sixteen, as in rows.  Pieces of 16 bytes are turned within their row, as memory fills it, so that reads of several
// rows lie in different banks.
template <bool ACROSS, int SIZE, int WAYS> struct side {
    static constexpr int F = SIZE / WAYS / 32, LOADS = SIZE / 32;  // fragments of a wave; its loads for a step, 1 KB each
    static constexpr int BYTES = SIZE * WS * 2;
    static_assert(!ACROSS || SIZE >= 128, "rows of 128 columns");
    __device__ static __forceinline__ int turn(int row) {
        return ACROSS ? (row & 3) << 2 | (row >> 2 & 3) : (row >> 1 & 1) << 2 | (row >> 2 & 3);
    }
    uint32_t read_at[ACROSS ? 2 * F : 4];  // bytes, of this lane's reads: by columns and rows, or by quarter steps
    uint32_t load_at[LOADS];               // bytes from the step's place in memory, of this lane's pieces
    int lane, wave;

    // which: the wave's part of the tile's outputs
    __device__ __forceinline__ side(int which, int lane_, int wave_) : lane(lane_), wave(wave_) {
        if (ACROSS) {
            const int row = 8 * (lane >> 5) + (lane & 15) / 4, c = 2 * (lane >> 4 & 1) + (lane & 3) / 2 + (SIZE == 128 ? 4 * F * which : 0);
#pragma unroll
            for (int u = 0; u < F; ++u)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    read_at[2 * u + k] = (SIZE == 256 ? which * 16384 : 0) + (row + 4 * k) * 256 + ((4 * u + c) ^ turn(row + 4 * k)) * 16 + 8 * (lane & 1);
        } else {
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
                read_at[kk] = which * (SIZE / WAYS * 128) + (lane & 31) * 128 + ((2 * kk + (lane >> 5)) ^ turn(lane & 31)) * 16;
        }
    }
    // Fragment u (32 outputs) of quarter step kk.
    __device__ __forceinline__ bf16x8 read(const DEAR_LDS char *s, int u, int kk) const {
        if (ACROSS) {
            const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((DEAR_LDS bf16x4 *)(s + read_at[2 * u] + 4096 * kk));
            const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((DEAR_LDS bf16x4 *)(s + read_at[2 * u + 1] + 4096 * kk));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
        return *(const DEAR_LDS bf16x8 *)(s + read_at[kk] + 4096 * u);
    }
    // Row of the operand's tile, and first value of the row, of this lane's load i; where the load puts this wave's pieces.
    __device__ __forceinline__ int first(int i) const {
        return ACROSS ? (SIZE == 256 ? wave % 2 * 32 : wave * 16) + 4 * i : wave * (SIZE / 4) + 8 * i;
    }
    __device__ __forceinline__ int row(int i) const { return first(i) + (ACROSS ? lane / 16 : lane / 8); }
    __device__ __forceinline__ int value(int i) const {
        return ACROSS ? (SIZE == 256 ? wave / 2 * 128 : 0) + (lane % 16 ^ turn(row(i))) * 8 : (lane % 8 ^ turn(row(i))) * 8;
    }
    __device__ __forceinline__ DEAR_LDS char *place(DEAR_LDS char *to, int i) const {
        return to + (ACROSS ? (SIZE == 256 ? wave / 2 * 16384 : 0) + first(i) * 256 : first(i) * 128);
    }
    // outputs: how many of the tile's there are, one at least; beyond them the last row, or the first values, again.  left: of the summed
    // index in the step, one at least; beyond it what is there already is read again, to be made zeros.
    __device__ __forceinline__ void aim(uint32_t stride, int outputs, int left) {
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const int r = min(row(i), (ACROSS ? left : outputs) - 1), v = value(i);
            load_at[i] = (uint32_t)r * stride + (v < (ACROSS ? outputs : left) ? v : 0) * 2;
        }
    }
    // Eighths from .. to of the loads.
    __device__ __forceinline__ void load(const char *at, DEAR_LDS char *s, int from, int to) const {
#pragma unroll
        for (int i = LOADS * from / 8; i < LOADS * to / 8; ++i) load_to_lds(at + load_at[i], place(s, i));
    }
    // Zeros behind the first `left` of the summed index, in the pieces that this lane has loaded.
    __device__ __forceinline__ void clear(DEAR_LDS char *to, int left) const {
#pragma unroll
        for (int i = 0; i < LOADS; ++i)
            if ((ACROSS ? row(i) : value(i)) >= left) *(DEAR_LDS u32x4 *)(place(to, i) + lane * 16) = u32x4{0, 0, 0, 0};
    }
};

// A tile: its operands' first step in memory and its place among the outputs.
struct wide_tile {
    const char *a, *b;
    int64_t sum;           // of the summed index
    int64_t out, row_end;  // first row of the outputs, behind the last (of a weight gradient in all experts' rows)
    int32_t col, a_rows, b_rows;
    bool none;
};

// A tile's sums to its outputs.  A lane has, of a row, columns apart: through 4 KB of LDS a wave, 32 rows of a line at a time, neighbouring lanes
// get a whole one.  Stored from the lanes they come as quarters of lines (16384 x 4096 x 1024 145 us, so 132); and past the caches, which the
// operands want (8192 x 8192 x 8192 weight gradient 830 us, so 798).  PARTS: outputs are fp32 sums.
template <int KIND, int SA, int SB, bool PARTS, int F, int G>
__device__ __forceinline__ void store_tile(const params &p, void *outputs, const wide_tile &t, const f32x16 (&acc)[F][G], DEAR_LDS char *lines, int lane, int wave) {
    constexpr int WAYS_A = SA == 32 ? 1 : 2, WAYS_B = 4 / WAYS_A, WAVE_A = SA / WAYS_A, WAVE_B = SB / WAYS_B;
    constexpr bool F32 = KIND == WEIGHT_GRAD || PARTS;
    typedef typename std::conditional<F32, float, bf16>::type O;
    constexpr int BLOCKS = F32 || G == 1 ? 1 : 2;                  // of 32 columns in a line
    constexpr int PIECES = BLOCKS * 32 * (int)sizeof(O) / 16;      // of 16 bytes
    constexpr int ROWS = 64 / PIECES;                              // of a store
    auto turned = [](int row, int piece) { return row * PIECES * 16 + (piece ^ (PIECES == 8 ? row & 7 : row >> 1 & 3)) * 16; };
    DEAR_LDS char *s = lines + wave * 4096;
    const int l = lane & 31, r = lane / PIECES, line_at = turned(r, lane % PIECES);
    const int rows = (int)min(t.row_end - t.out, (int64_t)SA), cols = min(p.n_b - t.col, SB), pitch = p.n_b * (int)sizeof(O);
    const int row0 = (wave / WAYS_B) * WAVE_A + r, col0 = (wave % WAYS_B) * WAVE_B + lane % PIECES * (int)(16 / sizeof(O));
    const uint32_t off = (uint32_t)row0 * (uint32_t)pitch + col0 * (uint32_t)sizeof(O);
    char *const at = (char *)((O *)outputs + t.out * p.n_b + t.col);
    const bool whole = rows == SA && cols == SB;
#pragma unroll
    for (int u = 0; u < F; ++u)
#pragma unroll
        for (int v = 0; v < G; v += BLOCKS) {
            auto put = [&](int piece, u32x4 x) { *(DEAR_LDS u32x4 *)(s + turned(l, piece)) = x; };
            if constexpr (F32) {
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    f32x4 x;
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[k] = acc[u][v][4 * q + k];
                    put(2 * q + (lane >> 5), __builtin_bit_cast(u32x4, x));
                }
            } else {
                // the halves of the wave exchange fours of columns, and have eight in a row each
#pragma unroll
                for (int w = 0; w < BLOCKS; ++w)
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        uint32_t x[2][2];
#pragma unroll
                        for (int h = 0; h < 2; ++h)
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const f32x16 &c = acc[u][v + w];
                                const bf16x2 y = {(bf16)c[8 * q + 4 * h + 2 * k], (bf16)c[8 * q + 4 * h + 2 * k + 1]};
                                x[h][k] = __builtin_bit_cast(uint32_t, y);
                            }
                        const auto w0 = __builtin_amdgcn_permlane32_swap(x[0][0], x[1][0], false, false);
                        const auto w1 = __builtin_amdgcn_permlane32_swap(x[0][1], x[1][1], false, false);
                        put(4 * w + 2 * q + (lane >> 5), u32x4{(uint32_t)w0[0], (uint32_t)w1[0], (uint32_t)w0[1], (uint32_t)w1[1]});
                    }
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int i = 0; i < 32 / ROWS; ++i) {
                const u32x4 x = *(DEAR_LDS u32x4 *)(s + i * 1024 + line_at);
                if (whole || (row0 + 32 * u + ROWS * i < rows && col0 + 32 * v < cols))
                    __builtin_nontemporal_store(x, (u32x4 *)(at + (int64_t)(32 * u + ROWS * i) * pitch + 32 * v * (int)sizeof(O) + off));
            }
            __builtin_amdgcn_wave_barrier();
        }
}

// The tiles of SA x SB outputs that next() gives, one after another.  xa, ya and xb, yb: the operands' places for steps in turn, arrays of
// their own, so that a read from one need not wait for what memory brings to another; lines: 4 KB a wave, or null where the second step's
// place is to serve for it as well.
template <int KIND, int SA, int SB, bool PARTS, typename NEXT>
__device__ __forceinline__ void run(const params &p, void *outputs, DEAR_LDS char *xa, DEAR_LDS char *ya, DEAR_LDS char *xb, DEAR_LDS char *yb,
                                    DEAR_LDS char *lines, NEXT next) {
    constexpr bool A_ACROSS = KIND == WEIGHT_GRAD, B_ACROSS = KIND != LINEAR;
    typedef side<A_ACROSS, SA, 2> side_a;
    typedef side<B_ACROSS, SB, 2> side_b;
    constexpr int F = side_a::F, G = side_b::F;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    side_a a(wave / 2, lane, wave);
    side_b b(wave % 2, lane, wave);
    const uint32_t a_stride = (uint32_t)p.a_stride * 2, b_stride = (uint32_t)p.b_stride * 2;
    const char *from_a = nullptr, *from_b = nullptr;
    int64_t left = 0;  // of the summed index, from the step that is loaded next on
    wide_tile now = next(), then = now, done = now;
    if (now.none) return;
    auto aim = [&](const wide_tile &t, int rows) {
        a.aim(a_stride, t.a_rows, rows);
        b.aim(b_stride, t.b_rows, rows);
    };
    auto begin = [&](const wide_tile &t) {
        from_a = t.a, from_b = t.b, left = t.sum;
        aim(t, (int)min(left, (int64_t)WS));
    };
    auto loaded = [&] {
        from_a += A_ACROSS ? (int64_t)WS * a_stride : WS * 2;
        from_b += B_ACROSS ? (int64_t)WS * b_stride : WS * 2;
        left -= WS;
    };
    auto load = [&](DEAR_LDS char *to_a, DEAR_LDS char *to_b, int from, int to) { a.load(from_a, to_a, from, to), b.load(from_b, to_b, from, to); };

    f32x16 acc[F][G];
    struct {
        bf16x8 a[F], b[G];
    } f, g;
    constexpr std::true_type yes;
    constexpr std::false_type no;
    auto read = [&](auto &x, const DEAR_LDS char *from_a, const DEAR_LDS char *from_b, int kk) {
#pragma unroll
        for (int u = 0; u < F; ++u) x.a[u] = a.read(from_a, u, kk);
#pragma unroll
        for (int u = 0; u < G; ++u) x.b[u] = b.read(from_b, u, kk);
    };
    auto multiply = [&](auto &x, auto first) {  // first: of a tile's sums
#pragma unroll
        for (int u = 0; u < F; ++u)
#pragma unroll
            for (int v = 0; v < G; ++v)  // a lane has one row of the outputs
                acc[u][v] = mma(x.b[v], x.a[u], decltype(first)::value ? f32x16{} : acc[u][v]);
    };
    // Beside the matrix instructions of a quarter step its reads, and `loads` loads.
    auto beside = [](auto loads) {
        constexpr int N = F * G, READS = F * (A_ACROSS ? 2 : 1) + G * (B_ACROSS ? 2 : 1), LOADS = decltype(loads)::value;
#pragma unroll
        for (int u = 0; u < N; ++u) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
#pragma unroll
            for (int k = u * READS / N; k < (u + 1) * READS / N; ++k) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
#pragma unroll
            for (int k = u * LOADS / N; k < (u + 1) * LOADS / N; ++k) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
        }
    };
    // The step in x and y is there, and all waves have read the one that is loaded over.  valid: of its part of the sum.
    auto ready = [&](DEAR_LDS char *x, DEAR_LDS char *y, int64_t valid) {
        __builtin_amdgcn_s_waitcnt(0x0070);
        if (valid < WS) {
            a.clear(x, (int)max(valid, (int64_t)0)), b.clear(y, (int)max(valid, (int64_t)0));
            __builtin_amdgcn_s_waitcnt(0xc07f);
        }
        __syncthreads();
    };
    // What comes behind this tile's whole steps: a part of one, or (sums are made of pairs of steps) nothing, for which its first again.
    auto rest = [&](const wide_tile &t) {
        if (left >= WS) return;
        if (left <= 0) from_a = t.a, from_b = t.b;
        aim(t, (int)(left > 0 ? left : 1));
    };
    // A step of a tile but its first: with the products that are left over from the step before.
    auto step = [&](DEAR_LDS char *x, DEAR_LDS char *y, DEAR_LDS char *to_a, DEAR_LDS char *to_b) {
        // half of the loads in the first quarter, and none in the last: all in the first one wait for one another's way (8192 x 8192 x 8192
        // 1013 us, so 947), and spread over all they come too late (988)
        constexpr int A = side_a::LOADS, B = side_b::LOADS;
        typedef std::integral_constant<int, A * 4 / 8 + B * 4 / 8> half;
        typedef std::integral_constant<int, A * 6 / 8 + B * 6 / 8 - half::value> fourth;
        typedef std::integral_constant<int, A + B - half::value - fourth::value> last;
        typedef std::integral_constant<int, 0> none;
        read(f, x, y, 0);
        load(to_a, to_b, 0, 4);
        multiply(g, no);
        beside(half());
        read(g, x, y, 1);
        load(to_a, to_b, 4, 6);
        multiply(f, no);
        beside(fourth());
        read(f, x, y, 2);
        load(to_a, to_b, 6, 8);
        multiply(g, no);
        beside(last());
        read(g, x, y, 3);
        multiply(f, no);
        beside(none());
        loaded();
    };

    begin(now);
    load(xa, ya, 0, 8);
    loaded();
    bool any = false;  // sums of a tile to store
    for (;;) {
        if (!now.none) rest(now);
        ready(xa, ya, left + WS);
        if (lines && !now.none) load(xb, yb, 0, 8);
        if (any) {
            multiply(g, no);
            store_tile<KIND, SA, SB, PARTS>(p, outputs, done, acc, lines ? lines : yb, lane, wave);
        }
        if (now.none) break;
        if (!lines) {
            if (any) __syncthreads();  // all waves' lines are out of the second step's place
            load(xb, yb, 0, 8);
        }
        loaded();
        read(f, xa, ya, 0);
        read(g, xa, ya, 1);
        multiply(f, yes);
        read(f, xa, ya, 2);
        multiply(g, no);
        read(g, xa, ya, 3);
        multiply(f, no);
        for (;;) {
            const int64_t valid = left + WS;
            const bool last = left <= 0;
            if (last) {
                then = next();
                begin(then.none ? now : then);  // (behind the last tile its first step again, which nothing reads)
            } else {
                rest(now);
            }
            ready(xb, yb, valid);
            step(xb, yb, xa, ya);
            if (last) break;
            const int64_t more = left + WS;
            rest(now);
            ready(xa, ya, more);
            step(xa, ya, xb, yb);
        }
        done = now, now = then, any = true;
    }
}

// What a workgroup knows of the experts: rows up to and with each one's, and its tiles or, of a weight gradient, experts by their rows.
struct experts_table {
    int32_t ends[TABLE], upto[TABLE];
};

template <int KIND, int SIZE> __device__ __forceinline__ void fill(experts_table &x, const params &p) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, rows = (int)p.rows;
    int32_t before = 0, tiles = 0;
    for (int e0 = 0; e0 < p.experts; e0 += 64) {  // each wave for itself, with the same values
        const int e = e0 + lane;
        int32_t end = e < p.experts ? min(max(p.ends[e], 0), rows) : 0;
        end = max(max_before(end, lane), before);
        int32_t begin = __shfl_up(end, 1);
        if (lane == 0) begin = before;
        const int32_t all = tiles + sum_before((int32_t)(((uint32_t)(end - begin) + SIZE - 1) / SIZE), lane);
        if (e < p.experts && wave == 0) {
            x.ends[e] = end;
            if (KIND != WEIGHT_GRAD) x.upto[e] = all;
        }
        before = __builtin_amdgcn_readfirstlane(__shfl(end, 63));
        tiles = __builtin_amdgcn_readfirstlane(__shfl(all, 63));
    }
    __syncthreads();
    if (KIND != WEIGHT_GRAD) return;
    // experts with most rows first, so that what is left in the end is short; of more than there are threads as they come
    for (int e = threadIdx.x; e < p.experts; e += THREADS) {
        int rank = e;
        if (p.experts <= THREADS) {
            const int mine = x.ends[e] - (e ? x.ends[e - 1] : 0);
            rank = 0;
            int begin = 0;
            for (int i = 0; i < p.experts; ++i) {
                const int end = x.ends[i], n = end - begin;
                rank += n > mine || (n == mine && i < e);
                begin = end;
            }
        }
        x.upto[rank] = e;
    }
    __syncthreads();
}

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Rows of no expert: zeros.
template <typename O> __device__ __forceinline__ void zero_rows(const params &p, O *outputs, int64_t first, int64_t behind) {
    constexpr int E = 16 / sizeof(O);
    const int64_t n = (behind - first) * (p.n_b / E);
    u32x4 *out = (u32x4 *)(outputs + first * p.n_b);
    for (int64_t i = (int64_t)blockIdx.x * THREADS + threadIdx.x; i < n; i += (int64_t)gridDim.x * THREADS) out[i] = u32x4{0, 0, 0, 0};
}

// Tile (a_tile, b_tile) of the experts' tiles of SA x SB, or a part of it: rows and columns from `down` and `across` on.  Its sum is 0 where
// there are no outputs.
template <int KIND, int SA, int SB>
__device__ __forceinline__ wide_tile tile_of(const experts_table &x, const params &p, int rank, int a_tile, int b_tile, int down, int across) {
    wide_tile t;
    t.none = false;
    t.col = b_tile * SB + across;
    t.b_rows = p.n_b - t.col;
    int expert = 0;
    if (KIND == WEIGHT_GRAD) {
        expert = uniform(x.upto[rank]);
        const int begin = expert ? uniform(x.ends[expert - 1]) : 0, row = a_tile * SA + down;
        t.sum = uniform(x.ends[expert]) - begin;
        t.a_rows = p.n_a - row;
        t.a = (const char *)p.a + ((int64_t)begin * p.a_stride + row) * 2;
        t.b = (const char *)p.b + ((int64_t)begin * p.b_stride + t.col) * 2;
        t.out = (int64_t)expert * p.n_a + row, t.row_end = (int64_t)(expert + 1) * p.n_a;
    } else {
        const int lane = threadIdx.x & 63;
        for (int e0 = 0; e0 < p.experts; e0 += 64) {
            const uint64_t found = __ballot(x.upto[min(e0 + lane, p.experts - 1)] > a_tile);
            if (found) {
                expert = e0 + (int)__builtin_ctzll(found);
                break;
            }
        }
        const int begin = expert ? uniform(x.ends[expert - 1]) : 0, end = uniform(x.ends[expert]);
        const int64_t first = begin + (int64_t)(a_tile - (expert ? uniform(x.upto[expert - 1]) : 0)) * SA + down;
        t.sum = p.sum;
        t.a_rows = (int)(end - first);
        t.a = (const char *)p.a + first * p.a_stride * 2;
        t.b = (const char *)p.b + ((int64_t)expert * p.sum * p.n_b + (KIND == LINEAR ? (int64_t)t.col * p.sum : t.col)) * 2;
        t.out = first, t.row_end = end;
    }
    if (t.a_rows <= 0 || t.b_rows <= 0) t.sum = 0;
    return t;
}

// A weight gradient's tile of an expert without rows.
template <int SIZE> __device__ __forceinline__ void zero_tile(const params &p, const wide_tile &t) {
    for (int i = threadIdx.x; i < SIZE * SIZE / 4; i += THREADS) {
        const int64_t row = t.out + i / (SIZE / 4);
        const int col = t.col + i % (SIZE / 4) * 4;
        if (row < t.row_end && col < p.n_b) *(u32x4 *)((float *)p.out + row * p.n_b + col) = u32x4{0, 0, 0, 0};
    }
}

// Item i of a column strip's order: strips four tiles wide, so that neighbours share rows and columns.
struct in_strips {
    int a, b;
    __device__ __forceinline__ in_strips(unsigned i, unsigned a_tiles, unsigned b_tiles) {
        const unsigned strip = i / (4u * a_tiles), wide = min(4u, b_tiles - 4 * strip), in = i - strip * 4 * a_tiles;
        a = (int)(in / wide), b = (int)(4 * strip + in % wide);
    }
};

// Tiles of SA x 128 outputs of splits of the sum, one after another.
template <int KIND, int SA, bool PARTS> __device__ __forceinline__ wide_tile few_tile(const experts_table &table, const params &p, unsigned &item) {
    const unsigned b_tiles = (unsigned)p.b_tiles, a_tiles = (unsigned)uniform(table.upto[p.experts - 1]), per = a_tiles * b_tiles;
    wide_tile t;
    t.none = item >= per * (PARTS ? p.splits : 1);
    if (t.none) return t;
    const unsigned split = PARTS ? item / per : 0;
    const in_strips at(item - split * per, a_tiles, b_tiles);
    t = tile_of<KIND, SA, 128>(table, p, 0, at.a, at.b, 0, 0);
    if (PARTS) {
        const int64_t begin = (int64_t)split * p.chunk;  // below the sum's end, as the host has it
        t.a += begin * 2;
        t.b += (KIND == LINEAR ? begin : begin * p.b_stride) * 2;
        t.sum = min((int64_t)p.chunk, t.sum - begin);
        const int64_t rows = (int64_t)split * p.rows;  // the split's outputs are as many rows further on
        t.out += rows, t.row_end += rows;
    }
    item += gridDim.x;
    return t;
}

// Zeros in the rows of no expert, in all splits' sums.
template <bool PARTS> __device__ __forceinline__ void few_rest(const experts_table &table, const params &p) {
    typedef typename std::conditional<PARTS, float, bf16>::type O;
    for (int s = 0; s < (PARTS ? p.splits : 1); ++s)
        zero_rows(p, PARTS ? (O *)p.parts + (int64_t)s * p.rows * p.n_b : (O *)p.out, uniform(table.ends[p.experts - 1]), p.rows);
}

// Waits for what is read or loaded, but for the last n times EACH loads, n <= MOST.
template <int MOST, int EACH> __device__ __forceinline__ void wait_for_all_but(int n) {
    if constexpr (MOST > 0)
        if (n < MOST) return wait_for_all_but<MOST - 1, EACH>(n);
    __builtin_amdgcn_s_waitcnt(0x0070 | (MOST * EACH & 15) | (MOST * EACH >> 4) << 14);
}

// The tiles of SA x 128 outputs that next() gives, with D - 1 steps under way.  A wave waits for its own loads by the count of those behind
// them, and the barrier is bare: __syncthreads() waits for all loads.  x, y: the operands' places for D steps in turn; the first of y holds
// 16 KB.
template <int KIND, int SA, bool PARTS, int D, typename NEXT>
__device__ __forceinline__ void run_ring(const params &p, void *outputs, DEAR_LDS char *const (&x)[D], DEAR_LDS char *const (&y)[D], NEXT next) {
    constexpr bool B_ACROSS = KIND == INPUT_GRAD;
    constexpr int SB = 128, WAYS_A = SA == 32 ? 1 : 2, WAYS_B = 4 / WAYS_A;
    typedef side<false, SA, WAYS_A> side_a;
    typedef side<B_ACROSS, SB, WAYS_B> side_b;
    constexpr int F = side_a::F, G = side_b::F;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    side_a a(wave / WAYS_B, lane, wave);
    side_b b(wave % WAYS_B, lane, wave);
    const uint32_t a_stride = (uint32_t)p.a_stride * 2, b_stride = (uint32_t)p.b_stride * 2;

    for (;;) {
        const wide_tile t = next();
        if (t.none) return;
        const int steps = (int)((t.sum + WS - 1) / WS), last = (int)(t.sum - (int64_t)(steps - 1) * WS);  // of the sum in the last step
        a.aim(a_stride, t.a_rows, WS), b.aim(b_stride, t.b_rows, WS);
        const char *from_a = t.a, *from_b = t.b;
        auto load = [&](int step, DEAR_LDS char *to_a, DEAR_LDS char *to_b) {
            if (step == steps - 1 && last < WS) a.aim(a_stride, t.a_rows, last), b.aim(b_stride, t.b_rows, last);
            a.load(from_a, to_a, 0, 8), b.load(from_b, to_b, 0, 8);
            from_a += WS * 2, from_b += B_ACROSS ? (int64_t)WS * b_stride : WS * 2;
        };
        __syncthreads();  // what is loaded over has been read
#pragma unroll
        for (int k = 0; k < D - 1; ++k)
            if (k < steps) load(k, x[k], y[k]);
        f32x16 acc[F][G] = {};
        struct {
            bf16x8 a[F], b[G];
        } q[4];
        auto read = [&](auto &q, const DEAR_LDS char *s, const DEAR_LDS char *r, int kk) {
#pragma unroll
            for (int u = 0; u < F; ++u) q.a[u] = a.read(s, u, kk);
#pragma unroll
            for (int u = 0; u < G; ++u) q.b[u] = b.read(r, u, kk);
        };
        auto multiply = [&](auto &q) {
#pragma unroll
            for (int u = 0; u < F; ++u)
#pragma unroll
                for (int v = 0; v < G; ++v) acc[u][v] = mma(q.b[v], q.a[u], acc[u][v]);
        };
        for (int base = 0; base < steps; base += D) {
#pragma unroll
            for (int k = 0; k < D; ++k) {
                const int step = base + k;
                if (step < steps) {
                    // this step is there, of all waves, and all have read the one that is loaded over: its own loads by the count of those behind them
                    wait_for_all_but<D - 2, side_a::LOADS + side_b::LOADS>(steps - 1 - step);
                    if (step == steps - 1 && last < WS) {
                        a.clear(x[k], last), b.clear(y[k], last);
                        __builtin_amdgcn_s_waitcnt(0xc07f);
                    }
                    asm volatile("" ::: "memory");
                    __builtin_amdgcn_s_barrier();
                    asm volatile("" ::: "memory");
                    // all of the step's reads before its products
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) read(q[kk], x[k], y[k], kk);
                    __builtin_amdgcn_sched_barrier(0);
                    if (step + D - 1 < steps) load(step + D - 1, x[(k + D - 1) % D], y[(k + D - 1) % D]);
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) multiply(q[kk]);
                }
            }
        }
        __syncthreads();
        store_tile<KIND, SA, SB, PARTS>(p, outputs, t, acc, y[0], lane, wave);
    }
}

// Tiles of 256.  Items go to the eight XCDs in runs of 32, one for each of its CUs; of a weight gradient, whose tiles differ, every other round
// backwards.  What fills a last round by half at most goes in quarters, tiles of 128: 256 of them take 0.38 of a round of tiles (sums of 4096:
// 40 of 106 us), so that one or two rounds of quarters are ahead of a round, and three are not (12288 x 1024 x 4096 126 against 106 us).  Where
// it fills no more than a sixteenth, 32 x 128 outputs a CU take 25 us in place of 40 (16385 x 4096 x 1024, input gradient, 148 to 132 us).
template <int KIND> __global__ __launch_bounds__(THREADS, 1) void experts_wide_kernel(params p) {
    constexpr int BYTES = 256 * WS * 2;
    __shared__ __attribute__((aligned(16))) char a0[BYTES], a1[BYTES], b0[BYTES], b1[BYTES], lines[THREADS / 64 * 4096];
    __shared__ experts_table table;
    fill<KIND, 256>(table, p);
    const unsigned b_tiles = (unsigned)p.b_tiles, a_tiles = KIND == WEIGHT_GRAD ? (unsigned)p.a_tiles : (unsigned)uniform(table.upto[p.experts - 1]);
    const unsigned per = a_tiles * b_tiles, items = KIND == WEIGHT_GRAD ? per * p.experts : per, over = items % CUS;
    const unsigned whole = over <= MOST_IN_QUARTERS ? items - over : items;
    if (KIND != WEIGHT_GRAD) zero_rows(p, (bf16 *)p.out, uniform(table.ends[p.experts - 1]), p.rows);
    auto xa = (DEAR_LDS char *)a0, ya = (DEAR_LDS char *)b0, xb = (DEAR_LDS char *)a1, yb = (DEAR_LDS char *)b1;
    unsigned round = 0;
    run<KIND, 256, 256, false>(p, p.out, xa, ya, xb, yb, (DEAR_LDS char *)lines, [&] {
        wide_tile t;
        for (;;) {
            const unsigned in_round = blockIdx.x % 8 * 32 + blockIdx.x / 8;
            const unsigned item = round * CUS + (KIND == WEIGHT_GRAD && round % 2 ? CUS - 1 - in_round : in_round);
            t.none = round * CUS >= whole;
            if (t.none) return t;
            ++round;
            if (item >= whole) continue;
            const in_strips at(item % per, a_tiles, b_tiles);
            t = tile_of<KIND, 256, 256>(table, p, (int)(item / per), at.a, at.b, 0, 0);
            if (t.sum > 0) return t;
            zero_tile<256>(p, t);
        }
    });
    if (whole == items) return;
    __syncthreads();
    if constexpr (KIND != WEIGHT_GRAD) {
        if (over <= MOST_SMALL) {
            constexpr int A = 32 * WS * 2;
            DEAR_LDS char *const x[4] = {xa, xb, ya, yb}, *const y[4] = {xa + A, xb + A, ya + A, yb + A};
            unsigned item = blockIdx.x;
            run_ring<KIND, 32, false, 4>(p, p.out, x, y, [&] {
                wide_tile t;
                for (;;) {
                    t.none = item >= 16 * over;
                    if (t.none) return t;
                    const in_strips at((whole + item / 16) % per, a_tiles, b_tiles);
                    t = tile_of<KIND, 256, 256>(table, p, 0, at.a, at.b, (int)(item / 2 % 8) * 32, (int)(item % 2) * 128);
                    item += CUS;
                    if (t.sum > 0) return t;
                }
            });
            return;
        }
    }
    round = 0;
    run<KIND, 128, 128, false>(p, p.out, xa, ya, xb, yb, (DEAR_LDS char *)lines, [&] {
        wide_tile t;
        for (;;) {
            const unsigned item = round * CUS + blockIdx.x;
            t.none = round * CUS >= 4 * over;
            if (t.none) return t;
            ++round;
            if (item >= 4 * over) continue;
            const in_strips at((whole + item / 4) % per, a_tiles, b_tiles);
            t = tile_of<KIND, 256, 256>(table, p, (int)((whole + item / 4) / per), at.a, at.b, (int)(item / 2 % 2) * 128, (int)(item % 2) * 128);
            if (t.sum > 0) return t;
            if (KIND == WEIGHT_GRAD && t.a_rows > 0 && t.b_rows > 0) zero_tile<128>(p, t);
        }
    });
}

// Tiles of 128 x 128 for fewer rows, two workgroups a CU, and sums in several splits (PARTS) where there are few tiles.
template <int KIND, bool PARTS> __global__ __launch_bounds__(THREADS, 2) void experts_few_kernel(params p) {
    __shared__ __attribute__((aligned(16))) char a0[128 * WS * 2], a1[128 * WS * 2], b0[128 * WS * 2], b1[128 * WS * 2];
    __shared__ experts_table table;
    fill<KIND, 128>(table, p);
    few_rest<PARTS>(table, p);
    unsigned item = blockIdx.x;
    run<KIND, 128, 128, PARTS>(p, PARTS ? (void *)p.parts : p.out, (DEAR_LDS char *)a0, (DEAR_LDS char *)b0, (DEAR_LDS char *)a1, (DEAR_LDS char *)b1,
                               nullptr, [&] { return few_tile<KIND, 128, PARTS>(table, p, item); });
}

// The same tiles, of 32 rows two a CU or of 128 one, with two steps under way where the third is multiplied: what they wait for is the weights'
// way from memory (32 rows, 4096 x 1024 over 8 14.8 us, 4.5 TB/s from HBM; 12.6 where the last cache holds them).  With one step under way
// 18.2 and 13.4 us, with five 15.3 and 14.4, with two pairs of steps 15.1 and 14.1.
template <int KIND, int SA, bool PARTS> __global__ __launch_bounds__(THREADS, SA == 32 ? 2 : 1) void experts_ring_kernel(params p) {
    constexpr int A = SA * WS * 2, B = 128 * WS * 2;
    // in arrays of their own: a read from one need not wait for what memory brings to another
    __shared__ __attribute__((aligned(16))) char a0[A], a1[A], a2[A], b0[B], b1[B], b2[B];
    __shared__ experts_table table;
    fill<KIND, SA>(table, p);
    few_rest<PARTS>(table, p);
    unsigned item = blockIdx.x;
    DEAR_LDS char *const x[3] = {(DEAR_LDS char *)a0, (DEAR_LDS char *)a1, (DEAR_LDS char *)a2};
    DEAR_LDS char *const y[3] = {(DEAR_LDS char *)b0, (DEAR_LDS char *)b1, (DEAR_LDS char *)b2};
    run_ring<KIND, SA, PARTS, 3>(p, PARTS ? (void *)p.parts : p.out, x, y, [&] { return few_tile<KIND, SA, PARTS>(table, p, item); });
}

// ------------------------------------------------------------------------------------ host
constexpr int64_t MAX_ROWS = INT32_MAX;
constexpr int32_t MAX_EXPERTS = 1 << 16, MAX_WIDTH = 1 << 20;

int size_of(int32_t dtype) { return dtype == DEAR_BF16 ? 2 : 4; }

int check(const dear_experts_t *x) {
    if (!x || (x->dtype != DEAR_F32 && x->dtype != DEAR_BF16) || x->rows < 0 || x->rows > MAX_ROWS) return DEAR_EINVAL;
    if (x->experts < 1 || x->experts > MAX_EXPERTS || x->outs < 1 || x->outs > MAX_WIDTH || x->ins < 1 || x->ins > MAX_WIDTH) return DEAR_EINVAL;
    return DEAR_OK;
}

int check_rows(const dear_experts_t &x, const void *p, int64_t stride, int64_t width) {
    if (x.rows > 0 && !p) return DEAR_EINVAL;
    if (x.rows > 1 && stride < width) return DEAR_EINVAL;
    return aligned(p, size_of(x.dtype)) ? DEAR_OK : DEAR_EALIGN;
}

bool vectors(const dear_experts_t &x, const void *p, int64_t stride, int64_t width) {
    const int n = size_of(x.dtype);
    return aligned(p, 16) && stride * n % 16 == 0 && width * n % 16 == 0;
}

// Whether memory can fill tiles directly: bf16 in whole vectors, with rows that 32-bit offsets reach.
template <int KIND> bool direct(const dear_experts_t &x, bool vec, const params &p) {
    const int64_t most = 1 << 22;
    if (x.dtype != DEAR_BF16 || !vec || !aligned(p.out, 16) || x.experts > TABLE || p.n_b % 8 || p.a_stride >= most || p.b_stride >= most) return false;
    const int64_t a_tiles = KIND == WEIGHT_GRAD ? ceil_div(x.outs, 256) * x.experts : x.rows / 32 + x.experts;
    return a_tiles * ceil_div(p.n_b, 128) <= INT32_MAX / 64;
}

template <int KIND> int64_t workspace_of(const dear_experts_t &x) {
    if (x.rows == 0) return 0;
    // what a call takes depends on its pointers
    const int any = choose_cut<KIND>(x, false).splits, direct = x.dtype == DEAR_BF16 ? choose_cut<KIND>(x, true).splits : 1;
    const int64_t most = any > direct ? any : direct;
    const int64_t outputs = KIND == WEIGHT_GRAD ? (int64_t)x.experts * x.outs * x.ins : x.rows * (KIND == LINEAR ? x.outs : x.ins);
    return most > 1 ? most * outputs * 4 : 0;
}

template <int KIND> int call(const dear_experts_t *x, hipStream_t stream) {
    if (int rc = check(x)) return rc;
    const bool weight = KIND != WEIGHT_GRAD;
    if (KIND != INPUT_GRAD)
        if (int rc = check_rows(*x, x->x, x->x_stride, x->ins)) return rc;
    if (KIND != LINEAR)
        if (int rc = check_rows(*x, x->dy, x->dy_stride, x->outs)) return rc;
    if (weight && x->rows == 0) return DEAR_OK;
    if (!x->ends || !x->out || (weight && !x->weight)) return DEAR_EINVAL;
    if (!aligned(x->ends, 4) || !aligned(x->out, KIND == WEIGHT_GRAD ? 4 : size_of(x->dtype)) || (weight && !aligned(x->weight, size_of(x->dtype))))
        return DEAR_EALIGN;
    const int64_t need = workspace_of<KIND>(*x);
    if (need && !x->workspace) return DEAR_EINVAL;
    if (need && !aligned(x->workspace, 256)) return DEAR_EALIGN;
    if (need > x->workspace_bytes) return DEAR_ETOOBIG;

    params p = {};
    p.ends = x->ends, p.rows = x->rows, p.experts = x->experts, p.out = x->out;
    bool vec;
    if (KIND == LINEAR) {
        p.a = x->x, p.a_stride = x->x_stride, p.b = x->weight, p.b_stride = x->ins, p.sum = x->ins, p.n_b = x->outs;
        vec = vectors(*x, p.a, p.a_stride, x->ins) && vectors(*x, p.b, p.b_stride, x->ins);
    } else if (KIND == INPUT_GRAD) {
        p.a = x->dy, p.a_stride = x->dy_stride, p.b = x->weight, p.b_stride = x->ins, p.sum = x->outs, p.n_b = x->ins;
        vec = vectors(*x, p.a, p.a_stride, x->outs) && vectors(*x, p.b, p.b_stride, x->ins);
    } else {
        p.a = x->dy, p.a_stride = x->dy_stride, p.b = x->x, p.b_stride = x->x_stride, p.n_a = x->outs, p.n_b = x->ins;
        vec = vectors(*x, p.a, p.a_stride, x->outs) && vectors(*x, p.b, p.b_stride, x->ins);
    }
    const bool is_direct = direct<KIND>(*x, vec, p);
    const choice c = choose_cut<KIND>(*x, is_direct);
    p.chunk = (int32_t)(ceil_div(ceil_div(p.sum, c.splits), WS) * WS);
    p.splits = KIND == WEIGHT_GRAD ? c.splits : (int32_t)ceil_div(p.sum, p.chunk), p.parts = (float *)x->workspace;
    if (c.how == WIDE) {
        p.a_tiles = (int32_t)ceil_div(p.n_a, 256), p.b_tiles = (int32_t)ceil_div(p.n_b, 256);
        experts_wide_kernel<KIND><<<CUS, THREADS, 0, stream>>>(p);
        return launch_status();
    }
    p.b_tiles = (int32_t)ceil_div(p.n_b, BB);
    // tiles of rows: each expert, and the rows behind the last, may have one that is not whole
    const int ba = c.how == RING32 || c.how == ANY32 ? 32 : c.how == ANY64 ? 64 : 128;
    p.a_tiles = (int32_t)(KIND == WEIGHT_GRAD ? ceil_div(x->outs, ba) : x->rows / ba + x->experts + 1);
    const int64_t groups = (int64_t)p.a_tiles * p.b_tiles * p.splits * (KIND == WEIGHT_GRAD ? x->experts : 1);
    if (groups * THREADS > MAX_THREADS) return DEAR_ETOOBIG;
    if constexpr (KIND != WEIGHT_GRAD) {
        if (is_direct) {
            const int64_t most = c.how == RING128 ? CUS : 2 * CUS;
            const unsigned n = (unsigned)(groups < most ? groups : most);
            auto by_parts = [&](auto parts) {
                constexpr bool PARTS = decltype(parts)::value;
                if (c.how == RING32) experts_ring_kernel<KIND, 32, PARTS><<<n, THREADS, 0, stream>>>(p);
                else if (c.how == RING128) experts_ring_kernel<KIND, 128, PARTS><<<n, THREADS, 0, stream>>>(p);
                else experts_few_kernel<KIND, PARTS><<<n, THREADS, 0, stream>>>(p);
            };
            if (p.splits > 1) by_parts(std::true_type());
            else by_parts(std::false_type());
        }
    }
    const unsigned n = (unsigned)groups;
    auto by_rows = [&](auto t, auto v) {
        typedef decltype(t) T;
        constexpr bool VEC = decltype(v)::value;
        if constexpr (KIND != WEIGHT_GRAD) {
            if (ba == 32) return experts_kernel<T, VEC, KIND, 32, 64><<<n, THREADS, 0, stream>>>(p);
            if (ba == 64) return experts_kernel<T, VEC, KIND, 64, 32><<<n, THREADS, 0, stream>>>(p);
        }
        // longer steps have half of the barriers, and are ahead in long sums: 16000 rows, 2001 x 1003 over 2, input gradient 161 and 138 us, weight
        // gradient 126 and 108, in fp32 636 and 571, 556 and 544; 8000 rows, 1001 x 999 over 5, 52 and 55, 49 and 42; 333 rows, weight gradient 11 and 13
        if ((KIND == WEIGHT_GRAD ? p.rows / p.experts / p.splits : p.chunk) > 1024)
            return experts_kernel<T, VEC, KIND, 128, 64><<<n, THREADS, 0, stream>>>(p);
        experts_kernel<T, VEC, KIND, 128, 32><<<n, THREADS, 0, stream>>>(p);
    };
    if (c.how >= ANY32) {
        if (x->dtype == DEAR_BF16) {
            if (vec) by_rows(bf16(), std::true_type());
            else by_rows(bf16(), std::false_type());
        } else {
            if (vec) by_rows(float(), std::true_type());
            else by_rows(float(), std::false_type());
        }
    }
    if (int rc = launch_status()) return rc;
    if (p.splits > 1) {
        const int64_t all = (KIND == WEIGHT_GRAD ? (int64_t)p.experts * p.n_a : p.rows) * p.n_b;
        const unsigned blocks = (unsigned)ceil_div(all, 256);
        if (x->dtype == DEAR_BF16 && KIND != WEIGHT_GRAD) parts_sum_kernel<<<blocks, 256, 0, stream>>>(p.parts, p.splits, all, (bf16 *)p.out);
        else parts_sum_kernel<<<blocks, 256, 0, stream>>>(p.parts, p.splits, all, (float *)p.out);
        return launch_status();
    }
    return DEAR_OK;
}

template <int KIND> int workspace(const dear_experts_t *x, int64_t *bytes) {
    if (!bytes) return DEAR_EINVAL;
    if (int rc = check(x)) return rc;
    *bytes = workspace_of<KIND>(*x);
    return DEAR_OK;
}

}  // namespace

extern "C" {

int dear_expert_linear(const dear_experts_t *args, void *hip_stream) { return call<LINEAR>(args, (hipStream_t)hip_stream); }
int dear_expert_input_grad(const dear_experts_t *args, void *hip_stream) { return call<INPUT_GRAD>(args, (hipStream_t)hip_stream); }
int dear_expert_weight_grad(const dear_experts_t *args, void *hip_stream) { return call<WEIGHT_GRAD>(args, (hipStream_t)hip_stream); }

int dear_expert_linear_workspace(const dear_experts_t *args, int64_t *bytes) { return workspace<LINEAR>(args, bytes); }
int dear_expert_input_grad_workspace(const dear_experts_t *args, int64_t *bytes) { return workspace<INPUT_GRAD>(args, bytes); }
int dear_expert_weight_grad_workspace(const dear_experts_t *args, int64_t *bytes) { return workspace<WEIGHT_GRAD>(args, bytes); }

}  // extern "C"
