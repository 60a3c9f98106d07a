// Attention and its backward pass (formulas: dear_ops.h).
//
// Forward: one pass over the keys with the running maximum m and sum l of a row; a step's scores s give p = exp(s - m), and what
// was summed before is multiplied by exp(m_before - m).  Backward: p = exp(s - lse) again from q, k and lse, so that no matrix of
// queries by keys is ever in memory; with delta = dout . out (its row sum), ds = p * (dout v' - delta):
//     dq = scale * ds k      dk = scale * ds' q      dv = p' dout
// dq sums over keys and dk, dv over queries: a kernel for each, that computes s and dout v' for itself (7 products for the 5 that
// one pass needs), as sums over workgroups would take atomics, whose order changes results, or fp32 copies in memory.
//
// Layout of products.  A wave owns 32 rows of one sequence, and a step's first products are taken with these as columns: a lane
// then holds values of one of its rows (with lane + 32 all of them), so that maxima, sums, lse and delta need one value a lane and
// the result, rounded to the type, is the next product's operand as it stands.  Operands that are summed over their rows are read
// from LDS with the transposing reads.
//
// Roundings.  Scores, p, ds, maxima and all sums are fp32.  In bf16 p and ds are rounded to bf16, as the matrix instructions take
// both operands in one type: at most 2^-8 of each, as the inputs' and the output's own roundings; two parts of each would take as
// many products again.  Outputs' error against 64 bits is 1.3 to 1.4 times that of all fp32 rounded once.  The sum l is of the p
// before their rounding.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "ops_common.h"

#pragma clang fp contract(fast)

namespace {

using namespace dear_ops;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int THREADS = 256, WAVES = THREADS / 64;
constexpr int BLOCK = 32 * WAVES;  // rows that a workgroup owns: 32 for each wave
constexpr int STEP = 64;           // rows of the other sequence that it takes at a time
constexpr int KEYS = 64;           // keys of a workgroup that computes dk and dv

// Waves of a SIMD that the kernels of this part are compiled for.  With two, one's products run beside the other's softmax; wide
// rows of fp32, and wide dk and dv with their operands, take the registers of both.
template <typename T, int W> constexpr int resident(bool dkv) {
    return sizeof(T) == 2 ? (dkv && W == 128 ? 1 : 2) : (W == 128 || dkv ? 1 : 2);
}

struct heads {
    char *data;
    int64_t batch, token, head;  // strides in bytes
};

struct params {
    int32_t q_heads, kv_heads, head_dim, causal;
    int32_t q_len, kv_len, batch, tiles, q_tiles;  // tiles: of this launch; q_tiles: BLOCKs of queries
    int32_t splits;      // of the sequence that a workgroup goes through
    float scale;
    const int32_t *q_lens, *kv_lens;
    heads q, k, v, out, dout, dq, dk, dv;
    float *lse;
    // backward, of the queries of all tiles: lse * log2(e), or infinity where no key is seen, and -delta
    float *powers, *deltas;
    // with several splits, of each: outputs that are not yet joined, fp32 [split, batch, head, token, head_dim], and, forward,
    // what the powers are taken against and their sums [split, batch, head, token]
    float *part, *part_base, *part_sum;
};

__device__ __forceinline__ char *at(const heads &t, int b, int h) {
    return t.data + b * t.batch + h * t.head;
}

__device__ __forceinline__ int length(const int32_t *lens, int b, int most) {
    return lens ? min(max(lens[b], 0), most) : most;
}

// STEP rows of W values, row by row in pieces of sixteen bytes, on their way from memory to LDS: rows at or beyond
// `valid` and values at or beyond head_dim are zeros, whatever stands there.
template <typename T, int W> struct stage {
    static constexpr int PER_ROW = W * sizeof(T) / 16, N = STEP * PER_ROW / THREADS;
    u32x4 piece[N];

    __device__ __forceinline__ void load(const char *p, int64_t token, int row0, int valid, int head_dim) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * THREADS, row = row0 + c / PER_ROW, byte = c % PER_ROW * 16;
            piece[i] = u32x4{0, 0, 0, 0};
            if (row < valid && byte < head_dim * (int)sizeof(T)) piece[i] = *(const u32x4 *)(p + row * token + byte);
        }
    }
    __device__ __forceinline__ void store(DEAR_LDS T *s) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * THREADS;
            *(DEAR_LDS u32x4 *)(s + c / PER_ROW * tile<T, W>::stride + c % PER_ROW * (16 / sizeof(T))) = piece[i];
        }
    }
};

// The 32 rows of one wave as fragments, from memory.
template <typename T, int W>
__device__ __forceinline__ void load_rows(frag<T> *f, const char *p, int64_t token, int row, int valid, int head_dim, int half) {
#pragma unroll
    for (int kk = 0; kk < W / 16; ++kk) {
        const int d = 16 * kk + 8 * half;
#pragma unroll
        for (int t = 0; t < 8; ++t) f[kk][t] = (T)0.f;
        if (row < valid && d < head_dim) f[kk] = *(const frag<T> *)(p + row * token + d * sizeof(T));
    }
}

// Rows 32 db + row_of(r, half) of column `token` of a transposed result, as rows of memory.
template <typename T, int W>
__device__ __forceinline__ void store_row(char *p, const f32x16 *x, float factor, int head_dim, int half) {
#pragma unroll
    for (int db = 0; db < W / 32; ++db)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int d = 32 * db + 8 * g + 4 * half;
            if (d < head_dim) {
                typedef T vec __attribute__((ext_vector_type(4)));
                vec o;
#pragma unroll
                for (int t = 0; t < 4; ++t) o[t] = (T)(x[db][4 * g + t] * factor);
                *(vec *)(p + d * sizeof(T)) = o;
            }
        }
}

// Workgroup -> (batch, head, tile, split), for `heads` heads of which `shared` neighbours read the same keys.  Workgroups go to
// the eight XCDs in turn.  Where it divides evenly an XCD gets whole groups of heads (every eighth, so that sequences of
// different lengths are spread), or at least whole heads; it takes them one after another with all their tiles, which find
// the other sequence in its L2 cache, or, in a causal call, whose tiles are numbered from the longest on, the same tile of
// all its heads and then the next, so that the shortest come last.
__device__ __forceinline__ void place(const params &a, unsigned heads, unsigned shared, int &b, int &h, int &t, int &split) {
    const unsigned pairs = heads * a.batch, tiles = a.tiles;
    unsigned pair, id = blockIdx.x % (pairs * tiles), xcd = 0, own = pairs;
    split = blockIdx.x / (pairs * tiles);
    if (pairs % 8 == 0) xcd = id % 8, id /= 8, own = pairs / 8;
    t = a.causal ? id / own : id % tiles;
    pair = a.causal ? id % own : id / tiles;
    if (pairs / shared % 8 == 0) pair = (pair / shared * 8 + xcd) * shared + pair % shared;
    else pair += xcd * own;
    b = pair / heads;
    h = pair % heads;
}

// The split's share of begin .. end: whole steps.
__device__ __forceinline__ void share(const params &a, int split, int &begin, int &end) {
    const int steps = (end - begin + STEP - 1) / STEP, each = (steps + a.splits - 1) / a.splits * STEP;
    begin += split * each;
    end = min(end, begin + each);
}

// Where the split's output of a row stands until all are joined.
__device__ __forceinline__ char *part_row(const params &a, int heads, int len, int split, int b, int h, int i) {
    return (char *)(a.part + ((((int64_t)split * a.batch + b) * heads + h) * len + i) * a.head_dim);
}

// ------------------------------------------------------------------------------------ forward
// fp32, and bf16 whose rows lie too far apart for the kernels below.  Tiles go through registers to LDS, a step's loads beside the
// products of the step before, two barriers a step.  3 x 385 queries and keys in fp32, 12 heads of 64, 38 us a call, four times what
// its products take at the rate of large ones (154 TFLOP/s).
template <typename T, int W> __global__ __launch_bounds__(THREADS, (resident<T, W>(false))) void attention_kernel(params a) {
    __shared__ __attribute__((aligned(16))) char lds[2 * tile<T, W>::bytes(STEP)];
    DEAR_LDS T *ks = (DEAR_LDS T *)lds, *vs = (DEAR_LDS T *)(lds + tile<T, W>::bytes(STEP));
    int b, h, t, split;
    place(a, a.q_heads, a.q_heads / a.kv_heads, b, h, t, split);
    if (a.causal) t = a.tiles - 1 - t;
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = threadIdx.x >> 6;
    const int nq = length(a.q_lens, b, a.q_len), nk = length(a.kv_lens, b, a.kv_len);
    const int kvh = h / (a.q_heads / a.kv_heads);
    const char *qp = at(a.q, b, h), *kp = at(a.k, b, kvh), *vp = at(a.v, b, kvh);
    const int i = t * BLOCK + wave * 32 + (lane & 31);  // this lane's query
    // keys 0 .. last are visible to it
    const int last = i < nq ? (a.causal ? min(nk - 1, i + nk - nq) : nk - 1) : -1;
    int begin = 0, end = t * BLOCK >= nq ? 0 : a.causal ? min(nk, min(t * BLOCK + BLOCK, nq) + nk - nq) : nk;
    share(a, split, begin, end);
    // the same of the whole wave: the fewest keys of a query, and the most
    const int wave_first = t * BLOCK + wave * 32;
    const int wave_least = wave_first + 31 < nq ? (a.causal ? min(nk - 1, wave_first + nk - nq) : nk - 1) : -1;

    frag<T> q[W / 16];
    load_rows<T, W>(q, qp, a.q.token, i, nq, a.head_dim, half);
    f32x16 o[W / 32] = {};
    float top = -INFINITY, sum = 0.f;
    const float c = a.scale * LOG2E;

    stage<T, W> kst, vst;
    if (begin < end) {
        kst.load(kp, a.k.token, begin, nk, a.head_dim);
        vst.load(vp, a.v.token, begin, nk, a.head_dim);
    }
    for (int j0 = begin; j0 < end; j0 += STEP) {
        __syncthreads();
        kst.store(ks);
        vst.store(vs);
        __syncthreads();
        if (j0 + STEP < end) {
            kst.load(kp, a.k.token, j0 + STEP, nk, a.head_dim);
            vst.load(vp, a.v.token, j0 + STEP, nk, a.head_dim);
        }
        f32x16 s[STEP / 32] = {};
#pragma unroll
        for (int kb = 0; kb < STEP / 32; ++kb)
#pragma unroll
            for (int kk = 0; kk < W / 16; ++kk) s[kb] = mma(straight<W>(ks, 32 * kb, kk, lane), q[kk], s[kb]);
        if (j0 + STEP - 1 > wave_least) {
#pragma unroll
            for (int kb = 0; kb < STEP / 32; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) s[kb][r] = j0 + 32 * kb + row_of(r, half) <= last ? s[kb][r] : -INFINITY;
        }
        float most = top;
#pragma unroll
        for (int kb = 0; kb < STEP / 32; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) most = fmaxf(most, s[kb][r]);
        most = halves_max(most);
        const float base = most == -INFINITY ? 0.f : most * c;
        const float keep = top == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(top * c - base);
        top = most;
        sum *= keep;
#pragma unroll
        for (int kb = 0; kb < STEP / 32; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                s[kb][r] = __builtin_amdgcn_exp2f(s[kb][r] * c - base);
                sum += s[kb][r];
            }
#pragma unroll
        for (int db = 0; db < W / 32; ++db) o[db] *= keep;
#pragma unroll
        for (int kb = 0; kb < STEP / 32; ++kb)
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                float x[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) x[u] = s[kb][8 * st + u];
                const frag<T> p = to_frag<T>(x);
#pragma unroll
                for (int db = 0; db < W / 32; ++db)
                    o[db] = mma(transposed<W>(vs, 32 * kb + 16 * st, 32 * db, lane), p, o[db]);
            }
    }
    if (i >= a.q_len) return;
    sum = halves_sum(sum);
    const bool none = top == -INFINITY && sum == 0.f;
    if (a.splits > 1) {
        store_row<float, W>(part_row(a, a.q_heads, a.q_len, split, b, h, i), o, 1.f, a.head_dim, half);
        const int64_t row = (((int64_t)split * a.batch + b) * a.q_heads + h) * a.q_len + i;
        if (half == 0) a.part_base[row] = top == -INFINITY ? 0.f : top * c, a.part_sum[row] = sum;
        return;
    }
    store_row<T, W>(at(a.out, b, h) + i * a.out.token, o, none ? 0.f : 1.f / sum, a.head_dim, half);
    if (half == 0)
        a.lse[((int64_t)b * a.q_heads + h) * a.q_len + i] = none ? -INFINITY : (top * c + __builtin_amdgcn_logf(sum)) * LN2;
}

// ------------------------------------------------------------------------------------ bf16, tiles filled directly
// Loads of STEP rows of W values that write LDS themselves.  A lane brings the same piece of every row that it has a part
// in; its offsets from the tile's first row are 32 bits (the host sees to it that they fit).  Rows at or beyond `valid`
// repeat the last one: what they stand for is masked, and their values are no others than those already read.  Values at
// or beyond head_dim are not loaded; `clear` has put zeros there.
template <int W, int WAVES> struct direct_loads {
    static constexpr int N = STEP / direct<W>::ROWS / WAVES;  // loads of a wave
    uint32_t piece, token, row;  // byte of the piece, bytes from row to row, first row of this lane
    bool some;

    __device__ __forceinline__ direct_loads(int64_t token_stride, int head_dim, int lane, int wave) {
        row = wave * direct<W>::ROWS + lane / direct<W>::PIECES;
        const int c = lane % direct<W>::PIECES ^ direct<W>::turn(row);  // `turn` is the same for all loads of the lane
        piece = c * 16, token = (uint32_t)token_stride, some = c * 8 < head_dim;
    }
    // p: the tile's first row; left >= 1: valid rows from there on
    __device__ __forceinline__ void load(const char *p, int left, DEAR_LDS bf16 *s, int wave) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint32_t r = row + i * WAVES * direct<W>::ROWS;
            if (left < STEP) r = min(r, (uint32_t)left - 1);
            if (some) load_to_lds(p + (r * token + piece), s + (i * WAVES + wave) * 512);
        }
    }
};

template <int W> __device__ __forceinline__ void clear(DEAR_LDS bf16 *s) {
    for (unsigned i = threadIdx.x; i < STEP * W / 8; i += blockDim.x) *(DEAR_LDS u32x4 *)(s + i * 8) = u32x4{0, 0, 0, 0};
}

// Scores of a step's keys to a running softmax.  `base` is what the powers are taken against: the running maximum, times
// scale * log2(e), of some step before.  It follows the maximum only when that has grown by more than GROWTH = 2^8, so
// that the sums are seldom rescaled; out = o / sum and lse do not depend on it.
constexpr float GROWTH = 8.f;

// Order of a block of N products with a fragment read for each: AHEAD reads first, then a product and a read in turn.
template <int N, int AHEAD> __device__ __forceinline__ void read_ahead() {
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD, 0);
#pragma unroll
    for (int n = 0; n < N - AHEAD; ++n) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, AHEAD, 0);
}

// Forward in bf16: 128 queries a workgroup, 32 a wave, two workgroups' waves a SIMD, steps of 64 keys in two buffers that are
// filled beside the products of the step before.  Rows of 128 are bound by the matrix instructions (busy 59 % of the time) and the
// softmax's instructions beside them (53 %); rows of 64, with half the products for as many scores, by the softmax's (61 and 28 %;
// waves wait 30 % of theirs).  Measured: 8192 queries and keys, causal, 16 heads of 128 for 4, 276 to 285 us = 963 TFLOP/s and more; 16
// sequences of 512 with ragged lengths, 16 heads of 64, 24 us = 2.3 TB/s; 128 queries and keys, 16 heads, 6 us.
template <int W> __global__ __launch_bounds__(THREADS, 2) void attention_direct_kernel(params a) {
    __shared__ __attribute__((aligned(16))) bf16 ks0[STEP * W], ks1[STEP * W], vs0[STEP * W], vs1[STEP * W];
    int b, h, t, split;
    place(a, a.q_heads, a.q_heads / a.kv_heads, b, h, t, split);
    if (a.causal) t = a.tiles - 1 - t;
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nq = length(a.q_lens, b, a.q_len), nk = length(a.kv_lens, b, a.kv_len);
    const int kvh = h / (a.q_heads / a.kv_heads);
    const int i = t * BLOCK + wave * 32 + (lane & 31);  // this lane's query
    // keys 0 .. last are visible to it
    const int last = i < nq ? (a.causal ? min(nk - 1, i + nk - nq) : nk - 1) : -1;
    int begin = 0, end = t * BLOCK >= nq ? 0 : a.causal ? min(nk, min(t * BLOCK + BLOCK, nq) + nk - nq) : nk;
    share(a, split, begin, end);
    const int wave_first = t * BLOCK + wave * 32;
    const int wave_least = wave_first + 31 < nq ? (a.causal ? min(nk - 1, wave_first + nk - nq) : nk - 1) : -1;
    const float c = a.scale * LOG2E;

    f32x16 o[W / 32] = {};
    float top = -INFINITY, base = 0.f, limit = -INFINITY, sum = 0.f;
    if (begin < end) {
        if (a.head_dim < W) {
            for (DEAR_LDS bf16 *s : {(DEAR_LDS bf16 *)ks0, (DEAR_LDS bf16 *)ks1, (DEAR_LDS bf16 *)vs0, (DEAR_LDS bf16 *)vs1}) clear<W>(s);
            __syncthreads();
        }
        const direct_loads<W, WAVES> kl(a.k.token, a.head_dim, lane, wave), vl(a.v.token, a.head_dim, lane, wave);
        const char *kp = at(a.k, b, kvh) + begin * a.k.token, *vp = at(a.v, b, kvh) + begin * a.v.token;
        int j0 = begin;
        auto load = [&](DEAR_LDS bf16 *ks, DEAR_LDS bf16 *vs, int j) {
            if (j < end) {
                kl.load(kp, nk - j, ks, wave);
                vl.load(vp, nk - j, vs, wave);
                kp += STEP * a.k.token, vp += STEP * a.v.token;
            }
        };
        load((DEAR_LDS bf16 *)ks0, (DEAR_LDS bf16 *)vs0, begin);
        frag<bf16> q[W / 16];
        load_rows<bf16, W>(q, at(a.q, b, h), a.q.token, i, nq, a.head_dim, half);
        direct<W> rd(lane);
        auto step = [&](const DEAR_LDS bf16 *ks, const DEAR_LDS bf16 *vs) {
            rd.renew();
            f32x16 s[STEP / 32] = {};
#pragma unroll
            for (int kk = 0; kk < W / 16; ++kk)
#pragma unroll
                for (int kb = 0; kb < STEP / 32; ++kb) s[kb] = mma(rd.straight(ks, 32 * kb, kk), q[kk], s[kb]);
            read_ahead<W / 16 * (STEP / 32), W == 128 ? 8 : 4>();
            if (j0 + STEP - 1 > wave_least) {
                __builtin_amdgcn_sched_barrier(0);  // keeps this a branch: as selects it would cost every step
#pragma unroll
                for (int kb = 0; kb < STEP / 32; ++kb)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[kb][r] = j0 + 32 * kb + row_of(r, half) <= last ? s[kb][r] : -INFINITY;
            }
            float most = s[0][0];
#pragma unroll
            for (int kb = 0; kb < STEP / 32; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) most = fmaxf(most, s[kb][r]);
            most = halves_max(most);
            if (__builtin_amdgcn_ballot_w64(most > limit)) {
                const float old = top == -INFINITY ? -INFINITY : base;  // nothing yet: what is kept is 0, far below 0 too
                top = fmaxf(top, most);
                base = top == -INFINITY ? 0.f : top * c;
                limit = top + GROWTH / c;
                const float keep = __builtin_amdgcn_exp2f(old - base);
                sum *= keep;
#pragma unroll
                for (int db = 0; db < W / 32; ++db) o[db] *= keep;
            }
#pragma unroll
            for (int kb = 0; kb < STEP / 32; ++kb)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    s[kb][r] = __builtin_amdgcn_exp2f(s[kb][r] * c - base);
                    sum += s[kb][r];
                }
#pragma unroll
            for (int kb = 0; kb < STEP / 32; ++kb)
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    float x[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u) x[u] = s[kb][8 * st + u];
                    const frag<bf16> p = to_frag<bf16>(x);
#pragma unroll
                    for (int db = 0; db < W / 32; ++db)
                        o[db] = mma(rd.transposed(vs, 32 * kb + 16 * st, db), p, o[db]);
                }
            j0 += STEP;
        };
        // one barrier a step: behind it this step's tiles are whole, and the other buffers are no longer read
        while (true) {
            loads_barrier();
            load((DEAR_LDS bf16 *)ks1, (DEAR_LDS bf16 *)vs1, j0 + STEP);
            step((DEAR_LDS bf16 *)ks0, (DEAR_LDS bf16 *)vs0);
            if (j0 >= end) break;
            loads_barrier();
            load((DEAR_LDS bf16 *)ks0, (DEAR_LDS bf16 *)vs0, j0 + STEP);
            step((DEAR_LDS bf16 *)ks1, (DEAR_LDS bf16 *)vs1);
            if (j0 >= end) break;
        }
    }
    if (i >= a.q_len) return;
    sum = halves_sum(sum);
    const bool none = top == -INFINITY && sum == 0.f;
    if (a.splits > 1) {
        store_row<float, W>(part_row(a, a.q_heads, a.q_len, split, b, h, i), o, 1.f, a.head_dim, half);
        const int64_t row = (((int64_t)split * a.batch + b) * a.q_heads + h) * a.q_len + i;
        if (half == 0) a.part_base[row] = base, a.part_sum[row] = sum;
        return;
    }
    store_row<bf16, W>(at(a.out, b, h) + i * a.out.token, o, none ? 0.f : 1.f / sum, a.head_dim, half);
    if (half == 0)
        a.lse[((int64_t)b * a.q_heads + h) * a.q_len + i] = none ? -INFINITY : (base + __builtin_amdgcn_logf(sum)) * LN2;
}

// ------------------------------------------------------------------------------------ backward: queries
// lse * log2(e) of query i, as what its powers are taken against: infinity where it sees no key, so that its probabilities
// are 0.  Kept, with -delta, for the kernel that computes dk and dv; there is a place for every query of every tile.
__device__ __forceinline__ float row_values(const params &a, int b, int h, int i, int split, int nq, int half, float delta) {
    const float z = i < nq ? a.lse[((int64_t)b * a.q_heads + h) * a.q_len + i] : -INFINITY;
    const float base = z == -INFINITY ? INFINITY : z * LOG2E;
    if (half == 0 && split == 0) {
        const int64_t row = ((int64_t)b * a.q_heads + h) * a.tiles * BLOCK + i;
        a.powers[row] = base;
        a.deltas[row] = -delta;
    }
    return base;
}

// dq of 32 queries a wave, over all keys.  As in the forward pass the results of the first products are taken
// transposed, a query to a lane, so that lse and delta are one value a lane.  It also writes delta for the other kernel.
// fp32, 3 x 385 with ragged lengths, 12 heads of 64, in seven splits: 44 us, and 6 to join them; its matrix instructions are busy
// 49 % of the time.
template <typename T, int W> __global__ __launch_bounds__(THREADS, (resident<T, W>(false))) void attention_dq_kernel(params a) {
    __shared__ __attribute__((aligned(16))) char lds[2 * tile<T, W>::bytes(STEP)];
    DEAR_LDS T *ks = (DEAR_LDS T *)lds, *vs = (DEAR_LDS T *)(lds + tile<T, W>::bytes(STEP));
    int b, h, t, split;
    place(a, a.q_heads, a.q_heads / a.kv_heads, b, h, t, split);
    if (a.causal) t = a.tiles - 1 - t;
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = threadIdx.x >> 6;
    const int nq = length(a.q_lens, b, a.q_len), nk = length(a.kv_lens, b, a.kv_len);
    const int kvh = h / (a.q_heads / a.kv_heads);
    const char *kp = at(a.k, b, kvh), *vp = at(a.v, b, kvh);
    const int i = t * BLOCK + wave * 32 + (lane & 31);
    const int last = i < nq ? (a.causal ? min(nk - 1, i + nk - nq) : nk - 1) : -1;
    int begin = 0, end = t * BLOCK >= nq ? 0 : a.causal ? min(nk, min(t * BLOCK + BLOCK, nq) + nk - nq) : nk;
    share(a, split, begin, end);
    const int wave_first = t * BLOCK + wave * 32;
    const int wave_least = wave_first + 31 < nq ? (a.causal ? min(nk - 1, wave_first + nk - nq) : nk - 1) : -1;

    frag<T> q[W / 16], g[W / 16];
    load_rows<T, W>(q, at(a.q, b, h), a.q.token, i, nq, a.head_dim, half);
    load_rows<T, W>(g, at(a.dout, b, h), a.dout.token, i, nq, a.head_dim, half);
    float delta = 0.f;
    {
        frag<T> out[W / 16];
        load_rows<T, W>(out, at(a.out, b, h), a.out.token, i, nq, a.head_dim, half);
#pragma unroll
        for (int kk = 0; kk < W / 16; ++kk)
#pragma unroll
            for (int u = 0; u < 8; ++u) delta += (float)g[kk][u] * (float)out[kk][u];
    }
    delta = halves_sum(delta);
    const float base = row_values(a, b, h, i, split, nq, half, delta), c = a.scale * LOG2E;

    f32x16 dq[W / 32] = {};
    stage<T, W> kst, vst;
    if (begin < end) {
        kst.load(kp, a.k.token, begin, nk, a.head_dim);
        vst.load(vp, a.v.token, begin, nk, a.head_dim);
    }
    for (int j0 = begin; j0 < end; j0 += STEP) {
        __syncthreads();
        kst.store(ks);
        vst.store(vs);
        __syncthreads();
        if (j0 + STEP < end) {
            kst.load(kp, a.k.token, j0 + STEP, nk, a.head_dim);
            vst.load(vp, a.v.token, j0 + STEP, nk, a.head_dim);
        }
#pragma unroll
        for (int kb = 0; kb < STEP / 32; ++kb) {
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int kk = 0; kk < W / 16; ++kk) {
                s = mma(straight<W>(ks, 32 * kb, kk, lane), q[kk], s);
                dp = mma(straight<W>(vs, 32 * kb, kk, lane), g[kk], dp);
            }
            const bool whole = j0 + 32 * kb + 31 <= wave_least;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const float p = __builtin_amdgcn_exp2f(s[r] * c - base);
                s[r] = whole || j0 + 32 * kb + row_of(r, half) <= last ? p * (dp[r] - delta) : 0.f;
            }
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                float x[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) x[u] = s[8 * st + u];
                const frag<T> ds = to_frag<T>(x);
#pragma unroll
                for (int db = 0; db < W / 32; ++db)
                    dq[db] = mma(transposed<W>(ks, 32 * kb + 16 * st, 32 * db, lane), ds, dq[db]);
            }
        }
    }
    if (i >= a.q_len) return;
    if (a.splits > 1) store_row<float, W>(part_row(a, a.q_heads, a.q_len, split, b, h, i), dq, 1.f, a.head_dim, half);
    else store_row<T, W>(at(a.dq, b, h) + i * a.dq.token, dq, a.scale, a.head_dim, half);
}

// ------------------------------------------------------------------------------------ backward: keys and values
// dk and dv of 32 keys a wave, over the queries of all heads that share them: one workgroup adds them all up, in order.
// Two waves have the same keys and take every other 32 queries; their sums are added at the end.  fp32, 3 x 385 with ragged
// lengths, 12 heads of 64: 51 us, one wave a SIMD, whose matrix instructions are busy 46 % of the time.
template <typename T, int W> __global__ __launch_bounds__(THREADS, (resident<T, W>(true))) void attention_dkv_kernel(params a) {
    __shared__ __attribute__((aligned(16))) char lds[2 * tile<T, W>::bytes(STEP)];
    __shared__ __attribute__((aligned(16))) float rows[2][STEP];  // what the queries' powers are taken against, and -delta
    DEAR_LDS T *qs = (DEAR_LDS T *)lds, *gs = (DEAR_LDS T *)(lds + tile<T, W>::bytes(STEP));
    int b, kvh, t, split;
    place(a, a.kv_heads, 1, b, kvh, t, split);
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = threadIdx.x >> 6;
    const int nq = length(a.q_lens, b, a.q_len), nk = length(a.kv_lens, b, a.kv_len);
    const int group = a.q_heads / a.kv_heads;
    const int turn = wave % 2, wave_first = t * KEYS + wave / 2 * 32, j = wave_first + (lane & 31);  // this lane's key
    // queries first .. nq - 1 see it
    const int first = j < nk ? (a.causal ? max(0, j - nk + nq) : 0) : nq;
    const int wave_last = wave_first + 31 < nk ? (a.causal ? max(0, wave_first + 31 - nk + nq) : 0) : nq;
    int begin = t * KEYS >= nk ? nq : a.causal ? max(0, t * KEYS - nk + nq) / STEP * STEP : 0, end = nq;
    share(a, split, begin, end);

    frag<T> k[W / 16], v[W / 16];
    load_rows<T, W>(k, at(a.k, b, kvh), a.k.token, j, nk, a.head_dim, half);
    load_rows<T, W>(v, at(a.v, b, kvh), a.v.token, j, nk, a.head_dim, half);
    f32x16 dk[W / 32] = {}, dv[W / 32] = {};
    const float c = a.scale * LOG2E;

    for (int h = kvh * group; h < (kvh + 1) * group; ++h) {
        const char *qp = at(a.q, b, h), *gp = at(a.dout, b, h);
        const int64_t row = ((int64_t)b * a.q_heads + h) * a.q_tiles * BLOCK;
        stage<T, W> qst, gst;
        float z = 0.f;
        // one value a thread: the first STEP threads take what powers are taken against, the next ones -delta
        auto load_z = [&](int i0) {
            const int64_t i = row + i0 + threadIdx.x % STEP;
            if (threadIdx.x < 2 * STEP) z = threadIdx.x < STEP ? a.powers[i] : a.deltas[i];
        };
        if (begin < end) {
            qst.load(qp, a.q.token, begin, nq, a.head_dim);
            gst.load(gp, a.dout.token, begin, nq, a.head_dim);
            load_z(begin);
        }
        for (int i0 = begin; i0 < end; i0 += STEP) {
            __syncthreads();
            qst.store(qs);
            gst.store(gs);
            if (threadIdx.x < 2 * STEP) rows[threadIdx.x / STEP][threadIdx.x % STEP] = z;
            __syncthreads();
            if (i0 + STEP < end) {
                qst.load(qp, a.q.token, i0 + STEP, nq, a.head_dim);
                gst.load(gp, a.dout.token, i0 + STEP, nq, a.head_dim);
                load_z(i0 + STEP);
            }
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int kk = 0; kk < W / 16; ++kk) {
                s = mma(straight<W>(qs, 32 * turn, kk, lane), k[kk], s);
                dp = mma(straight<W>(gs, 32 * turn, kk, lane), v[kk], dp);
            }
            const bool whole = i0 + 32 * turn >= wave_last && i0 + 32 * turn + 31 < nq;
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int n = 32 * turn + row_of(r, half);
                const float p = __builtin_amdgcn_exp2f(s[r] * c - rows[0][n]);
                s[r] = whole || (i0 + n >= first && i0 + n < nq) ? p : 0.f;
                dp[r] = s[r] * (dp[r] + rows[1][n]);
            }
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                float x[8], y[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) x[u] = s[8 * st + u], y[u] = dp[8 * st + u];
                const frag<T> p = to_frag<T>(x), ds = to_frag<T>(y);
#pragma unroll
                for (int db = 0; db < W / 32; ++db) {
                    dv[db] = mma(transposed<W>(gs, 32 * turn + 16 * st, 32 * db, lane), p, dv[db]);
                    dk[db] = mma(transposed<W>(qs, 32 * turn + 16 * st, 32 * db, lane), ds, dk[db]);
                }
            }
        }
    }
    DEAR_LDS float *sums = (DEAR_LDS float *)lds + wave / 2 * (W / 32 * 16 * 64);
    for (f32x16 *x : {dk, dv}) {
        __syncthreads();
#pragma unroll
        for (int db = 0; db < W / 32; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (turn == 1) sums[(db * 16 + r) * 64 + lane] = x[db][r];
        __syncthreads();
#pragma unroll
        for (int db = 0; db < W / 32; ++db)
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (turn == 0) x[db][r] += sums[(db * 16 + r) * 64 + lane];
    }
    if (turn == 1) return;
    if (j >= a.kv_len) return;
    if (a.splits > 1) {  // dk's come first, then dv's
        store_row<float, W>(part_row(a, a.kv_heads, a.kv_len, split, b, kvh, j), dk, 1.f, a.head_dim, half);
        store_row<float, W>(part_row(a, a.kv_heads, a.kv_len, a.splits + split, b, kvh, j), dv, 1.f, a.head_dim, half);
        return;
    }
    store_row<T, W>(at(a.dk, b, kvh) + j * a.dk.token, dk, a.scale, a.head_dim, half);
    store_row<T, W>(at(a.dv, b, kvh) + j * a.dv.token, dv, 1.f, a.head_dim, half);
}

// ------------------------------------------------------------------------------------ bf16 backward, tiles filled directly
// dq as above, its tiles as in the forward pass.  Bound by the matrix instructions where sequences are long: 2 x 4096,
// causal, 16 heads of 128 for 4, 201 us = 1026 TFLOP/s of its three products.  16 x 512, ragged, 16 heads of 64, 35 us:
// matrix instructions busy 28 %, vector instructions 40 %, and waves wait 42 % of their time.  Three waves a SIMD have too
// few registers (1 x 2048, causal, with dk and dv: 91 us for 84).
template <int W> __global__ __launch_bounds__(THREADS, 2) void attention_dq_direct_kernel(params a) {
    __shared__ __attribute__((aligned(16))) bf16 ks0[STEP * W], ks1[STEP * W], vs0[STEP * W], vs1[STEP * W];
    int b, h, t, split;
    place(a, a.q_heads, a.q_heads / a.kv_heads, b, h, t, split);
    if (a.causal) t = a.tiles - 1 - t;
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nq = length(a.q_lens, b, a.q_len), nk = length(a.kv_lens, b, a.kv_len);
    const int kvh = h / (a.q_heads / a.kv_heads);
    const int i = t * BLOCK + wave * 32 + (lane & 31);
    const int last = i < nq ? (a.causal ? min(nk - 1, i + nk - nq) : nk - 1) : -1;
    int begin = 0, end = t * BLOCK >= nq ? 0 : a.causal ? min(nk, min(t * BLOCK + BLOCK, nq) + nk - nq) : nk;
    share(a, split, begin, end);
    const int wave_first = t * BLOCK + wave * 32;
    const int wave_least = wave_first + 31 < nq ? (a.causal ? min(nk - 1, wave_first + nk - nq) : nk - 1) : -1;
    const float c = a.scale * LOG2E;
    const bool any = begin < end;

    const direct_loads<W, WAVES> kl(a.k.token, a.head_dim, lane, wave), vl(a.v.token, a.head_dim, lane, wave);
    const char *kp = at(a.k, b, kvh) + begin * a.k.token, *vp = at(a.v, b, kvh) + begin * a.v.token;
    auto load = [&](DEAR_LDS bf16 *ks, DEAR_LDS bf16 *vs, int j) {
        if (j < end) {
            kl.load(kp, nk - j, ks, wave);
            vl.load(vp, nk - j, vs, wave);
            kp += STEP * a.k.token, vp += STEP * a.v.token;
        }
    };
    if (any && a.head_dim < W) {
        for (DEAR_LDS bf16 *s : {(DEAR_LDS bf16 *)ks0, (DEAR_LDS bf16 *)ks1, (DEAR_LDS bf16 *)vs0, (DEAR_LDS bf16 *)vs1}) clear<W>(s);
        __syncthreads();
    }
    load((DEAR_LDS bf16 *)ks0, (DEAR_LDS bf16 *)vs0, begin);

    frag<bf16> q[W / 16], g[W / 16];
    load_rows<bf16, W>(q, at(a.q, b, h), a.q.token, i, nq, a.head_dim, half);
    load_rows<bf16, W>(g, at(a.dout, b, h), a.dout.token, i, nq, a.head_dim, half);
    float delta = 0.f;
    {
        frag<bf16> out[W / 16];
        load_rows<bf16, W>(out, at(a.out, b, h), a.out.token, i, nq, a.head_dim, half);
#pragma unroll
        for (int kk = 0; kk < W / 16; ++kk)
#pragma unroll
            for (int u = 0; u < 8; ++u) delta += (float)g[kk][u] * (float)out[kk][u];
    }
    delta = halves_sum(delta);
    const float base = row_values(a, b, h, i, split, nq, half, delta);

    f32x16 dq[W / 32] = {};
    int j0 = begin;
    direct<W> rd(lane);
    auto step = [&](const DEAR_LDS bf16 *ks, const DEAR_LDS bf16 *vs) {
        rd.renew();
#pragma unroll
        for (int kb = 0; kb < STEP / 32; ++kb) {
            f32x16 s = {}, dp;
#pragma unroll
            for (int r = 0; r < 16; ++r) dp[r] = -delta;
#pragma unroll
            for (int kk = 0; kk < W / 16; ++kk) {
                s = mma(rd.straight(ks, 32 * kb, kk), q[kk], s);
                dp = mma(rd.straight(vs, 32 * kb, kk), g[kk], dp);
            }
#pragma unroll
            for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(s[r] * c - base) * dp[r];
            if (j0 + 32 * kb + 31 > wave_least) {
                __builtin_amdgcn_sched_barrier(0);  // keeps this a branch: as selects it would cost every step
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = j0 + 32 * kb + row_of(r, half) <= last ? s[r] : 0.f;
            }
#pragma unroll
            for (int st = 0; st < 2; ++st) {
                float x[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) x[u] = s[8 * st + u];
                const frag<bf16> ds = to_frag<bf16>(x);
#pragma unroll
                for (int db = 0; db < W / 32; ++db)
                    dq[db] = mma(rd.transposed(ks, 32 * kb + 16 * st, db), ds, dq[db]);
            }
        }
        j0 += STEP;
    };
    while (any) {
        loads_barrier();
        load((DEAR_LDS bf16 *)ks1, (DEAR_LDS bf16 *)vs1, j0 + STEP);
        step((DEAR_LDS bf16 *)ks0, (DEAR_LDS bf16 *)vs0);
        if (j0 >= end) break;
        loads_barrier();
        load((DEAR_LDS bf16 *)ks0, (DEAR_LDS bf16 *)vs0, j0 + STEP);
        step((DEAR_LDS bf16 *)ks1, (DEAR_LDS bf16 *)vs1);
        if (j0 >= end) break;
    }
    if (i >= a.q_len) return;
    if (a.splits > 1) store_row<float, W>(part_row(a, a.q_heads, a.q_len, split, b, h, i), dq, 1.f, a.head_dim, half);
    else store_row<bf16, W>(at(a.dq, b, h) + i * a.dq.token, dq, a.scale, a.head_dim, half);
}

// dk and dv of 128 keys a workgroup, 32 a wave, for rows of 64 values: the operands and sums of both fit a wave beside a
// second one.  16 x 512, ragged, 16 heads: 44 us, matrix instructions busy 31 %, vector instructions 38 %, waves waiting 39 % of
// their time; in two kinds of waves as below 68 us.
__global__ __launch_bounds__(THREADS, 2) void attention_dkv_direct_kernel(params a) {
    constexpr int W = 64;
    __shared__ __attribute__((aligned(16))) bf16 qs0[STEP * W], qs1[STEP * W], gs0[STEP * W], gs1[STEP * W];
    __shared__ __attribute__((aligned(16))) float powers0[STEP], powers1[STEP], deltas0[STEP], deltas1[STEP];
    int b, kvh, t, split;
    place(a, a.kv_heads, 1, b, kvh, t, split);
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nq = length(a.q_lens, b, a.q_len), nk = length(a.kv_lens, b, a.kv_len);
    const int group = a.q_heads / a.kv_heads;
    const int wave_first = t * BLOCK + wave * 32, j = wave_first + (lane & 31);  // this lane's key
    // queries first .. nq - 1 see it; those beyond nq have probabilities of 0 by their powers
    const int first = j < nk ? (a.causal ? max(0, j - nk + nq) : 0) : nq;
    const int wave_last = wave_first + 31 < nk ? (a.causal ? max(0, wave_first + 31 - nk + nq) : 0) : nq;
    int begin = t * BLOCK >= nk ? nq : a.causal ? max(0, t * BLOCK - nk + nq) / STEP * STEP : 0, end = nq;
    share(a, split, begin, end);
    const int steps = begin < end ? (end - begin + STEP - 1) / STEP * group : 0;
    const float c = a.scale * LOG2E;

    f32x16 dk[W / 32] = {}, dv[W / 32] = {};
    if (steps > 0) {
        if (a.head_dim < W) {
            for (DEAR_LDS bf16 *s : {(DEAR_LDS bf16 *)qs0, (DEAR_LDS bf16 *)qs1, (DEAR_LDS bf16 *)gs0, (DEAR_LDS bf16 *)gs1}) clear<W>(s);
            __syncthreads();
        }
        const direct_loads<W, WAVES> ql(a.q.token, a.head_dim, lane, wave), gl(a.dout.token, a.head_dim, lane, wave);
        // the next step to be loaded: its queries, and its head's tensors
        int h = kvh * group, next = begin, loaded = 0;
        const char *qp = at(a.q, b, h) + begin * a.q.token, *gp = at(a.dout, b, h) + begin * a.dout.token;
        auto load = [&](DEAR_LDS bf16 *qs, DEAR_LDS bf16 *gs, DEAR_LDS float *powers, DEAR_LDS float *deltas) {
            if (loaded++ < steps) {
                ql.load(qp, nq - next, qs, wave);
                gl.load(gp, nq - next, gs, wave);
                const int64_t row = ((int64_t)b * a.q_heads + h) * a.q_tiles * BLOCK + next + lane;
                if (wave == 0) load_value_to_lds(a.powers + row, powers);
                if (wave == 1) load_value_to_lds(a.deltas + row, deltas);
                qp += STEP * a.q.token, gp += STEP * a.dout.token, next += STEP;
                if (next >= end) {
                    h += 1, next = begin;
                    qp = at(a.q, b, h) + begin * a.q.token, gp = at(a.dout, b, h) + begin * a.dout.token;
                }
            }
        };
#define DEAR_LOAD(n) load((DEAR_LDS bf16 *)qs##n, (DEAR_LDS bf16 *)gs##n, (DEAR_LDS float *)powers##n, (DEAR_LDS float *)deltas##n)
        DEAR_LOAD(0);
        frag<bf16> k[W / 16], v[W / 16];
        load_rows<bf16, W>(k, at(a.k, b, kvh), a.k.token, j, nk, a.head_dim, half);
        load_rows<bf16, W>(v, at(a.v, b, kvh), a.v.token, j, nk, a.head_dim, half);
        direct<W> rd(lane);
        int n = 0, i0 = begin;
        auto step = [&](const DEAR_LDS bf16 *qs, const DEAR_LDS bf16 *gs, const DEAR_LDS float *powers, const DEAR_LDS float *deltas) {
            rd.renew();
#pragma unroll
            for (int qb = 0; qb < STEP / 32; ++qb) {
                f32x16 s = {}, dp;
                if (i0 + 32 * qb < wave_last) {  // masked scores start, and stay, at -infinity
                    __builtin_amdgcn_sched_barrier(0);  // keeps this a branch
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = i0 + 32 * qb + row_of(r, half) >= first ? 0.f : -INFINITY;
                }
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const f32x4 d = *(const DEAR_LDS f32x4 *)(deltas + 32 * qb + row_of(r, half));
                    dp[r] = d[0], dp[r + 1] = d[1], dp[r + 2] = d[2], dp[r + 3] = d[3];
                }
#pragma unroll
                for (int kk = 0; kk < W / 16; ++kk) {
                    s = mma(rd.straight(qs, 32 * qb, kk), k[kk], s);
                    dp = mma(rd.straight(gs, 32 * qb, kk), v[kk], dp);
                }
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    float x[8], y[8];
#pragma unroll
                    for (int u = 0; u < 8; u += 4) {
                        const f32x4 e = *(const DEAR_LDS f32x4 *)(powers + 32 * qb + row_of(8 * st + u, half));
#pragma unroll
                        for (int w = 0; w < 4; ++w) {
                            x[u + w] = __builtin_amdgcn_exp2f(s[8 * st + u + w] * c - e[w]);
                            y[u + w] = x[u + w] * dp[8 * st + u + w];
                        }
                    }
                    const frag<bf16> p = to_frag<bf16>(x), ds = to_frag<bf16>(y);
#pragma unroll
                    for (int db = 0; db < W / 32; ++db) {
                        dv[db] = mma(rd.transposed(gs, 32 * qb + 16 * st, db), p, dv[db]);
                        dk[db] = mma(rd.transposed(qs, 32 * qb + 16 * st, db), ds, dk[db]);
                    }
                }
            }
            i0 += STEP;
            if (i0 >= end) i0 = begin;
            return ++n < steps;
        };
#define DEAR_STEP(n, other)  \
    loads_barrier();         \
    DEAR_LOAD(other);        \
    if (!step((DEAR_LDS bf16 *)qs##n, (DEAR_LDS bf16 *)gs##n, (DEAR_LDS float *)powers##n, (DEAR_LDS float *)deltas##n)) break;
        while (true) {
            DEAR_STEP(0, 1)
            DEAR_STEP(1, 0)
        }
#undef DEAR_STEP
#undef DEAR_LOAD
    }
    if (j >= a.kv_len) return;
    if (a.splits > 1) {  // dk's come first, then dv's
        store_row<float, W>(part_row(a, a.kv_heads, a.kv_len, split, b, kvh, j), dk, 1.f, a.head_dim, half);
        store_row<float, W>(part_row(a, a.kv_heads, a.kv_len, a.splits + split, b, kvh, j), dv, 1.f, a.head_dim, half);
        return;
    }
    store_row<bf16, W>(at(a.dk, b, kvh) + j * a.dk.token, dk, a.scale, a.head_dim, half);
    store_row<bf16, W>(at(a.dv, b, kvh) + j * a.dv.token, dv, 1.f, a.head_dim, half);
}

// dk and dv of 64 keys a workgroup of eight waves, for rows of 128 values.  Four compute probabilities and dv, four the
// gradients of the scores and dk: so each half needs the operands and sums of one of the two, two waves fit a SIMD, and there
// (waves w and w + 4) one of either kind runs beside the other.  Two waves of a kind have the same 32 keys and take every other
// 32 queries; their sums are added at the end.  Step n: the first kind computes s, p and dv of tile n and leaves p, in fp32, in
// LDS; the second takes p of tile n - 1, its dp from the step before, and computes dk of tile n - 1, then dp of tile n.
// Bound by the matrix instructions: 2 x 4096, causal, 16 heads of 128 for 4, 291 us = 945 TFLOP/s of its four products; all in
// one kind of waves, one a SIMD, 434 us.
constexpr int KV_WAVES = 8;

__global__ __launch_bounds__(64 * KV_WAVES, 2) void attention_dkv_halves_kernel(params a) {
    constexpr int W = 128;
    // Tiles in turn, three of the queries, as the one before is still read, and two of all else: arrays of their own, so that
    // the compiler sees that the loads under way are not what a step reads.
    __shared__ __attribute__((aligned(16))) bf16 qs0[STEP * W], qs1[STEP * W], qs2[STEP * W], gs0[STEP * W], gs1[STEP * W];
    __shared__ __attribute__((aligned(16))) float powers0[STEP], powers1[STEP], deltas0[STEP], deltas1[STEP];
    __shared__ __attribute__((aligned(16))) float ps[2][4][4][64 * 4];  // step, wave, quarter of its values: four a lane
    int b, kvh, t, split;
    place(a, a.kv_heads, 1, b, kvh, t, split);
    const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int nq = length(a.q_lens, b, a.q_len), nk = length(a.kv_lens, b, a.kv_len);
    const int group = a.q_heads / a.kv_heads, part = wave & 3, turn = part & 1;
    const bool second = wave >= 4;
    const int wave_first = t * KEYS + part / 2 * 32, j = wave_first + (lane & 31);  // this lane's key
    // queries first .. nq - 1 see it; those beyond nq have probabilities of 0 by their powers
    const int first = j < nk ? (a.causal ? max(0, j - nk + nq) : 0) : nq;
    const int wave_last = wave_first + 31 < nk ? (a.causal ? max(0, wave_first + 31 - nk + nq) : 0) : nq;
    int begin = t * KEYS >= nk ? nq : a.causal ? max(0, t * KEYS - nk + nq) / STEP * STEP : 0, end = nq;
    share(a, split, begin, end);
    const int steps = begin < end ? (end - begin + STEP - 1) / STEP * group : 0;
    const float c = a.scale * LOG2E;

    f32x16 sum[W / 32] = {};  // dv, or dk
    if (steps > 0) {
        if (a.head_dim < W) {
            for (DEAR_LDS bf16 *s : {(DEAR_LDS bf16 *)qs0, (DEAR_LDS bf16 *)qs1, (DEAR_LDS bf16 *)qs2, (DEAR_LDS bf16 *)gs0,
                                     (DEAR_LDS bf16 *)gs1})
                clear<W>(s);
            __syncthreads();
        }
        const direct_loads<W, KV_WAVES> ql(a.q.token, a.head_dim, lane, wave), gl(a.dout.token, a.head_dim, lane, wave);
        // the next step to be loaded: its queries, and its head's tensors
        int h = kvh * group, next = begin, loaded = 0;
        const char *qp = at(a.q, b, h) + begin * a.q.token, *gp = at(a.dout, b, h) + begin * a.dout.token;
        auto load = [&](DEAR_LDS bf16 *qs, DEAR_LDS bf16 *gs, DEAR_LDS float *powers, DEAR_LDS float *deltas) {
            if (loaded < steps) {
                ql.load(qp, nq - next, qs, wave);
                gl.load(gp, nq - next, gs, wave);
                const int64_t row = ((int64_t)b * a.q_heads + h) * a.q_tiles * BLOCK + next + lane;
                if (wave == 0) load_value_to_lds(a.powers + row, powers);
                if (wave == 4) load_value_to_lds(a.deltas + row, deltas);
                qp += STEP * a.q.token, gp += STEP * a.dout.token, next += STEP;
                if (next >= end) {
                    h += 1, next = begin;
                    qp = at(a.q, b, h) + begin * a.q.token, gp = at(a.dout, b, h) + begin * a.dout.token;
                }
            }
            ++loaded;
        };
#define DEAR_LOAD(q, g) load((DEAR_LDS bf16 *)qs##q, (DEAR_LDS bf16 *)gs##g, (DEAR_LDS float *)powers##g, (DEAR_LDS float *)deltas##g)
        DEAR_LOAD(0, 0);
        frag<bf16> kv[W / 16];  // the keys, or the values
        load_rows<bf16, W>(kv, second ? at(a.v, b, kvh) : at(a.k, b, kvh), second ? a.v.token : a.k.token, j, nk, a.head_dim, half);

        // with the place of the 32 queries that are this wave's turn
        direct<W> rd(lane);
        rd.move(64 * W * turn);
        if (!second) {
            int i0 = begin;
            auto step = [&](int n, const DEAR_LDS bf16 *qs, const DEAR_LDS bf16 *gs, const DEAR_LDS float *powers) {
                f32x16 s = {};
                if (i0 + 32 * turn < wave_last) {  // masked scores start, and stay, at -infinity
                    __builtin_amdgcn_sched_barrier(0);  // keeps this a branch
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = i0 + 32 * turn + row_of(r, half) >= first ? 0.f : -INFINITY;
                }
                i0 += STEP;
                if (i0 >= end) i0 = begin;
#pragma unroll
                for (int kk = 0; kk < W / 16; ++kk) s = mma(rd.straight(qs, 0, kk), kv[kk], s);
                frag<bf16> p[2];
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    float x[8];
#pragma unroll
                    for (int u = 0; u < 8; u += 4) {
                        const f32x4 e = *(const DEAR_LDS f32x4 *)(powers + 32 * turn + row_of(8 * st + u, half));
#pragma unroll
                        for (int w = 0; w < 4; ++w) x[u + w] = __builtin_amdgcn_exp2f(s[8 * st + u + w] * c - e[w]);
                        *(DEAR_LDS f32x4 *)(&ps[n & 1][part][2 * st + u / 4][lane * 4]) = f32x4{x[u], x[u + 1], x[u + 2], x[u + 3]};
                    }
                    p[st] = to_frag<bf16>(x);
                }
#pragma unroll
                for (int st = 0; st < 2; ++st)
#pragma unroll
                    for (int db = 0; db < W / 32; ++db) sum[db] = mma(rd.transposed(gs, 16 * st, db), p[st], sum[db]);
            };
            int n = 0;
#define DEAR_STEP(q, g, q_load, g_load)                                                      \
    loads_barrier();                                                                         \
    if (n == steps) break;                                                                   \
    DEAR_LOAD(q_load, g_load);                                                               \
    step(n, (DEAR_LDS bf16 *)qs##q, (DEAR_LDS bf16 *)gs##g, (DEAR_LDS float *)powers##g);     \
    ++n;
            while (true) {
                rd.renew();
                DEAR_STEP(0, 0, 1, 1)
                DEAR_STEP(1, 1, 2, 0)
                DEAR_STEP(2, 0, 0, 1)
                rd.renew();
                DEAR_STEP(0, 1, 1, 0)
                DEAR_STEP(1, 0, 2, 1)
                DEAR_STEP(2, 1, 0, 0)
            }
#undef DEAR_STEP
        } else {
            f32x16 dp;
            auto before = [&](int n, const DEAR_LDS bf16 *qs) {  // dk of tile n
#pragma unroll
                for (int st = 0; st < 2; ++st) {
                    float x[8];
#pragma unroll
                    for (int u = 0; u < 8; u += 4) {
                        const f32x4 p = *(const DEAR_LDS f32x4 *)(&ps[n & 1][part][2 * st + u / 4][lane * 4]);
#pragma unroll
                        for (int w = 0; w < 4; ++w) x[u + w] = p[w] * dp[8 * st + u + w];
                    }
                    const frag<bf16> ds = to_frag<bf16>(x);
#pragma unroll
                    for (int db = 0; db < W / 32; ++db) sum[db] = mma(rd.transposed(qs, 16 * st, db), ds, sum[db]);
                }
            };
            auto step = [&](const DEAR_LDS bf16 *gs, const DEAR_LDS float *deltas) {
#pragma unroll
                for (int u = 0; u < 16; u += 4) {
                    const f32x4 d = *(const DEAR_LDS f32x4 *)(deltas + 32 * turn + row_of(u, half));
                    dp[u] = d[0], dp[u + 1] = d[1], dp[u + 2] = d[2], dp[u + 3] = d[3];
                }
#pragma unroll
                for (int kk = 0; kk < W / 16; ++kk) dp = mma(rd.straight(gs, 0, kk), kv[kk], dp);
            };
            int n = 0;
            loads_barrier();
            DEAR_LOAD(1, 1);
            step((DEAR_LDS bf16 *)gs0, (DEAR_LDS float *)deltas0);
#define DEAR_STEP(q, g, q_load, g_load)                                     \
    loads_barrier();                                                        \
    before(n, (DEAR_LDS bf16 *)qs##q);                                      \
    if (++n == steps) break;                                                \
    DEAR_LOAD(q_load, g_load);                                              \
    step((DEAR_LDS bf16 *)gs##g, (DEAR_LDS float *)deltas##g);
            while (true) {
                rd.renew();
                DEAR_STEP(0, 1, 2, 0)
                DEAR_STEP(1, 0, 0, 1)
                DEAR_STEP(2, 1, 1, 0)
                rd.renew();
                DEAR_STEP(0, 0, 2, 1)
                DEAR_STEP(1, 1, 0, 0)
                DEAR_STEP(2, 0, 1, 1)
            }
#undef DEAR_STEP
#undef DEAR_LOAD
        }
        // the sums of the wave with the other turn, where the tiles were
        __syncthreads();
        static_assert(W / 32 * 16 * 64 * 4 <= STEP * W * 2, "the sums of 32 keys fit a tile");
        DEAR_LDS float *sums = second ? (part / 2 ? (DEAR_LDS float *)gs1 : (DEAR_LDS float *)gs0)
                                      : (part / 2 ? (DEAR_LDS float *)qs1 : (DEAR_LDS float *)qs0);
        if (turn == 1) {
#pragma unroll
            for (int db = 0; db < W / 32; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) sums[(db * 16 + r) * 64 + lane] = sum[db][r];
        }
        __syncthreads();
        if (turn == 0) {
#pragma unroll
            for (int db = 0; db < W / 32; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) sum[db][r] += sums[(db * 16 + r) * 64 + lane];
        }
    }
    if (turn == 1 || j >= a.kv_len) return;
    if (a.splits > 1) {  // dk's come first, then dv's
        store_row<float, W>(part_row(a, a.kv_heads, a.kv_len, second ? split : a.splits + split, b, kvh, j), sum, 1.f, a.head_dim, half);
        return;
    }
    const heads &out = second ? a.dk : a.dv;
    store_row<bf16, W>(at(out, b, kvh) + j * out.token, sum, second ? a.scale : 1.f, a.head_dim, half);
}

// ------------------------------------------------------------------------------------ splits joined
// Eight values of a row a thread; a row of the splits' outputs is [batch, head, token].
struct joined {
    int64_t row;
    int b, h, i, d;
    bool some;
    __device__ __forceinline__ joined(int batch, int heads, int len, int head_dim) {
        const int pieces = head_dim / 8;
        const int64_t n = (int64_t)blockIdx.x * THREADS + threadIdx.x, rows = (int64_t)batch * heads * len;
        row = n / pieces, d = (int)(n % pieces) * 8;
        some = row < rows;
        i = (int)(row % len), h = (int)(row / len % heads), b = (int)(row / len / heads);
    }
};

template <typename T> __device__ __forceinline__ void store_eight(char *p, int d, const float *x) { *(frag<T> *)(p + d * sizeof(T)) = to_frag<T>(x); }

template <typename T> __global__ __launch_bounds__(THREADS) void join_attention_kernel(params a) {
    const joined at_row(a.batch, a.q_heads, a.q_len, a.head_dim);
    if (!at_row.some) return;
    const int64_t rows = (int64_t)a.batch * a.q_heads * a.q_len, row = at_row.row;
    float most = -INFINITY;
    for (int s = 0; s < a.splits; ++s)
        if (a.part_sum[s * rows + row] != 0.f) most = fmaxf(most, a.part_base[s * rows + row]);
    float x[8] = {}, total = 0.f;
    for (int s = 0; s < a.splits; ++s) {
        const float sum = a.part_sum[s * rows + row];
        const float keep = sum == 0.f ? 0.f : __builtin_amdgcn_exp2f(a.part_base[s * rows + row] - most);
        const f32x8 o = *(const f32x8 *)(a.part + (s * rows + row) * a.head_dim + at_row.d);
        if (sum != 0.f) {
            total += sum * keep;
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] += o[u] * keep;
        }
    }
    const bool none = total == 0.f;
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] *= none ? 0.f : 1.f / total;
    store_eight<T>(at(a.out, at_row.b, at_row.h) + at_row.i * a.out.token, at_row.d, x);
    if (at_row.d == 0) a.lse[row] = none ? -INFINITY : (most + __builtin_amdgcn_logf(total)) * LN2;
}

// out = factor * the sum of the splits' rows.
template <typename T>
__global__ __launch_bounds__(THREADS) void join_sums_kernel(const float *part, int splits, heads out, int batch, int n_heads, int len, int head_dim,
                                                            float factor) {
    const joined at_row(batch, n_heads, len, head_dim);
    if (!at_row.some) return;
    const int64_t rows = (int64_t)batch * n_heads * len;
    float x[8] = {};
    for (int s = 0; s < splits; ++s) {
        const f32x8 o = *(const f32x8 *)(part + (s * rows + at_row.row) * head_dim + at_row.d);
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] += o[u];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] *= factor;
    store_eight<T>(at(out, at_row.b, at_row.h) + at_row.i * out.token, at_row.d, x);
}

// ------------------------------------------------------------------------------------ host
constexpr int64_t MAX_LEN = 1 << 30;

bool too_big(int64_t heads, int64_t batch, int64_t tiles) {
    return heads * batch > INT32_MAX || heads * batch * tiles > INT32_MAX;
}

int check_sizes(const dear_attention_t *p) {
    if (!p) return DEAR_EINVAL;
    if (p->batch < 0 || p->q_heads < 1 || p->kv_heads < 1 || p->q_heads % p->kv_heads) return DEAR_EINVAL;
    if (p->head_dim < 8 || p->head_dim > 128 || p->head_dim % 8) return DEAR_EINVAL;
    if (p->q_len < 0 || p->q_len > MAX_LEN || p->kv_len < 0 || p->kv_len > MAX_LEN) return DEAR_EINVAL;
    if (p->dtype != DEAR_F32 && p->dtype != DEAR_BF16) return DEAR_EINVAL;
    if ((p->causal != 0 && p->causal != 1) || p->reserved != 0) return DEAR_EINVAL;
    if (!(p->scale > 0.f) || !std::isfinite(p->scale)) return DEAR_EINVAL;
    if (too_big(p->q_heads, p->batch, ceil_div(p->q_len, BLOCK)) || too_big(p->kv_heads, p->batch, ceil_div(p->kv_len, KEYS)))
        return DEAR_ETOOBIG;
    return DEAR_OK;
}

// Whether a tensor of n tokens is there, and aligned; what is written has a place of its own for every element: from the shortest
// stride on each one is at least as long as what the axes before it span.
int check_heads(const dear_heads_t &t, const dear_attention_t *p, int64_t n, bool written) {
    if (p->batch == 0 || n == 0) return DEAR_OK;
    if (!t.data) return DEAR_EINVAL;
    const int64_t g = p->dtype == DEAR_BF16 ? 2 : 4;
    if (!aligned(t.data, 16) || t.batch_stride * g % 16 || t.token_stride * g % 16 || t.head_stride * g % 16) return DEAR_EALIGN;
    if (t.batch_stride < 0 || t.token_stride < 0 || t.head_stride < 0) return DEAR_EINVAL;
    if (written) {
        struct axis {
            int64_t stride, count;
        } axes[3] = {{t.batch_stride, p->batch}, {t.token_stride, n}, {t.head_stride, &t == &p->dk || &t == &p->dv ? p->kv_heads : p->q_heads}};
        std::sort(axes, axes + 3, [](const axis &a, const axis &b) { return a.stride < b.stride; });
        int64_t span = p->head_dim;
        for (const axis &a : axes) {
            if (a.count == 1) continue;
            if (a.stride < span || a.stride > (INT64_MAX - span) / a.count) return DEAR_EINVAL;
            span += (a.count - 1) * a.stride;
        }
    }
    return DEAR_OK;
}

params make(const dear_attention_t *p) {
    const int64_t g = p->dtype == DEAR_BF16 ? 2 : 4;
    auto t = [g](const dear_heads_t &x) {
        return heads{(char *)x.data, x.batch_stride * g, x.token_stride * g, x.head_stride * g};
    };
    params a = {};
    a.q_heads = p->q_heads, a.kv_heads = p->kv_heads, a.head_dim = p->head_dim, a.causal = p->causal;
    a.q_len = (int32_t)p->q_len, a.kv_len = (int32_t)p->kv_len, a.scale = p->scale, a.batch = p->batch;
    a.q_lens = p->q_lens, a.kv_lens = p->kv_lens;
    a.q = t(p->q), a.k = t(p->k), a.v = t(p->v), a.out = t(p->out);
    a.dout = t(p->dout), a.dq = t(p->dq), a.dk = t(p->dk), a.dv = t(p->dv);
    a.lse = p->lse;
    return a;
}

// Whether the rows of a step lie within 2^31 bytes, so that tiles can be filled directly.  With and without: 2 x 4096, causal, 16
// heads of 128 for 4, forward 160 and 185 us, backward 492 and 812; 16 x 512, 16 heads of 64, 30 and 33, 91 and 126.
bool near(const dear_attention_t *p, const dear_heads_t &t) { return p->dtype == DEAR_BF16 && t.token_stride < (1 << 30) / STEP; }

#define DEAR_BY_TYPE(p, kernel, grid, a, stream)                                                          \
    do {                                                                                                  \
        if ((p)->dtype == DEAR_BF16 && (p)->head_dim <= 64) kernel<bf16, 64><<<grid, THREADS, 0, stream>>>(a); \
        else if ((p)->dtype == DEAR_BF16) kernel<bf16, 128><<<grid, THREADS, 0, stream>>>(a);             \
        else if ((p)->head_dim <= 64) kernel<float, 64><<<grid, THREADS, 0, stream>>>(a);                 \
        else kernel<float, 128><<<grid, THREADS, 0, stream>>>(a);                                         \
    } while (0)

// Workgroups of a launch without splits, and the most threads that one has.
int64_t q_groups(const dear_attention_t *p) { return ceil_div(p->q_len, BLOCK) * p->batch * p->q_heads; }
int64_t kv_groups(const dear_attention_t *p, int keys) { return ceil_div(p->kv_len, keys) * p->batch * p->kv_heads; }
int kv_threads(const dear_attention_t *p) { return p->dtype == DEAR_BF16 && p->head_dim > 64 ? 64 * KV_WAVES : THREADS; }

// Splits of the sequence that workgroups go through, where there are too few of them for the chip: the number with the least
// time by this estimate, in microseconds.  The chip takes 256 * `resident` workgroups at a time; one goes through its share of
// the steps in `step` each (in a causal call the longest does, and all together half of them); joining the splits costs `join`,
// and 3 TB/s for `bytes` of output each.  Measured with and without: one query, 8 heads, 8192 keys of 128 values 29 and 164 us;
// 4 sequences of 656 with 2 key heads for 8, backward 45 and 88.
int splits_for(const dear_attention_t *p, int64_t groups, int threads, int64_t steps, double step, double resident, double join, double bytes) {
    int best = 1;
    double least = 0;
    // (joining takes a thread for eight values of 4 bytes)
    for (int64_t s = 1; s <= 16 && (s == 1 || (s <= steps && groups * s * threads <= MAX_THREADS && bytes <= 32. * MAX_THREADS)); ++s) {
        const double turns = (double)(groups * s) / (256 * resident), share = (double)ceil_div(steps, s) * step;
        const double t = (p->causal ? std::fmax(1, turns / 2) : std::ceil(turns)) * share + (s == 1 ? 0 : join + (double)s * bytes / 3e6);
        if (s == 1 || t < least) best = (int)s, least = t;
    }
    return best;
}

// A step of 64 keys or queries: bf16, waiting for its loads, 0.6 to 1.5 us; fp32, by its matrix instructions, 4.2 and, with the
// backward pass's products, 7.5 for each 64 values of a row.
int q_splits(const dear_attention_t *p, bool backward) {
    const bool wide = p->head_dim > 64, f32 = p->dtype == DEAR_F32;
    const double step = f32 ? (backward ? 7.5 : 4.2) * (wide ? 2 : 1) : (backward ? 0.8 : 0.6) * (wide ? 1.5 : 1);
    const int64_t rows = p->q_len * p->batch * p->q_heads;
    return splits_for(p, q_groups(p), THREADS, ceil_div(p->kv_len, STEP), step,
                      f32 ? 1 : wide || backward ? 2 : 4, 8, (double)(rows * p->head_dim * 4));
}
int kv_splits(const dear_attention_t *p, int keys) {
    const bool wide = p->head_dim > 64, f32 = p->dtype == DEAR_F32;
    const double step = (f32 ? 7.5 * (wide ? 2 : 1) : wide ? 1.2 : 1) * (p->q_heads / p->kv_heads);
    const int64_t rows = p->kv_len * p->batch * p->kv_heads;
    const int64_t seen = p->causal ? std::min(p->q_len, p->kv_len) : p->q_len;  // queries that a key is visible to, at most
    return splits_for(p, kv_groups(p, keys), kv_threads(p), ceil_div(seen, STEP), step, f32 || wide ? 1 : 2, 16,
                      (double)(2 * rows * p->head_dim * 4));
}

// What the splits' outputs take until they are joined.
int64_t forward_bytes(const dear_attention_t *p) {
    const int n = q_splits(p, false);
    return n > 1 ? ceil_div(n * p->q_len * p->batch * p->q_heads * (p->head_dim + 2) * 4, 256) * 256 : 0;
}
int64_t dq_bytes(const dear_attention_t *p) {
    const int n = q_splits(p, true);
    return n > 1 ? n * p->q_len * p->batch * p->q_heads * p->head_dim * 4 : 0;
}
int64_t dkv_bytes(const dear_attention_t *p, int keys) {
    const int n = kv_splits(p, keys);
    return n > 1 ? 2 * n * p->kv_len * p->batch * p->kv_heads * p->head_dim * 4 : 0;
}
int64_t rows_bytes(const dear_attention_t *p) { return ceil_div(p->q_len, BLOCK) * BLOCK * p->batch * p->q_heads * 8; }

int check_workspace(const dear_attention_t *p, int64_t need) {
    if (need == 0) return DEAR_OK;
    if (!p->workspace) return DEAR_EINVAL;
    if (!aligned(p->workspace, 256)) return DEAR_EALIGN;
    return p->workspace_bytes < need ? DEAR_ETOOBIG : DEAR_OK;
}

unsigned join_grid(const dear_attention_t *p, int64_t heads, int64_t len) {
    return (unsigned)ceil_div(p->batch * heads * len * (p->head_dim / 8), THREADS);
}

}  // namespace

extern "C" {

int dear_attention_workspace(const dear_attention_t *p, int64_t *bytes) {
    if (!bytes) return DEAR_EINVAL;
    if (int rc = check_sizes(p)) return rc;
    *bytes = forward_bytes(p);
    return DEAR_OK;
}

int dear_attention_backward_workspace(const dear_attention_t *p, int64_t *bytes) {
    if (!bytes) return DEAR_EINVAL;
    if (int rc = check_sizes(p)) return rc;
    // of every query of every tile two values, and the splits' outputs, dq's and then dk's and dv's; strides may call for
    // either width of tiles
    int64_t parts = dq_bytes(p);
    for (int keys : {KEYS, BLOCK})
        if (dkv_bytes(p, keys) > parts) parts = dkv_bytes(p, keys);
    *bytes = rows_bytes(p) + parts;
    return DEAR_OK;
}

int dear_attention(const dear_attention_t *p, void *hip_stream) {
    if (int rc = check_sizes(p)) return rc;
    if (int rc = check_heads(p->q, p, p->q_len, false)) return rc;
    if (int rc = check_heads(p->k, p, p->kv_len, false)) return rc;
    if (int rc = check_heads(p->v, p, p->kv_len, false)) return rc;
    if (int rc = check_heads(p->out, p, p->q_len, true)) return rc;
    if (p->batch == 0 || p->q_len == 0) return DEAR_OK;
    if (!p->lse) return DEAR_EINVAL;
    if (!aligned(p->lse, 4)) return DEAR_EALIGN;
    if (q_groups(p) * THREADS > MAX_THREADS) return DEAR_ETOOBIG;
    if (int rc = check_workspace(p, forward_bytes(p))) return rc;
    params a = make(p);
    a.tiles = (int32_t)ceil_div(p->q_len, BLOCK), a.splits = q_splits(p, false);
    const int64_t rows = p->q_len * p->batch * p->q_heads;
    a.part = (float *)p->workspace, a.part_base = a.part + a.splits * rows * p->head_dim, a.part_sum = a.part_base + a.splits * rows;
    const unsigned grid = (unsigned)a.tiles * p->q_heads * p->batch * a.splits;
    hipStream_t stream = (hipStream_t)hip_stream;
    const bool direct = near(p, p->k) && near(p, p->v);
    if (direct && p->head_dim <= 64) attention_direct_kernel<64><<<grid, THREADS, 0, stream>>>(a);
    else if (direct) attention_direct_kernel<128><<<grid, THREADS, 0, stream>>>(a);
    else DEAR_BY_TYPE(p, attention_kernel, grid, a, stream);
    if (int rc = launch_status()) return rc;
    if (a.splits > 1) {
        const unsigned join = join_grid(p, p->q_heads, p->q_len);
        if (p->dtype == DEAR_BF16) join_attention_kernel<bf16><<<join, THREADS, 0, stream>>>(a);
        else join_attention_kernel<float><<<join, THREADS, 0, stream>>>(a);
        return launch_status();
    }
    return DEAR_OK;
}

int dear_attention_backward(const dear_attention_t *p, void *hip_stream) {
    if (int rc = check_sizes(p)) return rc;
    for (const dear_heads_t *t : {&p->q, &p->out, &p->dout})
        if (int rc = check_heads(*t, p, p->q_len, false)) return rc;
    for (const dear_heads_t *t : {&p->k, &p->v})
        if (int rc = check_heads(*t, p, p->kv_len, false)) return rc;
    if (int rc = check_heads(p->dq, p, p->q_len, true)) return rc;
    for (const dear_heads_t *t : {&p->dk, &p->dv})
        if (int rc = check_heads(*t, p, p->kv_len, true)) return rc;
    if (p->batch == 0 || (p->q_len == 0 && p->kv_len == 0)) return DEAR_OK;
    if (p->q_len > 0) {
        if (!p->lse) return DEAR_EINVAL;
        if (!aligned(p->lse, 4)) return DEAR_EALIGN;
    }
    const bool direct = near(p, p->q) && near(p, p->dout) && near(p, p->k) && near(p, p->v);
    const int keys = direct && p->head_dim <= 64 ? BLOCK : KEYS;
    if (q_groups(p) * THREADS > MAX_THREADS || kv_groups(p, keys) * kv_threads(p) > MAX_THREADS) return DEAR_ETOOBIG;
    int64_t need = 0;
    (void)dear_attention_backward_workspace(p, &need);
    if (int rc = check_workspace(p, need)) return rc;
    params a = make(p);
    hipStream_t stream = (hipStream_t)hip_stream;
    const int64_t q_tiles = ceil_div(p->q_len, BLOCK), kv_tiles = ceil_div(p->kv_len, keys);
    a.q_tiles = (int32_t)q_tiles;
    a.powers = (float *)p->workspace, a.deltas = a.powers + q_tiles * BLOCK * p->batch * p->q_heads;
    a.part = (float *)((char *)p->workspace + rows_bytes(p));
    auto join = [&](const float *part, const heads &out, int n_heads, int64_t len, float factor) {
        const unsigned grid = join_grid(p, n_heads, len);
        if (p->dtype == DEAR_BF16)
            join_sums_kernel<bf16><<<grid, THREADS, 0, stream>>>(part, a.splits, out, p->batch, n_heads, (int)len, p->head_dim, factor);
        else
            join_sums_kernel<float><<<grid, THREADS, 0, stream>>>(part, a.splits, out, p->batch, n_heads, (int)len, p->head_dim, factor);
        return launch_status();
    };
    if (q_tiles) {
        a.tiles = (int32_t)q_tiles, a.splits = q_splits(p, true);
        const unsigned grid = (unsigned)q_tiles * p->q_heads * p->batch * a.splits;
        if (direct && p->head_dim <= 64) attention_dq_direct_kernel<64><<<grid, THREADS, 0, stream>>>(a);
        else if (direct) attention_dq_direct_kernel<128><<<grid, THREADS, 0, stream>>>(a);
        else DEAR_BY_TYPE(p, attention_dq_kernel, grid, a, stream);
        if (int rc = launch_status()) return rc;
        if (a.splits > 1)
            if (int rc = join(a.part, a.dq, p->q_heads, p->q_len, p->scale)) return rc;
    }
    if (kv_tiles) {
        a.tiles = (int32_t)kv_tiles, a.splits = kv_splits(p, keys);
        const unsigned grid = (unsigned)kv_tiles * p->kv_heads * p->batch * a.splits;
        if (direct && p->head_dim <= 64) attention_dkv_direct_kernel<<<grid, THREADS, 0, stream>>>(a);
        else if (direct) attention_dkv_halves_kernel<<<grid, 64 * KV_WAVES, 0, stream>>>(a);
        else DEAR_BY_TYPE(p, attention_dkv_kernel, grid, a, stream);
        if (int rc = launch_status()) return rc;
        if (a.splits > 1) {
            const int64_t all = a.splits * p->kv_len * p->batch * p->kv_heads * p->head_dim;
            if (int rc = join(a.part, a.dk, p->kv_heads, p->kv_len, p->scale)) return rc;
            if (int rc = join(a.part + all, a.dv, p->kv_heads, p->kv_len, 1.f)) return rc;
        }
    }
    return DEAR_OK;
}

}  // extern "C"
