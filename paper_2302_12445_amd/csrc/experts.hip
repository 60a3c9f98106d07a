// Products of rows with the weights of their experts, and both gradients (definitions: dear_ops.h).
//
//     y[m, n] = sum over k of x[m, k] w[e, n, k];  dx[m, k] = sum over n of dy[m, n] w[e, n, k]
//     dw[e, n, k] = sum over the rows m of e of dy[m, n] x[m, k]
//
// All three are sums of products of two operands that lie in memory either along the summed index (x and w for y, dy for dx) or across
// it (w for dx, both for dw); the former are read from LDS in rows, the latter with the transposing reads.  Rows of an expert start
// anywhere: a workgroup finds the expert of its tile from the ends, on the device, so that nothing waits for the host to know them.
#include <type_traits>

#include "ops_common.h"

#pragma clang fp contract(fast)

namespace {

using namespace dear_ops;

enum product { LINEAR, INPUT_GRAD, WEIGHT_GRAD };

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
constexpr int THREADS = 256;
constexpr int BA = 128, BB = 128, BS = 32;  // outputs' rows and columns of a workgroup, summed index of a step

// An operand's part of a step on its way from memory to LDS, in pieces of 16 bytes: BA rows of BS values along the summed index or, ACROSS
// it, BS rows of BA values.  Values beyond the sum are zeros in both operands, so that nothing that stands there counts; rows and columns
// beyond the outputs are whatever is there, and not stored.
template <typename T, bool VEC, bool ACROSS> struct stage {
    static constexpr int E = 16 / sizeof(T), N = BA * BS / E / THREADS, W = ACROSS ? BA : BS;
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
    typedef vec vec_anywhere __attribute__((aligned(sizeof(T))));  // global memory takes 16-byte loads from any element on
    vec v[N];

    // rows: of the operand in memory; row0, col0: the step's first; row_end, col_end: behind the last that may be read
    __device__ __forceinline__ void load(const T *data, int64_t stride, int64_t row0, int64_t row_end, int col0, int col_end) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * THREADS, col = col0 + c % (W / E) * E;
            const int64_t row = row0 + c / (W / E);
            const T *p = data + row * stride + col;
#pragma unroll
            for (int u = 0; u < E; ++u) v[i][u] = (T)0.f;
            if (row < row_end) {
                if (VEC) {
                    if (col < col_end) v[i] = *(const vec *)p;
                } else if (col + E <= col_end) {
                    v[i] = *(const vec_anywhere *)p;
                } else {
#pragma unroll
                    for (int u = 0; u < E - 1; ++u)
                        if (col + u < col_end) v[i][u] = p[u];
                }
            }
        }
    }
    __device__ __forceinline__ void store(DEAR_LDS T *s) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * THREADS;
            *(DEAR_LDS vec *)(s + c / (W / E) * tile<T, W>::stride + c % (W / E) * E) = v[i];
        }
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

// 128 x 128 outputs a workgroup, 64 x 64 a wave; a step's operands go through registers to LDS, the next one's loads beside its products.
template <typename T, bool VEC, int KIND> __global__ __launch_bounds__(THREADS, 2) void experts_kernel(params p) {
    constexpr bool A_ACROSS = KIND == WEIGHT_GRAD, B_ACROSS = KIND != LINEAR;
    typedef stage<T, VEC, A_ACROSS> stage_a;
    typedef stage<T, VEC, B_ACROSS> stage_b;
    constexpr int BYTES_A = tile<T, stage_a::W>::bytes(A_ACROSS ? BS : BA), BYTES_B = tile<T, stage_b::W>::bytes(B_ACROSS ? BS : BB);
    __shared__ __attribute__((aligned(16))) char lds[BYTES_A + BYTES_B];
    DEAR_LDS T *as = (DEAR_LDS T *)lds, *bs = (DEAR_LDS T *)(lds + BYTES_A);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned per = (unsigned)p.a_tiles * p.b_tiles;
    const unsigned id = KIND == WEIGHT_GRAD ? blockIdx.x % per : blockIdx.x;
    const part t = KIND == WEIGHT_GRAD ? rows_of(p, (int)(blockIdx.x / per)) : find<BA>(p, (int)(id / p.b_tiles));
    if (t.none) return;
    const int b0 = (int)(id % p.b_tiles) * BB, a0 = KIND == WEIGHT_GRAD ? (int)(id / p.b_tiles) * BA : 0;
    const bool behind = KIND != WEIGHT_GRAD && t.expert == p.experts;  // rows of no expert
    const int64_t begin = KIND == WEIGHT_GRAD ? t.begin : 0, end = behind ? 0 : KIND == WEIGHT_GRAD ? t.end : p.sum;
    const T *a = (const T *)p.a, *b = (const T *)p.b;
    if (KIND == LINEAR) b += (int64_t)t.expert * p.n_b * p.sum;
    if (KIND == INPUT_GRAD) b += (int64_t)t.expert * p.sum * p.n_b;
    f32x16 acc[2][2] = {};
    stage_a sa;
    stage_b sb;
    auto load = [&](int64_t s0) {
        if (KIND == WEIGHT_GRAD) sa.load(a, p.a_stride, s0, end, a0, p.n_a);
        else sa.load(a, p.a_stride, t.first, t.end, (int)s0, (int)end);
        if (B_ACROSS) sb.load(b, p.b_stride, s0, end, b0, p.n_b);
        else sb.load(b, p.b_stride, b0, p.n_b, (int)s0, (int)end);
    };
    if (begin < end) load(begin);
    for (int64_t s0 = begin; s0 < end; s0 += BS) {
        __syncthreads();
        sa.store(as);
        sb.store(bs);
        __syncthreads();
        if (s0 + BS < end) load(s0 + BS);
#pragma unroll
        for (int s = 0; s < BS / 16; ++s) {
            frag<T> f[2], g[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int row = (wave / 2) * 64 + 32 * u, col = (wave % 2) * 64 + 32 * u;
                f[u] = A_ACROSS ? transposed<stage_a::W>(as, 16 * s, row, lane) : along<stage_a::W>(as, row, s, lane);
                g[u] = B_ACROSS ? transposed<stage_b::W>(bs, 16 * s, col, lane) : along<stage_b::W>(bs, col, s, lane);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int w = 0; w < 2; ++w) acc[u][w] = mma(f[u], g[w], acc[u][w]);
        }
    }
    typedef typename std::conditional<KIND == WEIGHT_GRAD, float, T>::type O;
    const int64_t row0 = KIND == WEIGHT_GRAD ? a0 : t.first, row_end = KIND == WEIGHT_GRAD ? p.n_a : t.end;
    O *out = (O *)p.out + (KIND == WEIGHT_GRAD ? (int64_t)t.expert * p.n_a * p.n_b : 0);
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int col = b0 + (wave % 2) * 64 + 32 * w + (lane & 31);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int64_t row = row0 + (wave / 2) * 64 + 32 * u + row_of(r, lane >> 5);
                if (row < row_end && col < p.n_b) out[row * p.n_b + col] = (O)acc[u][w][r];
            }
        }
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

template <int KIND> int64_t workspace_of(const dear_experts_t &) { return 0; }

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
    // tiles of rows: each expert, and the rows behind the last, may have one that is not whole
    p.a_tiles = (int32_t)(KIND == WEIGHT_GRAD ? ceil_div(x->outs, BA) : x->rows / BA + x->experts + 1);
    p.b_tiles = (int32_t)ceil_div(p.n_b, BB);
    const int64_t groups = (int64_t)p.a_tiles * p.b_tiles * (KIND == WEIGHT_GRAD ? x->experts : 1);
    if (groups * THREADS > MAX_THREADS) return DEAR_ETOOBIG;
    const unsigned n = (unsigned)groups;
    if (x->dtype == DEAR_BF16) {
        if (vec) experts_kernel<bf16, true, KIND><<<n, THREADS, 0, stream>>>(p);
        else experts_kernel<bf16, false, KIND><<<n, THREADS, 0, stream>>>(p);
    } else {
        if (vec) experts_kernel<float, true, KIND><<<n, THREADS, 0, stream>>>(p);
        else experts_kernel<float, false, KIND><<<n, THREADS, 0, stream>>>(p);
    }
    return launch_status();
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
