// Gradient of a linear layer's weight from the checkpoint of its input (definitions: dear_ops.h).
//
//     dw[n, k] = sum over m of dy[m, n] * code[m, k] * 2^e[m, k / 32]
//
// The sum runs over the rows of both operands, so both are read from LDS with the transposing reads.  A checkpoint's
// value has 7 significant bits, so that it becomes an operand in bf16 without any rounding: products are exact, and what
// is rounded is the fp32 sum alone.
#include "ops_common.h"

#pragma clang fp contract(fast)

namespace {

using namespace dear_ops;

constexpr int THREADS = 256;
constexpr int BN = 128, BK = 128, BM = 32;  // outs and ins of a workgroup, rows of a step
constexpr int GROUP = DEAR_CHECKPOINT_GROUP;

struct params {
    const void *dy;
    const int8_t *codes;
    const uint8_t *exponents;
    int64_t dy_stride, rows, chunk;  // chunk: rows of one split
    int32_t outs, ins, padded, groups, n_tiles, k_tiles;
    float *out;  // [splits, outs, ins]
};

template <typename T, bool VEC> __global__ __launch_bounds__(THREADS) void weight_grad_kernel(params a) {
    __shared__ __attribute__((aligned(16))) char lds[tile<T, BN>::bytes(BM) + tile<T, BK>::bytes(BM)];
    DEAR_LDS T *ys = (DEAR_LDS T *)lds, *xs = (DEAR_LDS T *)(lds + tile<T, BN>::bytes(BM));
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const unsigned per_split = (unsigned)a.n_tiles * a.k_tiles, split = blockIdx.x / per_split, id = blockIdx.x % per_split;
    const int n0 = (int)(id / a.k_tiles) * BN, k0 = (int)(id % a.k_tiles) * BK;
    const int64_t begin = (int64_t)split * a.chunk, end = min(a.rows, begin + a.chunk);
    f32x16 acc[2][2] = {};
    for (int64_t m0 = begin; m0 < end; m0 += BM) {
        __syncthreads();
        constexpr int E = 16 / sizeof(T);
#pragma unroll
        for (int i = 0; i < BM * BN / E / THREADS; ++i) {
            const int c = threadIdx.x + i * THREADS, row = c / (BN / E), col = c % (BN / E) * E;
            typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
            vec v;
            const T *p = (const T *)a.dy + (m0 + row) * a.dy_stride + n0 + col;
#pragma unroll
            for (int u = 0; u < E; ++u) v[u] = (T)0.f;
            if (m0 + row < end) {
                if (VEC) {
                    if (n0 + col < a.outs) v = *(const vec *)p;
                } else {
#pragma unroll
                    for (int u = 0; u < E; ++u)
                        if (n0 + col + u < a.outs) v[u] = p[u];
                }
            }
            *(DEAR_LDS vec *)(ys + row * tile<T, BN>::stride + col) = v;
        }
        {
            // 16 codes a thread: one group's half
            const int row = threadIdx.x / (BK / 16), col = threadIdx.x % (BK / 16) * 16;
            u32x4 q = {0, 0, 0, 0};
            uint32_t e = 0;
            if (m0 + row < end && k0 + col < a.padded) {
                q = *(const u32x4 *)(a.codes + (m0 + row) * a.padded + k0 + col);
                e = a.exponents[(m0 + row) * a.groups + (k0 + col) / GROUP];
            }
            const float step = __uint_as_float(e << 23);
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float x[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) x[t] = (float)((int)(q[2 * w + t / 4] << (24 - 8 * (t % 4))) >> 24) * step;
                *(DEAR_LDS frag<T> *)(xs + row * tile<T, BK>::stride + col + 8 * w) = to_frag<T>(x);
            }
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < BM / 16; ++s) {
            frag<T> y[2], x[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                y[u] = transposed<BN>(ys, 16 * s, (wave / 2) * 64 + 32 * u, lane);
                x[u] = transposed<BK>(xs, 16 * s, (wave % 2) * 64 + 32 * u, lane);
            }
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int w = 0; w < 2; ++w) acc[u][w] = mma(y[u], x[w], acc[u][w]);
        }
    }
    float *out = a.out + (int64_t)split * a.outs * a.ins;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int k = k0 + (wave % 2) * 64 + 32 * w + (lane & 31);
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int n = n0 + (wave / 2) * 64 + 32 * u + row_of(r, lane >> 5);
                if (n < a.outs && k < a.ins) out[(int64_t)n * a.ins + k] = acc[u][w][r];
            }
        }
}

__global__ __launch_bounds__(256) void split_sum_kernel(const float *part, int splits, int64_t n, float *out) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float s = 0.f;
    for (int k = 0; k < splits; ++k) s += part[k * n + i];
    out[i] = s;
}

// ------------------------------------------------------------------------------------ host
constexpr int64_t MAX_WIDTH = 1 << 24, MAX_ROWS = (int64_t)1 << 40;

// Splits of the rows: as many as it takes for 512 workgroups, with no fewer than 256 rows each.
int splits_of(int64_t rows, int64_t outs, int64_t ins) {
    const int64_t tiles = ceil_div(outs, BN) * ceil_div(ins, BK);
    int64_t n = 512 / tiles;
    if (n > rows / 256) n = rows / 256;
    return n < 1 ? 1 : (int)n;
}

int check(int32_t dtype, int64_t rows, int64_t outs, int64_t ins) {
    if (dtype != DEAR_F32 && dtype != DEAR_BF16) return DEAR_EINVAL;
    if (rows < 0 || rows > MAX_ROWS || outs < 1 || outs > MAX_WIDTH || ins < 1 || ins > MAX_WIDTH) return DEAR_EINVAL;
    return DEAR_OK;
}

}  // namespace

extern "C" {

int dear_checkpoint_weight_grad_workspace(int32_t dtype, int64_t rows, int64_t outs, int64_t ins, int64_t *bytes) {
    if (!bytes) return DEAR_EINVAL;
    if (int rc = check(dtype, rows, outs, ins)) return rc;
    const int splits = splits_of(rows, outs, ins);
    *bytes = splits > 1 ? splits * outs * ins * 4 : 0;
    return DEAR_OK;
}

int dear_checkpoint_weight_grad(const void *dy, int32_t dtype, int64_t dy_stride, const int8_t *codes, const uint8_t *exponents,
                                int64_t rows, int64_t outs, int64_t ins, float *dw, void *workspace, int64_t workspace_bytes,
                                void *hip_stream) {
    int64_t need = 0;
    if (int rc = dear_checkpoint_weight_grad_workspace(dtype, rows, outs, ins, &need)) return rc;
    const int size = dtype == DEAR_BF16 ? 2 : 4;
    if (!dw || (rows > 0 && (!dy || !codes || !exponents)) || (need && !workspace)) return DEAR_EINVAL;
    if (rows > 1 && dy_stride < outs) return DEAR_EINVAL;
    if (!aligned(dw, 16) || !aligned(dy, size) || !aligned(codes, 16) || !aligned(workspace, 256)) return DEAR_EALIGN;
    if (need > workspace_bytes) return DEAR_ETOOBIG;
    hipStream_t stream = (hipStream_t)hip_stream;
    const int splits = splits_of(rows, outs, ins);
    params a = {};
    a.dy = dy, a.codes = codes, a.exponents = exponents, a.dy_stride = dy_stride, a.rows = rows;
    a.chunk = ceil_div(ceil_div(rows, splits), BM) * BM;
    a.outs = (int32_t)outs, a.ins = (int32_t)ins, a.groups = (int32_t)ceil_div(ins, GROUP), a.padded = a.groups * GROUP;
    a.n_tiles = (int32_t)ceil_div(outs, BN), a.k_tiles = (int32_t)ceil_div(ins, BK);
    a.out = splits > 1 ? (float *)workspace : dw;
    const int64_t groups = (int64_t)a.n_tiles * a.k_tiles * splits;
    if (groups > INT32_MAX || ceil_div(outs * ins, 256) > INT32_MAX) return DEAR_ETOOBIG;
    const unsigned grid = (unsigned)groups;
    const bool vec = aligned(dy, 16) && dy_stride * size % 16 == 0 && outs * size % 16 == 0;
    if (dtype == DEAR_BF16 && vec) weight_grad_kernel<bf16, true><<<grid, THREADS, 0, stream>>>(a);
    else if (dtype == DEAR_BF16) weight_grad_kernel<bf16, false><<<grid, THREADS, 0, stream>>>(a);
    else if (vec) weight_grad_kernel<float, true><<<grid, THREADS, 0, stream>>>(a);
    else weight_grad_kernel<float, false><<<grid, THREADS, 0, stream>>>(a);
    if (int rc = launch_status()) return rc;
    if (splits > 1) {
        split_sum_kernel<<<(unsigned)ceil_div(outs * ins, 256), 256, 0, stream>>>((const float *)workspace, splits, outs * ins, dw);
        return launch_status();
    }
    return DEAR_OK;
}

}  // extern "C"
