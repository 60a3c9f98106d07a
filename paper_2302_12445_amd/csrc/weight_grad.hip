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

// ------------------------------------------------------------------------------------ bf16, whole vectors
// A workgroup owns 128 x 128 outputs and each of its four waves sums all of them over rows of its own, 32 of every 128:
// a wave reads eight fragments for sixteen products, and the waves meet only at the end, to add their sums.
constexpr int WROWS = 32;                            // rows of a wave's step
constexpr int WSTEP = WROWS * (THREADS / 64);        // rows of a workgroup's step
constexpr int WTILE = WROWS * tile<bf16, 128>::stride;  // elements of one operand's tile

struct wave_step {
    u32x4 y[8], x[4];
    uint32_t e[4];
};

template <bool WHOLE>
__device__ __forceinline__ void load_step(wave_step &w, const char *y, const int8_t *x, const uint8_t *e, uint32_t y_off, uint32_t x_off,
                                          uint32_t e_off, uint32_t y_stride, uint32_t x_stride, uint32_t e_stride, int lane, int left) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int row = 4 * i + lane / 16;
        w.y[i] = *(const u32x4 *)(y + (y_off + (uint32_t)(WHOLE ? row : min(row, left - 1)) * y_stride));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int row = 8 * i + lane / 8, r = WHOLE ? row : min(row, left - 1);
        w.x[i] = *(const u32x4 *)(x + (x_off + (uint32_t)r * x_stride));
        w.e[i] = e[e_off + (uint32_t)r * e_stride];
        // rows beyond the last repeat it, times 0
        if (!WHOLE && row >= left) w.e[i] = 0;
    }
}

__device__ __forceinline__ void store_step(const wave_step &w, DEAR_LDS bf16 *ys, DEAR_LDS bf16 *xs, int lane) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        *(DEAR_LDS u32x4 *)(ys + (4 * i + lane / 16) * tile<bf16, 128>::stride + lane % 16 * 8) = w.y[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float step = __uint_as_float(w.e[i] << 23);
        u32x4 q[2];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const uint32_t c = w.x[i][k / 2];
            const float lo = (float)((int)(c << (24 - 16 * (k % 2))) >> 24) * step;
            const float hi = (float)((int)(c << (16 - 16 * (k % 2))) >> 24) * step;
            // both are bf16 values: their upper halves
            q[k / 4][k % 4] = __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
        }
        DEAR_LDS bf16 *p = xs + (8 * i + lane / 8) * tile<bf16, 128>::stride + lane % 8 * 16;
        *(DEAR_LDS u32x4 *)p = q[0];
        *(DEAR_LDS u32x4 *)(p + 8) = q[1];
    }
}

__device__ __forceinline__ void multiply_step(f32x16 (&acc)[4][4], const DEAR_LDS bf16 *ys, const DEAR_LDS bf16 *xs, int lane) {
#pragma unroll
    for (int s = 0; s < WROWS / 16; ++s) {
        bf16x8 y[4], x[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            y[u] = transposed<128>(ys, 16 * s, 32 * u, lane);
            x[u] = transposed<128>(xs, 16 * s, 32 * u, lane);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int v = 0; v < 4; ++v) acc[u][v] = mma(y[u], x[v], acc[u][v]);
    }
}

__global__ __launch_bounds__(THREADS, 1) void weight_grad_wide_kernel(params a) {
    // first two buffers of two tiles for each wave, then the waves' sums, two quarters at a time
    __shared__ __attribute__((aligned(16))) char lds[4 * 4 * WTILE * sizeof(bf16)];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const unsigned per_split = (unsigned)a.n_tiles * a.k_tiles, split = blockIdx.x / per_split, id = blockIdx.x % per_split;
    const int n0 = (int)(id % a.n_tiles) * 128, k0 = (int)(id / a.n_tiles) * 128;
    const int64_t begin = (int64_t)split * a.chunk + wave * WROWS, end = min(a.rows, (int64_t)(split + 1) * a.chunk);
    DEAR_LDS bf16 *const buf = (DEAR_LDS bf16 *)lds + wave * 4 * WTILE;

    f32x16 acc[4][4] = {};
    // outputs beyond the last repeat the first: they are not stored
    const uint32_t y_stride = (uint32_t)a.dy_stride * 2, x_stride = (uint32_t)a.padded, e_stride = (uint32_t)a.groups;
    const int yc = n0 + lane % 16 * 8, xc = k0 + lane % 8 * 16;
    const uint32_t y_off = (uint32_t)(yc < a.outs ? yc : 0) * 2, x_off = xc < a.padded ? xc : 0, e_off = x_off / GROUP;
    const char *y = (const char *)a.dy + begin * a.dy_stride * 2;
    const int8_t *x = a.codes + begin * a.padded;
    const uint8_t *e = a.exponents + begin * a.groups;
    const int64_t rows = end - begin, steps = rows > 0 ? (rows + WSTEP - 1) / WSTEP : 0;  // of this wave
    const int last = (int)(rows - (steps - 1) * WSTEP);  // rows from the last step on
    wave_step w;
    // step t: its operands go to LDS while the products of the step before run, and come from memory one step earlier
    auto load = [&](bool whole) {
        if (whole) load_step<true>(w, y, x, e, y_off, x_off, e_off, y_stride, x_stride, e_stride, lane, 0);
        else load_step<false>(w, y, x, e, y_off, x_off, e_off, y_stride, x_stride, e_stride, lane, last);
        y += (int64_t)WSTEP * y_stride, x += (int64_t)WSTEP * x_stride, e += (int64_t)WSTEP * e_stride;
    };
    if (steps > 0) {
        load(steps > 1);
        store_step(w, buf, buf + WTILE, lane);
        if (steps > 1) load(steps > 2);
        int64_t t = 0;
        DEAR_LDS bf16 *now = buf, *next = buf + 2 * WTILE;
        for (; t + 3 < steps; ++t) {
            multiply_step(acc, now, now + WTILE, lane);
            store_step(w, next, next + WTILE, lane);
            load(true);
            DEAR_LDS bf16 *const other = now;
            now = next, next = other;
        }
        for (; t < steps; ++t) {
            multiply_step(acc, now, now + WTILE, lane);
            if (t + 1 < steps) store_step(w, next, next + WTILE, lane);
            if (t + 2 < steps) load(false);
            DEAR_LDS bf16 *const other = now;
            now = next, next = other;
        }
    }

    float *out = a.out + (int64_t)split * a.outs * a.ins;
    DEAR_LDS float *sums = (DEAR_LDS float *)lds;  // [wave][64 rows][128]
    const bool vec = a.ins % 4 == 0;
#pragma unroll
    for (int pair = 0; pair < 2; ++pair) {
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    sums[(wave * 64 + 32 * u + row_of(r, lane >> 5)) * 128 + 32 * v + (lane & 31)] = acc[2 * pair + u][v][r];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = 8 * i + threadIdx.x / 32, col = threadIdx.x % 32 * 4;
            f32x4 t = *(DEAR_LDS f32x4 *)(sums + row * 128 + col);
#pragma unroll
            for (int k = 1; k < 4; ++k) t += *(DEAR_LDS f32x4 *)(sums + (k * 64 + row) * 128 + col);
            const int n = n0 + 64 * pair + row, k = k0 + col;
            if (n < a.outs) {
                float *p = out + (int64_t)n * a.ins + k;
                if (vec) {
                    if (k < a.ins) *(f32x4 *)p = t;
                } else {
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        if (k + q < a.ins) p[q] = t[q];
                }
            }
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

// Whether the wide kernel takes it: bf16 in whole vectors, with rows that 32-bit offsets reach.
bool wide(int32_t dtype, int64_t dy_stride, int64_t outs) {
    return dtype == DEAR_BF16 && outs % 8 == 0 && dy_stride < (1 << 24);
}

// Splits of the rows, each a sum of its own in the workspace: as many as it takes for 512 workgroups, with no fewer than
// 256 rows each.
int splits_of(int64_t rows, int64_t outs, int64_t ins) {
    const int64_t tiles = ceil_div(outs, BN) * ceil_div(ins, BK);
    int64_t n = 256 / tiles;
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
    a.chunk = ceil_div(ceil_div(rows, splits), WSTEP) * WSTEP;
    a.outs = (int32_t)outs, a.ins = (int32_t)ins, a.groups = (int32_t)ceil_div(ins, GROUP), a.padded = a.groups * GROUP;
    a.n_tiles = (int32_t)ceil_div(outs, BN), a.k_tiles = (int32_t)ceil_div(ins, BK);
    a.out = splits > 1 ? (float *)workspace : dw;
    const int64_t groups = (int64_t)a.n_tiles * a.k_tiles * splits;
    if (groups > INT32_MAX || ceil_div(outs * ins, 256) > INT32_MAX) return DEAR_ETOOBIG;
    const unsigned grid = (unsigned)groups;
    const bool vec = aligned(dy, 16) && dy_stride * size % 16 == 0 && outs * size % 16 == 0;
    if (vec && wide(dtype, dy_stride, outs)) weight_grad_wide_kernel<<<grid, THREADS, 0, stream>>>(a);
    else if (dtype == DEAR_BF16 && vec) weight_grad_kernel<bf16, true><<<grid, THREADS, 0, stream>>>(a);
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
