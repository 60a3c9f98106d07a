// Residual addition + root-mean-square norm with its backward pass, and checkpoints in 8 bits
// (definitions: dear_ops.h).  All of it is bound by HBM: each tensor is read or written once, in 16-byte pieces, a row of the
// norm staying in registers between its sum and its output.  All arithmetic is fp32; what is stored is rounded once, and codes
// are of y as it is stored, so that a checkpoint of y is the same whether the norm or encode wrote it.
#include <cmath>
#include <type_traits>

#include "ops_common.h"

#pragma clang fp contract(fast)

namespace {

using namespace dear_ops;

constexpr int GROUP = DEAR_CHECKPOINT_GROUP;
constexpr int LANE = 8;  // neighbours that a lane holds: four lanes share a group

// ------------------------------------------------------------------------------------ eight neighbours of a row
// Whole vectors, aligned where rows start on multiples of 16 bytes and hold a multiple of 8 values (VEC); otherwise from any
// element on, which global memory allows, and single values at the row's end.  Values beyond the row are zeros.
template <typename T> struct anywhere { typedef frag<T> type __attribute__((aligned(sizeof(T)))); };

template <typename T, bool VEC> __device__ __forceinline__ void load8(float *x, const T *row, int col, int cols) {
    if (VEC ? col < cols : col + LANE <= cols) {
        frag<T> f;
        if (VEC) f = *(const frag<T> *)(row + col);
        else f = *(const typename anywhere<T>::type *)(row + col);
#pragma unroll
        for (int t = 0; t < LANE; ++t) x[t] = (float)f[t];
    } else {
#pragma unroll
        for (int t = 0; t < LANE; ++t) x[t] = !VEC && col + t < cols ? (float)row[col + t] : 0.f;
    }
}

template <typename T, bool VEC> __device__ __forceinline__ void store8(T *row, const float *x, int col, int cols) {
    if (VEC) {
        if (col < cols) *(frag<T> *)(row + col) = to_frag<T>(x);
    } else if (col + LANE <= cols) {
        *(typename anywhere<T>::type *)(row + col) = to_frag<T>(x);
    } else {
#pragma unroll
        for (int t = 0; t < LANE; ++t)
            if (col + t < cols) row[col + t] = (T)x[t];
    }
}

// The values as T holds them.
template <typename T> __device__ __forceinline__ void round8(float *x) {
#pragma unroll
    for (int t = 0; t < LANE; ++t) x[t] = (float)(T)x[t];
}

// ------------------------------------------------------------------------------------ codes
// Codes of eight values and the exponent byte of the group that they share with the other three lanes of the quad.
// On bit patterns: with a = m 2^k, 1 <= m < 2, a <= 127 * 2^e = 1.984375 * 2^(e + 6) is e >= k - 6 for m <= 1.984375 and
// e >= k - 5 above, which the carry of the addition gives.  Of NaNs, infinities and finite values the larger pattern wins.
__device__ __forceinline__ u32x2 encode8(const float *x, uint32_t &exponent) {
    uint32_t a = 0;
#pragma unroll
    for (int t = 0; t < LANE; ++t) a = max(a, __float_as_uint(x[t]) & 0x7fffffffu);
    a = max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0xB1, 0xF, 0xF, true));  // quad_perm 1, 0, 3, 2
    a = max(a, (uint32_t)__builtin_amdgcn_mov_dpp((int)a, 0x4E, 0xF, 0xF, true));  // quad_perm 2, 3, 0, 1
    const bool broken = a >= 0x7f800000u;
    const int e = max(1, (int)((a + 0x1ffffu) >> 23) - 6);
    exponent = broken ? 255u : (uint32_t)e;
    const float inverse = __uint_as_float((uint32_t)(254 - e) << 23);
    u32x2 codes;
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        uint32_t c[4];
        // |x * inverse| <= 127: added to 1.5 * 2^23 it is rounded to an integer, halves to even, in the low bits
#pragma unroll
        for (int t = 0; t < 4; ++t) c[t] = __float_as_uint(__builtin_fmaf(x[4 * w + t], inverse, 12582912.f)) & 255u;
        const uint32_t word = c[0] | c[1] << 8 | c[2] << 16 | c[3] << 24;
        codes[w] = broken ? 0u : word;
    }
    return codes;
}

__device__ __forceinline__ void decode8(float *x, u32x2 codes, uint32_t exponent) {
    const float step = __uint_as_float(exponent << 23);  // of 255 an infinity: 0 * infinity is NaN
#pragma unroll
    for (int t = 0; t < LANE; ++t) x[t] = (float)((int)(codes[t / 4] << (24 - 8 * (t % 4))) >> 24) * step;
}

// Piece n of the rows: per_row pieces each, or, where per_row is 0, rows of whole groups that follow one another without gaps.
struct piece {
    uint32_t row;
    int col, cols;
    __device__ __forceinline__ piece(uint32_t n, uint32_t per_row, int32_t all) {
        if (per_row == 0) {
            row = n, col = 0, cols = LANE;
        } else {
            row = n / per_row, col = (int)(n - row * per_row) * LANE, cols = all;
        }
    }
};

// A vector of eight a thread, its group's magnitude by two exchanges within the quad.  8192 x 4096 in bf16: 16 us = 6.3 TB/s, the
// rate of a copy.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void encode_kernel(const T *x, int64_t row_stride, uint32_t total, int32_t cols, uint32_t per_row,
                                                     int8_t *codes, uint8_t *exponents) {
    const uint32_t n = blockIdx.x * 256 + threadIdx.x;
    if (n >= total) return;  // whole quads: per_row is a multiple of four
    const piece p(n, per_row, cols);
    float v[LANE];
    load8<T, VEC>(v, x + (int64_t)p.row * row_stride, p.col, p.cols);
    uint32_t e;
    const u32x2 c = encode8(v, e);
    *(u32x2 *)(codes + (int64_t)n * LANE) = c;
    if ((threadIdx.x & 3) == 0) exponents[n / 4] = (uint8_t)e;
}

// 8192 x 4096 to bf16: 15 us = 6.8 TB/s, the rate of a copy.
template <typename T, bool VEC>
__global__ __launch_bounds__(256) void decode_kernel(const int8_t *codes, const uint8_t *exponents, uint32_t total, int32_t cols,
                                                     uint32_t per_row, T *out, int64_t row_stride) {
    const uint32_t n = blockIdx.x * 256 + threadIdx.x;
    if (n >= total) return;
    const piece p(n, per_row, cols);
    float v[LANE];
    decode8(v, *(const u32x2 *)(codes + (int64_t)n * LANE), exponents[n / 4]);
    store8<T, VEC>(out + (int64_t)p.row * row_stride, v, p.col, p.cols);
}

// ------------------------------------------------------------------------------------ norm
// Sum over the threads of a row: 64, or all of the workgroup's.
template <int TPR> __device__ __forceinline__ float row_sum(float x) {
    x = wave_sum(x);
    if (TPR > 64) {
        __shared__ float part[TPR / 64];
        __syncthreads();  // the sums of the call before have been read
        if ((threadIdx.x & 63) == 0) part[threadIdx.x / 64] = x;
        __syncthreads();
        x = 0.f;
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) x += part[w];
    }
    return x;
}

constexpr int block_of(int tpr) { return tpr < 256 ? 256 : tpr; }

// A row stays in the registers of its TPR threads, V vectors of eight neighbours each: the sum of squares and the output take one
// read.  The output is written with its codes, which saves the read of y that encode would take.  8192 rows of 1024 in bf16, x and
// residual read, h, y and the checkpoint written: 13.4 us = 5.7 TB/s; with few rows it is the latency of one read and one write
// (128 rows 4 us).
template <typename T, int TPR, int V, bool VEC>
__global__ __launch_bounds__(block_of(TPR)) void norm_kernel(const T *x, int64_t x_stride, const T *residual, int64_t residual_stride,
                                                             const float *weight, int64_t rows, int32_t cols, float eps, T *h, T *y,
                                                             int8_t *codes, uint8_t *exponents, float *rstd) {
    constexpr int RPB = block_of(TPR) / TPR;
    const int tid = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR;
    if (row >= rows) return;  // with several rows a workgroup a whole wave, and no barrier follows
    float v[V][LANE], sum = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int col = (i * TPR + tid) * LANE;
        load8<T, VEC>(v[i], x + row * x_stride, col, cols);
        if (residual) {
            float r[LANE];
            load8<T, VEC>(r, residual + row * residual_stride, col, cols);
#pragma unroll
            for (int t = 0; t < LANE; ++t) v[i][t] += r[t];
            round8<T>(v[i]);
            store8<T, VEC>(h + row * cols, v[i], col, cols);
        }
#pragma unroll
        for (int t = 0; t < LANE; ++t) sum += v[i][t] * v[i][t];
    }
    const float r = 1.f / sqrtf(row_sum<TPR>(sum) / (float)cols + eps);
    if (tid == 0) rstd[row] = r;
    const int padded = (cols + GROUP - 1) / GROUP * GROUP;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int col = (i * TPR + tid) * LANE;
        float w[LANE];
        load8<float, VEC>(w, weight, col, cols);
#pragma unroll
        for (int t = 0; t < LANE; ++t) v[i][t] = v[i][t] * r * w[t];
        round8<T>(v[i]);
        if (y) store8<T, VEC>(y + row * cols, v[i], col, cols);
        if (codes) {
            uint32_t e;
            const u32x2 c = encode8(v[i], e);
            if (col < padded) {
                *(u32x2 *)(codes + row * padded + col) = c;
                if ((tid & 3) == 0) exponents[(row * padded + col) / GROUP] = (uint8_t)e;
            }
        }
    }
}

// Rows blockIdx, + grid, ...: the sum over them of dweight's terms stays in registers and becomes one row of `part`.  dx and
// dweight take the same read of dy and h.  8192 rows of 1024 in bf16, dy, h and dh read, dx written: 13.1 us = 5.1 TB/s.
template <typename T, int TPR, int V, bool VEC>
__global__ __launch_bounds__(block_of(TPR)) void norm_backward_kernel(const T *dy, int64_t dy_stride, const T *h, int64_t h_stride,
                                                                      const T *dh, int64_t dh_stride, const float *weight,
                                                                      const float *rstd, int64_t rows, int32_t cols, T *dx, float *part) {
    constexpr int RPB = block_of(TPR) / TPR;
    const int tid = threadIdx.x % TPR;
    // A row and the weights stay in registers, or, of the widest rows, come again for the second pass, from the L2 cache.
    constexpr bool HOLD = V <= 2 || TPR == 64;
    constexpr int H = HOLD ? V : 1;
    float w[H][LANE], g[H][LANE], n[H][LANE], dw[V][LANE];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (HOLD) load8<float, VEC>(w[i % H], weight, (i * TPR + tid) * LANE, cols);
#pragma unroll
        for (int t = 0; t < LANE; ++t) dw[i][t] = 0.f;
    }
    for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; row < rows; row += (int64_t)gridDim.x * RPB) {
        const float r = rstd[row];
        auto load = [&](int i) {  // n: the normed row, g: dy * weight
            const int col = (i * TPR + tid) * LANE, k = i % H;
            load8<T, VEC>(g[k], dy + row * dy_stride, col, cols);
            load8<T, VEC>(n[k], h + row * h_stride, col, cols);
            if (!HOLD) load8<float, VEC>(w[k], weight, col, cols);
        };
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int k = i % H;
            load(i);
#pragma unroll
            for (int t = 0; t < LANE; ++t) {
                n[k][t] *= r;
                dw[i][t] += g[k][t] * n[k][t];
                g[k][t] *= w[k][t];
                sum += g[k][t] * n[k][t];
            }
            if (!HOLD) __builtin_amdgcn_sched_barrier(0);  // one vector after another: their loads together do not fit
        }
        const float mean = row_sum<TPR>(sum) / (float)cols;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int col = (i * TPR + tid) * LANE, k = i % H;
            if (!HOLD) {
                load(i);
#pragma unroll
                for (int t = 0; t < LANE; ++t) n[k][t] *= r, g[k][t] *= w[k][t];
            }
            float d[LANE];
            if (dh) load8<T, VEC>(d, dh + row * dh_stride, col, cols);
#pragma unroll
            for (int t = 0; t < LANE; ++t) g[k][t] = (g[k][t] - n[k][t] * mean) * r + (dh ? d[t] : 0.f);
            store8<T, VEC>(dx + row * cols, g[k], col, cols);
            if (!HOLD) __builtin_amdgcn_sched_barrier(0);
        }
    }
    float *out = part + (int64_t)blockIdx.x * cols;
    if (RPB == 1) {
#pragma unroll
        for (int i = 0; i < V; ++i) store8<float, VEC>(out, dw[i], (i * TPR + tid) * LANE, cols);
        return;
    }
    __shared__ __attribute__((aligned(16))) float sums[RPB == 1 ? 1 : RPB][RPB == 1 ? 1 : V][RPB == 1 ? 1 : TPR * LANE];
#pragma unroll
    for (int i = 0; i < V; ++i)
#pragma unroll
        for (int t = 0; t < LANE; ++t) sums[threadIdx.x / TPR][i][tid * LANE + t] = dw[i][t];
    __syncthreads();
    for (int c = threadIdx.x; c < cols; c += block_of(TPR)) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < RPB; ++k) s += sums[k][c / (TPR * LANE)][c % (TPR * LANE)];
        out[c] = s;
    }
}

// Sum of n rows of `part`, 64 columns a workgroup: each of 16 waves adds every sixteenth row, and the waves' sums are
// added in order.  1024 rows of 1024 columns 4.2 us, the latency of its loads and of the launch.
constexpr int SUM_WAVES = 16;
__global__ __launch_bounds__(64 * SUM_WAVES) void column_sum_kernel(const float *part, int32_t n, int32_t cols, float *out) {
    __shared__ float sums[SUM_WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = blockIdx.x * 64 + lane;
    float s = 0.f;
    if (col < cols) {
        constexpr int U = 8;  // loads in flight
        int k = wave;
        for (; k + (U - 1) * SUM_WAVES < n; k += U * SUM_WAVES) {
            float x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) x[u] = part[(int64_t)(k + u * SUM_WAVES) * cols + col];
#pragma unroll
            for (int u = 0; u < U; ++u) s += x[u];
        }
        for (; k < n; k += SUM_WAVES) s += part[(int64_t)k * cols + col];
    }
    sums[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && col < cols) {
        s = 0.f;
#pragma unroll
        for (int w = 0; w < SUM_WAVES; ++w) s += sums[w][lane];
        out[col] = s;
    }
}

// ------------------------------------------------------------------------------------ host
int size_of(int32_t dtype) { return dtype == DEAR_BF16 ? 2 : 4; }
bool known(int32_t dtype) { return dtype == DEAR_BF16 || dtype == DEAR_F32; }

// Whether rows can be read in vectors of eight values of n bytes.
bool vectors(const void *p, int64_t stride, int64_t cols, int n) {
    return !p || (aligned(p, 16) && stride * n % 16 == 0 && cols % LANE == 0);
}

// Threads of a row: a wave up to 2048 columns, then as many as it takes for two vectors each, or for four of the widest.  A wave
// needs no barrier between its sum and its output: 32768 rows of 1024 in bf16, forward and backward, 53 and 45 us, with 256
// threads a row 73 and 72; 8192 rows of 4096 with 256 and 512 threads 56 and 54 against 55 and 59.
int threads_of_row(int64_t cols) { return cols <= 2048 ? 64 : cols <= 4096 ? 256 : cols <= 8192 ? 512 : 1024; }

// Workgroups of the backward pass, and rows of its workspace: as many as fill the chip with rows under way.  8192 rows of
// 1024 and 4096 columns: 512 / 1024 / 2048 workgroups 18.0 / 18.0 / 22.2 and 67 / 52 / 62 us.
int backward_groups(int64_t rows, int64_t cols) {
    const int64_t n = ceil_div(rows, cols <= 2048 ? 4 : 1), most = cols <= 4096 ? 1024 : 512;
    return (int)(n < most ? n : most);
}

template <typename T, int TPR, int V, bool VEC, typename F> void call(F f) { f.template operator()<T, TPR, V, VEC>(); }

// Calls f for the type, the threads of a row and its vectors.
template <typename T, bool VEC, typename F> void by_cols(int64_t cols, F f) {
    const int tpr = threads_of_row(cols), v = (int)ceil_div(cols, tpr * LANE);
    if (tpr == 64) {
        if (v == 1) return call<T, 64, 1, VEC>(f);
        if (v == 2) return call<T, 64, 2, VEC>(f);
        if (v == 3) return call<T, 64, 3, VEC>(f);
        return call<T, 64, 4, VEC>(f);
    }
    if (tpr == 256) return call<T, 256, 2, VEC>(f);
    if (tpr == 512) return call<T, 512, 2, VEC>(f);
    if (v <= 2) return call<T, 1024, 2, VEC>(f);
    if (v == 3) return call<T, 1024, 3, VEC>(f);
    return call<T, 1024, 4, VEC>(f);
}

template <typename F> void dispatch(int32_t dtype, bool vec, int64_t cols, F f) {
    if (dtype == DEAR_BF16) {
        if (vec) by_cols<bf16, true>(cols, f);
        else by_cols<bf16, false>(cols, f);
    } else {
        if (vec) by_cols<float, true>(cols, f);
        else by_cols<float, false>(cols, f);
    }
}

struct forward_call {
    const void *x, *residual;
    int64_t x_stride, residual_stride, rows;
    const float *weight;
    int32_t cols;
    float eps;
    void *h, *y;
    int8_t *codes;
    uint8_t *exponents;
    float *rstd;
    hipStream_t stream;
    template <typename T, int TPR, int V, bool VEC> void operator()() {
        constexpr int RPB = block_of(TPR) / TPR;
        const int64_t groups = ceil_div(cols, GROUP), most = MAX_THREADS / block_of(TPR) * RPB;  // rows of a launch
        for (int64_t first = 0; first < rows; first += most) {
            const int64_t n = rows - first < most ? rows - first : most;
            auto from = [&](const void *p, int64_t stride) { return p ? (T *)p + first * stride : nullptr; };
            norm_kernel<T, TPR, V, VEC><<<(unsigned)ceil_div(n, RPB), block_of(TPR), 0, stream>>>(
                from(x, x_stride), x_stride, from(residual, residual_stride), residual_stride, weight, n, cols, eps, from(h, cols),
                from(y, cols), codes ? codes + first * groups * GROUP : nullptr, exponents ? exponents + first * groups : nullptr,
                rstd + first);
        }
    }
};

struct backward_call {
    const void *dy, *h, *dh;
    int64_t dy_stride, h_stride, dh_stride, rows;
    const float *weight, *rstd;
    int32_t cols;
    void *dx;
    float *part;
    int groups;
    hipStream_t stream;
    template <typename T, int TPR, int V, bool VEC> void operator()() {
        norm_backward_kernel<T, TPR, V, VEC><<<groups, block_of(TPR), 0, stream>>>((const T *)dy, dy_stride, (const T *)h, h_stride,
                                                                                   (const T *)dh, dh_stride, weight, rstd, rows, cols,
                                                                                   (T *)dx, part);
    }
};

// The launches of a call on a checkpoint: as many rows at a time as 31 bits count the pieces of.  Calls
// f(first row, pieces, pieces of a row) for each; pieces of a row: 0 where rows without gaps (`dense`) are of whole groups.
template <typename F> int launches(int64_t rows, int64_t cols, bool dense, F f) {
    const int64_t per_row = ceil_div(cols, GROUP) * (GROUP / LANE), most = INT32_MAX / per_row;
    if (rows > INT64_MAX / 4 / per_row || ceil_div(rows * per_row, 256) > INT32_MAX) return DEAR_ETOOBIG;
    for (int64_t first = 0; first < rows; first += most) {
        const int64_t n = rows - first < most ? rows - first : most;
        f(first, (uint32_t)(n * per_row), dense && cols % GROUP == 0 ? 0u : (uint32_t)per_row);
    }
    return launch_status();
}

// Calls f with values of the type and of whether there are whole vectors.
template <typename F> void by_types(int32_t dtype, bool vec, F f) {
    auto by_vec = [&](auto t) {
        if (vec) f(t, std::true_type());
        else f(t, std::false_type());
    };
    if (dtype == DEAR_BF16) by_vec(bf16());
    else by_vec(float());
}

// A tensor that is read row by row.
int check_rows(const void *p, int64_t stride, int32_t dtype, int64_t rows, int64_t cols) {
    if (!p || (rows > 1 && stride < cols)) return DEAR_EINVAL;
    return aligned(p, size_of(dtype)) ? DEAR_OK : DEAR_EALIGN;
}

}  // namespace

extern "C" {

int dear_checkpoint_encode(const void *x, int32_t dtype, int64_t rows, int64_t cols, int64_t row_stride, int8_t *codes,
                           uint8_t *exponents, void *hip_stream) {
    if (!known(dtype) || rows < 0 || cols < 1 || cols > INT32_MAX - GROUP) return DEAR_EINVAL;
    if (rows == 0) return DEAR_OK;
    if (int rc = check_rows(x, row_stride, dtype, rows, cols)) return rc;
    if (!codes || !exponents) return DEAR_EINVAL;
    if (!aligned(codes, 16)) return DEAR_EALIGN;
    hipStream_t s = (hipStream_t)hip_stream;
    const bool vec = vectors(x, row_stride, cols, size_of(dtype));
    const int64_t groups = ceil_div(cols, GROUP);
    return launches(rows, cols, vec && (row_stride == cols || rows == 1), [&](int64_t first, uint32_t total, uint32_t per_row) {
        by_types(dtype, vec, [&](auto t, auto v) {
            typedef decltype(t) T;
            encode_kernel<T, decltype(v)::value><<<(total + 255) / 256, 256, 0, s>>>(
                (const T *)x + first * row_stride, per_row ? row_stride : LANE, total, (int32_t)cols, per_row,
                codes + first * groups * GROUP, exponents + first * groups);
        });
    });
}

int dear_checkpoint_decode(const int8_t *codes, const uint8_t *exponents, int64_t rows, int64_t cols, int32_t dtype, void *out,
                           void *hip_stream) {
    if (!known(dtype) || rows < 0 || cols < 1 || cols > INT32_MAX - GROUP) return DEAR_EINVAL;
    if (rows == 0) return DEAR_OK;
    if (!codes || !exponents || !out) return DEAR_EINVAL;
    if (!aligned(codes, 16) || !aligned(out, size_of(dtype))) return DEAR_EALIGN;
    hipStream_t s = (hipStream_t)hip_stream;
    const bool vec = vectors(out, cols, cols, size_of(dtype));
    const int64_t groups = ceil_div(cols, GROUP);
    return launches(rows, cols, vec, [&](int64_t first, uint32_t total, uint32_t per_row) {
        by_types(dtype, vec, [&](auto t, auto v) {
            typedef decltype(t) T;
            decode_kernel<T, decltype(v)::value><<<(total + 255) / 256, 256, 0, s>>>(
                codes + first * groups * GROUP, exponents + first * groups, total, (int32_t)cols, per_row, (T *)out + first * cols,
                per_row ? cols : LANE);
        });
    });
}

int dear_add_rms_norm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, const float *weight,
                      int32_t dtype, int64_t rows, int64_t cols, float eps, void *h, void *y, int8_t *codes, uint8_t *exponents,
                      float *rstd, void *hip_stream) {
    if (!known(dtype) || rows < 0 || cols < 1 || cols > DEAR_NORM_MAX_COLS || !(eps >= 0.f) || !std::isfinite(eps)) return DEAR_EINVAL;
    if (rows == 0) return DEAR_OK;
    if (int rc = check_rows(x, x_stride, dtype, rows, cols)) return rc;
    if (residual)
        if (int rc = check_rows(residual, residual_stride, dtype, rows, cols)) return rc;
    if (!residual != !h || !codes != !exponents || !weight || !rstd) return DEAR_EINVAL;
    const int n = size_of(dtype);
    if (!aligned(h, n) || !aligned(y, n) || !aligned(weight, 4) || !aligned(rstd, 4) || !aligned(codes, 16)) return DEAR_EALIGN;
    if (rows > INT32_MAX) return DEAR_ETOOBIG;
    const bool vec = vectors(x, x_stride, cols, n) && vectors(residual, residual_stride, cols, n) && vectors(h, cols, cols, n) &&
                     vectors(y, cols, cols, n) && vectors(weight, cols, cols, 4);
    dispatch(dtype, vec, cols, forward_call{x, residual, x_stride, residual_stride, rows, weight, (int32_t)cols, eps, h, y, codes,
                                            exponents, rstd, (hipStream_t)hip_stream});
    return launch_status();
}

int dear_add_rms_norm_backward_workspace(int32_t dtype, int64_t rows, int64_t cols, int64_t *bytes) {
    if (!bytes || !known(dtype) || rows < 0 || cols < 1 || cols > DEAR_NORM_MAX_COLS) return DEAR_EINVAL;
    *bytes = (int64_t)backward_groups(rows, cols) * cols * 4;
    return DEAR_OK;
}

int dear_add_rms_norm_backward(const void *dy, int64_t dy_stride, const void *h, int64_t h_stride, const void *dh, int64_t dh_stride,
                               const float *weight, const float *rstd, int32_t dtype, int64_t rows, int64_t cols, void *dx,
                               float *dweight, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    int64_t need = 0;
    if (int rc = dear_add_rms_norm_backward_workspace(dtype, rows, cols, &need)) return rc;
    if (!dweight) return DEAR_EINVAL;
    if (!aligned(dweight, 4)) return DEAR_EALIGN;
    hipStream_t stream = (hipStream_t)hip_stream;
    const int n = size_of(dtype), groups = backward_groups(rows, cols);
    if (rows > 0) {
        if (int rc = check_rows(dy, dy_stride, dtype, rows, cols)) return rc;
        if (int rc = check_rows(h, h_stride, dtype, rows, cols)) return rc;
        if (dh)
            if (int rc = check_rows(dh, dh_stride, dtype, rows, cols)) return rc;
        if (!weight || !rstd || !dx || !workspace) return DEAR_EINVAL;
        if (!aligned(dx, n) || !aligned(weight, 4) || !aligned(rstd, 4) || !aligned(workspace, 256)) return DEAR_EALIGN;
        if (workspace_bytes < need) return DEAR_ETOOBIG;
        const bool vec = vectors(dy, dy_stride, cols, n) && vectors(h, h_stride, cols, n) && vectors(dh, dh_stride, cols, n) &&
                         vectors(dx, cols, cols, n) && vectors(weight, cols, cols, 4);
        dispatch(dtype, vec, cols, backward_call{dy, h, dh, dy_stride, h_stride, dh_stride, rows, weight, rstd, (int32_t)cols, dx,
                                                 (float *)workspace, groups, stream});
        if (int rc = launch_status()) return rc;
    }
    column_sum_kernel<<<(unsigned)ceil_div(cols, 64), 64 * SUM_WAVES, 0, stream>>>((const float *)workspace, groups, (int32_t)cols, dweight);
    return launch_status();
}

}  // extern "C"
