// Gradient of a linear layer's weight from the checkpoint of its input (definitions: dear_ops.h).
//
//     dw[n, k] = sum over m of dy[m, n] * code[m, k] * 2^e[m, k / 32]
//
// The sum runs over the rows of both operands, so both are read from LDS with the transposing reads.  A checkpoint's
// value has 7 significant bits, so that it becomes an operand in bf16 without any rounding: products are exact, and what
// is rounded is the fp32 sum alone.
#include <cmath>
#include <type_traits>

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

// Workgroup -> split and tile.  Workgroups go to the eight XCDs in turn: each XCD gets a run of neighbours, in strips four
// tiles of outs wide, so that with 32 tiles under way it reads four tiles' columns of dy and eight of the codes.
__device__ __forceinline__ void place(const params &a, unsigned &split, unsigned &n_tile, unsigned &k_tile) {
    const unsigned total = gridDim.x, xcd = blockIdx.x % 8, least = total / 8, more = total % 8;
    const unsigned item = xcd * least + min(xcd, more) + blockIdx.x / 8;
    const unsigned per_split = (unsigned)a.n_tiles * a.k_tiles, id = item % per_split, strip = id / (4u * a.k_tiles);
    const unsigned wide = min(4u, a.n_tiles - 4 * strip), in_strip = id - strip * 4 * a.k_tiles;
    split = item / per_split;
    n_tile = 4 * strip + in_strip % wide;
    k_tile = in_strip / wide;
}

// A step's operands on their way from memory to LDS: pieces of 16 bytes of dy, and sixteen codes of a group a thread.
template <typename T, bool VEC> struct stage {
    static constexpr int E = 16 / sizeof(T), N = BM * BN / E / THREADS;
    typedef T vec __attribute__((ext_vector_type(16 / sizeof(T))));
    typedef vec vec_anywhere __attribute__((aligned(sizeof(T))));  // global memory takes 16-byte loads from any element on
    vec y[N];
    u32x4 x;
    uint32_t e;

    __device__ __forceinline__ void load(const params &a, int64_t m0, int64_t end, int n0, int k0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * THREADS, row = c / (BN / E), col = c % (BN / E) * E;
            const T *p = (const T *)a.dy + (m0 + row) * a.dy_stride + n0 + col;
#pragma unroll
            for (int u = 0; u < E; ++u) y[i][u] = (T)0.f;
            if (m0 + row < end) {
                if (VEC) {
                    if (n0 + col < a.outs) y[i] = *(const vec *)p;
                } else if (n0 + col + E <= a.outs) {
                    y[i] = *(const vec_anywhere *)p;
                } else {
#pragma unroll
                    for (int u = 0; u < E - 1; ++u)
                        if (n0 + col + u < a.outs) y[i][u] = p[u];
                }
            }
        }
        const int row = threadIdx.x / (BK / 16), col = threadIdx.x % (BK / 16) * 16;
        x = u32x4{0, 0, 0, 0}, e = 0;
        if (m0 + row < end && k0 + col < a.padded) {
            x = *(const u32x4 *)(a.codes + (m0 + row) * a.padded + k0 + col);
            e = a.exponents[(m0 + row) * a.groups + (k0 + col) / GROUP];
        }
    }
    __device__ __forceinline__ void store(DEAR_LDS T *ys, DEAR_LDS T *xs) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int c = threadIdx.x + i * THREADS;
            *(DEAR_LDS vec *)(ys + c / (BN / E) * tile<T, BN>::stride + c % (BN / E) * E) = y[i];
        }
        const int row = threadIdx.x / (BK / 16), col = threadIdx.x % (BK / 16) * 16;
        const float step = __uint_as_float(e << 23);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            float v[8];
#pragma unroll
            for (int t = 0; t < 8; ++t) v[t] = (float)((int)(x[2 * w + t / 4] << (24 - 8 * (t % 4))) >> 24) * step;
            *(DEAR_LDS frag<T> *)(xs + row * tile<T, BK>::stride + col + 8 * w) = to_frag<T>(v);
        }
    }
};

// fp32, odd sizes, few rows: 128 x 128 outputs a workgroup, 64 x 64 a wave; a step's operands go through registers to LDS, the
// next one's loads beside its products.  In fp32 the matrix instructions bound it, in bf16 the loads' latency: 1111 rows, 771 x 1003
// in fp32 33 us with 9 splits, and 6 to add them; 2048 rows, 4096 x 4096 in bf16 96 us.
template <typename T, bool VEC> __global__ __launch_bounds__(THREADS, 2) void weight_grad_kernel(params a) {
    __shared__ __attribute__((aligned(16))) char lds[tile<T, BN>::bytes(BM) + tile<T, BK>::bytes(BM)];
    DEAR_LDS T *ys = (DEAR_LDS T *)lds, *xs = (DEAR_LDS T *)(lds + tile<T, BN>::bytes(BM));
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    unsigned split, n_tile, k_tile;
    place(a, split, n_tile, k_tile);
    const int n0 = (int)n_tile * BN, k0 = (int)k_tile * BK;
    const int64_t begin = (int64_t)split * a.chunk, end = min(a.rows, begin + a.chunk);
    f32x16 acc[2][2] = {};
    stage<T, VEC> st;
    if (begin < end) st.load(a, begin, end, n0, k0);
    for (int64_t m0 = begin; m0 < end; m0 += BM) {
        __syncthreads();
        st.store(ys, xs);
        __syncthreads();
        if (m0 + BM < end) st.load(a, m0 + BM, end, n0, k0);
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
// A workgroup owns 128 x 128 outputs and each of its four waves sums all of them over rows of its own, 32 of every 128: a
// wave reads eight fragments for sixteen products, and the waves meet only at the end, to add their sums.  dy goes from
// memory to LDS by itself; codes come to registers, and as values to LDS, beside the products of the step before.  8192 rows,
// 1024 x 4096: 81 us a call = 850 TFLOP/s; with one wave a SIMD matrix instructions are busy 39 % of the time, the vector
// instructions that make values of codes 36 %, and 31 % of the LDS's cycles are bank conflicts.  The same outputs cut among
// the waves, 64 x 64 each, read twice as much from LDS and need a barrier a step: 186 us, and eight waves of 128 x 64 with a
// barrier a step 116.
constexpr int WROWS = 32;                      // rows of a wave's step
constexpr int WSTEP = WROWS * (THREADS / 64);  // rows of a workgroup's step
constexpr int WTILE = WROWS * 128;             // elements of one operand's tile

// Tiles have rows of 128 values without padding; piece c (16 bytes) of a row stands at c ^ turn(row), so that the four rows
// of a transposing read lie in different banks.  Values are written 32 bytes apart from lane to lane, which is what conflicts
// there are (attention's tiles, read alike and written in neighbouring pieces, have none).
__device__ __forceinline__ int turn(int row) { return (row & 3) << 2 | (row & 1); }

struct wave_codes {
    u32x4 x[4];
    uint32_t e[4];
};

// What a lane brings of a step: of dy row 4 i + lane / 16, of the codes row 8 i + lane / 8.
struct wave_loader {
    const char *y;
    const int8_t *x;
    const uint8_t *e;
    uint32_t y_stride, x_stride, e_stride;  // bytes
    uint32_t y_off, x_off, e_off;           // of the lane's piece

    // left: rows from the step's first on; those beyond are zeros (of the codes: the last row again, times 0)
    template <bool WHOLE> __device__ __forceinline__ void load_y(DEAR_LDS bf16 *s, int lane, int left) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = 4 * i + lane / 16;
            if (WHOLE || row < left) load_to_lds(y + (y_off + (uint32_t)row * y_stride), s + i * 512);
            else *(DEAR_LDS u32x4 *)(s + i * 512 + lane * 8) = u32x4{0, 0, 0, 0};
        }
        y += (int64_t)WSTEP * y_stride;
    }
    template <bool WHOLE> __device__ __forceinline__ void load_x(wave_codes &w, int lane, int left) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = 8 * i + lane / 8, r = WHOLE ? row : min(row, left - 1);
            w.x[i] = *(const u32x4 *)(x + (x_off + (uint32_t)r * x_stride));
            w.e[i] = e[e_off + (uint32_t)r * e_stride];
            if (!WHOLE && row >= left) w.e[i] = 0;
        }
        x += (int64_t)WSTEP * x_stride, e += (int64_t)WSTEP * e_stride;
    }
};

__device__ __forceinline__ void store_x(const wave_codes &w, DEAR_LDS bf16 *xs, int lane) {
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
        const int row = 8 * i + lane / 8;
#pragma unroll
        for (int k = 0; k < 2; ++k) *(DEAR_LDS u32x4 *)(xs + row * 128 + ((2 * (lane % 8) + k) ^ turn(row)) * 8) = q[k];
    }
}

struct wave_frags {
    bf16x8 y[4], x[4];
};

// column_at: of a lane's transposing reads, the byte of its piece in row 4 h + (lane % 16) / 4 for columns 32 u
__device__ __forceinline__ void read_frags(wave_frags &f, const DEAR_LDS bf16 *ys, const DEAR_LDS bf16 *xs, int s, const uint32_t (&column_at)[4]) {
    auto read = [&](const DEAR_LDS bf16 *t, int u) {
        const DEAR_LDS char *p = (const DEAR_LDS char *)(t + 16 * s * 128) + column_at[u];
        const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((DEAR_LDS bf16x4 *)p);
        const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((DEAR_LDS bf16x4 *)(p + 8 * 256));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    };
#pragma unroll
    for (int u = 0; u < 4; ++u) f.y[u] = read(ys, u), f.x[u] = read(xs, u);
}

__device__ __forceinline__ void multiply(f32x16 (&acc)[4][4], const wave_frags &f) {
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
        for (int v = 0; v < 4; ++v) acc[u][v] = mma(f.y[u], f.x[v], acc[u][v]);
}

__global__ __launch_bounds__(THREADS, 1) void weight_grad_wide_kernel(params a) {
    // tiles of even steps and of odd ones, in arrays of their own; at the end the waves' sums, two quarters at a time
    __shared__ __attribute__((aligned(16))) bf16 ys0[4 * WTILE], ys1[4 * WTILE], xs0[4 * WTILE], xs1[4 * WTILE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    unsigned split, n_tile, k_tile;
    place(a, split, n_tile, k_tile);
    const int n0 = (int)n_tile * 128, k0 = (int)k_tile * 128;
    const int64_t begin = (int64_t)split * a.chunk + wave * WROWS, end = min(a.rows, (int64_t)(split + 1) * a.chunk);

    f32x16 acc[4][4] = {};
    wave_loader in;
    in.y_stride = (uint32_t)a.dy_stride * 2, in.x_stride = (uint32_t)a.padded, in.e_stride = (uint32_t)a.groups;
    // outputs beyond the last repeat the first: they are not stored
    const int yc = n0 + (lane % 16 ^ turn(lane / 16)) * 8, xc = k0 + lane % 8 * 16;
    in.y_off = (uint32_t)(yc < a.outs ? yc : 0) * 2, in.x_off = xc < a.padded ? xc : 0, in.e_off = in.x_off / GROUP;
    in.y = (const char *)a.dy + begin * a.dy_stride * 2;
    in.x = a.codes + begin * a.padded;
    in.e = a.exponents + begin * a.groups;
    uint32_t column_at[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int row = 4 * (lane >> 5) + (lane & 15) / 4, c = 4 * u + 2 * (lane >> 4 & 1) + (lane & 3) / 2;
        column_at[u] = row * 256 + (c ^ turn(row)) * 16 + 8 * (lane & 1);
    }
    const int64_t rows = end - begin, steps = rows > 0 ? (rows + WSTEP - 1) / WSTEP : 0;  // of this wave
    const int last = (int)(rows - (steps - 1) * WSTEP);  // rows from the last step on
    if (steps > 0) {
        DEAR_LDS bf16 *const ya = (DEAR_LDS bf16 *)ys0 + wave * WTILE, *const yb = (DEAR_LDS bf16 *)ys1 + wave * WTILE;
        DEAR_LDS bf16 *const xa = (DEAR_LDS bf16 *)xs0 + wave * WTILE, *const xb = (DEAR_LDS bf16 *)xs1 + wave * WTILE;
        wave_codes w0, w1;
        wave_frags f, g;
        auto load_y = [&](DEAR_LDS bf16 *s, int64_t t) {
            if (t < steps - 1) in.load_y<true>(s, lane, 0);
            else if (t < steps) in.load_y<false>(s, lane, last);
        };
        auto load_x = [&](wave_codes &w, int64_t t) {
            if (t < steps - 1) in.load_x<true>(w, lane, 0);
            else if (t < steps) in.load_x<false>(w, lane, last);
        };
        load_y(ya, 0);
        load_x(w0, 0);
        store_x(w0, xa, lane);
        load_x(w1, 1);
        // Step t, in buffer t % 2: waits for its dy and for the codes of step t + 1, which are the wave's own loads, and for its
        // own reads of the buffer that is filled next (vmcnt 0 and lgkmcnt 0), reads its first fragments beside the products of the
        // second ones of the step before, and its second ones beside the products of the first.  MORE: steps to t + 2 are there
        // and whole.
        auto step = [&](auto more, int64_t t, const wave_codes &w, wave_codes &w_next, const DEAR_LDS bf16 *y, const DEAR_LDS bf16 *x,
                        DEAR_LDS bf16 *y_next, DEAR_LDS bf16 *x_next) {
            constexpr bool MORE = decltype(more)::value;
            __builtin_amdgcn_s_waitcnt(0x0070);
#pragma unroll
            for (int u = 0; u < 4; ++u) asm("" : "+v"(column_at[u]));
            if (MORE) in.load_y<true>(y_next, lane, 0), in.load_x<true>(w_next, lane, 0);
            else load_y(y_next, t + 1), load_x(w_next, t + 2);
            read_frags(f, y, x, 0, column_at);
            multiply(acc, g);
            read_frags(g, y, x, 1, column_at);
            multiply(acc, f);
            if (MORE || t + 1 < steps) store_x(w, x_next, lane);
            if (MORE) {
                // beside each product what else there is to do, in the order in which it is wanted
#pragma unroll
                for (int u = 0; u < 16; ++u) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 5, 0);
                }
#pragma unroll
                for (int u = 0; u < 16; ++u) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x002, 6, 0);
                    if (u % 2) __builtin_amdgcn_sched_group_barrier(0x200, 1, 0);
                }
            }
        };
        g = wave_frags{};  // before the first step
        int64_t t = 0;
        for (; t + 4 < steps; t += 2) {
            step(std::true_type{}, t, w1, w0, ya, xa, yb, xb);
            step(std::true_type{}, t + 1, w0, w1, yb, xb, ya, xa);
        }
        for (; t < steps; t += 2) {
            step(std::false_type{}, t, w1, w0, ya, xa, yb, xb);
            if (t + 1 < steps) step(std::false_type{}, t + 1, w0, w1, yb, xb, ya, xa);
        }
        multiply(acc, g);
    }

    DEAR_LDS float *const parts[4] = {(DEAR_LDS float *)ys0, (DEAR_LDS float *)ys1, (DEAR_LDS float *)xs0, (DEAR_LDS float *)xs1};
    DEAR_LDS float *const sums = wave < 2 ? (wave == 0 ? parts[0] : parts[1]) : (wave == 2 ? parts[2] : parts[3]);
    float *out = a.out + (int64_t)split * a.outs * a.ins;
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
                    sums[(32 * u + row_of(r, lane >> 5)) * 128 + 32 * v + (lane & 31)] = acc[2 * pair + u][v][r];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int row = 8 * i + threadIdx.x / 32, col = threadIdx.x % 32 * 4;
            f32x4 t = *(DEAR_LDS f32x4 *)(parts[0] + row * 128 + col);
#pragma unroll
            for (int k = 1; k < 4; ++k) t += *(DEAR_LDS f32x4 *)(parts[k] + row * 128 + col);
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

// Sum of the splits, in their order, eight loads in flight.
__global__ __launch_bounds__(256) void split_sum_kernel(const float *part, int splits, int64_t n, float *out) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i >= n) return;
    float s = 0.f;
    int k = 0;
    for (; k + 8 <= splits; k += 8) {
        float x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = part[(k + u) * n + i];
#pragma unroll
        for (int u = 0; u < 8; ++u) s += x[u];
    }
    for (; k < splits; ++k) s += part[k * n + i];
    out[i] = s;
}

// ------------------------------------------------------------------------------------ host
constexpr int64_t MAX_WIDTH = 1 << 24, MAX_ROWS = (int64_t)1 << 40;

// Whether the wide kernel can take it: bf16 in whole vectors, with rows that 32-bit offsets reach.
bool fits_wide(int32_t dtype, int64_t dy_stride, int64_t outs) {
    return dtype == DEAR_BF16 && outs % 8 == 0 && dy_stride < (1 << 24);
}

struct choice {
    bool wide;
    int splits;  // of the rows, each a sum of its own in the workspace
    double us;
};

// The kernel and the splits of the least time by this estimate, in microseconds.  A CU takes one workgroup of the wide kernel
// at a time, 8 and 1.2 for every 128 rows, or four (bf16) or three (fp32) of the other, 8 and 2.9 or 11 for 128 rows as
// long as loads are what it waits for, and a share of the CU's 1.5 or 8 (fp32 matrix instructions) when there are more.
// Several splits' sums are written, read and added, 5 TB/s, in another launch.  Measured, wide against the other: 8192 rows
// 4096 x 1024 84 and 186 us, 1024 x 1024 34 and 56; 2048 rows 4096 x 4096 109 and 96, 128 rows 35 and 17.
choice choose(int32_t dtype, bool can_wide, int64_t rows, int64_t outs, int64_t ins) {
    const int64_t tiles = ceil_div(outs, BN) * ceil_div(ins, BK), most = ceil_div(rows, 128) < 64 ? ceil_div(rows, 128) : 64;
    const double resident = dtype == DEAR_F32 ? 3 : 4, alone = dtype == DEAR_F32 ? 11 : 2.9, share = dtype == DEAR_F32 ? 8 : 1.5;
    choice best = {can_wide, 1, 0};
    for (int64_t s = 1; s == 1 || (s <= most && tiles * s * THREADS <= MAX_THREADS && outs * ins <= MAX_THREADS); ++s) {
        const double chunk = (double)ceil_div(ceil_div(rows, s), 128), a_cu = (double)ceil_div(tiles * s, 256);
        const double sums = s == 1 ? 0 : 4 + (double)(s + 1) * (double)outs * (double)ins * 4 / 5e6;
        const double wait = std::ceil(a_cu / resident) * chunk * alone, work = a_cu * chunk * share;
        const choice other = {false, (int)s, 8 + (wait > work ? wait : work) + sums};
        const choice wide = {true, (int)s, a_cu * (8 + 1.2 * chunk) + sums};
        if (best.us == 0 || other.us < best.us) best = other;
        if (can_wide && wide.us < best.us) best = wide;
    }
    return best;
}

int64_t sums_bytes(const choice &c, int64_t outs, int64_t ins) { return c.splits > 1 ? c.splits * outs * ins * 4 : 0; }

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
    // dy may be laid out so that the wide kernel cannot take it
    const int64_t any = sums_bytes(choose(dtype, false, rows, outs, ins), outs, ins);
    const int64_t wide = fits_wide(dtype, outs, outs) ? sums_bytes(choose(dtype, true, rows, outs, ins), outs, ins) : 0;
    *bytes = wide > any ? wide : any;
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
    const bool vec = aligned(dy, 16) && dy_stride * size % 16 == 0 && outs * size % 16 == 0;
    const choice c = choose(dtype, vec && fits_wide(dtype, dy_stride, outs), rows, outs, ins);
    const int splits = c.splits;
    params a = {};
    a.dy = dy, a.codes = codes, a.exponents = exponents, a.dy_stride = dy_stride, a.rows = rows;
    a.chunk = ceil_div(ceil_div(rows, splits), WSTEP) * WSTEP;
    a.outs = (int32_t)outs, a.ins = (int32_t)ins, a.groups = (int32_t)ceil_div(ins, GROUP), a.padded = a.groups * GROUP;
    a.n_tiles = (int32_t)ceil_div(outs, BN), a.k_tiles = (int32_t)ceil_div(ins, BK);
    a.out = splits > 1 ? (float *)workspace : dw;
    const int64_t groups = (int64_t)a.n_tiles * a.k_tiles * splits;
    if (groups * THREADS > MAX_THREADS) return DEAR_ETOOBIG;
    const unsigned grid = (unsigned)groups;
    if (c.wide) weight_grad_wide_kernel<<<grid, THREADS, 0, stream>>>(a);
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
