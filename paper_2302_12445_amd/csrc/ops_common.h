// What the training operators' kernels share: element types, matrix products of 32 x 32 blocks for bf16 and fp32
// operands, tiles in LDS and the fragments read from them.
//
// Fragments.  A 32 x 32 product step takes 16 values of the summed index.  Lane l holds, of either operand, row (or
// column) l % 32 and eight of the sixteen: slots t = 0 .. 7 of half h = l / 32.  In bf16 that is one
// v_mfma_f32_32x32x16_bf16; in fp32 eight v_mfma_f32_32x32x2_f32, one for each slot, on the same layout.  The order of
// the sixteen does not matter as long as both operands agree.  Of the result, lane l holds column l % 32 and the rows
//     row(r) = 8 * (r / 4) + 4 * h + r % 4,   r = 0 .. 15.
// Taken as slots of a second product, r = 8 s + t of step s is row 16 s + 8 * (t / 4) + 4 h + t % 4: a result becomes an
// operand without leaving the lane, if the other operand is read in the same order (`transposed`, below).
#ifndef DEAR_OPS_COMMON_H
#define DEAR_OPS_COMMON_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "dear_ops.h"

#pragma clang fp contract(fast)

namespace dear_ops {

typedef __bf16 bf16;
typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

#define DEAR_LDS __attribute__((address_space(3)))

template <typename T> struct frag_of;
template <> struct frag_of<bf16> { typedef bf16x8 type; };
template <> struct frag_of<float> { typedef f32x8 type; };
template <typename T> using frag = typename frag_of<T>::type;

__device__ __forceinline__ f32x16 mma(bf16x8 a, bf16x8 b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mma(f32x8 a, f32x8 b, f32x16 c) {
#pragma unroll
    for (int t = 0; t < 8; ++t) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[t], b[t], c, 0, 0, 0);
    return c;
}

// Eight fp32 values as a fragment; to bf16 rounded to nearest, halves to even.
template <typename T> __device__ __forceinline__ frag<T> to_frag(const float *x) {
    frag<T> f;
#pragma unroll
    for (int t = 0; t < 8; ++t) f[t] = (T)x[t];
    return f;
}

// The other half's value joined with one's own: both halves get the same result.
__device__ __forceinline__ float halves_max(float x) {
    auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(w[0]), __uint_as_float(w[1]));
}
__device__ __forceinline__ float halves_sum(float x) {
    auto w = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(w[0]) + __uint_as_float(w[1]);
}


// Sum over the wave, the same in all lanes: quads, eights and sixteens by moves within a row of sixteen lanes, then
// across the rows.
template <int CTRL> __device__ __forceinline__ float plus_moved(float x) {
    return x + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float wave_sum(float x) {
    x = plus_moved<0xB1>(x);   // quad_perm 1, 0, 3, 2
    x = plus_moved<0x4E>(x);   // quad_perm 2, 3, 0, 1
    x = plus_moved<0x141>(x);  // row_half_mirror
    x = plus_moved<0x140>(x);  // row_mirror
    auto w = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return halves_sum(__uint_as_float(w[0]) + __uint_as_float(w[1]));
}

__device__ __forceinline__ int row_of(int r, int half) { return 8 * (r / 4) + 4 * half + r % 4; }

// A tile of rows of W values in LDS.  Rows are padded so that the sixteen-byte pieces of eight rows, and the
// 32-byte pieces of four rows, lie in different banks: by 32 bytes in bf16, by 16 in fp32.
template <typename T, int W> struct tile {
    static constexpr int stride = W + (sizeof(T) == 2 ? 16 : 4);  // elements
    static constexpr int bytes(int rows) { return rows * stride * (int)sizeof(T); }
};

// Rows row0 .. +31, slots of step kk: values 16 kk + 8 h + t of the row.
template <int W> __device__ __forceinline__ bf16x8 straight(const DEAR_LDS bf16 *s, int row0, int kk, int lane) {
    return *(const DEAR_LDS bf16x8 *)(s + (row0 + (lane & 31)) * tile<bf16, W>::stride + 16 * kk + 8 * (lane >> 5));
}
template <int W> __device__ __forceinline__ f32x8 straight(const DEAR_LDS float *s, int row0, int kk, int lane) {
    const DEAR_LDS float *p = s + (row0 + (lane & 31)) * tile<float, W>::stride + 16 * kk + 8 * (lane >> 5);
    const f32x4 a = *(const DEAR_LDS f32x4 *)p, b = *(const DEAR_LDS f32x4 *)(p + 4);
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Columns col0 .. +31, slots: rows row0 + 8 * (t / 4) + 4 h + t % 4 (row0 a multiple of 16: the order of a result).
// In bf16 the LDS transposes: of 16 lanes, lane i names four values of row i / 4 and gets the four rows of column i.
template <int W> __device__ __forceinline__ bf16x8 transposed(const DEAR_LDS bf16 *s, int row0, int col0, int lane) {
    const DEAR_LDS bf16 *p = s + (row0 + 4 * (lane >> 5) + (lane & 15) / 4) * tile<bf16, W>::stride + col0 +
                             16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((DEAR_LDS bf16x4 *)p);
    const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((DEAR_LDS bf16x4 *)(p + 8 * tile<bf16, W>::stride));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}
template <int W> __device__ __forceinline__ f32x8 transposed(const DEAR_LDS float *s, int row0, int col0, int lane) {
    const DEAR_LDS float *p = s + (row0 + 4 * (lane >> 5)) * tile<float, W>::stride + col0 + (lane & 31);
    f32x8 f;
#pragma unroll
    for (int t = 0; t < 8; ++t) f[t] = p[(8 * (t / 4) + t % 4) * tile<float, W>::stride];
    return f;
}

// ------------------------------------------------------------------------------------ tiles that memory fills directly
// Rows of W bf16 values without padding, brought by loads that write LDS themselves: a wave's load puts 64 pieces of 16
// bytes in a row, so that the order of the pieces is what keeps reads apart in the banks.  Piece c of a row stands at
// c ^ turn(row): for 128 values (256 bytes, one line of all banks) the eight rows that a quarter of a straight read
// touches, and the four rows of a transposing one, differ; for 64 values two rows share a line, and pairs of rows differ.
template <int W> struct direct {
    static constexpr int PIECES = W / 8;                     // of a row
    static constexpr int ROWS = 64 / PIECES;                 // of a wave's load
    __device__ static __forceinline__ int turn(int row) {
        return W == 128 ? (row & 3) << 2 | (row >> 2 & 3) : (row >> 1 & 1) << 2 | (row >> 2 & 3);
    }
    // Offset in bytes of piece c of a row.
    __device__ static __forceinline__ uint32_t at(int row, int c) { return row * (2 * W) + (c ^ turn(row)) * 16; }

    // A lane's offsets from a tile's start, of straight reads by step and of transposing ones by columns and rows.  `renew`
    // tells the compiler once a step that they may have changed: otherwise it keeps the sum of each with the place of
    // each tile, which is a constant of the instruction, in a register of its own.
    uint32_t row_at[W / 16], column_at[W / 32][2];
    __device__ __forceinline__ direct(int lane) {
#pragma unroll
        for (int kk = 0; kk < W / 16; ++kk) row_at[kk] = at(lane & 31, 2 * kk + (lane >> 5));
        const int row = 4 * (lane >> 5) + (lane & 15) / 4, c = 2 * (lane >> 4 & 1) + (lane & 3) / 2;
#pragma unroll
        for (int db = 0; db < W / 32; ++db)
#pragma unroll
            for (int u = 0; u < 2; ++u) column_at[db][u] = at(row + 8 * u, 4 * db + c) + 8 * (lane & 1);
    }
    __device__ __forceinline__ void renew() {
#pragma unroll
        for (int kk = 0; kk < W / 16; ++kk) asm("" : "+v"(row_at[kk]));
#pragma unroll
        for (int db = 0; db < W / 32; ++db) asm("" : "+v"(column_at[db][0]), "+v"(column_at[db][1]));
    }
    // By n bytes: a multiple of 32 rows.
    __device__ __forceinline__ void move(int n) {
#pragma unroll
        for (int kk = 0; kk < W / 16; ++kk) row_at[kk] += n;
#pragma unroll
        for (int db = 0; db < W / 32; ++db) column_at[db][0] += n, column_at[db][1] += n;
    }

    // Rows row0 .. +31 (a multiple of 32), slots of step kk, as `straight`.
    __device__ __forceinline__ bf16x8 straight(const DEAR_LDS bf16 *s, int row0, int kk) const {
        return *(const DEAR_LDS bf16x8 *)((const DEAR_LDS char *)(s + row0 * W) + row_at[kk]);
    }
    // Columns 32 db .. +31, slots of rows row0 .. +15 (a multiple of 16), as `transposed`.
    __device__ __forceinline__ bf16x8 transposed(const DEAR_LDS bf16 *s, int row0, int db) const {
        const DEAR_LDS char *p = (const DEAR_LDS char *)(s + row0 * W);
        const bf16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((DEAR_LDS bf16x4 *)(p + column_at[db][0]));
        const bf16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((DEAR_LDS bf16x4 *)(p + column_at[db][1]));
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

__device__ __forceinline__ void load_to_lds(const char *p, DEAR_LDS void *s) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)p, s, 16, 0, 0);
}

// One value a lane.
__device__ __forceinline__ void load_value_to_lds(const float *p, DEAR_LDS float *s) {
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)p, s, 4, 0, 0);
}

// Barrier behind which the tiles that this workgroup's waves have loaded to LDS are whole: each wave first waits for its
// own loads (vmcnt 0), which a barrier by itself does not.
__device__ __forceinline__ void loads_barrier() {
    __builtin_amdgcn_s_waitcnt(0x0f70);
    __syncthreads();
}

// HIP takes fewer than 2^32 threads along a dimension of a launch.
constexpr int64_t MAX_THREADS = 0xffffffff;

inline bool aligned(const void *p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
inline int launch_status() { return hipGetLastError() == hipSuccess ? DEAR_OK : DEAR_EHIP; }

}  // namespace dear_ops
#endif
