// Gated linear recurrence along the steps of each sequence, forward and backward (definitions: dear_ops.h).
//
//     a = sigmoid(gate);  s[t] = a[t] s[t-1] + (1 - a[t]) x[t]
//     G[t] = dh[t] + e[t+1],  e[t] = a[t] G[t];  dx = (1 - a) G;  dgate = G (s[t-1] - x) a (1 - a)
//
// A stretch of steps is a map s -> A s + H with A the product of its a; two stretches in a row are again one:
// (A2 A1, A2 H1 + H2).  Backward the map is e -> A e + E with the same A, from the last step to the first.  So a tile of
// 256 steps is cut into strips of sixteen: a lane joins its own steps, lanes and waves join theirs, and a second
// walk over the strip, from the state before it, gives the outputs; every tensor is read once.  Of sequences of several
// tiles each tile has a workgroup of its own, which tells the others its map and joins those of the tiles before
// it.  The backward pass needs the states before each step as well: it computes them again, in fp32, from the states that the
// forward pass kept at each tile's first step, which takes less traffic than to read h, and no rounding.
//
// What it reads and writes, 6 bytes of bf16 an element forward and 10 backward, and the vector instructions, which issue 64 and 72 % of the time, bound it
// together: single tiles, 64 x 256 x 1024 bf16, 18.6 and 32.7 us, where 15 and 25 are what a large copy would take (calls in a row find about half
// of it in the last cache); tiles that are joined, 2 x 8192 x 1024, with the launch that clears their maps 25.5 and 40.1.
#include <cfloat>
#include <type_traits>

#include "ops_common.h"

#pragma clang fp contract(fast)

namespace {

using namespace dear_ops;

constexpr int KEPT = DEAR_RECURRENCE_KEPT;  // steps from one kept state to the next: a whole tile
constexpr int R = 16;                       // steps of a lane's strip
constexpr int N = 2;                        // channels of a lane
constexpr int ROW_LANES = 32;               // lanes across the channels; the halves of a wave are two strips
constexpr int STRIPS = 64 / ROW_LANES;
constexpr int WAVE_STEPS = STRIPS * R;
constexpr int CG = N * ROW_LANES;           // channels of a workgroup: in bf16 128 bytes of a row, a line of the cache
constexpr int WAVES = KEPT / WAVE_STEPS;    // that a tile fills
static_assert(KEPT % WAVE_STEPS == 0, "a tile is made of whole waves");

struct rows_t {
    const void *data;
    int64_t batch_stride, step_stride;
};

struct params {
    rows_t x, gate, h, dh, dx, dgate;
    const float *state, *dlast;
    float *last, *dstate, *kept;
    const int32_t *lens;
    uint32_t *tickets;  // workgroups that have begun of those that share a sequence's channels, one count a line of the cache
    uint64_t *maps;     // of their tiles, [batch, tiles, width]: C and H, or E, of the tiles in their order; at first all ones
    int64_t steps;
    int32_t width, groups, tiles;
};

// a = sigmoid(g) and b = 1 - a: with t = exp(-g) they are 1 / (1 + t) and t / (1 + t).  exp2's argument y is rounded, by |g| 2^-24 and more, which
// is an error of t's.  Of fp32 gates, t is mended by what y leaves of -g, so that a and b are right to 8 units of 2^-24 (exp2 and the reciprocal 2 each,
// four roundings); where gates are bf16 that would cost 4 to 5 % of the time (64 x 256 x 1024 18.6 us, so 19.4, backward 32.7 and 34.4; of fp32 gates less than 1), and
// results of bf16 are rounded by 2^15 units.  Where fp32 has no more: below gates of -87.3, where t stops so that 1 + t has a reciprocal, a is some 2^-126, and above
// 87.3 b may be 0.  A NaN stays one.
template <typename T> __device__ __forceinline__ void gates(float g, float &a, float &b, float &t) {
    if (sizeof(T) == 4) {
        const float f = __builtin_elementwise_maximum(__builtin_elementwise_minimum(g, 128.f), -87.3365f), y = f * -0x1.715476p+0f;
        const float r = __builtin_fmaf(y, 0x1.05c61p-29f, __builtin_fmaf(y, -0x1.62e43p-1f, -f));
        t = __builtin_amdgcn_exp2f(y);
        t = __builtin_fmaf(t, r, t);
    } else {
        t = __builtin_amdgcn_exp2f(__builtin_elementwise_minimum(g * -1.44269504088896f, 126.f));
    }
    a = __builtin_amdgcn_rcpf(1.f + t);
    b = t * a;
}
template <typename T> __device__ __forceinline__ void gates(float g, float &a, float &b) {
    float t;
    gates<T>(g, a, b, t);
}

// The halves' values of x: the earlier strip's and the later one's.
__device__ __forceinline__ void halves(float x, float &earlier, float &later) {
    const uint32_t u = __float_as_uint(x);
    auto w = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    earlier = __uint_as_float(w[0]), later = __uint_as_float(w[1]);
}

// What a map keeps of the state, A, is told on as one number C: A itself below a half, from there on -(1 - A), with the sign, by which the state
// goes on as s + (H - (1 - A) s).  An A near 1 that is rounded by itself is wrong by the same 2^-25 each time that a gate stays, which adds up over
// all that a channel remembers, to 2^-25 / (1 - a) (of fp32 steps with a gate of 9, 4e-4); by C the state goes to where H and 1 - A say, however
// long the sequence is.  So go states from tile to tile and from call to call (2 x 8192 x 1024 bf16 forward 27.1 us, so 27.9); within a tile, from a
// state that is at hand, they go by A.  -0 leaves a state as it is.
__device__ __forceinline__ float coefficient(float A, float B) { return B <= 0.5f ? -B : A; }
__device__ __forceinline__ bool by_complement(float C) { return (int32_t)__float_as_uint(C) < 0; }
__device__ __forceinline__ float whole(float C) { return by_complement(C) ? 1.f + C : C; }
__device__ __forceinline__ float complement(float C) { return by_complement(C) ? -C : 1.f - C; }
// (An infinite state stays one: only what is subtracted is kept finite.)
__device__ __forceinline__ float through(float C, float H, float s) {
    const bool less = by_complement(C);
    const float t = less ? __builtin_amdgcn_fmed3f(s, -FLT_MAX, FLT_MAX) : s;
    return __builtin_fmaf(C, t, H) + (less ? s : 0.f);
}
// A, B = 1 - A and H of several stretches in a row (or A, B and E from the last to the first).  H, which starts from 0, goes by A: it is off by a
// rounding a stretch, whatever the state is.
struct stretches {
    float A = 1.f, B = 0.f, H = 0.f;
    __device__ __forceinline__ void add(float A1, float B1, float H1) {
        H = A1 * H + H1;
        B += A * B1;
        A *= A1;
    }
};

// Joins the strips of a wave.  q: of a strip 1 / A is the product of its 1 + t, and q what that is above 1, q = (1 + t) q + t from step to step: a sum
// of nothing below 0, out of which A and, where it is near 1, B = 1 - A come as exactly as it is.  (A large q has no inverse that fp32 holds, or is
// infinite, or 0 of that and so a NaN: A is 0 there.)  H and E become the wave's.  before: the map from the wave's first step to the strip's, behind:
// backward from the wave's last step to the strip's, by A.
template <bool FORWARD, bool BACKWARD>
__device__ __forceinline__ void join(float q, float &A, float &B, float &H, float &E, float &before_A, float &before_H, float &behind_A, float &behind_E,
                                     int lane) {
    float q0, q1;
    halves(q, q0, q1);
    const float A0 = __builtin_amdgcn_rcpf(1.f + q0), A1 = __builtin_amdgcn_rcpf(1.f + q1);
    const bool later = lane & 32;
    if (FORWARD) {
        float H0, H1;
        halves(H, H0, H1);
        before_A = later ? A0 : 1.f;
        before_H = later ? H0 : 0.f;
        H = A1 * H0 + H1;
    }
    if (BACKWARD) {
        float E0, E1;
        halves(E, E0, E1);
        behind_A = later ? 1.f : A1;
        behind_E = later ? 0.f : E1;
        E = A0 * E1 + E0;
    }
    A = A0 * A1;
    const float all = q1 * (1.f + q0) + q0;
    B = all <= 1.f ? all * A : 1.f - A;
}

// How a lane's N channels lie in memory.
enum { SINGLE, ANYWHERE, ALIGNED };

// First of a workgroup's N channels number `pair`.  Lanes behind the last channel take the last ones over again, with the same results, so that no
// lane needs a branch.
template <int MODE> __device__ __forceinline__ int first_of(const params &a, int group, int pair) {
    const int col = group * CG + pair * N;
    return MODE != SINGLE ? min(col, a.width - N) : col;
}
// Where a lane stands: its channels, its strip and, of a tile, its first step.
struct place {
    int64_t b;
    int lane, wave, group, col, step;
    template <int MODE> __device__ __forceinline__ place(const params &a, uint32_t sequence_group, std::integral_constant<int, MODE>) {
        lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        b = sequence_group / a.groups;
        group = (int)(sequence_group % a.groups);
        col = first_of<MODE>(a, group, lane % ROW_LANES);
        step = wave * WAVE_STEPS + lane / ROW_LANES * R;
    }
};

__device__ __forceinline__ int64_t length(const params &a, int64_t b) {
    return a.lens ? min(max((int64_t)a.lens[b], (int64_t)0), a.steps) : a.steps;
}

// A lane's channels of a step as they are in memory, in whole registers: two values of bf16 are one.
typedef uint32_t u32;
template <typename T> struct raw_of { typedef u32 type; };
template <> struct raw_of<float> { typedef f32x2 type; };
template <typename T> using raw = typename raw_of<T>::type;
template <typename R> struct anywhere_of { typedef R type __attribute__((aligned(2))); };  // global memory takes it
template <> struct anywhere_of<f32x2> { typedef f32x2 type __attribute__((aligned(4))); };

__device__ __forceinline__ float get(u32 x, int c) { return __uint_as_float(c ? x & 0xffff0000u : x << 16); }
__device__ __forceinline__ float get(f32x2 x, int c) { return x[c]; }
// To bf16 rounded to nearest, halves to even.
template <typename T> __device__ __forceinline__ raw<T> both(float x, float y) {
    if constexpr (sizeof(T) == 2) return __builtin_bit_cast(u32, bf16x2{(bf16)x, (bf16)y});
    else return f32x2{x, y};
}

// at: the row, or bytes before it that are the same for the whole workgroup, and off the others.
template <typename T, int MODE> __device__ __forceinline__ raw<T> load(const char *at, uint32_t off, int col, int cols) {
    if (MODE == ALIGNED) return *(const raw<T> *)(at + (off + (uint32_t)(col * (int)sizeof(T))));
    if (MODE == ANYWHERE) return *(const typename anywhere_of<raw<T>>::type *)(at + (off + (uint32_t)(col * (int)sizeof(T))));
    const T x = *(const T *)(at + (off + (uint32_t)(min(col, cols - 1) * (int)sizeof(T))));
    const T y = *(const T *)(at + (off + (uint32_t)(min(col + 1, cols - 1) * (int)sizeof(T))));
    return both<T>((float)x, (float)y);
}
template <typename T, int MODE> __device__ __forceinline__ void store(char *at, uint32_t off, raw<T> v, int col, int cols) {
    if (MODE == ALIGNED) *(raw<T> *)(at + (off + (uint32_t)(col * (int)sizeof(T)))) = v;
    else if (MODE == ANYWHERE) *(typename anywhere_of<raw<T>>::type *)(at + (off + (uint32_t)(col * (int)sizeof(T)))) = v;
    else
#pragma unroll
        for (int c = 0; c < N; ++c) *(T *)(at + (off + (uint32_t)(min(col + c, cols - 1) * (int)sizeof(T)))) = (T)get(v, c);
}

// Of a tensor the R rows of a lane's strip in a tile that starts at `at` (the same for the whole workgroup, so that a lane's address is
// 32 bits beside it).  Only `valid` rows of the tile, one at least, are read: behind them the last one again.
template <typename T> __device__ __forceinline__ char *tile_at(const rows_t &t, int64_t b, int tile) {
    return (char *)t.data + (b * t.batch_stride + (int64_t)tile * KEPT * t.step_stride) * (int64_t)sizeof(T);
}
template <typename T, int MODE>
__device__ __forceinline__ void load_strip(raw<T> (&v)[R], const rows_t &from, int tile, const place &p, int valid, int cols) {
    const char *at = tile_at<T>(from, p.b, tile);
    const uint32_t stride = (uint32_t)from.step_stride * (uint32_t)sizeof(T), last = (uint32_t)(valid - 1) * stride, off = (uint32_t)p.step * stride;
    if (valid == KEPT) {
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = load<T, MODE>(at + (int64_t)r * stride, off, p.col, cols);
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) v[r] = load<T, MODE>(at, min(off + (uint32_t)r * stride, last), p.col, cols);
    }
}
template <typename T, int MODE>
__device__ __forceinline__ void store_strip(const raw<T> (&v)[R], const rows_t &to, int tile, const place &p, int there, int cols) {
    char *at = tile_at<T>(to, p.b, tile);
    const uint32_t stride = (uint32_t)to.step_stride * (uint32_t)sizeof(T), off = (uint32_t)p.step * stride;
    if (there == KEPT) {
#pragma unroll
        for (int r = 0; r < R; ++r) store<T, MODE>(at + (int64_t)r * stride, off, v[r], p.col, cols);
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (p.step + r < there) store<T, MODE>(at + (int64_t)r * stride, off, v[r], p.col, cols);
    }
}
// Of the steps left from a tile's first on, those within it.
__device__ __forceinline__ int within(int64_t steps, int tile) {
    return (int)min(max(steps - (int64_t)tile * KEPT, (int64_t)0), (int64_t)KEPT);
}

// A row of states.
template <int MODE> __device__ __forceinline__ void load_state(float *s, const float *row, int col, int cols) {
    const f32x2 v = load<float, MODE>((const char *)row, 0, col, cols);
#pragma unroll
    for (int c = 0; c < N; ++c) s[c] = v[c];
}
template <int MODE> __device__ __forceinline__ void store_state(float *row, const float *s, int col, int cols) {
    store<float, MODE>((char *)row, 0, f32x2{s[0], s[1]}, col, cols);
}

// The map of a tile's steps before the last wave has been joined: each wave's in LDS, [wave][A, 1 - A, H or E][channel].
enum { MAP_A, MAP_B, MAP_H, MAP_E };
template <int W> struct wave_maps_of { typedef float type[W][4][CG] __attribute__((aligned(16))); };
template <int W> using wave_maps = typename wave_maps_of<W>::type;

// s through a wave's map, of H or E, within a tile: by A alone, as in a strip.  One wave's after another, as all of them at once take registers.
template <int WHICH, int W> __device__ __forceinline__ void pass(float *s, const wave_maps<W> &maps, int w, const place &p) {
    const f32x2 A = *(const f32x2 *)&maps[w][MAP_A][p.lane % ROW_LANES * N], H = *(const f32x2 *)&maps[w][WHICH][p.lane % ROW_LANES * N];
#pragma unroll
    for (int c = 0; c < N; ++c) s[c] = A[c] * s[c] + H[c];
    __builtin_amdgcn_sched_barrier(0);
}
// s through all waves' maps, joined before.
template <int WHICH, int W> __device__ __forceinline__ void pass_all(float *s, const wave_maps<W> &maps, const place &p) {
    stretches all[N];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const int w = WHICH == MAP_H ? i : W - 1 - i, at = p.lane % ROW_LANES * N;
        const f32x2 A = *(const f32x2 *)&maps[w][MAP_A][at], B = *(const f32x2 *)&maps[w][MAP_B][at], H = *(const f32x2 *)&maps[w][WHICH][at];
#pragma unroll
        for (int c = 0; c < N; ++c) all[c].add(A[c], B[c], H[c]);
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int c = 0; c < N; ++c) s[c] = through(coefficient(all[c].A, all[c].B), all[c].H, s[c]);
}

constexpr uint64_t UNTOLD = ~(uint64_t)0;
constexpr int TICKET = 32;  // counts of workgroups lie 128 bytes apart

// What workgroups share, before they begin: maps, and a copy of the state that they start from, as its place may be the last one's too.
__global__ __launch_bounds__(256) void untold_kernel(uint64_t *maps, int64_t n, uint32_t *tickets, const float *from, float *state, int64_t states,
                                                     int64_t counts) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) maps[i] = UNTOLD;
    if (i < states) state[i] = from ? from[i] : 0.f;
    if (i < counts) tickets[i * TICKET] = 0;
}

// The workgroup's place among those that have begun on the same channels, which is its tile: whoever has a smaller number has begun before,
// and tells its map without waiting for anyone, so that every wait for a smaller number ends, in whatever order workgroups are started.
__device__ __forceinline__ int take_ticket(uint32_t *ticket) {
    __shared__ uint32_t mine;
    if (threadIdx.x == 0) mine = __hip_atomic_fetch_add(ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    return (int)__builtin_amdgcn_readfirstlane(mine);
}

// A map as one word, so that who reads it reads all of it, and needs no fence.
__device__ __forceinline__ uint64_t *map_at(const params &a, int64_t b, int order, int col, int c) {
    return a.maps + (b * a.tiles + order) * a.width + min(col + c, a.width - 1);
}
// A tile's map from its waves', of H or E: a lane of the first wave takes one channel.
template <int WHICH, int MODE, int W> __device__ __forceinline__ void tell(const params &a, const place &p, int order, const wave_maps<W> &maps) {
    static_assert(CG == 64, "a channel a lane");
    stretches all;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const int w = WHICH == MAP_H ? i : W - 1 - i;
        all.add(maps[w][MAP_A][p.lane], maps[w][MAP_B][p.lane], maps[w][WHICH][p.lane]);
    }
    const float C = coefficient(all.A, all.B);
    const uint32_t x = C != C ? 0x7fc00000u : __float_as_uint(C);  // (some NaN is all ones)
    __hip_atomic_store(map_at(a, p.b, order, first_of<MODE>(a, p.group, p.lane / N), p.lane % N), (uint64_t)__float_as_uint(all.H) << 32 | x, __ATOMIC_RELAXED,
                       __HIP_MEMORY_SCOPE_AGENT);
}

// s through the maps of the tiles before `order`: strips take a run of tiles each, and are joined as a tile's are.  The order in which maps
// are joined does not depend on when they are told.
template <int W> __device__ __forceinline__ void through_earlier(float *s, const params &a, const place &p, int order, wave_maps<W> &maps) {
    const int each = (order + W * STRIPS - 1) / (W * STRIPS), first = (p.wave * STRIPS + p.lane / ROW_LANES) * each;
    stretches before[N];
    for (int i = first; i < min(first + each, order); ++i) {
        uint64_t x[N];
        for (;;) {
            bool told = true;
#pragma unroll
            for (int c = 0; c < N; ++c) {
                x[c] = __hip_atomic_load(map_at(a, p.b, i, p.col, c), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                told = told && x[c] != UNTOLD;
            }
            if (told) break;
            __builtin_amdgcn_s_sleep(1);
        }
#pragma unroll
        for (int c = 0; c < N; ++c) {
            const float mine = __uint_as_float((uint32_t)x[c]);
            const float H = through(mine, __uint_as_float((uint32_t)(x[c] >> 32)), before[c].H);  // (of any number of stretches)
            before[c].add(whole(mine), complement(mine), 0.f);
            before[c].H = H;
        }
    }
#pragma unroll
    for (int c = 0; c < N; ++c) {
        stretches both, later;
        halves(before[c].A, both.A, later.A), halves(before[c].B, both.B, later.B), halves(before[c].H, both.H, later.H);
        both.add(later.A, later.B, later.H);
        if (p.lane < ROW_LANES) {
            maps[p.wave][MAP_A][p.lane * N + c] = both.A;
            maps[p.wave][MAP_B][p.lane * N + c] = both.B;
            maps[p.wave][MAP_H][p.lane * N + c] = both.H;
        }
    }
    __syncthreads();
    pass_all<MAP_H, W>(s, maps, p);
}

// Steps behind the last one: a = 1 and nothing added, by gates of infinity and values of 0.
template <typename T> __device__ __forceinline__ void still(raw<T> (&g)[R], raw<T> (&x)[R], const place &p, int valid) {
    asm volatile("");  // in a branch of its own: whole tiles are to pass it by
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool in = p.step + r < valid;
        g[r] = in ? g[r] : both<T>(__builtin_inff(), __builtin_inff());
        x[r] = in ? x[r] : raw<T>{};
    }
}
template <typename T> __device__ __forceinline__ void zero_behind(raw<T> (&x)[R], const place &p, int valid) {
    asm volatile("");
#pragma unroll
    for (int r = 0; r < R; ++r) x[r] = p.step + r < valid ? x[r] : raw<T>{};
}

// A workgroup of W waves takes one tile, all of a sequence's steps or (SHARED) those that its ticket says; the second set of maps is for the
// tiles before.
template <typename T, int W, int MODE, bool SHARED> __global__ __launch_bounds__(64 * W, 4) void recurrence_kernel(params a) {
    __shared__ wave_maps<W> lds[SHARED ? 2 : 1];
    const uint32_t id = SHARED ? blockIdx.x % (gridDim.x / a.tiles) : blockIdx.x;  // a sequence and its channels: neighbours take neighbouring ones
    const place p(a, id, std::integral_constant<int, MODE>());
    const int tile = SHARED ? take_ticket(a.tickets + id * TICKET) : 0;
    const int64_t end = length(a, p.b);
    const bool speaks = threadIdx.x < ROW_LANES;  // stores states
    float carry[N] = {};
    if (a.state) load_state<MODE>(carry, a.state + p.b * a.width, p.col, a.width);
    const int valid = within(end, tile), there = within(a.steps, tile);
    raw<T> g[R], x[R];
    if (valid > 0) {
        load_strip<T, MODE>(g, a.gate, tile, p, valid, a.width);
        load_strip<T, MODE>(x, a.x, tile, p, valid, a.width);
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) g[r] = x[r] = raw<T>{};
    }
    if (valid < WAVE_STEPS * W) still<T>(g, x, p, valid);
    auto &maps = lds[0];
    float ga[R][N], gx[R][N], before_A[N], before_H[N];
#pragma unroll
    for (int c = 0; c < N; ++c) {
        float q = 0.f, A, B, H = 0.f, none = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float gb, t;
            gates<T>(get(g[r], c), ga[r][c], gb, t);
            gx[r][c] = gb * get(x[r], c);
            q = (1.f + t) * q + t;
            H = ga[r][c] * H + gx[r][c];
        }
        join<true, false>(q, A, B, H, none, before_A[c], before_H[c], none, none, p.lane);
        if (p.lane < ROW_LANES) {
            maps[p.wave][MAP_A][p.lane * N + c] = A;
            maps[p.wave][MAP_B][p.lane * N + c] = B;
            maps[p.wave][MAP_H][p.lane * N + c] = H;
        }
        __builtin_amdgcn_sched_barrier(0);  // one channel after another: together they take registers that waves could have
    }
    __syncthreads();
    if (SHARED) {
        if (p.wave == 0 && tile + 1 < a.tiles) tell<MAP_H, MODE, W>(a, p, tile, maps);
        if (tile > 0) through_earlier<W>(carry, a, p, tile, lds[SHARED ? 1 : 0]);
    }
    if (speaks && a.kept) store_state<MODE>(a.kept + (p.b * a.tiles + tile) * a.width, carry, p.col, a.width);
    float s[N];
#pragma unroll
    for (int c = 0; c < N; ++c) s[c] = carry[c];
    if (p.wave == 0 && tile == a.tiles - 1) {
        pass_all<MAP_H, W>(carry, maps, p);
    } else {
#pragma unroll
        for (int w = 0; w < W - 1; ++w)
            if (w < p.wave) pass<MAP_H, W>(s, maps, w, p);
    }
#pragma unroll
    for (int c = 0; c < N; ++c) s[c] = before_A[c] * s[c] + before_H[c];
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int c = 0; c < N; ++c) s[c] = ga[r][c] * s[c] + gx[r][c];
        x[r] = both<T>(s[0], s[1]);
    }
    if (valid < there) zero_behind<T>(x, p, valid);
    store_strip<T, MODE>(x, a.h, tile, p, there, a.width);
    if (speaks && a.last && tile == a.tiles - 1) store_state<MODE>(a.last + p.b * a.width, carry, p.col, a.width);
}

// One step, as of sequences that are continued token by token: a lane has two channels of a sequence, and nothing to join (of launches in a row 16 x 1
// x 1024 bf16 2.3 us, 256 x 1 x 1024 2.6; by the kernel above, whose lanes have sixteen steps, 3.9 and 7.4).
template <typename T, int MODE> __global__ __launch_bounds__(256) void recurrence_step_kernel(params a, uint32_t pairs, uint32_t all) {
    const uint32_t i = blockIdx.x * 256 + threadIdx.x;
    if (i >= all) return;
    const int64_t b = i / pairs;
    int col = (int)(i % pairs) * N;
    if (MODE != SINGLE) col = min(col, a.width - N);
    const raw<T> g = load<T, MODE>(tile_at<T>(a.gate, b, 0), 0, col, a.width), x = load<T, MODE>(tile_at<T>(a.x, b, 0), 0, col, a.width);
    float s[N] = {}, h[N] = {};
    if (a.state) load_state<MODE>(s, a.state + b * a.width, col, a.width);
    if (a.kept) store_state<MODE>(a.kept + b * a.width, s, col, a.width);
    if (length(a, b) > 0)
#pragma unroll
        for (int c = 0; c < N; ++c) {
            float ga, gb;
            gates<T>(get(g, c), ga, gb);
            const float y = through(coefficient(ga, gb), gb * get(x, c), s[c]);
            h[c] = s[c] = y;
        }
    store<T, MODE>(tile_at<T>(a.h, b, 0), 0, both<T>(h[0], h[1]), col, a.width);
    if (a.last) store_state<MODE>(a.last + b * a.width, s, col, a.width);
}

// As recurrence_kernel, from the last tile to the first; the states before the tile's steps come from the kept one.
template <typename T, int W, int MODE, bool SHARED> __global__ __launch_bounds__(64 * W, sizeof(T) == 2 ? 4 : 2) void recurrence_backward_kernel(params a) {
    __shared__ wave_maps<W> lds[SHARED ? 2 : 1];
    const uint32_t id = SHARED ? blockIdx.x % (gridDim.x / a.tiles) : blockIdx.x;  // a sequence and its channels: neighbours take neighbouring ones
    const place p(a, id, std::integral_constant<int, MODE>());
    const int order = SHARED ? take_ticket(a.tickets + id * TICKET) : 0, tile = a.tiles - 1 - order;
    const int64_t end = length(a, p.b);
    const bool speaks = threadIdx.x < ROW_LANES;
    float carry[N] = {};
    if (a.dlast) load_state<MODE>(carry, a.dlast + p.b * a.width, p.col, a.width);
    const int valid = within(end, tile), there = within(a.steps, tile);
    raw<T> g[R], x[R], dh[R];
    if (valid > 0) {
        load_strip<T, MODE>(g, a.gate, tile, p, valid, a.width);
        load_strip<T, MODE>(x, a.x, tile, p, valid, a.width);
        load_strip<T, MODE>(dh, a.dh, tile, p, valid, a.width);
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) g[r] = x[r] = dh[r] = raw<T>{};
    }
    if (valid < WAVE_STEPS * W) still<T>(g, x, p, valid), zero_behind<T>(dh, p, valid);
    float s[N];
    load_state<MODE>(s, a.kept + (p.b * a.tiles + tile) * a.width, p.col, a.width);
    auto &maps = lds[0];
    float before_A[N], before_H[N], behind_A[N], behind_E[N];
#pragma unroll
    for (int c = 0; c < N; ++c) {
        float q = 0.f, A, B, H = 0.f, E = 0.f, ga[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float gb, t;
            gates<T>(get(g[r], c), ga[r], gb, t);
            q = (1.f + t) * q + t;
            H = ga[r] * H + gb * get(x[r], c);
        }
#pragma unroll
        for (int r = R - 1; r >= 0; --r) E = ga[r] * E + ga[r] * get(dh[r], c);
        join<true, true>(q, A, B, H, E, before_A[c], before_H[c], behind_A[c], behind_E[c], p.lane);
        if (p.lane < ROW_LANES) {
            maps[p.wave][MAP_A][p.lane * N + c] = A;
            maps[p.wave][MAP_B][p.lane * N + c] = B;
            maps[p.wave][MAP_H][p.lane * N + c] = H;
            maps[p.wave][MAP_E][p.lane * N + c] = E;
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
    if (SHARED) {
        if (p.wave == 0 && tile > 0) tell<MAP_E, MODE, W>(a, p, order, maps);
        if (order > 0) through_earlier<W>(carry, a, p, order, lds[SHARED ? 1 : 0]);
    }
    float e[N];
#pragma unroll
    for (int c = 0; c < N; ++c) e[c] = carry[c];
#pragma unroll
    for (int w = W - 1; w > 0; --w)
        if (w > p.wave) pass<MAP_E, W>(e, maps, w, p);
#pragma unroll
    for (int w = 0; w < W - 1; ++w)
        if (w < p.wave) pass<MAP_H, W>(s, maps, w, p);
    if (p.wave == 0 && tile == 0) pass_all<MAP_E, W>(carry, maps, p);
    // the gates are computed again, channel by channel, and the gradients take the inputs' places: kept from above they would take 64 registers
#pragma unroll
    for (int r = 0; r < R; ++r) asm("" : "+v"(g[r]), "+v"(x[r]), "+v"(dh[r]));
    float dx[N][R], dg[N][R];
#pragma unroll
    for (int c = 0; c < N; ++c) {
        s[c] = before_A[c] * s[c] + before_H[c];
        e[c] = behind_A[c] * e[c] + behind_E[c];
        float ga[R], gb[R], q[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            gates<T>(get(g[r], c), ga[r], gb[r]);
            q[r] = (s[c] - get(x[r], c)) * ga[r];
            s[c] = ga[r] * s[c] + gb[r] * get(x[r], c);
        }
#pragma unroll
        for (int r = R - 1; r >= 0; --r) {
            const float G = get(dh[r], c) + e[c];
            dx[c][r] = gb[r] * G;
            dg[c][r] = q[r] * dx[c][r];
            e[c] = ga[r] * G;
        }
        __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) x[r] = both<T>(dx[0][r], dx[1][r]), g[r] = both<T>(dg[0][r], dg[1][r]);
    if (valid < there) zero_behind<T>(x, p, valid), zero_behind<T>(g, p, valid);
    store_strip<T, MODE>(x, a.dx, tile, p, there, a.width);
    store_strip<T, MODE>(g, a.dgate, tile, p, there, a.width);
    if (speaks && a.dstate && tile == 0) store_state<MODE>(a.dstate + p.b * a.width, carry, p.col, a.width);
}

// ------------------------------------------------------------------------------------ host
constexpr int64_t MAX_STEPS = (int64_t)1 << 30;
constexpr int32_t MAX_WIDTH = 1 << 24;
constexpr int64_t MAX_STEP_STRIDE = 1 << 22;  // so that 32 bits reach the rows of a tile

int size_of(int32_t dtype) { return dtype == DEAR_BF16 ? 2 : 4; }

// Channels of a workgroup.
int64_t groups_of(const dear_recurrence_t &r) { return ceil_div(r.width, CG); }

// Whether workgroups share a sequence's channels, a tile each, which takes a launch more.
bool shares(const dear_recurrence_t &r) { return r.steps > KEPT; }

int check(const dear_recurrence_t *r) {
    if (!r || (r->dtype != DEAR_F32 && r->dtype != DEAR_BF16) || r->batch < 0 || r->steps < 0 || r->steps > MAX_STEPS) return DEAR_EINVAL;
    if (r->width < 1 || r->width > MAX_WIDTH || r->reserved != 0) return DEAR_EINVAL;
    return DEAR_OK;
}

// Whether a launch would have more threads than it takes.  Asked by division, as products of the sizes may pass 64 bits; what is below the limit,
// workspaces among it, stays far from that.
bool too_many(const dear_recurrence_t &r) {
    if (r.batch == 0 || r.steps == 0) return false;
    return groups_of(r) * ceil_div(r.steps, KEPT) > MAX_THREADS / (64 * WAVES) / r.batch;
}

// A tensor of the structure, which is read or, where it is written, has a place of its own for each element.
int check_tensor(const dear_recurrence_t &r, const dear_steps_t &t, bool written) {
    if (!t.data || t.batch_stride < 0 || t.step_stride < 0) return DEAR_EINVAL;
    if (r.steps > 1 && t.step_stride >= MAX_STEP_STRIDE) return DEAR_ETOOBIG;
    const int64_t sequence = r.width + (r.steps > 1 ? (r.steps - 1) * t.step_stride : 0);
    if (r.batch > 1 && t.batch_stride > (INT64_MAX / 4 - sequence) / (r.batch - 1)) return DEAR_EINVAL;  // (4 bytes an element)
    if (written) {
        const int64_t batch = r.batch, steps = r.steps;
        const bool by_batch = t.batch_stride >= t.step_stride;  // which of the axes lies further apart
        const int64_t inner = by_batch ? t.step_stride : t.batch_stride, outer = by_batch ? t.batch_stride : t.step_stride;
        const int64_t inner_n = by_batch ? steps : batch, outer_n = by_batch ? batch : steps;
        int64_t span = r.width;
        if (inner_n > 1) {
            if (inner < span) return DEAR_EINVAL;
            if (inner > (INT64_MAX - span) / inner_n) return DEAR_EINVAL;
            span += (inner_n - 1) * inner;
        }
        if (outer_n > 1 && outer < span) return DEAR_EINVAL;
    }
    return aligned(t.data, size_of(r.dtype)) ? DEAR_OK : DEAR_EALIGN;
}

int64_t workspace_of(const dear_recurrence_t &r) {
    return r.batch && shares(r) ? r.batch * (groups_of(r) * TICKET * 4 + (ceil_div(r.steps, KEPT) + 1) * r.width * 8) : 0;
}

bool vectors(const dear_recurrence_t &r, const dear_steps_t &t) {
    const int n = size_of(r.dtype);
    return aligned(t.data, N * n) && t.batch_stride % N == 0 && t.step_stride % N == 0;
}

int check_call(const dear_recurrence_t *r, bool backward) {
    if (int rc = check(r)) return rc;
    if (r->batch == 0) return DEAR_OK;
    if (too_many(*r)) return DEAR_ETOOBIG;
    if (!aligned(r->lens, 4) || !aligned(r->state, 4) || !aligned(r->last, 4) || !aligned(r->kept, 4) || !aligned(r->dlast, 4) ||
        !aligned(r->dstate, 4))
        return DEAR_EALIGN;
    if (r->steps > 0) {
        if (backward && !r->kept) return DEAR_EINVAL;
        if (int rc = check_tensor(*r, r->x, false)) return rc;
        if (int rc = check_tensor(*r, r->gate, false)) return rc;
        if (!backward)
            if (int rc = check_tensor(*r, r->h, true)) return rc;
        if (backward) {
            if (int rc = check_tensor(*r, r->dh, false)) return rc;
            if (int rc = check_tensor(*r, r->dx, true)) return rc;
            if (int rc = check_tensor(*r, r->dgate, true)) return rc;
        }
        const int64_t need = workspace_of(*r);
        if (need && !r->workspace) return DEAR_EINVAL;
        if (need && !aligned(r->workspace, 256)) return DEAR_EALIGN;
        if (need > r->workspace_bytes) return DEAR_ETOOBIG;
    }
    return DEAR_OK;
}

// The state of sequences without steps.
__global__ __launch_bounds__(256) void copy_state_kernel(const float *from, float *to, int64_t n) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < n) to[i] = from ? from[i] : 0.f;
}

template <typename T, int MODE, bool BACKWARD> void launch(params a, int64_t batch, bool shared, void *workspace, hipStream_t stream) {
    const int64_t groups = batch * a.groups;
    auto by_waves = [&](auto waves) {
        constexpr int W = decltype(waves)::value;
        if (BACKWARD) recurrence_backward_kernel<T, W, MODE, false><<<(unsigned)groups, 64 * W, 0, stream>>>(a);
        else recurrence_kernel<T, W, MODE, false><<<(unsigned)groups, 64 * W, 0, stream>>>(a);
    };
    if (shared) {
        const int64_t states = batch * a.width, n = states * a.tiles;
        a.tickets = (uint32_t *)workspace, a.maps = (uint64_t *)(a.tickets + groups * TICKET);
        float *copy = (float *)(a.maps + n);
        untold_kernel<<<(unsigned)ceil_div(n, 256), 256, 0, stream>>>(a.maps, n, a.tickets, BACKWARD ? a.dlast : a.state, copy, states, groups);
        a.state = a.dlast = copy;
        const unsigned all = (unsigned)(groups * a.tiles);
        if (BACKWARD) recurrence_backward_kernel<T, WAVES, MODE, true><<<all, 64 * WAVES, 0, stream>>>(a);
        else recurrence_kernel<T, WAVES, MODE, true><<<all, 64 * WAVES, 0, stream>>>(a);
    } else if (a.steps == 1 && !BACKWARD) {
        const int64_t pairs = ceil_div(a.width, N), all = batch * pairs;
        recurrence_step_kernel<T, MODE><<<(unsigned)ceil_div(all, 256), 256, 0, stream>>>(a, (uint32_t)pairs, (uint32_t)all);
    } else {
        // waves that no step would fill take time all the same: 256 x 32 x 1024 bf16 11.3 us with one, 18 with three, 40 with eight; 128 x 128 x 1024
        // 19.1 with four, 26.1 with eight; 64 x 192 x 1024 18.2 with six, 17.8 with eight
        const int64_t waves = ceil_div(a.steps, WAVE_STEPS);
        if (waves <= 1) by_waves(std::integral_constant<int, 1>());
        else if (waves <= 2) by_waves(std::integral_constant<int, 2>());
        else if (waves <= 3) by_waves(std::integral_constant<int, 3>());
        else if (waves <= 4) by_waves(std::integral_constant<int, 4>());
        else by_waves(std::integral_constant<int, WAVES>());
    }
}

int call(const dear_recurrence_t *r, bool backward, hipStream_t stream) {
    if (int rc = check_call(r, backward)) return rc;
    if (r->batch == 0) return DEAR_OK;
    if (r->steps == 0) {
        const float *from = backward ? r->dlast : r->state;
        float *to = backward ? r->dstate : r->last;
        const int64_t n = (int64_t)r->batch * r->width;
        if (!to || to == from) return DEAR_OK;
        if (n > MAX_THREADS) return DEAR_ETOOBIG;
        copy_state_kernel<<<(unsigned)ceil_div(n, 256), 256, 0, stream>>>(from, to, n);
        return launch_status();
    }
    auto rows = [](const dear_steps_t &t) { return rows_t{t.data, t.batch_stride, t.step_stride}; };
    params a = {};
    a.x = rows(r->x), a.gate = rows(r->gate), a.h = rows(r->h), a.dh = rows(r->dh), a.dx = rows(r->dx), a.dgate = rows(r->dgate);
    a.state = r->state, a.dlast = r->dlast, a.last = r->last, a.dstate = r->dstate, a.kept = r->kept, a.lens = r->lens;
    a.steps = r->steps, a.width = r->width;
    a.groups = (int32_t)groups_of(*r), a.tiles = (int32_t)ceil_div(r->steps, KEPT);
    bool vec = r->width % N == 0 && vectors(*r, r->x) && vectors(*r, r->gate);
    vec = vec && (backward ? vectors(*r, r->dh) && vectors(*r, r->dx) && vectors(*r, r->dgate) : vectors(*r, r->h));
    vec = vec && aligned(r->state, 8) && aligned(r->last, 8) && aligned(r->kept, 8) && aligned(r->dlast, 8) && aligned(r->dstate, 8);
    auto by_mode = [&](auto t, auto mode) {
        typedef decltype(t) T;
        if (backward) launch<T, decltype(mode)::value, true>(a, r->batch, shares(*r), r->workspace, stream);
        else launch<T, decltype(mode)::value, false>(a, r->batch, shares(*r), r->workspace, stream);
    };
    // Of an odd width the last channel but one is taken twice, by two workgroups or, of one step, perhaps two waves, with the same results.  Where
    // the state before is overwritten with the one behind, the second could find the latter: there each channel is taken by one lane.
    const bool over_itself = backward ? r->dstate && r->dstate == r->dlast : r->last && r->last == r->state;
    const bool apart = over_itself && r->width % N && (r->width > CG || r->steps == 1) && !shares(*r);
    auto by_type = [&](auto t) {
        if (vec) by_mode(t, std::integral_constant<int, ALIGNED>());
        else if (r->width >= N && !apart) by_mode(t, std::integral_constant<int, ANYWHERE>());
        else by_mode(t, std::integral_constant<int, SINGLE>());
    };
    if (r->dtype == DEAR_BF16) by_type(bf16());
    else by_type(float());
    return launch_status();
}

}  // namespace

extern "C" {

int dear_recurrence(const dear_recurrence_t *args, void *hip_stream) { return call(args, false, (hipStream_t)hip_stream); }

int dear_recurrence_backward(const dear_recurrence_t *args, void *hip_stream) { return call(args, true, (hipStream_t)hip_stream); }

int dear_recurrence_workspace(const dear_recurrence_t *args, int64_t *bytes) {
    if (!bytes) return DEAR_EINVAL;
    if (int rc = check(args)) return rc;
    if (too_many(*args)) return DEAR_ETOOBIG;
    *bytes = workspace_of(*args);
    return DEAR_OK;
}

}  // extern "C"
