// The norm over all gradients of a model, and the gradients scaled down to a largest norm (definitions: dear_ops.h).
//
//     norm = sqrt(sum of g^2 over all tensors);  out = g * min(1, max_norm / norm)
//
// HBM bounds it: one read for the sum, then one read and one write for what is scaled (334 M fp32 gradients: 198 us, with some of it in the last
// cache, and 464 = 5.8 TB/s; in bf16, into fp32, 497 for both).  The tensors are taken as one sequence of elements in pieces of 8192, of which workgroups
// take every 2048th: neither many small tensors nor a few large ones leave the chip unevenly loaded, and at any time the chip is in one
// stretch of memory (a span of its own for each workgroup: 745 us instead of 697).  Sums are in 64 bits: no square overflows or vanishes,
// and the sum of any number of them rounds far below the result's 32 bits.  The parts are added in an order that does not change, by
// every workgroup of the second launch for itself: that costs each a read of 16 KB from the cache, and saves a launch.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "ops_common.h"

#pragma clang fp contract(fast)

namespace {

using namespace dear_ops;

constexpr int THREADS = 256;
constexpr int MOST = 120;        // tensors whose places are arguments of a launch, 4 KB at most
constexpr int64_t PARTS = 2048;  // workgroups, and parts of the sum
constexpr int64_t PIECE = 8192;  // elements that a workgroup takes at a time
constexpr int64_t MAX_TENSORS = 1 << 20;
constexpr int64_t MAX_ELEMENTS = (int64_t)1 << 56;

struct entry {
    const void *in;
    void *out;
    int64_t end;     // elements up to and with this tensor's
    int32_t bf16s;   // 1: in is bf16, 2: out is
    int32_t reserved;
};
struct table {
    entry e[MOST];
    int32_t count;
};
static_assert(sizeof(table) <= 4000, "with the other arguments 4 KB");

// Longer lists go to the workspace first, MOST at a time, so that one launch has all of them: several launches for a pass leave the chip
// half empty at each one's end (334 M elements in 390 tensors 817 us, so 775).
__global__ __launch_bounds__(128) void table_kernel(const table t, entry *to) {
    const int i = threadIdx.x;
    if (i < t.count) to[i] = t.e[i];
}

template <typename T, int N> struct vec_of { typedef T type __attribute__((ext_vector_type(N), aligned(sizeof(T)))); };
template <typename T, int N> using vec = typename vec_of<T, N>::type;  // from any element on, which global memory takes

// Calls f(tensor, first element, elements) for what this workgroup has of the tensors: of all elements every gridDim-th piece.
template <bool HERE, typename F> __device__ __forceinline__ void each(const table &t, const entry *far, F f) {
    auto at_ = [&](int i) -> const entry & { return HERE ? t.e[i] : far[i]; };
    const int64_t total = at_(t.count - 1).end;
    int i = 0;
    for (int64_t piece = blockIdx.x; piece * PIECE < total; piece += gridDim.x) {
        int64_t at = piece * PIECE;
        const int64_t behind = min(at + PIECE, total);
        // the first tensor that ends behind `at`: near the one before, mostly
        int lo = i, hi = i, step = 1;
        while (at_(hi).end <= at) lo = hi + 1, hi = min(hi + step, t.count - 1), step *= 2;
        while (lo < hi) {
            const int mid = (lo + hi) / 2;
            if (at_(mid).end > at) hi = mid;
            else lo = mid + 1;
        }
        for (i = lo;; ++i) {
            const entry e = at_(i);
            const int64_t begin = i ? at_(i - 1).end : 0, n = min(e.end, behind) - at;
            f(e, at - begin, n);
            at += n;
            if (at >= behind) break;
        }
    }
}

__device__ __forceinline__ double square(float x) { return (double)x * (double)x; }

// Of four fp32 values in 64 bits.
__device__ __forceinline__ void add_squares(double &s, vec<float, 4> v) {
#pragma unroll
    for (int k = 0; k < 4; ++k) s = __builtin_fma((double)v[k], (double)v[k], s);
}
// Of eight bf16 values: their squares are exact in fp32, and are added there, as 64 bits would take longer than memory (seven roundings, less
// than 2^-21 of the group's sum), unless fp32 does not hold what there is, or does not hold all of it.
__device__ __forceinline__ void add_squares(double &s, vec<bf16, 8> v) {
    float t = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) t = __builtin_fmaf((float)v[k], (float)v[k], t);
    if (t >= 0x1p-60f && t < __builtin_inff()) {
        s += (double)t;
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) s = __builtin_fma((double)(float)v[k], (double)(float)v[k], s);
    }
}

// Read past the caches: of a model's gradients nothing is left of them when they are scaled (334 M fp32 251 us, so 222).
template <typename T> __device__ __forceinline__ double squares(const T *p, int64_t n) {
    constexpr int V = 16 / sizeof(T), U = 4;  // values of a vector, vectors in flight
    constexpr int64_t STEP = THREADS * V;
    double s = 0.;
    int64_t i = (int64_t)threadIdx.x * V;
    for (; i + (U - 1) * STEP + V <= n; i += U * STEP) {
        vec<T, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = __builtin_nontemporal_load((const vec<T, V> *)(p + i + u * STEP));
#pragma unroll
        for (int u = 0; u < U; ++u) add_squares(s, v[u]);
    }
    for (; i + V <= n; i += STEP) add_squares(s, *(const vec<T, V> *)(p + i));
    if (i < n)
        for (int k = 0; k < V - 1 && i + k < n; ++k) s += square((float)p[i + k]);
    return s;
}

__device__ __forceinline__ double block_sum(double s) {
    __shared__ double lds[THREADS];
    lds[threadIdx.x] = s;
#pragma unroll
    for (int n = THREADS / 2; n > 0; n /= 2) {
        __syncthreads();
        if ((int)threadIdx.x < n) lds[threadIdx.x] += lds[threadIdx.x + n];
    }
    __syncthreads();
    return lds[0];
}

template <bool HERE> __global__ __launch_bounds__(THREADS) void squares_kernel(const table t, const entry *far, double *parts) {
    double s = 0.;
    each<HERE>(t, far, [&](const entry &e, int64_t first, int64_t n) {
        s += e.bf16s & 1 ? squares((const bf16 *)e.in + first, n) : squares((const float *)e.in + first, n);
    });
    s = block_sum(s);
    if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

// The norm from the parts of the sum, the same in all threads.
__device__ __forceinline__ double norm_of(const double *parts, int n) {
    double s = 0.;
    for (int i = threadIdx.x; i < n; i += THREADS) s += parts[i];
    return sqrt(block_sum(s));
}

__global__ __launch_bounds__(THREADS) void norm_kernel(const double *parts, int n, float *norm) {
    const double whole = norm_of(parts, n);
    if (threadIdx.x == 0) *norm = (float)whole;
}

// One rounding: of the product, or to bf16.  Vectors of 16 bytes of the wider type, so that neighbouring lanes write without gaps, and past the
// caches (334 M bf16 into fp32 540 us, so 497).
template <typename T, typename O> __device__ __forceinline__ void scale(const T *p, O *o, int64_t n, float by) {
    constexpr int V = sizeof(T) + sizeof(O) == 4 ? 8 : 4, U = 4;
    constexpr int64_t STEP = THREADS * V;
    auto write = [&](int64_t i, vec<T, V> v) {
        vec<O, V> w;
#pragma unroll
        for (int k = 0; k < V; ++k) w[k] = (O)((float)v[k] * by);
        __builtin_nontemporal_store(w, (vec<O, V> *)(o + i));
    };
    int64_t i = (int64_t)threadIdx.x * V;
    for (; i + (U - 1) * STEP + V <= n; i += U * STEP) {
        vec<T, V> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = __builtin_nontemporal_load((const vec<T, V> *)(p + i + u * STEP));
#pragma unroll
        for (int u = 0; u < U; ++u) write(i + u * STEP, v[u]);
    }
    for (; i + V <= n; i += STEP) write(i, *(const vec<T, V> *)(p + i));
    if (i < n)
        for (int k = 0; k < V - 1 && i + k < n; ++k) o[i + k] = (O)((float)p[i + k] * by);
}
// By a factor that fp32 does not hold in full: gradients near the largest number, scaled to a norm of 1, which is too rare to be fast.
template <typename T, typename O> __device__ __forceinline__ void scale(const T *p, O *o, int64_t n, double by) {
#pragma unroll 1
    for (int64_t i = threadIdx.x; i < n; i += THREADS) o[i] = (O)(float)((double)(float)p[i] * by);
}

template <bool HERE>
__global__ __launch_bounds__(THREADS) void scale_kernel(const table t, const entry *far, const double *parts, int n, float max_norm, float *norm) {
    const double whole = norm_of(parts, n);
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)whole;
    const bool clip = !(whole <= (double)max_norm);  // (a NaN clips, so that it shows in every gradient)
    const double by = clip ? (double)max_norm / whole : 1.;
    auto scale_all = [&](auto by) {
        each<HERE>(t, far, [&](const entry &e, int64_t first, int64_t count) {
            if (!clip && e.in == e.out) return;  // is what it is to be
            if (e.bf16s == 0) scale((const float *)e.in + first, (float *)e.out + first, count, by);
            else if (e.bf16s == 1) scale((const bf16 *)e.in + first, (float *)e.out + first, count, by);
            else if (e.bf16s == 2) scale((const float *)e.in + first, (bf16 *)e.out + first, count, by);
            else scale((const bf16 *)e.in + first, (bf16 *)e.out + first, count, by);
        });
    };
    if (by > 0. && by < 0x1p-126) scale_all(by);  // (0 is that of an infinite norm, as steps that overflow have)
    else scale_all((float)by);
}

// ------------------------------------------------------------------------------------ host
int size_of(int32_t dtype) { return dtype == DEAR_BF16 ? 2 : 4; }
bool known(int32_t dtype) { return dtype == DEAR_BF16 || dtype == DEAR_F32; }

int check(const dear_grad_t *g, int64_t count, bool clip, int64_t *total) {
    if (count < 0 || count > MAX_TENSORS || (count && !g)) return DEAR_EINVAL;
    *total = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (g[i].elements < 0 || g[i].elements > MAX_ELEMENTS || !known(g[i].dtype) || (clip && !known(g[i].out_dtype))) return DEAR_EINVAL;
        if (g[i].elements == 0) continue;
        if (!g[i].data || (clip && !g[i].out)) return DEAR_EINVAL;
        if (!aligned(g[i].data, size_of(g[i].dtype)) || (clip && !aligned(g[i].out, size_of(g[i].out_dtype)))) return DEAR_EALIGN;
        if (*total > MAX_ELEMENTS - g[i].elements) return DEAR_EINVAL;
        *total += g[i].elements;
    }
    return DEAR_OK;
}

// Whether each output has its place to itself, but for its own input: the same address and type.
int check_places(const dear_grad_t *g, int64_t count) {
    struct place {
        uintptr_t begin, end;
        int64_t i;
    };
    try {
        std::vector<place> outs;
        outs.reserve(count);
        for (int64_t i = 0; i < count; ++i)
            if (g[i].elements) outs.push_back({(uintptr_t)g[i].out, (uintptr_t)g[i].out + g[i].elements * size_of(g[i].out_dtype), i});
        std::sort(outs.begin(), outs.end(), [](const place &a, const place &b) { return a.begin < b.begin; });
        for (size_t k = 1; k < outs.size(); ++k)
            if (outs[k].begin < outs[k - 1].end) return DEAR_EINVAL;
        for (int64_t i = 0; i < count; ++i) {
            if (!g[i].elements) continue;
            const uintptr_t begin = (uintptr_t)g[i].data, end = begin + g[i].elements * size_of(g[i].dtype);
            auto k = std::upper_bound(outs.begin(), outs.end(), begin, [](uintptr_t b, const place &p) { return b < p.end; });
            for (; k != outs.end() && k->begin < end; ++k)
                if (k->i != i || k->begin != begin || g[i].dtype != g[i].out_dtype) return DEAR_EINVAL;
        }
    } catch (const std::bad_alloc &) {
        return DEAR_ENOMEM;
    }
    return DEAR_OK;
}

int64_t workspace_of(int64_t count) { return (PARTS) * (int64_t)sizeof(double) + (count > MOST ? count * (int64_t)sizeof(entry) : 0); }

int norm_and_clip(const dear_grad_t *g, int64_t count, bool clip, float max_norm, float *norm, void *workspace, int64_t bytes, hipStream_t s) {
    int64_t total = 0;
    if (int rc = check(g, count, clip, &total)) return rc;
    if (!norm || !workspace || (clip && !(max_norm > 0.f))) return DEAR_EINVAL;
    if (!aligned(norm, 4) || !aligned(workspace, 256)) return DEAR_EALIGN;
    if (bytes < workspace_of(count)) return DEAR_ETOOBIG;
    if (clip)
        if (int rc = check_places(g, count)) return rc;
    double *parts = (double *)workspace;
    entry *far = (entry *)(parts + PARTS);
    if (total == 0) {
        norm_kernel<<<1, THREADS, 0, s>>>(parts, 0, norm);
        return launch_status();
    }
    table t;
    const bool here = count <= MOST;
    int64_t end = 0, in = 0;  // entries in the workspace
    int n = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (!g[i].elements) continue;
        end += g[i].elements;
        t.e[n++] = entry{g[i].data, g[i].out, end, (g[i].dtype == DEAR_BF16 ? 1 : 0) | (clip && g[i].out_dtype == DEAR_BF16 ? 2 : 0), 0};
        if (n == MOST && !here) {
            t.count = n;
            table_kernel<<<1, 128, 0, s>>>(t, far + in);
            in += n, n = 0;
        }
    }
    t.count = n;
    if (!here) {
        if (n) table_kernel<<<1, 128, 0, s>>>(t, far + in);
        t.count = (int32_t)(in + n);
    }
    const int64_t pieces = ceil_div(end, PIECE);
    const unsigned groups = (unsigned)(pieces < PARTS ? pieces : PARTS);
    if (here) squares_kernel<true><<<groups, THREADS, 0, s>>>(t, nullptr, parts);
    else squares_kernel<false><<<groups, THREADS, 0, s>>>(t, far, parts);
    if (int rc = launch_status()) return rc;
    if (!clip) norm_kernel<<<1, THREADS, 0, s>>>(parts, (int)groups, norm);
    else if (here) scale_kernel<true><<<groups, THREADS, 0, s>>>(t, nullptr, parts, (int)groups, max_norm, norm);
    else scale_kernel<false><<<groups, THREADS, 0, s>>>(t, far, parts, (int)groups, max_norm, norm);
    return launch_status();
}

}  // namespace

extern "C" {

int dear_grad_norm_workspace(int64_t count, int64_t *bytes) {
    if (!bytes || count < 0 || count > MAX_TENSORS) return DEAR_EINVAL;
    *bytes = workspace_of(count);
    return DEAR_OK;
}

int dear_grad_norm(const dear_grad_t *grads, int64_t count, float *norm, void *workspace, int64_t workspace_bytes, void *hip_stream) {
    return norm_and_clip(grads, count, false, 0.f, norm, workspace, workspace_bytes, (hipStream_t)hip_stream);
}

int dear_clip_grads(const dear_grad_t *grads, int64_t count, float max_norm, float *norm, void *workspace, int64_t workspace_bytes,
                    void *hip_stream) {
    return norm_and_clip(grads, count, true, max_norm, norm, workspace, workspace_bytes, (hipStream_t)hip_stream);
}

}  // extern "C"
