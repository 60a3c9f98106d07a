// The norm over all gradients of a model, and the gradients scaled down to a largest norm (definitions: dear_ops.h).
//
//     norm = sqrt(sum of g^2 over all tensors);  out = g * min(1, max_norm / norm)
//
// HBM bounds it: one read for the sum, then one read and one write for what is scaled.  The tensors are taken as one
// sequence of elements that is cut into equal spans, one a workgroup, so that neither many small tensors nor a few large ones
// leave the chip unevenly loaded.  Squares are added in 64 bits: none overflows or vanishes, and the sum of any number of them
// rounds far below the result's 32 bits.  The parts are added in an order that does not change, by every workgroup of the second
// launch for itself: that costs each a read of some 16 KB from the cache, and saves a launch.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "ops_common.h"

#pragma clang fp contract(fast)

namespace {

using namespace dear_ops;

constexpr int THREADS = 256;
constexpr int MOST = 150;        // tensors of a launch: their places are its arguments, 4 KB at most
constexpr int64_t PARTS = 2048;  // spans that all elements are cut into, and one for each launch
constexpr int64_t LEAST = 2048;  // elements of a span
constexpr int64_t MAX_TENSORS = 1 << 20;
constexpr int64_t MAX_ELEMENTS = (int64_t)1 << 56;

struct table {
    const void *in[MOST];
    void *out[MOST];
    int64_t end[MOST];     // elements of the launch up to and with this tensor's
    uint8_t bf16s[MOST];   // 1: in is bf16, 2: out is
    int32_t count;
    int64_t span;
};
static_assert(sizeof(table) <= 4000, "with the other arguments 4 KB");

template <typename T> struct vec_of { typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T)))); };
template <typename T> using vec = typename vec_of<T>::type;  // 16 bytes from any element on, which global memory takes
template <typename T> constexpr int V = 16 / sizeof(T);

// Calls f(tensor, first element, elements) for each tensor that the workgroup's span reaches into.
template <typename F> __device__ __forceinline__ void each(const table &t, F f) {
    int64_t at = (int64_t)blockIdx.x * t.span;
    const int64_t behind = min(at + t.span, t.end[t.count - 1]);
    int lo = 0, hi = t.count - 1;  // the first tensor that ends behind `at`
    while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (t.end[mid] > at) hi = mid;
        else lo = mid + 1;
    }
    for (int i = lo; at < behind; ++i) {
        const int64_t begin = i ? t.end[i - 1] : 0, n = min(t.end[i], behind) - at;
        if (n > 0) f(i, at - begin, n);
        at += n;
    }
}

template <typename T> __device__ __forceinline__ double squares(const T *p, int64_t n) {
    double s = 0.;
    auto add = [&](vec<T> v) {
#pragma unroll
        for (int k = 0; k < V<T>; ++k) s = __builtin_fma((double)(float)v[k], (double)(float)v[k], s);
    };
    constexpr int U = 4;  // vectors in flight
    constexpr int64_t STEP = THREADS * V<T>;
    int64_t i = (int64_t)threadIdx.x * V<T>;
    for (; i + (U - 1) * STEP + V<T> <= n; i += U * STEP) {
        vec<T> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = *(const vec<T> *)(p + i + u * STEP);
#pragma unroll
        for (int u = 0; u < U; ++u) add(v[u]);
    }
    for (; i + V<T> <= n; i += STEP) add(*(const vec<T> *)(p + i));
    if (i < n)
        for (int k = 0; k < V<T> - 1 && i + k < n; ++k) s = __builtin_fma((double)(float)p[i + k], (double)(float)p[i + k], s);
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

__global__ __launch_bounds__(THREADS) void squares_kernel(const table t, double *parts) {
    double s = 0.;
    each(t, [&](int i, int64_t first, int64_t n) {
        s += t.bf16s[i] & 1 ? squares((const bf16 *)t.in[i] + first, n) : squares((const float *)t.in[i] + first, n);
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

// One rounding: of the product, or to bf16.
template <typename T, typename O> __device__ __forceinline__ void scale(const T *p, O *o, int64_t n, float by) {
    typedef O ovec __attribute__((ext_vector_type(V<T>), aligned(sizeof(O))));
    auto write = [&](int64_t i, vec<T> v) {
        ovec w;
#pragma unroll
        for (int k = 0; k < V<T>; ++k) w[k] = (O)((float)v[k] * by);
        *(ovec *)(o + i) = w;
    };
    constexpr int U = 4;
    constexpr int64_t STEP = THREADS * V<T>;
    int64_t i = (int64_t)threadIdx.x * V<T>;
    for (; i + (U - 1) * STEP + V<T> <= n; i += U * STEP) {
        vec<T> v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = *(const vec<T> *)(p + i + u * STEP);
#pragma unroll
        for (int u = 0; u < U; ++u) write(i + u * STEP, v[u]);
    }
    for (; i + V<T> <= n; i += STEP) write(i, *(const vec<T> *)(p + i));
    if (i < n)
        for (int k = 0; k < V<T> - 1 && i + k < n; ++k) o[i + k] = (O)((float)p[i + k] * by);
}

__global__ __launch_bounds__(THREADS) void scale_kernel(const table t, const double *parts, int n, float max_norm, float *norm) {
    const double whole = norm_of(parts, n);
    if (norm && blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)whole;
    const bool clip = !(whole <= (double)max_norm);  // (a NaN clips, so that it shows in every gradient)
    const float by = clip ? (float)((double)max_norm / whole) : 1.f;
    each(t, [&](int i, int64_t first, int64_t count) {
        const int types = t.bf16s[i];
        if (!clip && t.in[i] == t.out[i]) return;  // is what it is to be
        if (types == 0) scale((const float *)t.in[i] + first, (float *)t.out[i] + first, count, by);
        else if (types == 1) scale((const bf16 *)t.in[i] + first, (float *)t.out[i] + first, count, by);
        else if (types == 2) scale((const float *)t.in[i] + first, (bf16 *)t.out[i] + first, count, by);
        else scale((const bf16 *)t.in[i] + first, (bf16 *)t.out[i] + first, count, by);
    });
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

// Elements of a span.
int64_t span_of(int64_t total) {
    const int64_t n = ceil_div(ceil_div(total, PARTS), 1024) * 1024;
    return n < LEAST ? LEAST : n;
}
int64_t most_parts(int64_t count) { return PARTS + ceil_div(count, MOST); }

// Calls f(table, workgroups) for the launches of a list.
template <typename F> void launches(const dear_grad_t *g, int64_t count, int64_t total, F f) {
    table t;
    t.span = span_of(total);
    int64_t end = 0;
    t.count = 0;
    auto flush = [&] {
        if (t.count) f(t, (unsigned)ceil_div(end, t.span));
        t.count = 0, end = 0;
    };
    for (int64_t i = 0; i < count; ++i) {
        if (!g[i].elements) continue;
        end += g[i].elements;
        t.in[t.count] = g[i].data, t.out[t.count] = g[i].out, t.end[t.count] = end;
        t.bf16s[t.count] = (uint8_t)((g[i].dtype == DEAR_BF16 ? 1 : 0) | (g[i].out_dtype == DEAR_BF16 ? 2 : 0));
        if (++t.count == MOST) flush();
    }
    flush();
}

int norm_and_clip(const dear_grad_t *g, int64_t count, bool clip, float max_norm, float *norm, void *workspace, int64_t bytes, hipStream_t s) {
    int64_t total = 0;
    if (int rc = check(g, count, clip, &total)) return rc;
    if (!norm || !workspace || (clip && !(max_norm > 0.f))) return DEAR_EINVAL;
    if (!aligned(norm, 4) || !aligned(workspace, 256)) return DEAR_EALIGN;
    if (bytes < most_parts(count) * (int64_t)sizeof(double)) return DEAR_ETOOBIG;
    if (clip)
        if (int rc = check_places(g, count)) return rc;
    double *parts = (double *)workspace;
    int n = 0;
    launches(g, count, total, [&](const table &t, unsigned groups) {
        squares_kernel<<<groups, THREADS, 0, s>>>(t, parts + n);
        n += (int)groups;
    });
    if (int rc = launch_status()) return rc;
    if (!clip || total == 0) {
        norm_kernel<<<1, THREADS, 0, s>>>(parts, n, norm);
    } else {
        float *said = norm;
        launches(g, count, total, [&](const table &t, unsigned groups) {
            scale_kernel<<<groups, THREADS, 0, s>>>(t, parts, n, max_norm, said);
            said = nullptr;
        });
    }
    return launch_status();
}

}  // namespace

extern "C" {

int dear_grad_norm_workspace(int64_t count, int64_t *bytes) {
    if (!bytes || count < 0 || count > MAX_TENSORS) return DEAR_EINVAL;
    *bytes = most_parts(count) * (int64_t)sizeof(double);
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
