// The norm of all gradients together, and clipping by it.
//   norm = sqrt of the sum of the squares of all elements of all tensors;  out = grad * (max_norm / norm) if norm is finite and above max_norm, else grad
#include <float.h>
#include <stdlib.h>

#include "row_ops.h"

namespace sol {
namespace {

// The tensors of one launch, by value: no copy to the device, nothing to keep alive, and a captured graph holds them.  A tensor is cut into chunks, so that a workgroup's share is even.
constexpr int TABLE = 112, CHUNK = 8192, MAX_GROUPS = 1024;
struct GradTable {
    const void *grad[TABLE];
    void *out[TABLE];
    uint64_t count[TABLE];
    uint32_t first[TABLE + 1];      // chunks in front of each tensor
    uint32_t bf16[(TABLE + 31) / 32];
    int n;
};

struct Chunk {
    int tensor;
    uint64_t at;                    // its first element
    int len;
};
__device__ __forceinline__ Chunk find_chunk(const GradTable &t, uint32_t i) {
    int lo = 0, hi = t.n;           // first[lo] <= i < first[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= i) lo = mid;
        else hi = mid;
    }
    const uint64_t at = (uint64_t)(i - t.first[lo]) * CHUNK, left = t.count[lo] - at;
    return {lo, at, (int)(left < CHUNK ? left : CHUNK)};
}
__device__ __forceinline__ bool is_bf16(const GradTable &t, int k) { return t.bf16[k >> 5] >> (k & 31) & 1; }

__device__ __forceinline__ double block_sum(double v, double *red) {        // 256 threads; in all of them
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
}

template <typename T> __device__ __forceinline__ double squares(const T *g, int len) {
    double s = 0.0;
    for (int i = threadIdx.x * 8; i < len; i += 2048) {
        float v[8];
        load8_any<T>(g + i, v, len - i);
#pragma unroll
        for (int e = 0; e < 8; e++) s += (double)v[e] * (double)v[e];
    }
    return s;
}

// Workgroup b takes the chunks b, b + grid, ... and writes the sum of their squares to part[b]
__global__ void __launch_bounds__(256) grad_squares_kernel(const GradTable t, double *part) {
    __shared__ double red[4];
    double s = 0.0;
    for (uint32_t i = blockIdx.x; i < t.first[t.n]; i += gridDim.x) {
        const Chunk c = find_chunk(t, i);
        if (is_bf16(t, c.tensor)) s += squares<bf16_t>(static_cast<const bf16_t *>(t.grad[c.tensor]) + c.at, c.len);
        else s += squares<float>(static_cast<const float *>(t.grad[c.tensor]) + c.at, c.len);
    }
    s = block_sum(s, red);
    if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__device__ __forceinline__ double sum_of_parts(const double *part, int parts, double *red) {
    double s = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) s += part[i];
    return block_sum(s, red);
}

__global__ void __launch_bounds__(256) grad_norm_kernel(const double *part, int parts, float *norm) {
    __shared__ double red[4];
    const double s = sum_of_parts(part, parts, red);
    if (threadIdx.x == 0) *norm = (float)sqrt(s);
}

template <typename T> __device__ __forceinline__ void scaled(const T *g, T *out, int len, float f) {
    for (int i = threadIdx.x * 8; i < len; i += 2048) {
        float v[8];
        load8_any<T>(g + i, v, len - i);
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] *= f;
        store8_any<T>(out + i, v, len - i);
    }
}

// The norm comes in 32 bits from grad_norm_kernel in front.  Where nothing is clipped the elements are copied as they are, or left where they are in place.
__global__ void __launch_bounds__(256) grad_scale_kernel(const GradTable t, const float *norm, float max_norm) {
    const float n = *norm;
    const bool clip = n > max_norm && n <= FLT_MAX;
    const float f = clip ? max_norm / n : 1.f;
    for (uint32_t i = blockIdx.x; i < t.first[t.n]; i += gridDim.x) {
        const Chunk c = find_chunk(t, i);
        if (!clip && t.grad[c.tensor] == t.out[c.tensor]) continue;
        if (is_bf16(t, c.tensor)) scaled<bf16_t>(static_cast<const bf16_t *>(t.grad[c.tensor]) + c.at, static_cast<bf16_t *>(t.out[c.tensor]) + c.at, c.len, f);
        else scaled<float>(static_cast<const float *>(t.grad[c.tensor]) + c.at, static_cast<float *>(t.out[c.tensor]) + c.at, c.len, f);
    }
}

uint64_t chunks_of(const sol_grad &g) { return (g.count + CHUNK - 1) / CHUNK; }

// Calls f(table, first part) for each launch's share of the tensors
template <typename F> sol_status each_table(const sol_grad *grads, int tensors, F f) {
    GradTable t;
    int part = 0;
    t.n = 0;
    t.first[0] = 0;
    memset(t.bf16, 0, sizeof(t.bf16));
    auto flush = [&]() -> sol_status {
        if (t.n == 0) return SOL_OK;
        const int groups = (int)min(t.first[t.n], (uint32_t)MAX_GROUPS);
        SOL_TRY(f(t, groups, part));
        part += groups;
        t.n = 0;
        memset(t.bf16, 0, sizeof(t.bf16));
        return SOL_OK;
    };
    for (int i = 0; i < tensors; i++) {
        const sol_grad &g = grads[i];
        if (g.count == 0) continue;
        if (t.n == TABLE || (t.n && t.first[t.n] + chunks_of(g) > 0x7fffffffu)) SOL_TRY(flush());
        t.grad[t.n] = g.grad; t.out[t.n] = g.out; t.count[t.n] = g.count;
        t.bf16[t.n >> 5] |= (g.dtype == SOL_BF16 ? 1u : 0u) << (t.n & 31);
        t.first[t.n + 1] = t.first[t.n] + (uint32_t)chunks_of(g);
        t.n++;
    }
    return flush();
}

int total_parts(const sol_grad *grads, int tensors) {
    int parts = 0;
    each_table(grads, tensors, [&](const GradTable &, int groups, int) { parts += groups; return SOL_OK; });
    return parts;
}

struct Span { uintptr_t at, end; int i; };
int by_start(const void *p, const void *q) {
    const Span *a = static_cast<const Span *>(p), *b = static_cast<const Span *>(q);
    return a->at < b->at ? -1 : a->at > b->at ? 1 : a->i - b->i;
}

sol_status check_grads(const sol_grad *grads, int tensors, bool out) {
    SOL_REQUIRE(tensors >= 0, SOL_ERR_SHAPE, "%d tensors", tensors);
    SOL_REQUIRE(grads || tensors == 0, SOL_ERR_NULL, "the list of gradients is NULL");
    for (int i = 0; i < tensors; i++) {
        const sol_grad &g = grads[i];
        SOL_REQUIRE(g.dtype == SOL_F32 || g.dtype == SOL_BF16, SOL_ERR_DTYPE, "gradient %d: unknown dtype %d", i, g.dtype);
        if (g.count == 0) continue;
        SOL_REQUIRE(g.count < (1ull << 40), SOL_ERR_UNSUPPORTED, "gradient %d: 2^40 elements or more", i);
        SOL_REQUIRE(g.grad && (g.out || !out), SOL_ERR_NULL, "gradient %d: a pointer is NULL", i);
        const uintptr_t mask = dtype_size(g.dtype) - 1;
        SOL_REQUIRE(!(reinterpret_cast<uintptr_t>(g.grad) & mask) && (!out || !(reinterpret_cast<uintptr_t>(g.out) & mask)), SOL_ERR_ALIGN, "gradient %d is not aligned to its elements", i);
    }
    if (!out || tensors == 0) return SOL_OK;
    // No two of the buffers may share memory: a tensor listed twice would be scaled twice, an output on another gradient would change it before it is read.
    Span few[256], *spans = 2 * (size_t)tensors <= 256 ? few : static_cast<Span *>(malloc(2 * (size_t)tensors * sizeof(Span)));
    SOL_REQUIRE(spans, SOL_ERR_UNSUPPORTED, "no memory for a list of %d gradients", tensors);
    int n = 0;
    for (int i = 0; i < tensors; i++) {
        const sol_grad &g = grads[i];
        const uintptr_t bytes = g.count * dtype_size(g.dtype), at = reinterpret_cast<uintptr_t>(g.grad), to = reinterpret_cast<uintptr_t>(g.out);
        if (bytes) spans[n++] = Span{at, at + bytes, i};
        if (bytes && at != to) spans[n++] = Span{to, to + bytes, i};
    }
    qsort(spans, (size_t)n, sizeof(Span), by_start);
    int a = -1, b = -1;
    for (int k = 1; k < n && a < 0; k++)
        if (spans[k].at < spans[k - 1].end) { a = spans[k - 1].i; b = spans[k].i; }
    if (spans != few) free(spans);
    SOL_REQUIRE(a < 0, SOL_ERR_UNSUPPORTED, "gradients %d and %d, or what is written for them, share memory", a, b);
    return SOL_OK;
}

sol_status launch_norm_of(const sol_grad *grads, int tensors, float *norm, void *workspace, hipStream_t st) {
    double *part = static_cast<double *>(workspace);
    int parts = 0;
    SOL_TRY(each_table(grads, tensors, [&](const GradTable &t, int groups, int first) -> sol_status {
        hipLaunchKernelGGL(grad_squares_kernel, dim3((unsigned)groups), dim3(256), 0, st, t, part + first);
        SOL_HIP(hipGetLastError());
        parts = first + groups;
        return SOL_OK;
    }));
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(256), 0, st, part, parts, norm);
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

sol_status check_norm_out(const float *norm) {
    SOL_REQUIRE(norm, SOL_ERR_NULL, "norm must not be NULL");
    SOL_REQUIRE((reinterpret_cast<uintptr_t>(norm) & 3u) == 0, SOL_ERR_ALIGN, "norm must be 4-byte aligned");
    return SOL_OK;
}

}  // namespace
}  // namespace sol

using namespace sol;

extern "C" {

size_t sol_grad_workspace_bytes(const sol_grad *grads, int tensors) {
    return check_grads(grads, tensors, false) == SOL_OK ? (size_t)total_parts(grads, tensors) * 8 : 0;
}

sol_status sol_grad_norm(const sol_grad *grads, int tensors, float *norm, void *workspace, size_t workspace_bytes, void *stream) {
    SOL_TRY(check_grads(grads, tensors, false));
    SOL_TRY(check_norm_out(norm));
    SOL_TRY(check_scratch(workspace, workspace_bytes, (size_t)total_parts(grads, tensors) * 8));
    return launch_norm_of(grads, tensors, norm, workspace, (hipStream_t)stream);
}

sol_status sol_grad_clip(const sol_grad *grads, int tensors, float max_norm, float *norm, void *workspace, size_t workspace_bytes, void *stream) {
    SOL_TRY(check_grads(grads, tensors, true));
    SOL_TRY(check_norm_out(norm));
    SOL_REQUIRE(max_norm > 0.f, SOL_ERR_SHAPE, "max_norm %g is not positive", (double)max_norm);       // refuses a NaN too
    SOL_TRY(check_scratch(workspace, workspace_bytes, (size_t)total_parts(grads, tensors) * 8));
    hipStream_t st = (hipStream_t)stream;
    SOL_TRY(launch_norm_of(grads, tensors, norm, workspace, st));
    return each_table(grads, tensors, [&](const GradTable &t, int groups, int) -> sol_status {
        hipLaunchKernelGGL(grad_scale_kernel, dim3((unsigned)groups), dim3(256), 0, st, t, norm, max_norm);
        SOL_HIP(hipGetLastError());
        return SOL_OK;
    });
}

}  // extern "C"
