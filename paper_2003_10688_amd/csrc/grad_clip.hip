// The norm of all gradients together, and clipping by it.
//   norm = sqrt of the sum of the squares of all elements of all tensors;  out = grad * (max_norm / norm) if norm is finite and above max_norm, else grad
#include <float.h>
#include <stdlib.h>

#include <algorithm>

#include "row_ops.h"

namespace sol {
namespace {

// The tensors of one launch, by value: no copy to the device, nothing to keep alive, and a captured graph holds them.  A tensor is cut into chunks, so that a workgroup's share is even.
// 170 tensors fill the 4 KB of a kernel's arguments, so that a network of that many takes one launch and not two.
constexpr int TABLE = 170, CHUNK = 8192, MAX_GROUPS = 1024;
constexpr int MAX_TENSORS = 1 << 15, MAX_JOIN = 4096;
struct GradTable {
    const void *grad[TABLE];
    void *out[TABLE];
    uint32_t first[TABLE + 1];      // chunks in front of each tensor
    uint16_t last[TABLE];           // elements of its last chunk - 1
    uint32_t bf16[(TABLE + 31) / 32];
    int n;
};
static_assert(sizeof(GradTable) <= 4096 - 64, "kernel arguments");

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
    return {lo, (uint64_t)(i - t.first[lo]) * CHUNK, i + 1 == t.first[lo + 1] ? t.last[lo] + 1 : CHUNK};
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

// Both passes take a chunk in pieces of 16 bytes a thread, all of a chunk's under way at a time; the ends of tensors element by element.
template <typename T> constexpr int WIDTH = 16 / sizeof(T);
template <typename T> constexpr int PIECES = CHUNK / (256 * WIDTH<T>);      // of a thread
template <typename T> __device__ __forceinline__ void load_chunk(const T *g, RawPiece<T, WIDTH<T>> (&r)[PIECES<T>]) {
#pragma unroll
    for (int k = 0; k < PIECES<T>; k++) r[k].load(g + (k * 256 + threadIdx.x) * WIDTH<T>, WIDTH<T>);
}

// A product of two fp32 values is exact in 64 bits, and sums of them neither overflow nor lose small terms.  It costs nothing beside the memory: 2^28 bf16 elements 112 us (4.8 TB/s), 110 with fp32
// sums; 2^26 fp32 elements 44 us (6.1 TB/s) either way.
template <typename T> __device__ __forceinline__ double squares(const T *g, int len) {
    double s = 0.0;
    if (len == CHUNK) {
        RawPiece<T, WIDTH<T>> r[PIECES<T>];
        load_chunk<T>(g, r);
#pragma unroll
        for (int k = 0; k < PIECES<T>; k++)
#pragma unroll
            for (int e = 0; e < WIDTH<T>; e++) {
                const double v = r[k].get(e);
                s += v * v;
            }
    } else {
        for (int i = threadIdx.x * WIDTH<T>; i < len; i += 256 * WIDTH<T>) {
            RawPiece<T, WIDTH<T>> r;
            r.load(g + i, len - i);
#pragma unroll
            for (int e = 0; e < WIDTH<T>; e++) {
                const double v = r.get(e);
                s += v * v;
            }
        }
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

// max_norm / norm as the product of two factors.  Where fp32 holds the quotient with all its digits the second is 1, and so without effect; where the quotient lies below 2^-126 (an exploded norm of
// 1e38 and a max_norm of 1e-3, whose results fp32 holds all the same), the first is the power of two that brings the norm into 2 .. 4, which rounds nothing, and the second max_norm over that.
struct Factor { float first, then; };
__device__ __forceinline__ Factor clip_factor(float max_norm, float norm) {
    const float q = max_norm / norm;
    if (q >= FLT_MIN) return {q, 1.f};
    int k;
    frexpf(norm, &k);
    const float first = ldexpf(1.f, 2 - k);
    return {first, max_norm / (norm * first)};
}

template <bool STREAM, typename T> __device__ __forceinline__ void scaled(const T *g, T *out, int len, Factor f) {
    if (len == CHUNK) {
        RawPiece<T, WIDTH<T>> r[PIECES<T>];
        load_chunk<T>(g, r);
#pragma unroll
        for (int k = 0; k < PIECES<T>; k++) {
            float v[WIDTH<T>];
#pragma unroll
            for (int e = 0; e < WIDTH<T>; e++) v[e] = r[k].get(e) * f.first * f.then;
            if constexpr (STREAM) stream_piece<T, WIDTH<T>>(out + (k * 256 + threadIdx.x) * WIDTH<T>, v);
            else store_piece<T, WIDTH<T>>(out + (k * 256 + threadIdx.x) * WIDTH<T>, v, WIDTH<T>);
        }
    } else {
        for (int i = threadIdx.x * WIDTH<T>; i < len; i += 256 * WIDTH<T>) {
            RawPiece<T, WIDTH<T>> r;
            r.load(g + i, len - i);
            float v[WIDTH<T>];
#pragma unroll
            for (int e = 0; e < WIDTH<T>; e++) v[e] = r.get(e) * f.first * f.then;
            store_piece<T, WIDTH<T>>(out + i, v, len - i);
        }
    }
}

// Every workgroup joins the parts itself, which takes a launch less, and the first leaves the norm (each launch's first, the same one); parts = 0: the norm is there.  Where nothing is clipped the elements are copied as they are, or left where they are in place.
// The chunks are taken from the last on: what the pass in front read last is still in the caches, and stays there where the results are written past them (STREAM): 2^28 bf16 elements
// 300 us, both passes together, 333 with ordinary stores; 2^26 fp32 elements 123 and 147.  The 102 MB of a ResNet-50-shaped network's gradients 57 us.
template <bool STREAM> __global__ void __launch_bounds__(256) grad_scale_kernel(const GradTable t, const double *part, int parts, float *norm, float max_norm) {
    __shared__ double red[4];
    const float n = parts ? (float)sqrt(sum_of_parts(part, parts, red)) : *norm;
    if (parts && blockIdx.x == 0 && threadIdx.x == 0) *norm = n;
    const bool clip = n > max_norm && n <= FLT_MAX;
    const Factor f = clip ? clip_factor(max_norm, n) : Factor{1.f, 1.f};
    for (uint32_t j = blockIdx.x; j < t.first[t.n]; j += gridDim.x) {
        const Chunk c = find_chunk(t, t.first[t.n] - 1 - j);
        if (!clip && t.grad[c.tensor] == t.out[c.tensor]) continue;
        if (is_bf16(t, c.tensor)) scaled<STREAM, bf16_t>(static_cast<const bf16_t *>(t.grad[c.tensor]) + c.at, static_cast<bf16_t *>(t.out[c.tensor]) + c.at, c.len, f);
        else scaled<STREAM, float>(static_cast<const float *>(t.grad[c.tensor]) + c.at, static_cast<float *>(t.out[c.tensor]) + c.at, c.len, f);
    }
}

uint64_t chunks_of(const sol_grad &g) { return (g.count + CHUNK - 1) / CHUNK; }

// How many tensors from `at` on fit one launch; *chunks: theirs (2^27 at most, from fewer than 2^40 elements)
int table_end(const sol_grad *grads, int tensors, int at, uint64_t *chunks) {
    int n = 0;
    *chunks = 0;
    for (; at < tensors; at++) {
        const uint64_t k = chunks_of(grads[at]);
        if (k == 0) continue;
        if (n == TABLE) break;
        *chunks += k;
        n++;
    }
    return at;
}
int groups_of(uint64_t chunks) { return (int)(chunks < MAX_GROUPS ? chunks : MAX_GROUPS); }

// The tensors from `at` to `end`
void fill_table(const sol_grad *grads, int at, int end, GradTable *t) {
    t->n = 0;
    t->first[0] = 0;
    memset(t->bf16, 0, sizeof(t->bf16));
    for (; at < end; at++) {
        const sol_grad &g = grads[at];
        if (g.count == 0) continue;
        const int i = t->n++;
        t->grad[i] = g.grad; t->out[i] = g.out;
        t->bf16[i >> 5] |= (g.dtype == SOL_BF16 ? 1u : 0u) << (i & 31);
        t->first[i + 1] = t->first[i] + (uint32_t)chunks_of(g);
        t->last[i] = (uint16_t)((g.count - 1) % CHUNK);
    }
}

int total_parts(const sol_grad *grads, int tensors) {
    int parts = 0;
    uint64_t chunks;
    for (int at = 0; at < tensors;) {
        at = table_end(grads, tensors, at, &chunks);
        parts += groups_of(chunks);
    }
    return parts;
}

struct Buffer { uintptr_t at, end; int i; };      // i = -1: the norm

// out: the results and the norm are looked at too
sol_status check_grads(const sol_grad *grads, int tensors, bool out, const float *norm = nullptr) {
    SOL_REQUIRE(tensors >= 0, SOL_ERR_SHAPE, "%d tensors", tensors);
    SOL_REQUIRE(grads || tensors == 0, SOL_ERR_NULL, "the list of gradients is NULL");
    SOL_REQUIRE(tensors <= MAX_TENSORS, SOL_ERR_UNSUPPORTED, "more than 2^15 tensors: %d", tensors);
    uint64_t total = 0;
    for (int i = 0; i < tensors; i++) {
        const sol_grad &g = grads[i];
        SOL_REQUIRE(g.dtype == SOL_F32 || g.dtype == SOL_BF16, SOL_ERR_DTYPE, "gradient %d: unknown dtype %d", i, g.dtype);
        if (g.count == 0) continue;
        SOL_REQUIRE(g.count < (1ull << 40) && (total += g.count) < (1ull << 40), SOL_ERR_UNSUPPORTED, "gradients up to %d: 2^40 elements or more", i);
        SOL_REQUIRE(g.grad && (g.out || !out), SOL_ERR_NULL, "gradient %d: a pointer is NULL", i);
        const uintptr_t mask = dtype_size(g.dtype) - 1;
        SOL_REQUIRE(!(reinterpret_cast<uintptr_t>(g.grad) & mask) && (!out || !(reinterpret_cast<uintptr_t>(g.out) & mask)), SOL_ERR_ALIGN, "gradient %d is not aligned to its elements", i);
    }
    if (!out || tensors == 0) return SOL_OK;
    // No two of the buffers may share memory: a tensor listed twice would be scaled twice, an output on another gradient would change it before it is read, and so would the norm.
    Buffer few[513], *spans = 2 * tensors <= 512 ? few : static_cast<Buffer *>(malloc((2 * (size_t)tensors + 1) * sizeof(Buffer)));
    SOL_REQUIRE(spans, SOL_ERR_UNSUPPORTED, "no memory for a list of %d gradients", tensors);
    int n = 0;
    if (norm) spans[n++] = Buffer{reinterpret_cast<uintptr_t>(norm), reinterpret_cast<uintptr_t>(norm + 1), -1};
    for (int i = 0; i < tensors; i++) {
        const sol_grad &g = grads[i];
        const uintptr_t bytes = g.count * dtype_size(g.dtype), at = reinterpret_cast<uintptr_t>(g.grad), to = reinterpret_cast<uintptr_t>(g.out);
        if (bytes) spans[n++] = Buffer{at, at + bytes, i};
        if (bytes && at != to) spans[n++] = Buffer{to, to + bytes, i};
    }
    std::sort(spans, spans + n, [](const Buffer &p, const Buffer &q) { return p.at < q.at; });       // in place, without memory of its own
    int a = 0, b = 0;
    bool shared = false;
    for (int k = 1; k < n && !shared; k++)
        if (spans[k].at < spans[k - 1].end) { a = spans[k - 1].i; b = spans[k].i; shared = true; }
    if (spans != few) free(spans);
    SOL_REQUIRE(!shared || (a >= 0 && b >= 0), SOL_ERR_UNSUPPORTED, "the norm and gradient %d, or what is written for it, share memory", max(a, b));
    SOL_REQUIRE(!shared, SOL_ERR_UNSUPPORTED, "gradients %d and %d, or what is written for them, share memory", a, b);
    return SOL_OK;
}

sol_status launch_squares(const sol_grad *grads, int tensors, double *part, hipStream_t st) {
    GradTable t;
    uint64_t chunks;
    for (int at = 0; at < tensors;) {
        const int end = table_end(grads, tensors, at, &chunks), groups = groups_of(chunks);
        fill_table(grads, at, end, &t);
        at = end;
        if (groups == 0) continue;
        hipLaunchKernelGGL(grad_squares_kernel, dim3((unsigned)groups), dim3(256), 0, st, t, part);
        SOL_HIP(hipGetLastError());
        part += groups;
    }
    return SOL_OK;
}

// The sums that a call writes into its scratch may lie on no gradient, on no result and not on the norm, which others of its workgroups read or write meanwhile.
sol_status check_parts(const sol_grad *grads, int tensors, bool out, const float *norm, const void *workspace, size_t bytes) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(workspace), end = at + bytes;
    auto meets = [&](const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) < end && at < reinterpret_cast<uintptr_t>(p) + n; };
    SOL_REQUIRE(bytes == 0 || !meets(norm, sizeof(*norm)), SOL_ERR_UNSUPPORTED, "the workspace and the norm share memory");
    for (int i = 0; i < tensors && bytes; i++) {
        const size_t n = grads[i].count * dtype_size(grads[i].dtype);
        SOL_REQUIRE(n == 0 || (!meets(grads[i].grad, n) && (!out || !meets(grads[i].out, n))), SOL_ERR_UNSUPPORTED, "the workspace and gradient %d, or what is written for it, share memory", i);
    }
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
    const int parts = total_parts(grads, tensors);
    SOL_TRY(check_scratch(workspace, workspace_bytes, (size_t)parts * 8));
    SOL_TRY(check_parts(grads, tensors, false, norm, workspace, (size_t)parts * 8));
    hipStream_t st = (hipStream_t)stream;
    SOL_TRY(launch_squares(grads, tensors, static_cast<double *>(workspace), st));
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(256), 0, st, static_cast<const double *>(workspace), parts, norm);
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

sol_status sol_grad_clip(const sol_grad *grads, int tensors, float max_norm, float *norm, void *workspace, size_t workspace_bytes, void *stream) {
    SOL_TRY(check_norm_out(norm));
    SOL_TRY(check_grads(grads, tensors, true, norm));
    SOL_REQUIRE(max_norm > 0.f, SOL_ERR_SHAPE, "max_norm %g is not positive", (double)max_norm);       // refuses a NaN too
    const int parts = total_parts(grads, tensors);
    SOL_TRY(check_scratch(workspace, workspace_bytes, (size_t)parts * 8));
    SOL_TRY(check_parts(grads, tensors, true, norm, workspace, (size_t)parts * 8));
    hipStream_t st = (hipStream_t)stream;
    double *part = static_cast<double *>(workspace);
    SOL_TRY(launch_squares(grads, tensors, part, st));
    const bool join = parts > MAX_JOIN || parts == 0;
    if (join) {
        hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(256), 0, st, part, parts, norm);
        SOL_HIP(hipGetLastError());
    }
    // from the last tensors to the first: what the first pass read last is still in the caches
    int starts[MAX_TENSORS / TABLE + 2], tables = 0;
    uint64_t chunks;
    for (int at = 0; at < tensors; at = table_end(grads, tensors, at, &chunks)) starts[tables++] = at;
    starts[tables] = tensors;
    size_t bytes = 0;
    for (int i = 0; i < tensors; i++) bytes += grads[i].count * dtype_size(grads[i].dtype);
    const bool stream_out = bytes >= STREAM_BYTES;
    GradTable t;
    for (int k = tables - 1; k >= 0; k--) {
        const int groups = groups_of((table_end(grads, starts[k + 1], starts[k], &chunks), chunks));
        if (groups == 0) continue;
        fill_table(grads, starts[k], starts[k + 1], &t);
        if (stream_out) hipLaunchKernelGGL(grad_scale_kernel<true>, dim3((unsigned)groups), dim3(256), 0, st, t, part, join ? 0 : parts, norm, max_norm);
        else hipLaunchKernelGGL(grad_scale_kernel<false>, dim3((unsigned)groups), dim3(256), 0, st, t, part, join ? 0 : parts, norm, max_norm);
        SOL_HIP(hipGetLastError());
    }
    return SOL_OK;
}

}  // extern "C"
