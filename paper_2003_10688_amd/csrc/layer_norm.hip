// Layer norm and its backward pass.
//   forward   mean and rstd = 1 / sqrt(variance + eps) of each row;  y = (x - mean) * rstd * gamma + beta
//   backward  h = (x - mean) * rstd,  g = dy * gamma;  dx = rstd * (g - mean(g) - h * mean(g h)) + residual;  dgamma = column sums of dy h, dbeta of dy
#include <float.h>

#include "row_ops.h"

namespace sol {
namespace {

struct NormArgs {
    const void *x, *dy, *residual;
    const float *gamma, *beta, *mean_in, *rstd_in;
    void *y;                    // backward: dx
    float *mean, *rstd;
    long ldx, ldy;              // backward: of dy
    int rows, cols;
    float eps, inv_cols;
};

// gamma's (beta's) 8 values from column c on; `none` where there are none
__device__ __forceinline__ void load_weight8(const float *w, int c, int nv, float none, float v[8]) {
    if (w) load8_any<float>(w + c, v, nv);
    else {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = none;
    }
}

// sum / n with the reciprocal and one correction, so that equal elements whose sum is exact have their own value for a mean
__device__ __forceinline__ float mean_of(float sum, float n, float inv) {
    const float m = sum * inv;
    return fmaf(fmaf(-m, n, sum), inv, m);
}

// Means and squared deviations of the waves, put together: mean = sum n_w mean_w / n, deviations = sum (d_w + n_w (mean_w - mean)^2) (Chan, Golub, LeVeque).
// One barrier a row; two sets of slots in turn, so that the next row's values do not meet readers of this one's.
template <int TPR, int G, typename T>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_kernel(const NormArgs a) {
    constexpr int BLOCK = TPR < 256 ? 256 : TPR, RPB = BLOCK / TPR, WAVES = TPR / 64;
    __shared__ float4 red[2][WAVES];
    const int lane = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    float gm[G][8], bt[G][8];
    int nv[G], n_wave = 0;
#pragma unroll
    for (int k = 0; k < G; k++) {
        const int c = (lane + k * TPR) * 8;
        nv[k] = min(8, a.cols - c);
        load_weight8(a.gamma, c, nv[k], 1.f, gm[k]);
        load_weight8(a.beta, c, nv[k], 0.f, bt[k]);
        n_wave += max(0, min(512, a.cols - (lane / 64 * 64 + k * TPR) * 8));
    }
    const float inv_wave = n_wave ? 1.f / (float)n_wave : 0.f;
    int phase = 0;
    for (long row = (long)blockIdx.x * RPB + slot; row < a.rows; row += (long)gridDim.x * RPB) {      // with TPR > 64 a workgroup has one row at a time: every thread meets every barrier
        const T *x = static_cast<const T *>(a.x) + row * a.ldx;
        float v[G][8], s = 0.f;
#pragma unroll
        for (int k = 0; k < G; k++) {
            load8_any<T>(x + (lane + k * TPR) * 8, v[k], nv[k]);
#pragma unroll
            for (int e = 0; e < 8; e++) s += v[k][e];
        }
        float mean = mean_of(wave_sum(s), (float)n_wave, inv_wave), m2 = 0.f;
#pragma unroll
        for (int k = 0; k < G; k++)
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float d = e < nv[k] ? v[k][e] - mean : 0.f;
                m2 += d * d;
            }
        m2 = wave_sum(m2);
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) red[phase][lane / 64] = make_float4(mean, m2, (float)n_wave, 0.f);
            __syncthreads();
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; w++) sum += red[phase][w].x * red[phase][w].z;
            mean = mean_of(sum, (float)a.cols, a.inv_cols);
            m2 = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; w++) {
                const float4 p = red[phase][w];
                m2 += p.y + p.z * (p.x - mean) * (p.x - mean);
            }
            phase ^= 1;
        }
        const float rstd = __builtin_amdgcn_rsqf(m2 * a.inv_cols + a.eps);
        T *y = static_cast<T *>(a.y) + row * a.ldy;
#pragma unroll
        for (int k = 0; k < G; k++) {
#pragma unroll
            for (int e = 0; e < 8; e++) v[k][e] = (v[k][e] - mean) * rstd * gm[k][e] + bt[k][e];
            store8_any<T>(y + (lane + k * TPR) * 8, v[k], nv[k]);
        }
        if (lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

// A sum over a workgroup of 1024 threads, in all of them
__device__ __forceinline__ float block_sum(float v, float *red) {
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x / 64] = v;
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < 16; w++) s += red[w];
    return s;
}

// Rows that registers do not hold: three passes over a row, of which the second and third find it in the caches
template <typename T> __global__ void __launch_bounds__(1024) norm_long_kernel(const NormArgs a) {
    __shared__ float red[16];
    for (long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.ldx;
        T *y = static_cast<T *>(a.y) + row * a.ldy;
        float v[8], s = 0.f;
        for (int c = threadIdx.x * 8; c < a.cols; c += 8192) {
            load8_any<T>(x + c, v, a.cols - c);
#pragma unroll
            for (int e = 0; e < 8; e++) s += v[e];
        }
        const float mean = mean_of(block_sum(s, red), (float)a.cols, a.inv_cols);
        s = 0.f;
        for (int c = threadIdx.x * 8; c < a.cols; c += 8192) {
            load8_any<T>(x + c, v, a.cols - c);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float d = e < a.cols - c ? v[e] - mean : 0.f;
                s += d * d;
            }
        }
        const float rstd = __builtin_amdgcn_rsqf(block_sum(s, red) * a.inv_cols + a.eps);
        for (int c = threadIdx.x * 8; c < a.cols; c += 8192) {
            const int nv = min(8, a.cols - c);
            float g[8], b[8];
            load8_any<T>(x + c, v, nv);
            load_weight8(a.gamma, c, nv, 1.f, g);
            load_weight8(a.beta, c, nv, 0.f, b);
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = (v[e] - mean) * rstd * g[e] + b[e];
            store8_any<T>(y + c, v, nv);
        }
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
    }
}

template <int TPR, int G, typename T>
__global__ void __launch_bounds__(TPR < 256 ? 256 : TPR) norm_dx_kernel(const NormArgs a) {
    constexpr int BLOCK = TPR < 256 ? 256 : TPR, RPB = BLOCK / TPR, WAVES = TPR / 64;
    __shared__ float2 red[2][WAVES];
    const int lane = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    float gm[G][8];
    int nv[G];
#pragma unroll
    for (int k = 0; k < G; k++) {
        const int c = (lane + k * TPR) * 8;
        nv[k] = min(8, a.cols - c);
        load_weight8(a.gamma, c, nv[k], 1.f, gm[k]);
    }
    int phase = 0;
    for (long row = (long)blockIdx.x * RPB + slot; row < a.rows; row += (long)gridDim.x * RPB) {
        const T *x = static_cast<const T *>(a.x) + row * a.ldx, *dy = static_cast<const T *>(a.dy) + row * a.ldy;
        const float mean = a.mean_in[row], rstd = a.rstd_in[row];
        float h[G][8], g[G][8], s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int k = 0; k < G; k++) {
            load8_any<T>(x + (lane + k * TPR) * 8, h[k], nv[k]);
            load8_any<T>(dy + (lane + k * TPR) * 8, g[k], nv[k]);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                h[k][e] = e < nv[k] ? (h[k][e] - mean) * rstd : 0.f;
                g[k][e] *= gm[k][e];
                s1 += g[k][e];
                s2 += g[k][e] * h[k][e];
            }
        }
        s1 = wave_sum(s1);
        s2 = wave_sum(s2);
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) red[phase][lane / 64] = make_float2(s1, s2);
            __syncthreads();
            s1 = s2 = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; w++) { s1 += red[phase][w].x; s2 += red[phase][w].y; }
            phase ^= 1;
        }
        const float c1 = s1 * a.inv_cols, c2 = s2 * a.inv_cols;
        const size_t out = (size_t)row * a.cols;
#pragma unroll
        for (int k = 0; k < G; k++) {
            const int c = (lane + k * TPR) * 8;
#pragma unroll
            for (int e = 0; e < 8; e++) g[k][e] = rstd * (g[k][e] - c1 - h[k][e] * c2);
            if (a.residual) {
                load8_any<T>(static_cast<const T *>(a.residual) + out + c, h[k], nv[k]);
#pragma unroll
                for (int e = 0; e < 8; e++) g[k][e] += h[k][e];
            }
            store8_any<T>(static_cast<T *>(a.y) + out + c, g[k], nv[k]);
        }
    }
}

template <typename T> __global__ void __launch_bounds__(1024) norm_dx_long_kernel(const NormArgs a) {
    __shared__ float red[16];
    for (long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.x) + row * a.ldx, *dy = static_cast<const T *>(a.dy) + row * a.ldy;
        const float mean = a.mean_in[row], rstd = a.rstd_in[row];
        float h[8], g[8], w[8], s1 = 0.f, s2 = 0.f;
        for (int c = threadIdx.x * 8; c < a.cols; c += 8192) {
            const int nv = min(8, a.cols - c);
            load8_any<T>(x + c, h, nv);
            load8_any<T>(dy + c, g, nv);
            load_weight8(a.gamma, c, nv, 1.f, w);
#pragma unroll
            for (int e = 0; e < 8; e++) {
                const float ge = g[e] * w[e];
                s1 += ge;
                s2 += e < nv ? ge * ((h[e] - mean) * rstd) : 0.f;
            }
        }
        const float c1 = block_sum(s1, red) * a.inv_cols, c2 = block_sum(s2, red) * a.inv_cols;
        const size_t out = (size_t)row * a.cols;
        for (int c = threadIdx.x * 8; c < a.cols; c += 8192) {
            const int nv = min(8, a.cols - c);
            load8_any<T>(x + c, h, nv);
            load8_any<T>(dy + c, g, nv);
            load_weight8(a.gamma, c, nv, 1.f, w);
#pragma unroll
            for (int e = 0; e < 8; e++) g[e] = rstd * (g[e] * w[e] - c1 - (h[e] - mean) * rstd * c2);
            if (a.residual) {
                load8_any<T>(static_cast<const T *>(a.residual) + out + c, h, nv);
#pragma unroll
                for (int e = 0; e < 8; e++) g[e] += h[e];
            }
            store8_any<T>(static_cast<T *>(a.y) + out + c, g, nv);
        }
    }
}

// Column sums of a chunk of rows: 32 groups of 8 columns x 32 rows at a time.
struct NormColumns {
    const void *dy, *x;
    const float *mean, *rstd;
    long ldy, ldx;
    int rows, cols, per_chunk, tiles;
    float *dgamma, *dbeta;      // parts [chunk][cols], or the sums themselves; NULL: not wanted
};
template <typename T> __global__ void __launch_bounds__(1024) norm_columns_kernel(const NormColumns a) {
    __shared__ float red[2][32][256 + 4];
    const int tile = (int)blockIdx.x % a.tiles, chunk = (int)blockIdx.x / a.tiles;
    const int gl = threadIdx.x & 31, rl = threadIdx.x >> 5, c = (tile * 32 + gl) * 8, nv = min(8, a.cols - c);
    const int r0 = chunk * a.per_chunk, r1 = min(a.rows, r0 + a.per_chunk);
    float sg[8], sb[8];
#pragma unroll
    for (int e = 0; e < 8; e++) sg[e] = sb[e] = 0.f;
    if (nv > 0) {
        for (int r = r0 + rl; r < r1; r += 32) {
            float h[8], g[8];
            load8_any<T>(static_cast<const T *>(a.x) + r * a.ldx + c, h, nv);
            load8_any<T>(static_cast<const T *>(a.dy) + r * a.ldy + c, g, nv);
            const float mean = a.mean[r], rstd = a.rstd[r];
#pragma unroll
            for (int e = 0; e < 8; e++) {
                sg[e] += g[e] * ((h[e] - mean) * rstd);
                sb[e] += g[e];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; e++) { red[0][rl][gl * 8 + e] = sg[e]; red[1][rl][gl * 8 + e] = sb[e]; }
    __syncthreads();
    const int which = threadIdx.x >> 8, col = tile * 256 + (threadIdx.x & 255);
    float *out = which == 0 ? a.dgamma : a.dbeta;
    if (which > 1 || col >= a.cols || !out) return;
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < 32; r++) s += red[which][r][threadIdx.x & 255];
    out[(size_t)chunk * a.cols + col] = s;
}

// Two workgroups per CU, each with 32 rows or more
int rows_per_chunk(int rows, int cols) {
    const int want = max(1, 512 / ceil_div(cols, 256));
    return rows <= 64 ? 64 : (int)round_up((size_t)max(1, (rows + want - 1) / want), 32);
}
int norm_chunks(int rows, int cols) { return rows > 0 ? (int)(((long)rows + rows_per_chunk(rows, cols) - 1) / rows_per_chunk(rows, cols)) : 0; }

sol_status check_norm(const sol_layer_norm_desc *nd, sol_layer_norm_desc *n) {
    SOL_REQUIRE(nd, SOL_ERR_NULL, "layer norm descriptor is NULL");
    *n = *nd;
    SOL_REQUIRE(n->dtype == SOL_F32 || n->dtype == SOL_BF16, SOL_ERR_DTYPE, "layer norm: unknown dtype %d", n->dtype);
    SOL_REQUIRE(n->rows >= 0 && n->cols > 0, SOL_ERR_SHAPE, "bad layer norm shape [%d,%d]", n->rows, n->cols);
    SOL_REQUIRE(n->cols <= MAX_COLS, SOL_ERR_UNSUPPORTED, "more than 2^20 columns: %d", n->cols);
    SOL_TRY(check_row_pitch("x", n->cols, &n->ldx));
    SOL_TRY(check_row_pitch("y", n->cols, &n->ldy));
    return SOL_OK;
}

enum { NORM_FORWARD, NORM_DX };
template <int TPR, int G, typename T> void launch_rows(int kind, const NormArgs &a, hipStream_t st) {
    constexpr int BLOCK = TPR < 256 ? 256 : TPR, RPB = BLOCK / TPR;
    const dim3 grid((unsigned)min(((long)a.rows + RPB - 1) / RPB, 2048l));
    if (kind == NORM_FORWARD) hipLaunchKernelGGL((norm_kernel<TPR, G, T>), grid, dim3(BLOCK), 0, st, a);
    else hipLaunchKernelGGL((norm_dx_kernel<TPR, G, T>), grid, dim3(BLOCK), 0, st, a);
}
template <typename T> sol_status launch_norm(int kind, const NormArgs &a, hipStream_t st) {
    const int groups = ceil_div(a.cols, 8);
    if (groups <= 64) launch_rows<64, 1, T>(kind, a, st);
    else if (groups <= 128) launch_rows<64, 2, T>(kind, a, st);
    else if (groups <= 256) launch_rows<256, 1, T>(kind, a, st);
    else if (groups <= 512) launch_rows<256, 2, T>(kind, a, st);
    else if (groups <= 1024) launch_rows<512, 2, T>(kind, a, st);
    else {
        const dim3 grid((unsigned)min(a.rows, 1024));
        if (kind == NORM_FORWARD) hipLaunchKernelGGL(norm_long_kernel<T>, grid, dim3(1024), 0, st, a);
        else hipLaunchKernelGGL(norm_dx_long_kernel<T>, grid, dim3(1024), 0, st, a);
    }
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

}  // namespace
}  // namespace sol

using namespace sol;

extern "C" {

sol_status sol_layer_norm(const sol_layer_norm_desc *nd, const void *x, const float *gamma, const float *beta, void *y, float *mean, float *rstd, void *stream) {
    sol_layer_norm_desc n;
    SOL_TRY(check_norm(nd, &n));
    SOL_REQUIRE(n.eps >= FLT_MIN && n.eps <= FLT_MAX, SOL_ERR_SHAPE, "layer norm: eps %g is not in 2^-126 .. 2^128", (double)n.eps);       // refuses a NaN too
    if (n.rows == 0) return SOL_OK;
    SOL_REQUIRE(x && y, SOL_ERR_NULL, "x and y must not be NULL");
    SOL_REQUIRE(aligned16(x) && aligned16(gamma) && aligned16(beta) && aligned16(y) && aligned16(mean) && aligned16(rstd), SOL_ERR_ALIGN, "device pointers must be 16-byte aligned");
    SOL_REQUIRE(y != x || n.ldx == n.ldy, SOL_ERR_UNSUPPORTED, "layer norm: y in the place of x needs its pitch");
    const void *const outs[3] = {y, mean, rstd}, *const ins[3] = {gamma, beta, x};
    for (int i = 0; i < 3; i++) {
        for (int j = 0; j < (i ? 3 : 2); j++) SOL_REQUIRE(!outs[i] || outs[i] != ins[j], SOL_ERR_UNSUPPORTED, "layer norm: outputs must not alias inputs");
        for (int j = 0; j < i; j++) SOL_REQUIRE(!outs[i] || outs[i] != outs[j], SOL_ERR_UNSUPPORTED, "layer norm: outputs must not alias each other");
    }
    NormArgs a{};
    a.x = x; a.gamma = gamma; a.beta = beta; a.y = y; a.mean = mean; a.rstd = rstd;
    a.ldx = n.ldx; a.ldy = n.ldy; a.rows = n.rows; a.cols = n.cols; a.eps = n.eps; a.inv_cols = 1.f / (float)n.cols;
    return n.dtype == SOL_BF16 ? launch_norm<bf16_t>(NORM_FORWARD, a, (hipStream_t)stream) : launch_norm<float>(NORM_FORWARD, a, (hipStream_t)stream);
}

size_t sol_layer_norm_backward_workspace_bytes(const sol_layer_norm_desc *nd) {
    sol_layer_norm_desc n;
    if (check_norm(nd, &n) != SOL_OK) return 0;
    const int chunks = norm_chunks(n.rows, n.cols);
    return chunks > 1 ? (size_t)2 * chunks * n.cols * 4 : 0;
}

sol_status sol_layer_norm_backward(const sol_layer_norm_desc *nd, const void *dy, const void *x, const float *gamma, const float *mean, const float *rstd, const void *residual, void *dx,
                                   float *dgamma, float *dbeta, void *workspace, size_t workspace_bytes, void *stream) {
    sol_layer_norm_desc n;
    SOL_TRY(check_norm(nd, &n));
    SOL_REQUIRE(aligned16(dy) && aligned16(x) && aligned16(gamma) && aligned16(mean) && aligned16(rstd) && aligned16(residual) && aligned16(dx) && aligned16(dgamma) && aligned16(dbeta),
                SOL_ERR_ALIGN, "device pointers must be 16-byte aligned");
    hipStream_t st = (hipStream_t)stream;
    SumJobs sums{};
    if (n.rows == 0) {
        if (dgamma) sums.add(nullptr, 0, n.cols, dgamma, SOL_F32);
        if (dbeta) sums.add(nullptr, 0, n.cols, dbeta, SOL_F32);
        return launch_sums(sums, st);
    }
    SOL_REQUIRE(dy && x && mean && rstd, SOL_ERR_NULL, "dy, x, mean and rstd must not be NULL");
    const void *const outs[3] = {dx, dgamma, dbeta}, *const ins[6] = {dy, x, gamma, mean, rstd, residual};
    for (int i = 0; i < 3; i++) {
        for (int j = 0; j < (i ? 6 : 5); j++) SOL_REQUIRE(!outs[i] || outs[i] != ins[j], SOL_ERR_UNSUPPORTED, "layer norm backward: outputs must not alias inputs");
        for (int j = 0; j < i; j++) SOL_REQUIRE(!outs[i] || outs[i] != outs[j], SOL_ERR_UNSUPPORTED, "layer norm backward: outputs must not alias each other");
    }
    SOL_TRY(check_scratch(workspace, workspace_bytes, sol_layer_norm_backward_workspace_bytes(&n)));
    if (dgamma || dbeta) {
        const int chunks = norm_chunks(n.rows, n.cols);
        float *pg = static_cast<float *>(workspace), *pb = pg + (size_t)chunks * n.cols;
        NormColumns c{dy, x, mean, rstd, n.ldy, n.ldx, n.rows, n.cols, rows_per_chunk(n.rows, n.cols), ceil_div(n.cols, 256), dgamma, dbeta};
        if (chunks > 1) {
            if (dgamma) { c.dgamma = pg; sums.add(pg, chunks, n.cols, dgamma, SOL_F32); }
            if (dbeta) { c.dbeta = pb; sums.add(pb, chunks, n.cols, dbeta, SOL_F32); }
        }
        const dim3 grid((unsigned)(c.tiles * chunks));
        if (n.dtype == SOL_BF16) hipLaunchKernelGGL(norm_columns_kernel<bf16_t>, grid, dim3(1024), 0, st, c);
        else hipLaunchKernelGGL(norm_columns_kernel<float>, grid, dim3(1024), 0, st, c);
        SOL_HIP(hipGetLastError());
    }
    if (dx) {
        NormArgs a{};
        a.x = x; a.dy = dy; a.residual = residual; a.gamma = gamma; a.mean_in = mean; a.rstd_in = rstd; a.y = dx;
        a.ldx = n.ldx; a.ldy = n.ldy; a.rows = n.rows; a.cols = n.cols; a.inv_cols = 1.f / (float)n.cols;
        SOL_TRY(n.dtype == SOL_BF16 ? launch_norm<bf16_t>(NORM_DX, a, st) : launch_norm<float>(NORM_DX, a, st));
    }
    return launch_sums(sums, st);
}

}  // extern "C"
