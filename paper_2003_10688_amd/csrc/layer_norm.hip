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
// of a span; 0 in the places that are not the thread's own
template <int W> __device__ __forceinline__ void load_weight(const float *w, const Span<W> &sp, float none, float v[W]) {
    RawPiece<float, W> raw;
    if (w) sp.template load<false>(w, raw);
#pragma unroll
    for (int e = 0; e < W; e++) v[e] = !sp.has(e) ? 0.f : w ? raw.get(e) : none;
}
// A row for TPR threads, 8 to 1024: workgroups of 256 where a row's threads are in one wave and none waits for another, else one row a workgroup
template <int TPR> constexpr int ROW_BLOCK = TPR <= 64 ? 256 : TPR;
template <int TPR> constexpr int ROW_WAVES = TPR <= 64 ? 1 : TPR / 64;

// sum / n with the reciprocal and one correction, so that equal elements whose sum is exact have their own value for a mean
__device__ __forceinline__ float mean_of(float sum, float n, float inv) {
    const float m = sum * inv;
    return fmaf(fmaf(-m, n, sum), inv, m);
}

// Sums and squared deviations of the waves, put together: mean = sum s_w / n, deviations = sum (d_w + n_w (mean_w - mean)^2) (Chan, Golub, LeVeque).
// One barrier a row; two sets of slots in turn, so that the next row's values do not meet readers of this one's.
// A row stays in registers between its only reading and its writing, gamma and beta for all rows of a workgroup.  Bound by memory: 16384 x 4096 bf16 43 us (6.2 TB/s; 52, 5.2 TB/s, with inputs that the last cache does not hold), 2^20 x 64 43 us with 8 threads a
// row (162 with a wave's 64), 16384 x 8192 84 us with results past the caches (100 without); one row of 2048 2.2 us, a launch and one round trip.
template <int TPR, int G, bool WHOLE, bool STREAM, typename T>
__global__ void __launch_bounds__(ROW_BLOCK<TPR>) norm_kernel(const NormArgs a) {
    constexpr int BLOCK = ROW_BLOCK<TPR>, RPB = BLOCK / TPR, WAVES = ROW_WAVES<TPR>, W = 16 / sizeof(T), P = G * 8 / W;
    __shared__ float4 red[2][WAVES];
    const int lane = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    const Spans<W, P> sp(lane * W, TPR * W, a.cols);
    float gm[P][W], bt[P][W];
    int n_wave = 0;
#pragma unroll
    for (int k = 0; k < P; k++) {
        load_weight(a.gamma, sp[k], 1.f, gm[k]);
        load_weight(a.beta, sp[k], 0.f, bt[k]);
        n_wave += max(0, min((TPR < 64 ? TPR : 64) * W, a.cols - (lane / 64 * 64 + k * TPR) * W));
    }
    const float inv_wave = n_wave ? 1.f / (float)n_wave : 0.f;
    int phase = 0;
    for (long row = (long)blockIdx.x * RPB + slot; row < a.rows; row += (long)gridDim.x * RPB) {      // above 64 threads a row a workgroup has one at a time: every thread meets every barrier
        const T *x = static_cast<const T *>(a.x) + row * a.ldx;
        float v[P][W], s = 0.f;
#pragma unroll
        for (int k = 0; k < P; k++) {
            RawPiece<T, W> raw;
            sp[k].template load<WHOLE>(x, raw);
#pragma unroll
            for (int e = 0; e < W; e++) {
                v[k][e] = raw.get(e);
                s += WHOLE || sp[k].has(e) ? v[k][e] : 0.f;     // zeros where there is nothing
            }
        }
        s = group_sum<TPR>(s);
        float mean = mean_of(s, (float)n_wave, inv_wave), m2 = 0.f;
#pragma unroll
        for (int k = 0; k < P; k++)
#pragma unroll
            for (int e = 0; e < W; e++) {
                const float d = (WHOLE ? sp[k].some() : sp[k].has(e)) ? v[k][e] - mean : 0.f;
                m2 += d * d;
            }
        m2 = group_sum<TPR>(m2);
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) red[phase][lane / 64] = make_float4(mean, m2, (float)n_wave, s);
            __syncthreads();
            float sum = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; w++) sum += red[phase][w].w;
            mean = mean_of(sum, (float)a.cols, a.inv_cols);
            m2 = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; w++) {
                const float4 p = red[phase][w];
                m2 += p.y + p.z * (p.x - mean) * (p.x - mean);
            }
            phase ^= 1;
        }
        const float rstd = __builtin_amdgcn_rsqf(m2 * a.inv_cols + a.eps);      // within 1 ulp: half an ulp more than a rounded root, beside sums over a row
        T *y = static_cast<T *>(a.y) + row * a.ldy;
#pragma unroll
        for (int k = 0; k < P; k++) {
#pragma unroll
            for (int e = 0; e < W; e++) v[k][e] = (v[k][e] - mean) * rstd * gm[k][e] + bt[k][e];
            sp[k].template store<WHOLE, STREAM>(y, v[k]);
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

// Rows that registers do not hold beside gamma and beta: three passes over a row, of which the second and third find it in the caches.  4096 x 16384 bf16 62 us, 4.3 TB/s, as with all of a row in
// the registers of 1024 threads, which leave one workgroup a CU.
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
        const float rstd = __builtin_amdgcn_rsqf(block_sum(s, red) * a.inv_cols + a.eps);       // within 1 ulp, as above
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

// Column sums of a chunk of rows, by the workgroup `block` of tiles * chunks.
struct NormColumns {
    const void *dy, *x;
    const float *mean, *rstd;
    long ldy, ldx;
    int rows, cols, per_chunk, tiles, blocks;
    float *dgamma, *dbeta;      // parts [chunk][cols], or the sums themselves; NULL: not wanted
};
// GROUPS groups of 8 columns x LANES rows at a time, four rows of a thread under way
template <int GROUPS, int LANES, typename T> __device__ __forceinline__ void column_sums(const NormColumns &a, int block, float (*red)[LANES][GROUPS * 8 + 4]) {
    const int tile = block % a.tiles, chunk = block / a.tiles;
    const int gl = threadIdx.x % GROUPS, rl = threadIdx.x / GROUPS, first = (tile * GROUPS + gl) * 8;
    const int r0 = chunk * a.per_chunk, r1 = min(a.rows, r0 + a.per_chunk);
    const Span<8> sp(first, a.cols);
    float sg[8], sb[8];
#pragma unroll
    for (int e = 0; e < 8; e++) sg[e] = sb[e] = 0.f;
    if (sp.some()) {
        for (int r = r0 + rl; r < r1; r += 4 * LANES) {
            RawPiece<T, 8> h[4], g[4];
            float mean[4], rstd[4];
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const int q = min(r + u * LANES, r1 - 1);
                sp.template load<false>(static_cast<const T *>(a.x) + q * a.ldx, h[u]);
                sp.template load<false>(static_cast<const T *>(a.dy) + q * a.ldy, g[u]);
                mean[u] = a.mean[q];
                rstd[u] = a.rstd[q];
            }
#pragma unroll
            for (int u = 0; u < 4; u++)
                if (r + u * LANES < r1) {
#pragma unroll
                    for (int e = 0; e < 8; e++) {
                        sg[e] += g[u].get(e) * ((h[u].get(e) - mean[u]) * rstd[u]);
                        sb[e] += g[u].get(e);
                    }
                }
        }
    }
#pragma unroll
    for (int e = 0; e < 8; e++)
        if (sp.has(e)) {
            const int lc = sp.c + e - tile * GROUPS * 8;
            red[0][rl][lc] = sg[e];
            red[1][rl][lc] = sb[e];
        }
    __syncthreads();
    const int which = threadIdx.x / (GROUPS * 8), lc = threadIdx.x % (GROUPS * 8), col = tile * GROUPS * 8 + lc;
    float *out = which == 0 ? a.dgamma : a.dbeta;
    if (which > 1 || col >= a.cols || !out) return;
    float s = 0.f;
#pragma unroll
    for (int r = 0; r < LANES; r++) s += red[which][r][lc];
    out[(size_t)chunk * a.cols + col] = s;
}
template <typename T> __global__ void __launch_bounds__(1024) norm_columns_kernel(const NormColumns a) {
    __shared__ float red[2][32][256 + 4];
    column_sums<32, 32, T>(a, (int)blockIdx.x, red);
}

// The row's part of the backward pass, from g = dy gamma and h: gamma, and so g, is 0 in places that are not the thread's own.  A piece without columns is left out all the same: its h is -mean * rstd,
// which may be more than fp32 holds where the row's own h are not, and 0 * inf would make the row's sums NaN.  (Places behind the end of rows shorter than a piece hold the row's last element again,
// whose h is one of the row's own.)  A select a piece, in front of the sum and not on h: 16384 x 4096 bf16 with a residual 102.0 us without it, 102.5 with it, 105.5 with h itself selected.
template <int P, int W> __device__ __forceinline__ void row_products(const Spans<W, P> &sp, const float (&g)[P][W], const float (&h)[P][W], float &s1, float &s2) {
    s1 = s2 = 0.f;
#pragma unroll
    for (int k = 0; k < P; k++) {
        float s = s2;
#pragma unroll
        for (int e = 0; e < W; e++) {
            s1 += g[k][e];
            s += g[k][e] * h[k][e];
        }
        s2 = sp[k].some() ? s : s2;
    }
}

// dx, a row for TPR threads; the workgroups in front sum the columns where there are few rows, so that both take one launch: the data is read twice, but the second time from the caches.
// 64 x 2048 bf16 3.8 us (two launches 7.2); dx alone of 4096 x 16384 84 us, 4.8 TB/s.
template <int TPR, int G, bool WHOLE, bool STREAM, typename T>
__global__ void __launch_bounds__(ROW_BLOCK<TPR>) norm_dx_kernel(const NormArgs a, const NormColumns cols) {
    constexpr int BLOCK = ROW_BLOCK<TPR>, RPB = BLOCK / TPR, WAVES = ROW_WAVES<TPR>, W = 16 / sizeof(T), P = G * 8 / W;
    __shared__ union {
        float columns[2][BLOCK / 8][64 + 4];
        float2 red[2][WAVES];
    } s;
    if ((int)blockIdx.x < cols.blocks) {
        column_sums<8, BLOCK / 8, T>(cols, (int)blockIdx.x, s.columns);
        return;
    }
    const int lane = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    const Spans<W, P> sp(lane * W, TPR * W, a.cols);
    float gm[P][W];
#pragma unroll
    for (int k = 0; k < P; k++) load_weight(a.gamma, sp[k], 1.f, gm[k]);
    int phase = 0;
    for (long row = (long)(blockIdx.x - cols.blocks) * RPB + slot; row < a.rows; row += (long)(gridDim.x - cols.blocks) * RPB) {
        const T *x = static_cast<const T *>(a.x) + row * a.ldx, *dy = static_cast<const T *>(a.dy) + row * a.ldy;
        const float mean = a.mean_in[row], rstd = a.rstd_in[row];
        float h[P][W], g[P][W], s1, s2;
#pragma unroll
        for (int k = 0; k < P; k++) {
            RawPiece<T, W> rx, ry;
            sp[k].template load<WHOLE, true>(x, rx);
            sp[k].template load<WHOLE>(dy, ry);
#pragma unroll
            for (int e = 0; e < W; e++) {
                h[k][e] = (rx.get(e) - mean) * rstd;
                g[k][e] = ry.get(e) * gm[k][e];
            }
        }
        row_products(sp, g, h, s1, s2);
        s1 = group_sum<TPR>(s1);
        s2 = group_sum<TPR>(s2);
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) s.red[phase][lane / 64] = make_float2(s1, s2);
            __syncthreads();
            s1 = s2 = 0.f;
#pragma unroll
            for (int w = 0; w < WAVES; w++) { s1 += s.red[phase][w].x; s2 += s.red[phase][w].y; }
            phase ^= 1;
        }
        const float c1 = s1 * a.inv_cols, c2 = s2 * a.inv_cols;
        const size_t out = (size_t)row * a.cols;
#pragma unroll
        for (int k = 0; k < P; k++) {
#pragma unroll
            for (int e = 0; e < W; e++) g[k][e] = rstd * (g[k][e] - c1 - h[k][e] * c2);
            if (a.residual) {       // dx may be in its place: a thread uses its own elements alone
                RawPiece<T, W> res;
                sp[k].template load<WHOLE>(static_cast<const T *>(a.residual) + out, res);
#pragma unroll
                for (int e = 0; e < W; e++) g[k][e] += res.get(e);
            }
            sp[k].template store<WHOLE, STREAM>(static_cast<T *>(a.y) + out, g[k]);
        }
    }
}

// dx and the columns' sums in one pass over the data: workgroups stay, take SLOTS rows at a time, with the next ones' loads under way, and keep the sums of their rows' columns in
// registers; parts [workgroup][cols] at the end.  Bound by memory: 16384 x 4096 bf16 with a residual 98 us and 5 for the parts (5.5 TB/s; two passes over the data 184), 1021 x 1531 fp32 9.7 and 4.
// Threads of a workgroup: 1024 with one piece each where rows are whole pieces, which 128 registers hold, so that one workgroup a CU is enough and fewer parts are left (16384 x 4096 bf16 104 us; 512
// threads with two pieces each 111).  Ends of rows take more registers.
template <bool WHOLE> constexpr int GRAD_BLOCK = WHOLE ? 1024 : 512;
template <int TPR, int G, bool WHOLE, bool STREAM, typename T>
__global__ void __launch_bounds__(GRAD_BLOCK<WHOLE>) norm_grad_kernel(const NormArgs a, float *dgamma, float *dbeta) {
    constexpr int SLOTS = GRAD_BLOCK<WHOLE> / TPR, WAVES = ROW_WAVES<TPR>, W = 16 / sizeof(T), P = G * 8 / W;
    __shared__ float2 red[2][GRAD_BLOCK<WHOLE> / 64];
    __shared__ float sums[SLOTS > 1 ? SLOTS : 1][SLOTS > 1 ? TPR * G * 8 : 1];
    const int lane = threadIdx.x % TPR, slot = threadIdx.x / TPR;
    const Spans<W, P> sp(lane * W, TPR * W, a.cols);
    float gm[P][W], sg[P][W], sb[P][W];
#pragma unroll
    for (int k = 0; k < P; k++) {
        load_weight(a.gamma, sp[k], 1.f, gm[k]);
#pragma unroll
        for (int e = 0; e < W; e++) sg[k][e] = sb[k][e] = 0.f;
    }
    RawPiece<T, W> xr[P], yr[P];
    float mean = 0.f, rstd = 0.f;
    auto fetch = [&](long row) {
        if (row >= a.rows) return;
#pragma unroll
        for (int k = 0; k < P; k++) {
            sp[k].template load<WHOLE, true>(static_cast<const T *>(a.x) + row * a.ldx, xr[k]);
            sp[k].template load<WHOLE>(static_cast<const T *>(a.dy) + row * a.ldy, yr[k]);
        }
        mean = a.mean_in[row];
        rstd = a.rstd_in[row];
    };
    int phase = 0;
    long row = (long)blockIdx.x * SLOTS + slot;
    fetch(row);
    for (long first = (long)blockIdx.x * SLOTS; first < a.rows; first += (long)gridDim.x * SLOTS) {      // the same for every thread: each meets every barrier
        const bool there = row < a.rows;
        float h[P][W], g[P][W], s1 = 0.f, s2 = 0.f;
        const float r = rstd;
        if (there) {
#pragma unroll
            for (int k = 0; k < P; k++)
#pragma unroll
                for (int e = 0; e < W; e++) {
                    h[k][e] = (xr[k].get(e) - mean) * rstd;
                    const float d = yr[k].get(e);
                    sb[k][e] += d;
                    sg[k][e] += d * h[k][e];
                    g[k][e] = d * gm[k][e];
                }
        }
        RawPiece<T, W> res[P];
        const size_t out = (size_t)row * a.cols;
        if (there && a.residual) {
#pragma unroll
            for (int k = 0; k < P; k++) sp[k].template load<WHOLE>(static_cast<const T *>(a.residual) + out, res[k]);
        }
        row += (long)gridDim.x * SLOTS;
        fetch(row);
        if (a.y) {
            if (there) row_products(sp, g, h, s1, s2);
            s1 = group_sum<TPR>(s1);
            s2 = group_sum<TPR>(s2);
            if constexpr (WAVES > 1) {
                if ((threadIdx.x & 63) == 0) red[phase][threadIdx.x / 64] = make_float2(s1, s2);
                __syncthreads();
                s1 = s2 = 0.f;
#pragma unroll
                for (int w = 0; w < WAVES; w++) { s1 += red[phase][slot * WAVES + w].x; s2 += red[phase][slot * WAVES + w].y; }
                phase ^= 1;
            }
            const float c1 = s1 * a.inv_cols, c2 = s2 * a.inv_cols;
            if (there) {
#pragma unroll
                for (int k = 0; k < P; k++) {
#pragma unroll
                    for (int e = 0; e < W; e++) {
                        g[k][e] = r * (g[k][e] - c1 - h[k][e] * c2);
                        if (a.residual) g[k][e] += res[k].get(e);
                    }
                    sp[k].template store<WHOLE, STREAM>(static_cast<T *>(a.y) + out, g[k]);
                }
            }
        }
    }
    // the slots' sums, in their order, a column a thread
#pragma unroll
    for (int which = 0; which < 2; which++) {
        float (&s)[P][W] = which == 0 ? sg : sb;
        float *part = which == 0 ? dgamma : dbeta;
        if (!part) continue;
        part += (size_t)blockIdx.x * a.cols;
        if constexpr (SLOTS == 1) {
#pragma unroll
            for (int k = 0; k < P; k++) sp[k].template store<WHOLE>(part, s[k]);
        } else {
            __syncthreads();
#pragma unroll
            for (int k = 0; k < P; k++)
#pragma unroll
                for (int e = 0; e < W; e++)
                    if (sp[k].has(e)) sums[slot][sp[k].c + e] = s[k][e];
            __syncthreads();
            for (int c = threadIdx.x; c < a.cols; c += GRAD_BLOCK<WHOLE>) {
                float v = 0.f;
#pragma unroll
                for (int q = 0; q < SLOTS; q++) v += sums[q][c];
                part[c] = v;
            }
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

enum { NORM_FORWARD, NORM_DX, NORM_GRAD };
// Groups of 8 columns that a row may have in registers: where dx alone is computed, and where gamma and beta or the columns' sums are kept beside it
constexpr int MAX_DX_GROUPS = 2048, MAX_GROUPS = 1024;
// Few rows: columns are summed by workgroups of their own, beside the rows', in the same launch.  us, that launch against one pass and a launch for its parts, calls of a graph with a residual and
// changing inputs:     64 columns        512             2048            8192
//   bf16   512 rows    5.8 and  8.3     6.3 and  8.1    8.2 and 11.0   11.6 and 16.2
//         1024         9.1 and  8.5    11.7 and  9.9   13.7 and 14.2   20.2 and 24.8
//         1536        13.1 and  9.1    17.1 and 11.1   18.7 and 15.7   29.0 and 30.2
//   fp32   512         5.6 and  8.9     7.3 and  7.6    9.1 and 11.6   19.5 and 21.2
//          768         8.3 and  9.4    10.0 and 10.1   12.2 and 13.8   27.5 and 28.7
//         1024        10.6 and  9.2    12.4 and 10.7   15.2 and 14.9   34.3 and 34.7
// One border for all widths: at it narrow bf16 rows lose 0.6 to 1.8 us, and behind it wide ones would still gain up to 1.2.
bool few_rows(int rows, int dt) { return (size_t)rows * dtype_size(dt) <= 2048; }

// Threads that a row takes in norm_grad_kernel: one for each group of 8 columns, or two groups a thread for long rows that are no whole pieces (see GRAD_BLOCK)
int grad_threads(int groups, bool whole) {
    int t = 8;
    while (t < groups) t *= 2;
    return !whole && t > 256 ? t / 2 : t;
}

struct NormLaunch {
    int kind;
    NormArgs a;
    NormColumns cols;           // NORM_DX: what the workgroups in front sum
    int groups;                 // NORM_GRAD: workgroups
    float *dgamma, *dbeta;      // and their parts
};
template <int TPR, int G, bool WHOLE, bool STREAM, typename T> void launch_rows_of(const NormLaunch &l, hipStream_t st) {
    constexpr int BLOCK = ROW_BLOCK<TPR>, RPB = BLOCK / TPR;
    const int rows = (int)min(((long)l.a.rows + RPB - 1) / RPB, 2048l);
    if constexpr (TPR * G <= MAX_GROUPS) {
        if (l.kind == NORM_FORWARD) {
            hipLaunchKernelGGL((norm_kernel<TPR, G, WHOLE, STREAM, T>), dim3((unsigned)rows), dim3(BLOCK), 0, st, l.a);
            return;
        }
    }
    hipLaunchKernelGGL((norm_dx_kernel<TPR, G, WHOLE, STREAM, T>), dim3((unsigned)(l.cols.blocks + (l.a.y ? rows : 0))), dim3(BLOCK), 0, st, l.a, l.cols);
}
template <typename T> bool whole_rows(int cols) { return cols % (16 / sizeof(T)) == 0; }
template <typename T> bool streamed(const NormArgs &a) { return (size_t)a.rows * a.cols * sizeof(T) >= STREAM_BYTES; }
template <int TPR, int G, typename T> void launch_rows(const NormLaunch &l, hipStream_t st) {
    if (!whole_rows<T>(l.a.cols)) launch_rows_of<TPR, G, false, false, T>(l, st);
    else if (streamed<T>(l.a)) launch_rows_of<TPR, G, true, true, T>(l, st);
    else launch_rows_of<TPR, G, true, false, T>(l, st);
}
template <int TPR, int G, bool WHOLE, typename T> void launch_grad(const NormLaunch &l, hipStream_t st) {
    const dim3 grid((unsigned)l.groups), block(GRAD_BLOCK<WHOLE>);
    if constexpr (WHOLE) {
        if (streamed<T>(l.a)) hipLaunchKernelGGL((norm_grad_kernel<TPR, G, true, true, T>), grid, block, 0, st, l.a, l.dgamma, l.dbeta);
        else hipLaunchKernelGGL((norm_grad_kernel<TPR, G, true, false, T>), grid, block, 0, st, l.a, l.dgamma, l.dbeta);
    } else {
        hipLaunchKernelGGL((norm_grad_kernel<TPR, G, false, false, T>), grid, block, 0, st, l.a, l.dgamma, l.dbeta);
    }
}
template <bool WHOLE, typename T> void launch_grad_rows(const NormLaunch &l, int groups, hipStream_t st) {
    switch (grad_threads(groups, WHOLE)) {
    case 8: return launch_grad<8, 1, WHOLE, T>(l, st);
    case 16: return launch_grad<16, 1, WHOLE, T>(l, st);
    case 32: return launch_grad<32, 1, WHOLE, T>(l, st);
    case 64: return launch_grad<64, 1, WHOLE, T>(l, st);
    case 128: return launch_grad<128, 1, WHOLE, T>(l, st);
    case 256:
        if constexpr (!WHOLE)
            if (groups > 256) return launch_grad<256, 2, false, T>(l, st);
        return launch_grad<256, 1, WHOLE, T>(l, st);
    case 512: return launch_grad<512, WHOLE ? 1 : 2, WHOLE, T>(l, st);
    default:
        if constexpr (WHOLE) launch_grad<1024, 1, true, T>(l, st);
    }
}
template <typename T> sol_status launch_norm(const NormLaunch &l, hipStream_t st) {
    const int groups = ceil_div(l.a.cols, 8);
    if (groups > (l.kind == NORM_DX ? MAX_DX_GROUPS : MAX_GROUPS)) {
        const dim3 grid((unsigned)min(l.a.rows, 1024));
        if (l.kind == NORM_FORWARD) hipLaunchKernelGGL(norm_long_kernel<T>, grid, dim3(1024), 0, st, l.a);
        else hipLaunchKernelGGL(norm_dx_long_kernel<T>, grid, dim3(1024), 0, st, l.a);
    } else if (l.kind != NORM_GRAD) {
        if (groups <= 8) launch_rows<8, 1, T>(l, st);
        else if (groups <= 16) launch_rows<16, 1, T>(l, st);
        else if (groups <= 32) launch_rows<32, 1, T>(l, st);
        else if (groups <= 64) launch_rows<64, 1, T>(l, st);
        else if (groups <= 128) launch_rows<128, 1, T>(l, st);
        else if (groups <= 256) launch_rows<256, 1, T>(l, st);
        else if (groups <= 512) launch_rows<256, 2, T>(l, st);
        else if (groups <= 1024) launch_rows<512, 2, T>(l, st);
        else launch_rows<1024, 2, T>(l, st);
    } else if (whole_rows<T>(l.a.cols)) launch_grad_rows<true, T>(l, groups, st);
    else launch_grad_rows<false, T>(l, groups, st);
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}
sol_status launch_norm(const NormLaunch &l, int dt, hipStream_t st) { return dt == SOL_BF16 ? launch_norm<bf16_t>(l, st) : launch_norm<float>(l, st); }

// Parts that dgamma and dbeta are summed in: 1 where workgroups beside the rows' sum whole columns
int norm_parts(int rows, int cols, int dt) {
    const int groups = ceil_div(cols, 8);
    if (groups <= MAX_DX_GROUPS && few_rows(rows, dt)) return 1;
    if (groups > MAX_GROUPS) return norm_chunks(rows, cols);
    const bool whole = cols % (16 / (int)dtype_size(dt)) == 0;
    const int slots = (whole ? GRAD_BLOCK<true> : GRAD_BLOCK<false>) / grad_threads(groups, whole);
    const long rounds = ((long)rows + slots - 1) / slots, most = min(rounds, groups <= 256 && !whole ? 512l : 256l);
    // A round of rows costs a workgroup about what 32 more parts cost the launch that sums them: 32 rounds = parts^2 makes the sum of both least.  Up to a GPU full of workgroups.
    // us for both launches with 4, 16, 32, 64 and 512 in place of 32: 1021 x 1531 fp32 19.9, 15.6, 13.8, 14.6, 19.6 (46 to 511 parts); 2048 x 2048 bf16 24.8, 18.5, 16.2, 16.4, 16.5 (46 to 256);
    // 4096 x 512 bf16 17.7, 13.5, 13.6, 12.3, 13.0; 4096 x 1024 fp32 37.8, 25.9, 21.2, 21.2, 20.3; 4096 x 4096 bf16 56.3, 39.0, 34.3, 34.2, 34.2; 20000 x 1001 fp32 77.6, 81.9, 69.7, 68.3, 68.4.
    long parts = 1;
    while (parts * parts < 32 * rounds && parts < most) parts++;
    return (int)parts;
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
    NormLaunch l{};
    l.kind = NORM_FORWARD;
    NormArgs &a = l.a;
    a.x = x; a.gamma = gamma; a.beta = beta; a.y = y; a.mean = mean; a.rstd = rstd;
    a.ldx = n.ldx; a.ldy = n.ldy; a.rows = n.rows; a.cols = n.cols; a.eps = n.eps; a.inv_cols = 1.f / (float)n.cols;
    return launch_norm(l, n.dtype, (hipStream_t)stream);
}

size_t sol_layer_norm_backward_workspace_bytes(const sol_layer_norm_desc *nd) {
    sol_layer_norm_desc n;
    if (check_norm(nd, &n) != SOL_OK) return 0;
    const int parts = norm_parts(n.rows, n.cols, n.dtype);
    return parts > 1 ? (size_t)2 * parts * n.cols * 4 : 0;
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
    NormLaunch l{};
    NormArgs &a = l.a;
    a.x = x; a.dy = dy; a.residual = residual; a.gamma = gamma; a.mean_in = mean; a.rstd_in = rstd; a.y = dx;
    a.ldx = n.ldx; a.ldy = n.ldy; a.rows = n.rows; a.cols = n.cols; a.inv_cols = 1.f / (float)n.cols;
    const bool columns = dgamma || dbeta, few = ceil_div(n.cols, 8) <= MAX_DX_GROUPS && few_rows(n.rows, n.dtype), wide = ceil_div(n.cols, 8) > MAX_GROUPS && !few;
    if (!columns && !dx) return SOL_OK;
    // where the columns' sums go: parts, which a launch behind puts together, or their own place
    const int parts = norm_parts(n.rows, n.cols, n.dtype);
    float *pg = dgamma, *pb = dbeta;
    if (parts > 1) {
        float *ws = static_cast<float *>(workspace);
        if (dgamma) { pg = ws; sums.add(pg, parts, n.cols, dgamma, SOL_F32); }
        if (dbeta) { pb = ws + (size_t)parts * n.cols; sums.add(pb, parts, n.cols, dbeta, SOL_F32); }
    }
    if (columns) l.cols = NormColumns{dy, x, mean, rstd, n.ldy, n.ldx, n.rows, n.cols, n.rows, ceil_div(n.cols, 64), ceil_div(n.cols, 64), pg, pb};
    if (wide) {
        if (columns) {
            l.cols.per_chunk = rows_per_chunk(n.rows, n.cols);
            l.cols.tiles = ceil_div(n.cols, 256);
            const dim3 grid((unsigned)(l.cols.tiles * parts));
            if (n.dtype == SOL_BF16) hipLaunchKernelGGL(norm_columns_kernel<bf16_t>, grid, dim3(1024), 0, st, l.cols);
            else hipLaunchKernelGGL(norm_columns_kernel<float>, grid, dim3(1024), 0, st, l.cols);
            SOL_HIP(hipGetLastError());
            l.cols = NormColumns{};
        }
        l.kind = NORM_DX;
        if (dx) SOL_TRY(launch_norm(l, n.dtype, st));
    } else {
        l.kind = columns && !few ? NORM_GRAD : NORM_DX;
        l.groups = parts;
        l.dgamma = pg;
        l.dbeta = pb;
        SOL_TRY(launch_norm(l, n.dtype, st));
    }
    return launch_sums(sums, st);
}

}  // extern "C"
