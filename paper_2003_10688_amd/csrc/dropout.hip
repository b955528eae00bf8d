// Memory-bound passes beside the linear layer's products: dropout, the gradient in front of the products (activation's slope and dropout's
// mask in one pass, with the column sums that are the bias gradient), partial sums put together, rows copied to an aligned pitch.
#include "linear_ops.h"

namespace sol {

// y = dropout(x) + residual.  One group of 8 columns per thread and step: one call of the generator (about 75 instructions, 20 of them 32-bit multiplications at a quarter of the
// rate), which 16 bits per element keep below the memory's time: 16384 x 8192 bf16 with a residual 149 us, 5.4 TB/s, a copy's rate; 12544 x 1366 18 us.  Small ones are a launch: 2.6 us.
template <typename T>
__global__ void __launch_bounds__(256) dropout_kernel(const T *x, const T *res, T *y, int cols, uint32_t groups, FastDiv dg, uint32_t total, const DropArgs d) {
    const uint32_t step = drop_step(d);
    for (uint32_t i = blockIdx.x * 256u + threadIdx.x; i < total; i += gridDim.x * 256u) {
        uint32_t row, g;
        dg.divmod(i, row, g);
        const size_t at = (size_t)row * cols + g * 8;
        const int nv = min(8, cols - (int)g * 8);
        float v[8], r[8];
        load8_any<T>(x + at, v, nv);
        if (res) load8_any<T>(res + at, r, nv);
        if (d.t) drop8(d, step, row, g, v);
        if (res) {
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] += r[e];
        }
        store8_any<T>(y + at, v, nv);
    }
}

sol_status launch_dropout(const void *x, const void *res, void *y, int rows, int cols, int dt, const DropArgs &d, hipStream_t st) {
    const uint32_t groups = (uint32_t)ceil_div(cols, 8), total = (uint32_t)rows * groups;
    const dim3 grid((unsigned)min((total + 255u) / 256u, 256u * 32u));
    if (dt == SOL_BF16)
        hipLaunchKernelGGL(dropout_kernel<bf16_t>, grid, dim3(256), 0, st, (const bf16_t *)x, (const bf16_t *)res, (bf16_t *)y, cols, groups, FastDiv(groups), total, d);
    else
        hipLaunchKernelGGL(dropout_kernel<float>, grid, dim3(256), 0, st, (const float *)x, (const float *)res, (float *)y, cols, groups, FastDiv(groups), total, d);
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

// Rows copied to an aligned pitch.  3904 x 5265 bf16 at any alignment: 14 us, 5.9 TB/s; 1021 x 1531 5.3 us, of which a launch and two round trips (whole groups, ends of rows) are most.
template <typename T> struct PadArgs {
    const T *x;
    T *out;
    long ld, ldo;
    int cols;
    uint32_t total;
    FastDiv dg;
    explicit PadArgs(const PadRows &p)
        : x(static_cast<const T *>(p.x)), out(static_cast<T *>(p.out)), ld(p.ld), ldo(p.ldo), cols(p.cols), total((uint32_t)p.rows * (uint32_t)(p.ldo / 8)), dg((uint32_t)(p.ldo / 8)) {}
};
template <typename T> __device__ __forceinline__ void pad_rows(const PadArgs<T> &p, uint32_t first, uint32_t stride) {
    for (uint32_t i = first; i < p.total; i += stride) {
        uint32_t row, g;
        p.dg.divmod(i, row, g);
        float v[8];
        load8_any<T>(p.x + row * p.ld + g * 8, v, min(8, p.cols - (int)g * 8));       // zeros where there are none
        store8_any<T>(p.out + row * p.ldo + g * 8, v, 8);
    }
}

// dz = act'(z) * dropout(dy), and sums of its columns in 32 bits before it is rounded.  A workgroup takes 256 columns of a chunk of rows: 32 groups of 8
// columns x 32 rows at a time, so that one round trip to memory serves 32 rows (with 8 rows at a time, us: 777 x 509 fp32 13.6, now 6.4; 2048 x 8192 bf16 21.4, now 19.1; four
// rows of a thread loaded together, with the code of five activations unrolled four times, 17.5 and 23.8).  Bound by memory where it is large: 2048 x 8192
// with SiLU 5.3 TB/s, 8192 x 16384 with GELU and dropout 157 us, 5.1 TB/s.
constexpr int DZ_ROWS = 32;
template <typename T>
__global__ void __launch_bounds__(32 * DZ_ROWS) linear_dz_kernel(const T *__restrict__ dy, long lddy, const T *__restrict__ z, T *__restrict__ dz, long ldz, int rows, int cols,
                                                                 int rows_per_chunk, int act, const DropArgs d, float *__restrict__ part, int tiles, int chunks,
                                                                 const PadArgs<T> pad) {
    if ((int)blockIdx.x >= tiles * chunks) {        // the copy of x that dW will read runs beside it
        pad_rows(pad, (blockIdx.x - (uint32_t)(tiles * chunks)) * (32u * DZ_ROWS) + threadIdx.x, (gridDim.x - (uint32_t)(tiles * chunks)) * (32u * DZ_ROWS));
        return;
    }
    const int tile = (int)blockIdx.x % tiles, chunk = (int)blockIdx.x / tiles;
    __shared__ float red[DZ_ROWS][256 + 4];
    const int gl = threadIdx.x & 31, rl = threadIdx.x >> 5, n = (tile * 32 + gl) * 8, nv = min(8, cols - n);
    const int r0 = chunk * rows_per_chunk, r1 = min(rows, r0 + rows_per_chunk);
    const uint32_t step = drop_step(d);
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; e++) sum[e] = 0.f;
    if (nv > 0 || (dz && n < ldz)) {
        for (int r = r0 + rl; r < r1; r += DZ_ROWS) {
            float v[8], s[8];
            load8_any<T>(dy + r * lddy + n, v, nv);
            if (act != SOL_ACT_NONE) load8_any<T>(z + (size_t)r * cols + n, s, nv);
            if (d.t) drop8(d, step, (uint32_t)r, (uint32_t)n >> 3, v);
            switch (act) {
#define SOL_ACT_CASE(A) case A: { _Pragma("unroll") for (int e = 0; e < 8; e++) v[e] *= act_slope(A, s[e]); break; }
                SOL_ACT_CASE(SOL_ACT_RELU)
                SOL_ACT_CASE(SOL_ACT_GELU)
                SOL_ACT_CASE(SOL_ACT_GELU_TANH)
                SOL_ACT_CASE(SOL_ACT_SILU)
#undef SOL_ACT_CASE
                default: break;
            }
#pragma unroll
            for (int e = 0; e < 8; e++) {
                v[e] = e < nv ? v[e] : 0.f;         // the columns behind the last are zeros in dz: the products' reduction runs over them
                sum[e] += v[e];
            }
            if (dz) store8_any<T>(dz + r * ldz + n, v, 8);
        }
    }
    if (!part) return;
#pragma unroll
    for (int e = 0; e < 8; e++) red[rl][gl * 8 + e] = sum[e];
    __syncthreads();
    const int c = tile * 256 + threadIdx.x;
    if (threadIdx.x >= 256 || c >= cols) return;
    float t = 0.f;
#pragma unroll
    for (int r = 0; r < DZ_ROWS; r++) t += red[r][threadIdx.x];
    part[(size_t)chunk * cols + c] = t;
}

// Two workgroups per CU, each with 32 rows or more; up to 64 rows are one chunk, whose sums are db themselves.
static int dz_rows_per_chunk(int rows, int cols) {
    const int want = max(1, 512 / ceil_div(cols, 256));
    return rows <= 64 ? 64 : (int)round_up((size_t)max(1, ceil_div(rows, want)), DZ_ROWS);
}
int linear_dz_chunks(int rows, int cols) { return rows > 0 ? ceil_div(rows, dz_rows_per_chunk(rows, cols)) : 0; }

sol_status launch_linear_dz(const void *dy, long lddy, const void *z, void *dz, long ldz, int rows, int cols, int act, const DropArgs &d, int dt, float *part, const PadRows &pad,
                            hipStream_t st) {
    const int rpc = dz_rows_per_chunk(rows, cols), tiles = ceil_div(dz ? (int)ldz : cols, 256), chunks = linear_dz_chunks(rows, cols), block = 32 * DZ_ROWS;
    const dim3 grid((unsigned)(tiles * chunks + (pad.x ? (int)min(((long)rows * (pad.ldo / 8) + block - 1) / block, 2048l) : 0)));
    if (dt == SOL_BF16)
        hipLaunchKernelGGL(linear_dz_kernel<bf16_t>, grid, dim3(block), 0, st, (const bf16_t *)dy, lddy, (const bf16_t *)z, (bf16_t *)dz, ldz, rows, cols, rpc, act, d, part, tiles,
                           chunks, PadArgs<bf16_t>(pad));
    else
        hipLaunchKernelGGL(linear_dz_kernel<float>, grid, dim3(block), 0, st, (const float *)dy, lddy, (const float *)z, (float *)dz, ldz, rows, cols, rpc, act, d, part, tiles,
                           chunks, PadArgs<float>(pad));
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

__global__ void __launch_bounds__(256) sums_kernel(const SumJobs jobs) {
    __shared__ float red[256];
    const int b = (int)blockIdx.x, k = b >= jobs.first[2] ? 2 : b >= jobs.first[1] ? 1 : 0;
    sum_parts(jobs.job[k], b - jobs.first[k], jobs.first[k + 1] - jobs.first[k], red);
}

sol_status launch_sums(SumJobs jobs, hipStream_t st) {
    jobs.first[0] = 0;
    for (int k = 0; k < 3; k++) {
        jobs.first[k + 1] = jobs.first[k] + (k < jobs.count ? sum_blocks(jobs.job[k]) : 0);
    }
    if (jobs.first[3] == 0) return SOL_OK;
    hipLaunchKernelGGL(sums_kernel, dim3((unsigned)jobs.first[3]), dim3(256), 0, st, jobs);
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

template <typename T> __global__ void __launch_bounds__(256) pad_rows_kernel(const PadArgs<T> p) { pad_rows(p, blockIdx.x * 256u + threadIdx.x, gridDim.x * 256u); }

sol_status launch_pad_rows(const PadRows &p, int dt, hipStream_t st) {
    const uint32_t total = (uint32_t)p.rows * (uint32_t)(p.ldo / 8);
    const dim3 grid((unsigned)min((total + 255u) / 256u, 256u * 32u));
    if (dt == SOL_BF16) hipLaunchKernelGGL(pad_rows_kernel<bf16_t>, grid, dim3(256), 0, st, PadArgs<bf16_t>(p));
    else hipLaunchKernelGGL(pad_rows_kernel<float>, grid, dim3(256), 0, st, PadArgs<float>(p));
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

}  // namespace sol
