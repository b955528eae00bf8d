// The linear layer with its epilogue, its backward pass, and dropout: what their kernels share (internal).
//   forward   y = dropout(act(z)) + residual,  z = x W^T + bias
//   backward  dz = act'(z) * dropout(dy);  dx = dz W,  dW = dz^T x,  db = column sums of dz
#pragma once
#include "conv_common.h"

namespace sol {

// ---- dropout: a mask that is drawn wherever it is needed and stored nowhere ------------------------------------------------
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw: Parallel random numbers: as easy as 1, 2, 3, SC 2011).  One call gives the numbers of
// 8 neighbouring columns of one row, 16 bits each: key = seed, counter = (col / 8, row, call, step).  16 bits are enough for a
// probability (it is rounded to a multiple of 2^-16, and the factor of what is kept follows the rounded one, so the expectation is
// exact) and halve the generator's work, which otherwise costs more than the memory traffic of an elementwise pass.
struct DropArgs {
    uint32_t k0, k1, call;
    const uint32_t *step;       // device value, read by the kernel: a captured graph draws another mask when it changes; NULL: 0
    uint32_t t;                 // an element is kept if its 16 bits are >= t; 0: no dropout, 65536: nothing is kept
    float scale;                // 65536 / (65536 - t)
};

struct Philox4 { uint32_t w[4]; };

__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) {       // one instruction
#if defined(__HIP_DEVICE_COMPILE__)
    return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
#else
    return a ^ b ^ c;
#endif
}

__device__ __forceinline__ Philox4 philox(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
    for (int r = 0; r < 10; r++) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = xor3((uint32_t)(b >> 32), c1, k0);
        c2 = xor3((uint32_t)(a >> 32), c3, k1);
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

__device__ __forceinline__ uint32_t drop_step(const DropArgs &d) { return d.t && d.step ? *d.step : 0u; }

// v[e] = kept ? v[e] * scale : 0 for columns 8 * group .. + 7 of a row.  A select: what is dropped is 0 even where v is not finite.
__device__ __forceinline__ void drop8(const DropArgs &d, uint32_t step, uint32_t row, uint32_t group, float v[8]) {
    if (d.t >= 65536u) {
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = 0.f;
        return;
    }
    const Philox4 p = philox(group, row, d.call, step, d.k0, d.k1);
    const uint32_t th = d.t << 16;
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const uint32_t bits = e & 1 ? p.w[e >> 1] : p.w[e >> 1] << 16;      // the 16 bits on top; what is below them cannot change the comparison with th
        v[e] = bits >= th ? v[e] * d.scale : 0.f;
    }
}

// ---- activations ---------------------------------------------------------------------------------------------------------------
// Infinite z give the limits (silu(-inf) = -0, not NaN); a NaN stays one, except that ReLU maps it to 0 as in every other kernel here.
__device__ __forceinline__ float fast_exp(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }
__device__ __forceinline__ float half_exp(float s) { return __builtin_amdgcn_exp2f(s * -0.72134752044448170f); }     // exp(-s / 2)
__device__ __forceinline__ float at_least(float z, float lo) { return z < lo ? lo : z; }          // keeps a NaN
__device__ __forceinline__ float within(float z, float lim) { return z > lim ? lim : z < -lim ? -lim : z; }

// The normal distribution's tail, Q(a) = erfc(a / sqrt 2) / 2 = e * P(t) for a >= 0, with e = exp(-a^2 / 2) and t = 1 / (1 + 0.3 a).
// P is a polynomial fitted here to erfcx for the smallest relative error on [0, 14]: 1.64e-7 (1.9e-7 with its constants rounded to 32 bits), so the far negative side of GELU keeps
// its digits.  One exponential, one reciprocal and ten multiply-adds.
__device__ __forceinline__ float normal_tail(float a, float e) {
    const float t = __builtin_amdgcn_rcpf(1.f + 0.3f * a);
    float p = 0.03567459061741829f;
    p = p * t - 0.15720225870609283f;
    p = p * t + 0.20635199546813965f;
    p = p * t - 0.05368218198418617f;
    p = p * t + 0.12856081128120422f;
    p = p * t + 0.09991374611854553f;
    p = p * t + 0.12075391411781311f;
    p = p * t + 0.11962930113077164f;
    return p * t * e;
}
__device__ __forceinline__ float sigmoid(float u) { return __builtin_amdgcn_rcpf(1.f + fast_exp(-u)); }

constexpr float TANH_2C = 1.5957691216057308f, TANH_CUBE = 0.044715f;      // gelu_tanh(z) = z sigmoid(2 sqrt(2 / pi) (z + 0.044715 z^3))

__device__ __forceinline__ float act_forward(int act, float z) {
    switch (act) {
        case SOL_ACT_RELU: return __builtin_fmaxf(z, 0.f);
        case SOL_ACT_GELU: {                                                // max(z, 0) - |z| Q(|z|)
            const float a = __builtin_fminf(__builtin_fabsf(z), 100.f);
            return __builtin_fmaf(-a, normal_tail(a, half_exp(a * a)), at_least(z, 0.f));
        }
        case SOL_ACT_GELU_TANH: z = at_least(z, -100.f); return z * sigmoid(TANH_2C * (z + TANH_CUBE * z * z * z));
        case SOL_ACT_SILU: z = at_least(z, -100.f); return z * sigmoid(z);
        default: return z;
    }
}

// act'(z); beyond +-100 every slope is 0 or 1 in 32 bits, and the powers of z in the formulas stay finite
__device__ __forceinline__ float act_slope(int act, float z) {
    switch (act) {
        case SOL_ACT_RELU: return z > 0.f ? 1.f : 0.f;
        case SOL_ACT_GELU: {
            z = within(z, 100.f);
            const float e = half_exp(z * z), q = normal_tail(__builtin_fabsf(z), e);
            return (z < 0.f ? q : 1.f - q) + z * e * 0.3989422804014327f;
        }
        case SOL_ACT_GELU_TANH: {
            z = within(z, 100.f);
            const float s = sigmoid(TANH_2C * (z + TANH_CUBE * z * z * z));
            return s + z * s * (1.f - s) * TANH_2C * (1.f + 3.f * TANH_CUBE * z * z);
        }
        case SOL_ACT_SILU: {
            z = within(z, 100.f);
            const float s = sigmoid(z);
            return s + z * s * (1.f - s);
        }
        default: return 1.f;
    }
}

// ---- 8 neighbouring elements of a row at any alignment ------------------------------------------------------------------------
// Rows of odd length start at addresses that divide by the element size only.  Global loads and stores of 16 bytes need no more than
// that on this target (unaligned access mode), so the ends of rows are the only elements that travel one by one.
typedef lds_pipe::u32x4_t u32x4_any __attribute__((aligned(2)));

template <typename T> __device__ __forceinline__ void load8_any(const T *p, float v[8], int nv) {
    if (nv >= 8) {
        if constexpr (sizeof(T) == 2) {
            const lds_pipe::u32x4_t w = *reinterpret_cast<const u32x4_any *>(p);
#pragma unroll
            for (int e = 0; e < 4; e++) { v[2 * e] = __uint_as_float(w[e] << 16); v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u); }
        } else {
            const lds_pipe::u32x4_t a = reinterpret_cast<const u32x4_any *>(p)[0], b = reinterpret_cast<const u32x4_any *>(p)[1];
#pragma unroll
            for (int e = 0; e < 4; e++) { v[e] = __uint_as_float(a[e]); v[4 + e] = __uint_as_float(b[e]); }
        }
    } else {                                                   // no branch between the loads, so that they are under way together
#pragma unroll
        for (int e = 0; e < 8; e++) v[e] = 0.f;
        if (nv > 0) {
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = Elem<T>::load(p + min(e, nv - 1));
#pragma unroll
            for (int e = 1; e < 8; e++) v[e] = e < nv ? v[e] : 0.f;
        }
    }
}
template <typename T> __device__ __forceinline__ void store8_any(T *p, const float v[8], int nv) {
    if (nv >= 8) {
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<u32x4_any *>(p) = lds_pipe::u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
        } else {
            reinterpret_cast<u32x4_any *>(p)[0] = lds_pipe::u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
            reinterpret_cast<u32x4_any *>(p)[1] = lds_pipe::u32x4_t{__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])};
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++)
            if (e < nv) Elem<T>::store(p + e, v[e]);
    }
}

// ---- the epilogue of the forward product ----------------------------------------------------------------------------------------
struct LinearEpi {
    const float *bias;          // NULL: none
    const void *res;            // NULL: none
    void *y, *pre;              // pre: where z is stored, dense [M][N]; NULL: nowhere
    long ldr, ldy;
    int act;
    DropArgs drop;
};

// v: 8 sums of row m, columns n .. n + 7 (nv of them exist) -> z -> y.  bias8: the columns' bias.
template <typename T>
__device__ __forceinline__ void finish8(const LinearEpi &e, uint32_t step, int m, int n, int N, int nv, float v[8], const float bias8[8]) {
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] += bias8[i];
    if (e.pre) store8_any<T>(static_cast<T *>(e.pre) + (size_t)m * N + n, v, nv);
    if (e.act != SOL_ACT_NONE) {
        switch (e.act) {        // one uniform branch for 8 elements
#define SOL_ACT_CASE(A) case A: { _Pragma("unroll") for (int i = 0; i < 8; i++) v[i] = act_forward(A, v[i]); break; }
            SOL_ACT_CASE(SOL_ACT_RELU)
            SOL_ACT_CASE(SOL_ACT_GELU)
            SOL_ACT_CASE(SOL_ACT_GELU_TANH)
            SOL_ACT_CASE(SOL_ACT_SILU)
#undef SOL_ACT_CASE
        }
    }
    if (e.drop.t) drop8(e.drop, step, (uint32_t)m, (uint32_t)n >> 3, v);
    if (e.res) {
        float r[8];
        load8_any<T>(static_cast<const T *>(e.res) + m * e.ldr + n, r, nv);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] += r[i];
    }
    store8_any<T>(static_cast<T *>(e.y) + m * e.ldy + n, v, nv);
}
// n is a multiple of 8 and the bias 16-byte aligned
__device__ __forceinline__ void load_bias8(const float *bias, int n, int nv, float b[8]) {
    if (bias && nv >= 8) {
        const float4 lo = *reinterpret_cast<const float4 *>(bias + n), hi = *reinterpret_cast<const float4 *>(bias + n + 4);
        b[0] = lo.x; b[1] = lo.y; b[2] = lo.z; b[3] = lo.w; b[4] = hi.x; b[5] = hi.y; b[6] = hi.z; b[7] = hi.w;
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) b[e] = bias && e < nv ? bias[n + e] : 0.f;
    }
}

// The same for two groups of one product's results at once, whose arithmetic is independent and fills the waits of one another: columns n .. n + 7 and n + 32 .. n + 39 of row m (BESIDE:
// both halves of a 128-byte line of bf16 are stored one behind the other), or of rows m and m + 16.
template <typename T, bool BESIDE>
__device__ __forceinline__ void finish_two(const LinearEpi &e, uint32_t step, int m, int n, int M, int N, float (&v)[2][8]) {
    const int m1 = BESIDE ? m : m + 16, n1 = BESIDE ? n + 32 : n;
    const int nv0 = m < M ? min(8, N - n) : 0, nv1 = m1 < M ? min(8, N - n1) : 0;
    const size_t zat = (size_t)m * N + n, yat = (size_t)m * e.ldy + n, rat = (size_t)m * e.ldr + n;
    const size_t zto = BESIDE ? 32 : (size_t)16 * N, yto = BESIDE ? 32 : (size_t)16 * e.ldy, rto = BESIDE ? 32 : (size_t)16 * e.ldr;
    float b[2][8];
    load_bias8(e.bias, n, min(8, N - n), b[0]);
    if constexpr (BESIDE) load_bias8(e.bias, n1, min(8, N - n1), b[1]);
#pragma unroll
    for (int c = 0; c < 8; c++) { v[0][c] += b[0][c]; v[1][c] += b[BESIDE][c]; }
    if (e.pre) {
        if (nv0 > 0) store8_any<T>(static_cast<T *>(e.pre) + zat, v[0], nv0);
        if (nv1 > 0) store8_any<T>(static_cast<T *>(e.pre) + zat + zto, v[1], nv1);
    }
    if (e.act != SOL_ACT_NONE) {
        switch (e.act) {
#define SOL_ACT_CASE(A) case A: { _Pragma("unroll") for (int i = 0; i < 16; i++) v[i >> 3][i & 7] = act_forward(A, v[i >> 3][i & 7]); break; }
            SOL_ACT_CASE(SOL_ACT_RELU)
            SOL_ACT_CASE(SOL_ACT_GELU)
            SOL_ACT_CASE(SOL_ACT_GELU_TANH)
            SOL_ACT_CASE(SOL_ACT_SILU)
#undef SOL_ACT_CASE
        }
    }
    if (e.drop.t) {
        drop8(e.drop, step, (uint32_t)m, (uint32_t)n >> 3, v[0]);
        drop8(e.drop, step, (uint32_t)m1, (uint32_t)n1 >> 3, v[1]);
    }
    if (e.res) {
        float r[2][8];
        load8_any<T>(static_cast<const T *>(e.res) + rat, r[0], nv0);
        load8_any<T>(static_cast<const T *>(e.res) + rat + rto, r[1], nv1);
#pragma unroll
        for (int c = 0; c < 8; c++) { v[0][c] += r[0][c]; v[1][c] += r[1][c]; }
    }
    if (nv0 > 0) store8_any<T>(static_cast<T *>(e.y) + yat, v[0], nv0);
    if (nv1 > 0) store8_any<T>(static_cast<T *>(e.y) + yat + yto, v[1], nv1);
}

// ---- launchers --------------------------------------------------------------------------------------------------------------------
// D[p][c] = sum_k A(p, k) B(c, k) for p < M, c < N, k < K.  An operand is stored along k ([p][k], ld elements between its rows) or across
// it ([k][p]).  Base addresses and pitches are multiples of 16 bytes; an operand stored along k ends its rows with zeros up to a multiple of
// 128 bytes, or has K a multiple of 16 bytes' worth of elements and a_cut set.
struct GemmPlan {
    int tile;                   // 64, 128 or 256 rows and columns
    int split;                  // > 1: the reduction in so many parts; part s goes to `part` + s * M * N (fp32, dense), nothing else is written
    double us;                  // estimate of the time
};
struct GemmArgs {
    const void *a, *b;
    long lda, ldb;
    int a_row, b_row;           // bytes of a row that may be read (the pitch where it is this library's own buffer)
    int a_cut;                  // A, stored along k: elements >= K of a row are not zeros and have to be masked
    int M, N, K;
    GemmPlan plan;
    float *part;
    void *out; long ldo; int out_dt;    // plain result (no epilogue)
    LinearEpi epi;
    int ntp, ntc, steps;        // set by the launcher: tiles of rows and columns; stages of a part
};
enum GemmKind { GEMM_FORWARD, GEMM_DX, GEMM_DW };
GemmPlan plan_gemm(int M, int N, int K, int dt, bool may_split);
// whether dx and dW are faster in one launch than as planned one by one; *px, *pw: their plans then
bool plan_pair(int m, int in_f, int out_f, int dt, const GemmPlan &dx, const GemmPlan &dw, GemmPlan *px, GemmPlan *pw);
sol_status launch_linear_gemm(const GemmArgs &a, int dt, GemmKind kind, hipStream_t st);
int &linear_tile_of_thread(GemmKind kind);                     // sol_debug_linear_tile
double linear_rows_time(const GemmArgs &a, int dt);            // forward, weights streamed past few rows (linear.hip): estimate of its time, negative where it cannot run
sol_status launch_linear_rows(const GemmArgs &a, int dt, hipStream_t st);
// A copy of [rows][cols] (pitch ld, any alignment) to dense rows of ldo elements, the rest of each row zeros
struct PadRows {
    const void *x;
    void *out;
    long ld, ldo;               // ldo: a multiple of 8
    int rows, cols;
};
constexpr size_t MAX_PAD_GROUPS = 0x100000000ull - 0x200000ull;         // rows * (ldo / 8) at most: counted in 32 bits, and a grid has 2^21 threads at most
sol_status launch_pad_rows(const PadRows &p, int dt, hipStream_t st);
sol_status launch_dropout(const void *x, const void *res, void *y, int rows, int cols, int dt, const DropArgs &d, hipStream_t st);
// dz = act'(z) * dropout(dy) into rows of ldz elements (zeros behind the columns) unless dz is NULL; column sums of dz over every chunk of rows into part
// [linear_dz_chunks][cols] unless that is NULL; in the same launch the copy `pad` of as many rows, unless its x is NULL
sol_status launch_linear_dz(const void *dy, long lddy, const void *z, void *dz, long ldz, int rows, int cols, int act, const DropArgs &d, int dt, float *part, const PadRows &pad,
                            hipStream_t st);
int linear_dz_chunks(int rows, int cols);
// Sums of parts: out[i] = part[0][i] + part[1][i] + ..., in an order that the shape alone fixes; zeros where there are no parts.
struct SumJob {
    const float *part;
    int nsplit;
    long n;
    void *out;
    int out_dt;
};
// Parts are read once, coalesced.  256 threads sum 256 elements, or, where there are more than 16 parts (column sums), 32 elements in eight groups that take the parts in turn
// (8192 columns, 64 parts: 4.6 us, 10.8 with one thread per column).
inline int sum_blocks(const SumJob &j) { const int wide = j.nsplit > 16 ? 32 : 256; return (int)min((j.n + wide - 1) / wide, 8192l); }
__device__ __forceinline__ void sum_parts(const SumJob &j, int block, int blocks, float *red) {        // red: 256 floats of LDS
    const int groups = j.nsplit > 16 ? 8 : 1, wide = 256 / groups, lane = threadIdx.x & (wide - 1), group = threadIdx.x / wide;
    const long n = j.n;
    for (long i0 = (long)block * wide; i0 < n; i0 += (long)blocks * wide) {
        const long i = i0 + lane;
        const float *p = j.part + i;
        float s = 0.f;
        if (i < n) {
            int q = group;
            for (; q + 3 * groups < j.nsplit; q += 4 * groups) {          // four loads under way at a time
                const float v0 = p[q * n], v1 = p[(q + groups) * n], v2 = p[(q + 2 * groups) * n], v3 = p[(q + 3 * groups) * n];
                s += v0;
                s += v1;
                s += v2;
                s += v3;
            }
            for (; q < j.nsplit; q += groups) s += p[q * n];
        }
        if (groups > 1) {
            red[group * 32 + lane] = s;
            __syncthreads();
            s = 0.f;
            for (int g = 0; g < groups; g++) s += red[g * 32 + lane];
            __syncthreads();
        }
        if (group == 0 && i < n) {
            if (j.out_dt == SOL_BF16) Elem<bf16_t>::store(static_cast<bf16_t *>(j.out) + i, s);
            else static_cast<float *>(j.out)[i] = s;
        }
    }
}
struct SumJobs {                // up to three of them in one launch
    SumJob job[3];
    int first[4];               // set by the launcher: workgroups in front of each job
    int count;
    void add(const float *part, int nsplit, long n, void *out, int out_dt) { job[count++] = SumJob{part, nsplit, n, out, out_dt}; }
};
sol_status launch_sums(SumJobs jobs, hipStream_t st);
// dx and dW as plan_pair has them, and a sum whose parts are there already, in one launch
sol_status launch_linear_pair(GemmArgs dx, GemmArgs dw, const SumJob &sum, int dt, hipStream_t st);

}  // namespace sol
