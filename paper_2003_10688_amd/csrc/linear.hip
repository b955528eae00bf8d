// Linear layer for small batches:  y[m][o] = act( scale[o] * sum_i x[m][i] w[o][i] + shift[o] + res[m][o] ).
//
// With a batch of a few dozen rows the GEMM has one or two pixel tiles, so the convolution kernels, which
// parallelise over output tiles, leave most of the chip idle and walk the whole reduction in one workgroup.
// Here a workgroup owns 32 rows x 32 output features and its eight waves split the reduction between them;
// MFMA fragments (16 bytes of consecutive reduction elements of one row) are loaded straight from global
// memory into registers, sixteen steps in flight per wave (the kernel is latency-bound: for 2048 inputs that is
// the whole reduction in one round trip) -- x is tiny and
// L2-resident -- and the eight partial accumulators are added through LDS in a fixed order behind one barrier.
#include "linear_ops.h"

namespace sol {

template <typename T>
__global__ void __launch_bounds__(512) linear_kernel(const ConvArgs a) {
    constexpr int EPC = 16 / (int)sizeof(T);       // reduction elements per fragment
    constexpr int UN = 16, NWV = 8;                // k-steps in flight per wave; waves per workgroup
    __shared__ float red[NWV][32][33];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, lr = lane & 31, lh = lane >> 5;
    const int n0 = blockIdx.x * 32, m0 = blockIdx.y * 32;
    const int M = a.P, K = a.C, N = a.Cout;
    const T *__restrict__ xg = static_cast<const T *>(a.x);
    const T *__restrict__ wg = static_cast<const T *>(a.w);

    const bool wok = n0 + lr < N, xok = m0 + lr < M;
    const T *wp = wg + (size_t)(wok ? n0 + lr : 0) * a.Kp;
    const T *xp = xg + (size_t)(xok ? m0 + lr : 0) * K;
    const uint4 zero = make_uint4(0, 0, 0, 0);

    f32x16_t acc;
#pragma unroll
    for (int e = 0; e < 16; e++) acc[e] = 0.f;

    const int nsteps = (K + 2 * EPC - 1) / (2 * EPC);   // one step = 2*EPC reduction elements (both lane halves); K % EPC == 0
    for (int s0 = wave * UN; s0 < nsteps; s0 += NWV * UN) {
        // Every lane loads every step, from a clamped address (the start of a valid row), and what it must not use is
        // replaced by zeros after the last load is issued: a load behind a condition, or a use of its value between
        // the loads, makes the compiler wait for it before it issues the next one.
        uint4 fa[UN], fb[UN];
        auto k_of = [&](int u) { return (s0 + u) * 2 * EPC + lh * EPC; };   // < K, or: past the end / ragged last step
#pragma unroll
        for (int u = 0; u < UN; u++) {
            const int k = k_of(u), kk = k < K ? k : 0;
            fa[u] = *reinterpret_cast<const uint4 *>(wp + kk);
            fb[u] = *reinterpret_cast<const uint4 *>(xp + kk);
        }
        __builtin_amdgcn_sched_barrier(0);             // all 2 * UN loads are in flight before the first value is needed
#pragma unroll
        for (int u = 0; u < UN; u++) {
            const bool ok = k_of(u) < K;
            Mma<T>::run(acc, (ok && wok) ? fa[u] : zero, (ok && xok) ? fb[u] : zero);
        }
    }

    // accumulator register e of lane l: feature 8*(e/4) + 4*(l/32) + e%4, row l%32.  Every wave parks its partial
    // block, then each of the first 256 threads adds the eight partials of 4 outputs in wave order.
#pragma unroll
    for (int e = 0; e < 16; e++) red[wave][lr][8 * (e / 4) + 4 * lh + e % 4] = acc[e];
    __syncthreads();

    if (tid >= 256) return;
    const int row = tid >> 3, f0 = (tid & 7) * 4;
    const int m = m0 + row;
    if (m >= M) return;
    T *__restrict__ yg = static_cast<T *>(a.y);
    const T *__restrict__ resg = static_cast<const T *>(a.res);
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const int o = n0 + f0 + e;
        if (o >= N) break;
        float t = 0.f;
#pragma unroll
        for (int w = 0; w < NWV; w++) t += red[w][row][f0 + e];
        t = t * (a.scale ? a.scale[o] : 1.f) + (a.shift ? a.shift[o] : 0.f);
        if (resg) t += Elem<T>::load(resg + (size_t)m * N + o);
        if (a.act == SOL_ACT_RELU) t = __builtin_fmaxf(t, 0.f);
        Elem<T>::store(yg + (size_t)m * a.ldy + o, t);
    }
}

// unpadded 1x1 "convolution" over a [rows,1,1,C] tensor with few rows, rows a whole number of 16-byte fragments.  The
// kernel reads x as P dense rows: with padding a [n,1,1,C] input has more output pixels than input rows (the padding
// pixels hold act(shift + residual)), which the gather kernels handle.
bool linear_kernel_applies(const ConvArgs &a, int dt) {
    const int frag = 16 / (int)dtype_size(dt);     // a fragment is 16 bytes of one row: rows must be whole fragments
    return a.R == 1 && a.S == 1 && a.H == 1 && a.W == 1 && a.ph == 0 && a.pw == 0 && a.Ho == 1 && a.Wo == 1 && a.P == a.N &&
           a.pool == 0 && a.P <= 1024 && a.C % frag == 0;
}

sol_status launch_linear(const ConvArgs &a, int dt, hipStream_t st) {
    const dim3 grid(ceil_div(a.Cout, 32), ceil_div(a.P, 32));
    if (dt == SOL_BF16)
        hipLaunchKernelGGL(linear_kernel<bf16_t>, grid, dim3(512), 0, st, a);
    else
        hipLaunchKernelGGL(linear_kernel<float>, grid, dim3(512), 0, st, a);
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

// ---- weight streaming ---------------------------------------------------------------------------------------------
//   y[m][o] as above, for up to 128 rows (FUSED: for as many as the times at linear_rows_time say).  PB x CB blocks of 16 rows x 16 features per workgroup; eight waves split the
// reduction.  The job is to stream the weights at the rate of HBM, so their loads must be whole lines and many of them must be
// in flight: a wave loads 128 bytes of 8 weight rows per instruction into REGISTERS, NS stages ahead (with the rows of x in
// the LDS ring as well, LDS would hold one stage of both), turns them into MFMA fragments through a strip of LDS of its own, and
// takes the rows of x (resident in L2) by LDS DMA.  No wave waits for another before the partial sums meet.
// Measured, every layer on weights that no cache holds (us; before: 32-row linear_kernel below 16 MB of weights, the ring kernel
// of conv_gemm8.hip above): bf16 8192x8192, 64 rows 48.5 -> 35.6, 1 row 43.9 -> 30.2 (4.4 TB/s; the launch, the first round trip and
// the last sums are about 7 us of it); bf16 2048x1000, 64 rows 10.4 -> 7.9; 5000x5000, 37 rows 36.0 -> 23.4; fp32 4096x4096, 64
// rows 49.8 -> 30.2, 1 row 36.3 -> 18.2.  With 64 rows the rows of x are twice the bytes of the weights on the way into a CU.
// Weights packed so that a workgroup's stream is one contiguous run: 28.1 instead of 30.2 us with 1 row, 38.4 instead of 35.6
// with 64 (so the pitch of the rows is not what bounds it).
// FUSED: the epilogue of sol_linear_fused (activation, dropout, residual, z) in the place of scale, shift and ReLU.  It costs nothing that shows: 8 rows, 8192 -> 8192 with GELU and a
// residual 30.9 us (4.3 TB/s); 64 rows fp32 4096 -> 4096 with SiLU and a residual 24.5 us, where the products alone take 14.
template <typename T, int PB, int CB, int NS, bool FUSED>
__global__ void __launch_bounds__(512) linear_stream_kernel(const ConvArgs a, const LinearEpi epi, int nrt, int nft) {
#if defined(__HIP_DEVICE_COMPILE__)
    using namespace lds_pipe;
    constexpr int ES = (int)sizeof(T), BP = PB * 16, BC = CB * 16, NW = 8;
    constexpr int ROWB = 128, XL = BP / 8, WL = BC / 8, L = XL + WL;   // bytes of a row per stage; loads (8 rows each) per stage
    constexpr int XST = BP * ROWB, WST = BC * ROWB, LSTR = 68;
    constexpr int LDSB = NW * (NS * XST + WST), REDB = NW * PB * CB * 4 * LSTR * 4;
    static_assert(LDSB <= 160 * 1024 && REDB <= 160 * 1024 && (NS - 1) * L < 64, "LDS, vmcnt");
    __shared__ __align__(1024) unsigned char lds[LDSB > REDB ? LDSB : REDB];

    // the row tiles of one feature tile run on one XCD at the same time: the second finds the weights in L2
    const int grp = (int)blockIdx.x / (8 * nrt), in = (int)blockIdx.x - grp * 8 * nrt;
    const int ft = grp * 8 + (in & 7), m0 = (in >> 3) * BP, n0 = ft * BC;
    if (ft >= nft) return;

    const int tid = threadIdx.x, lane = tid & 63, lr = lane & 15, lg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lslot = lane & 7, lrow = lane >> 3;
    // rows of a length that 16 bytes do not divide lie in a padded copy: their last piece is read whole
    const unsigned xbytes = (unsigned)(a.P - 1) * a.ldx * ES + (((unsigned)a.C * ES + 15u) & ~15u), wbytes = (unsigned)a.Cout * a.Kp * ES;
    const __amdgpu_buffer_rsrc_t xr = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(a.x), 0, (int)xbytes, 0x00020000);
    const __amdgpu_buffer_rsrc_t wr = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(a.w), 0, (int)wbytes, 0x00020000);
    const __amdgpu_buffer_rsrc_t xnull = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(a.x), 0, 0, 0x00020000);
    const __amdgpu_buffer_rsrc_t wnull = __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(a.w), 0, 0, 0x00020000);

    // rows beyond the tensor get an out-of-range offset, which the hardware answers with zeros
    unsigned xo[XL], wo[WL];
#pragma unroll
    for (int i = 0; i < XL; i++) {
        const int row = i * 8 + lrow;
        xo[i] = m0 + row < a.P ? (unsigned)(m0 + row) * a.ldx * ES + ((lslot ^ swz<ROWB>(row)) << 4) : 0xffffffffu;
    }
#pragma unroll
    for (int i = 0; i < WL; i++) {
        const int row = i * 8 + lrow;
        wo[i] = n0 + row < a.Cout ? (unsigned)(n0 + row) * a.Kp * ES + (lslot << 4) : 0xffffffffu;
    }
    const int nst = (a.C * ES + ROWB - 1) / ROWB, tail = a.C * ES - (nst - 1) * ROWB;    // stages; bytes of the last one
    const int s0 = (int)((long)nst * wave / NW), s1 = (int)((long)nst * (wave + 1) / NW);
    const int n = s1 - s0;
    // the workgroups start at different stages: 39.1 -> 35.6 us (64 rows, 8192x8192), or all ask for the same columns of x at once.
    // The row tiles of one feature tile start at the same one, so that equal rows give equal bits (one stage apart was up to
    // 6 % faster with 65 to 128 rows: 65, bf16 3072 -> 16384, 44.3 against 47.1; 128, 8192 -> 8192, 54.9 against 55.9)
    int s = n > 0 ? s0 + (grp + wave) % n : s0, left = n;
    unsigned char *ring = lds + wave * (NS * XST), *strip = lds + NW * NS * XST + wave * WST;

    u32x4_t wq[NS][WL];
    auto issue = [&](auto B) {                             // stage s into slot B; beyond s1 through a size-0 resource -> zeros
        constexpr int buf = decltype(B)::value;
        const bool real = left > 0, last = s == nst - 1;     // the last stage of a row may be ragged (16-byte pieces)
        const __amdgpu_buffer_rsrc_t xq = real ? xr : xnull, wb = real ? wr : wnull;
#pragma unroll
        for (int i = 0; i < XL; i++) {
            const unsigned cut = (last && ((lslot ^ (int)swz<ROWB>(i * 8 + lrow)) << 4) >= tail) ? 0xffffffffu : 0u;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(xq, (__attribute__((address_space(3))) void *)(ring + buf * XST + i * 1024), 16, xo[i] | cut, s * ROWB, 0, 0);
        }
        const unsigned cut = (last && (lslot << 4) >= tail) ? 0xffffffffu : 0u;
#pragma unroll
        for (int i = 0; i < WL; i++) wq[buf][i] = __builtin_amdgcn_raw_buffer_load_b128(wb, wo[i] | cut, s * ROWB, 0);
        --left;
        if (++s == s1) s = s0;
    };
    f32x4_t acc[CB][PB];
#pragma unroll
    for (int i = 0; i < CB; i++)
#pragma unroll
        for (int j = 0; j < PB; j++) acc[i][j] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    const unsigned fsw = swz<ROWB>(lr);                    // block row bases are multiples of 16: the swizzle depends on lr only
    const unsigned fo0 = lr * ROWB + ((lg ^ fsw) << 4), fo1 = lr * ROWB + (((lg + 4) ^ fsw) << 4);
    const unsigned xb = lds_addr(ring), sb = lds_addr(strip);
    unsigned wst[WL];                                      // where this lane's piece of a weight row goes in the strip
#pragma unroll
    for (int i = 0; i < WL; i++) wst[i] = sb + (i * 8 + lrow) * ROWB + ((lslot ^ swz<ROWB>(i * 8 + lrow)) << 4);

    if (s0 < s1) {
        static_for<NS>([&](auto B) { issue(B); });
        const int rounds = (s1 - s0 + NS - 1) / NS;        // a wave ends on a whole round: its last stages may be zeros
        for (int r = 0; r < rounds; r++) {
            static_for<NS>([&](auto B) {
                constexpr int buf = decltype(B)::value;
                wait_vmcnt<(NS - 1) * L>();                // this stage has landed once only the NS - 1 behind it are outstanding
#pragma unroll
                for (int i = 0; i < WL; i++) asm volatile("ds_write_b128 %0, %1" ::"v"(wst[i]), "v"(wq[buf][i]) : "memory");
                u32x4_t fw[2][CB], fx[2][PB];
                static_for<PB>([&](auto J) { lds_read16<buf * XST + decltype(J)::value * 16 * ROWB>(fx[0][decltype(J)::value], xb + fo0); });
                static_for<PB>([&](auto J) { lds_read16<buf * XST + decltype(J)::value * 16 * ROWB>(fx[1][decltype(J)::value], xb + fo1); });
                // the wave's own writes: LDS operations of one wave are carried out in order
                static_for<CB>([&](auto I) { lds_read16<decltype(I)::value * 16 * ROWB>(fw[0][decltype(I)::value], sb + fo0); });
                static_for<CB>([&](auto I) { lds_read16<decltype(I)::value * 16 * ROWB>(fw[1][decltype(I)::value], sb + fo1); });
                wait_lgkmcnt<0>();
                static_for<2>([&](auto H) {
                    static_for<CB>([&](auto I) { landed(fw[decltype(H)::value][decltype(I)::value]); });
                    static_for<PB>([&](auto J) { landed(fx[decltype(H)::value][decltype(J)::value]); });
                });
                issue(B);                                  // the slot's data is in registers: refill it
#pragma unroll
                for (int h = 0; h < 2; h++)
#pragma unroll
                    for (int i = 0; i < CB; i++)
#pragma unroll
                        for (int j = 0; j < PB; j++) Mma16<T>::run(acc[i][j], fw[h][i], fx[h][j]);
            });
        }
        wait_vmcnt<0>();                                   // the zero-fill DMAs of the tail
    }
    __syncthreads();                                       // every ring is dead: the LDS becomes the parking place of the partial sums
    typedef float Block[4 * LSTR];
    Block *red = reinterpret_cast<Block *>(lds);           // [wave][block]

    // accumulator register e of lane l: feature 4 * (l / 16) + e, row l % 16 of its block
#pragma unroll
    for (int i = 0; i < CB; i++)
#pragma unroll
        for (int j = 0; j < PB; j++)
            *reinterpret_cast<float4 *>(&red[wave * PB * CB + j * CB + i][lg * LSTR + lr * 4]) = make_float4(acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]);
    __syncthreads();

    if constexpr (FUSED) {
        const uint32_t step = drop_step(epi.drop);
        for (int it = tid; it < BP * (BC / 8); it += NW * 64) {   // eight features of one row per thread, the waves' sums added in order
            const int cg = it % (BC / 8), row = it / (BC / 8), o = n0 + cg * 8, m = m0 + row, nv = min(8, a.Cout - o);
            if (nv <= 0 || m >= a.P) continue;
            const int blk = (row >> 4) * CB + (cg >> 1), at = (cg & 1) * 2 * LSTR + (row & 15) * 4;
            float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, bias8[8];
            load_bias8(epi.bias, o, nv, bias8);
#pragma unroll
            for (int w = 0; w < NW; w++) {
                const float4 p = *reinterpret_cast<const float4 *>(&red[w * PB * CB + blk][at]), q = *reinterpret_cast<const float4 *>(&red[w * PB * CB + blk][at + LSTR]);
                v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
                v[4] += q.x; v[5] += q.y; v[6] += q.z; v[7] += q.w;
            }
            finish8<T>(epi, step, m, o, a.Cout, nv, v, bias8);
        }
        return;
    }
    T *__restrict__ yg = static_cast<T *>(a.y);
    const T *__restrict__ resg = static_cast<const T *>(a.res);
    for (int it = tid; it < BP * (BC / 4); it += NW * 64) {   // four features of one row per thread, the waves' sums added in order
        const int cg = it % (BC / 4), row = it / (BC / 4), o = n0 + cg * 4, m = m0 + row, nv = min(4, a.Cout - o);
        if (nv <= 0 || m >= a.P) continue;
        const int blk = (row >> 4) * CB + (cg >> 2), at = (cg & 3) * LSTR + (row & 15) * 4;
        float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < NW; w++) {
            const float4 q = *reinterpret_cast<const float4 *>(&red[w * PB * CB + blk][at]);
            v[0] += q.x; v[1] += q.y; v[2] += q.z; v[3] += q.w;
        }
#pragma unroll
        for (int e = 0; e < 4; e++) {
            if (e >= nv) break;
            float t = v[e] * (a.scale ? a.scale[o + e] : 1.f) + (a.shift ? a.shift[o + e] : 0.f);
            if (resg) t += Elem<T>::load(resg + (size_t)m * a.Cout + o + e);
            v[e] = a.act == SOL_ACT_RELU ? __builtin_fmaxf(t, 0.f) : t;
        }
        T *yp = yg + (size_t)m * a.ldy + o;
        if (nv == 4 && ((a.ldy | a.Cout) & 3) == 0) {
            if constexpr (ES == 2) *reinterpret_cast<uint2 *>(yp) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
            else *reinterpret_cast<float4 *>(yp) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (e < nv) Elem<T>::store(yp + e, v[e]);
        }
    }
#endif
}

// Matrices of 16 MB and more belong to the ring kernel when the rows are many for the length of the reduction: x is most of what
// a workgroup fetches, and 64 features share it there, 32 here.  Each side counts for as much as the rounds of 256 workgroups that
// it makes are full.  The line is a fit to 624 timed layers (33..128 rows, 2048..8192 -> 4096..16384 in steps of 512), on which the choice
// is 0.6 % slower than the better of the two on average and 14 % at worst; always here: 2.9 % and 27 %.  bf16, ring kernel
// against here, us: 128 rows, 2048 -> 6656 16.4, 20.5; 2048 -> 8192 17.8, 20.9; 2048 -> 12800 30.1, 38.1; 4096 -> 8192 30.2, 32.7;
// 4096 -> 16384 65.5, 63.4; 8192 -> 8192 55.0, 54.5; 64 rows, 2048 -> 12800 21.1, 23.4; 4096 -> 8192 25.1, 21.7; 4096 -> 12800 37.2, 38.2.
// Features in multiples of 512: eight sets of tiles, one per XCD (128 rows, 2048 -> 6400, where every XCD reads the whole matrix:
// 39.4, 20.2).
static bool ring_kernel_is_better(const ConvArgs &a, int dt) {
    if (dt != SOL_BF16 || a.C % 128 != 0 || a.Cout % 512 != 0 || a.P <= 32 || (double)a.Cout * a.Kp * 2.0 < 16.0 * 1048576) return false;
    const auto fill = [](int n) { return (float)n / (float)(256 * ceil_div(n, 256)); };      // of the rounds that n workgroups make
    const int here = ceil_div(a.P, 64) * ceil_div(a.Cout, 32), tiles = ceil_div(a.P, 64) * ceil_div(a.Cout, 64);
    if (tiles < 200 && here <= 256) return false;
    const float e = here <= 256 ? 1.f : fill(here), er = fill(tiles);
    return (float)a.C * e * e * e <= (float)(tiles <= 256 ? 44 * a.P : 32 * a.P + 512) * er * er;
}

// Up to 128 rows (above, the 64-row tiles re-read the weights too often), and reductions that linear_kernel does not finish in
// one round trip: from 4 KB per row in bf16 (64 rows: 1024 -> 1000 features 6.6 against 6.3 us here, 2048 -> 1000 10.4 against 7.9;
// 13 rows, 512 -> 1000: 4.2 against 5.2; 128 rows, 1528 -> 1528: 7.7 against 8.5), from 2 KB in fp32, where its 32x32 blocks are a
// long chain of matrix instructions (9 rows, 512 -> 1000: 7.3 against 5.5; 64 rows, 128 -> 10: 4.8 against 5.6).
bool linear_stream_applies(const ConvArgs &a, int dt) {
    const double es = (double)dtype_size(dt);
    return linear_kernel_applies(a, dt) && a.P <= 128 && !ring_kernel_is_better(a, dt) && a.C * (int)es >= (dt == SOL_BF16 ? 4096 : 2048) && (double)a.P * a.C * es < 2147483648.0 && (double)a.Cout * a.Kp * es < 2147483648.0;
}

struct StreamGrid { int pb, nrt, nft; bool wide; };
static StreamGrid stream_grid(int rows, int features) {
    const int pb = rows <= 16 ? 1 : rows <= 32 ? 2 : 4, nrt = ceil_div(rows, pb * 16);
    // 32 features per workgroup, or 16 when that takes fewer row loads in the rounds that 256 workgroups of one per CU make
    const int n32 = ceil_div(features, 32), n16 = ceil_div(features, 16);
    const bool wide = (long)ceil_div(n32 * nrt, 256) * (pb * 16 + 32) <= (long)ceil_div(n16 * nrt, 256) * (pb * 16 + 16);
    return StreamGrid{pb, nrt, wide ? n32 : n16, wide};
}

template <typename T, bool FUSED> static sol_status launch_stream_typed(const ConvArgs &a, const LinearEpi &epi, hipStream_t st) {
    const StreamGrid sg = stream_grid(a.P, a.Cout);
    const int pb = sg.pb, nrt = sg.nrt, nft = sg.nft;
    const bool wide = sg.wide;
    const dim3 grid(ceil_div(nft, 8) * 8 * nrt), block(512);
#define STREAM(PB, CB, NS) hipLaunchKernelGGL((linear_stream_kernel<T, PB, CB, NS, FUSED>), grid, block, 0, st, a, epi, nrt, nft)
    if (wide) {
        if (pb == 1) STREAM(1, 2, 4);
        else if (pb == 2) STREAM(2, 2, 4);
        else STREAM(4, 2, 2);
    } else {
        if (pb == 1) STREAM(1, 1, 4);
        else if (pb == 2) STREAM(2, 1, 4);
        else STREAM(4, 1, 2);
    }
#undef STREAM
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

sol_status launch_linear_stream(const ConvArgs &a, int dt, hipStream_t st) {
    return dt == SOL_BF16 ? launch_stream_typed<bf16_t, false>(a, LinearEpi{}, st) : launch_stream_typed<float, false>(a, LinearEpi{}, st);
}

// The same with the epilogue of sol_linear_fused.  Rows of x and of the packed weights are whole fragments of 16 bytes.
// The time in us that tells it from the tile kernels (plan_gemm's is made the same way), negative where its 32-bit offsets do not reach: every round of 32 workgroups of an
// XCD (which has every eighth tile of features) costs a start, a sum over the waves and the stages of the longest wave.  Fitted to 150 products of 1 .. 256 rows,
// 64 .. 8192 -> 32 .. 16384, and held against 260 more of up to 4000 rows: the choice between the two kinds is 0.5 % slower than the better one on average and 35 % at worst
// (1500 rows, 1792 -> 80, bf16: 11.1 for 8.2).  Tile kernel against here, us: one row bf16 512 -> 1632 4.4, 4.7; 1728 -> 1200 7.8, 4.7; 48 rows 1024 -> 10272 6.4, 13.8;
// 3904 -> 3856 17.2, 12.0; 256 rows fp32 896 -> 3856 20.8, 27.7; 4544 -> 96 81, 25; 16 rows fp32 7040 -> 7552 125, 34.
double linear_rows_time(const GemmArgs &g, int dt) {
    const double es = (double)dtype_size(dt);
    if ((double)g.M * g.lda * es >= 2147483648.0 || (double)g.N * g.ldb * es >= 2147483648.0) return -1.0;
    static const double cost[2][3][2][2] = {                   // [fp32][16, 32 or 64 rows][16 or 32 features] a round, a stage
        {{{1.36, 0.28}, {1.65, 0.90}}, {{1.77, 0.38}, {2.07, 1.07}}, {{1.41, 0.70}, {2.53, 1.05}}},
        {{{1.61, 0.33}, {2.55, 0.84}}, {{3.28, 0.54}, {5.06, 1.14}}, {{2.31, 1.15}, {4.65, 2.09}}},
    };
    const StreamGrid sg = stream_grid(g.M, g.N);
    const double *c = cost[dt == SOL_F32][sg.pb >> 1][sg.wide];
    const long rounds = ((long)ceil_div(sg.nft, 8) * sg.nrt + 31) / 32, stages = ceil_div(ceil_div(g.K * (int)es, 128), 8);
    return rounds * (c[0] + c[1] * stages);
}
sol_status launch_linear_rows(const GemmArgs &g, int dt, hipStream_t st) {
    linear_tile_of_thread(GEMM_FORWARD) = 0;
    ConvArgs a{};
    a.x = g.a; a.w = g.b;
    a.P = g.M; a.C = g.K; a.ldx = (int)g.lda; a.Cout = g.N; a.Kp = (int)g.ldb;
    return dt == SOL_BF16 ? launch_stream_typed<bf16_t, true>(a, g.epi, st) : launch_stream_typed<float, true>(a, g.epi, st);
}

}  // namespace sol
