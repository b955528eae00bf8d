// The matrix products of the linear layer, forward and backward:  D[p][c] = sum_k A(p, k) B(c, k).
//
//   forward  z = x W^T     A = x  [m][in]   along k    B = W  [out][in]  along k
//   dx       = dz W        A = dz [m][out]  along k    B = W  [out][in]  across k
//   dW       = dz^T x      A = dz [m][out]  across k   B = x  [m][in]    across k
//
// One kernel for the three.  Four waves share a tile of rows x columns; stages of 64 bytes of reduction per row (32 bf16, 16 fp32)
// travel memory -> LDS by DMA through a ring of NS stages, each wave multiplies its quarter with 32x32 matrix instructions.
// An operand along k lies in LDS as rows of 64 bytes, read as 16-byte fragments; one across k lies as it is in memory, rows of
// columns, and is transposed on the way to registers (ds_read_b64_tr_b16 for bf16, four 4-byte reads for fp32), so no transposed copy of W, dz or x is
// ever made.  Slots are permuted on the global side of the DMA so that neither kind of read meets a bank twice.
//
// Why two workgroups of four waves per CU, and not one of eight on a tile twice as large: every wave of a workgroup waits at the
// same barrier, starts up and writes its results at the same time, and nothing multiplies meanwhile; two workgroups drift apart, and one's
// epilogue (activation, dropout's generator: up to 15 % of the products' time on the vector units) runs beside the other's products.
#include "linear_ops.h"

namespace sol {

using namespace lds_pipe;

typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));

// One fragment: 16 bytes of reduction of one row or column per lane.  bf16 across k arrives in two halves.
template <typename T, bool ACROSS> struct Frag;
template <typename T> struct Frag<T, false> {
    u32x4_t v;
    template <int OFF, int RB> __device__ __forceinline__ void read(unsigned addr) { lds_read16<OFF>(v, addr); }
    __device__ __forceinline__ void land() { landed(v); }
    __device__ __forceinline__ u32x4_t get() const { return v; }
    static constexpr int READS = 1;
};
template <> struct Frag<bf16_t, true> {
    u32x2_t lo, hi;
    // lane s of 16 names 8 bytes of row s / 4; lane i receives column i of rows 0..3 (lo) and of rows 4..7 (hi)
    template <int OFF, int RB> __device__ __forceinline__ void read(unsigned addr) {
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=&v"(lo) : "v"(addr), "n"(OFF));
        asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=&v"(hi) : "v"(addr), "n"(OFF + 4 * RB));
    }
    __device__ __forceinline__ void land() { asm volatile("" : "+v"(lo), "+v"(hi)); }
    __device__ __forceinline__ u32x4_t get() const { return u32x4_t{lo.x, lo.y, hi.x, hi.y}; }
    static constexpr int READS = 2;
};
template <> struct Frag<float, true> {
    unsigned e0, e1, e2, e3;
    template <int OFF, int RB> __device__ __forceinline__ void read(unsigned addr) {
        asm volatile("ds_read_b32 %0, %1 offset:%2" : "=&v"(e0) : "v"(addr), "n"(OFF));
        asm volatile("ds_read_b32 %0, %1 offset:%2" : "=&v"(e1) : "v"(addr), "n"(OFF + RB));
        asm volatile("ds_read_b32 %0, %1 offset:%2" : "=&v"(e2) : "v"(addr), "n"(OFF + 2 * RB));
        asm volatile("ds_read_b32 %0, %1 offset:%2" : "=&v"(e3) : "v"(addr), "n"(OFF + 3 * RB));
    }
    __device__ __forceinline__ void land() { asm volatile("" : "+v"(e0), "+v"(e1), "+v"(e2), "+v"(e3)); }
    __device__ __forceinline__ u32x4_t get() const { return u32x4_t{e0, e1, e2, e3}; }
    static constexpr int READS = 4;
};

// Where one operand's tile lies: BR rows (or columns) of the product, 64 bytes of reduction.
template <typename T, bool ACROSS, int BR> struct Tile {
    static constexpr int ES = (int)sizeof(T), BK = 64 / ES, RB = ACROSS ? BR * ES : 64;     // bytes of a row in LDS
    static constexpr int BYTES = BR * 64, SEGS = BYTES / 1024;                              // DMA instructions of 64 lanes x 16 bytes

    // permutation of the 16-byte slots of a row across k: transposing reads take 64 bytes of four neighbouring rows at once, 4-byte reads
    // 128 bytes of rows k and k + 4
    static __device__ __forceinline__ int permute(int k) {
        if constexpr (ES == 2) return RB >= 256 ? (k & 3) << 2 : ((k >> 1) & 1) << 2;
        else return RB >= 256 ? ((k >> 2) & 1) << 3 : 0;
    }
    // byte offset, from the tile's corner in memory, of what this lane's part of DMA instruction `seg` brings
    static __device__ __forceinline__ unsigned offset(int seg, int lane, unsigned pitch) {
        if constexpr (ACROSS) {
            const int at = seg * 1024 + lane * 16, k = at / RB, slot = (at % RB) / 16;
            return (unsigned)k * pitch + (unsigned)((slot ^ permute(k)) << 4);
        } else {
            const int row = seg * 16 + (lane >> 2);
            return (unsigned)row * pitch + (unsigned)(((lane & 3) ^ swz<64>(row)) << 4);
        }
    }
    // LDS offset of this lane's fragment of the first k-step for the 32-wide block `blk`
    static __device__ __forceinline__ unsigned frag(int blk, int lane) {
        const int lr = lane & 31, lh = lane >> 5;
        if constexpr (!ACROSS) {
            return (unsigned)((blk * 32 + lr) * 64 + ((lh ^ swz<64>(lr)) << 4));
        } else if constexpr (ES == 2) {
            const int s = lane & 15, k = 8 * lh + (s >> 2), slot = blk * 4 + ((lane >> 4) & 1) * 2 + ((s & 3) >> 1);
            return (unsigned)(k * RB + ((slot ^ permute(k)) << 4) + (s & 1) * 8);
        } else {
            const int k = 4 * lh, slot = blk * 8 + (lr >> 2);
            return (unsigned)(k * RB + ((slot ^ permute(k)) << 4) + (lr & 3) * 4);
        }
    }
};

// KIND: GEMM_FORWARD (A, B along k), GEMM_DX (B across), GEMM_DW (both across).  WP x WC = 4 waves of TP x TC blocks of 32 x 32.
template <typename T, GemmKind KIND, int WP, int WC, int TP, int TC, int NS, int PERCU>
__global__ void __launch_bounds__(256, PERCU) linear_gemm_kernel(const GemmArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool AX = KIND == GEMM_DW, BX = KIND != GEMM_FORWARD;
    constexpr int NW = 4, ES = (int)sizeof(T), BP = WP * TP * 32, BC = WC * TC * 32, BK = 64 / ES;
    using TA = Tile<T, AX, BP>;
    using TB = Tile<T, BX, BC>;
    using FA = Frag<T, AX>;
    using FB = Frag<T, BX>;
    constexpr int STAGE = TA::BYTES + TB::BYTES, XL = TA::SEGS / NW, WL = TB::SEGS / NW, L = XL + WL;
    constexpr int READS = TP * FA::READS + TC * FB::READS;     // LDS instructions of a k-step
    constexpr int ERS = TC * 32 + 4;                           // floats of a row in the epilogue's strips
    static_assert(WP * WC == NW && TA::SEGS % NW == 0 && TB::SEGS % NW == 0, "waves");
    static_assert(NW * 32 * ERS * 4 <= NS * STAGE && NS >= 3 && (NS - 2) * L < 64, "strips in the ring; vmcnt");
    __shared__ __align__(1024) unsigned char lds[NS * STAGE];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wc = wave / WP;

    // Tile order.  Workgroups go to the eight XCDs in turn; each XCD takes a contiguous run of a sequence that walks the columns of eight rows
    // of tiles, so that what runs on it at one time is a block of about eight by eight tiles and shares its operands in that L2.
    const int ntiles = a.ntp * a.ntc, per = (ntiles + 7) >> 3;
    const int split = (int)blockIdx.x / (per * 8), bid = (int)blockIdx.x - split * per * 8;
    const int t = (bid & 7) * per + (bid >> 3);
    if ((bid >> 3) >= per || t >= ntiles) return;
    const int g = t / (8 * a.ntc), in = t - g * 8 * a.ntc, rows = min(8, a.ntp - g * 8);
    const int p0 = (g * 8 + in % rows) * BP, c0 = (in / rows) * BC;

    const int nk = (a.K + BK - 1) / BK, s0 = split * a.steps, s1 = min(nk, s0 + a.steps);   // this part's stages

    // The operands' corners move along the reduction as scalars, and so does the number of bytes left behind them: what lies behind the last
    // row, or behind the last stage, is out of range and arrives as zeros.
    const unsigned apitch = (unsigned)(a.lda * ES), bpitch = (unsigned)(a.ldb * ES);
    const size_t astep = AX ? (size_t)BK * apitch : 64, bstep = BX ? (size_t)BK * bpitch : 64;
    const size_t a0 = (AX ? (size_t)p0 * ES : (size_t)p0 * apitch) + s0 * astep, b0 = (BX ? (size_t)c0 * ES : (size_t)c0 * bpitch) + s0 * bstep;
    const unsigned char *ap = static_cast<const unsigned char *>(a.a) + a0, *bp = static_cast<const unsigned char *>(a.b) + b0;
    long aleft = (long)a.a_bytes - (long)a0, bleft = (long)a.b_bytes - (long)b0;

    unsigned ao[XL], bo[WL];
#pragma unroll
    for (int i = 0; i < XL; i++) ao[i] = TA::offset(wave * XL + i, lane, apitch);
#pragma unroll
    for (int i = 0; i < WL; i++) bo[i] = TB::offset(wave * WL + i, lane, bpitch);
    // A along k whose rows do not end with zeros: the slots of the last stage that lie behind K (the row permutation is the same for every i)
    unsigned cut = 0;
    if constexpr (!AX) cut = a.a_cut && (nk - 1) * 64 + (((lane & 3) ^ swz<64>(lane >> 2)) << 4) >= a.K * ES ? 0xffffffffu : 0u;

    int left = s1 - s0, at = s0;                               // stages not yet requested; the next one
    __amdgpu_buffer_rsrc_t ar, br;
    unsigned acut = 0;
    auto next_stage = [&]() {                                  // resources of the next stage to request
        const bool real = left > 0;
        const unsigned an = real && aleft > 0 ? (unsigned)min(aleft, 0xfffffff0L) : 0u, bn = real && bleft > 0 ? (unsigned)min(bleft, 0xfffffff0L) : 0u;
        ar = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(ap), 0, (int)an, 0x00020000);
        br = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(bp), 0, (int)bn, 0x00020000);
        if constexpr (!AX) acut = at == nk - 1 ? cut : 0u;
        ap += astep; bp += bstep; aleft -= (long)astep; bleft -= (long)bstep;
        --left; ++at;
    };
    auto request = [&](auto I, int buf) {                      // the I-th DMA of this wave for that stage
        constexpr int i = decltype(I)::value;
        unsigned char *la = lds + buf * STAGE, *lb = la + TA::BYTES;
        if constexpr (i < XL)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ar, (__attribute__((address_space(3))) void *)(la + (wave * XL + i) * 1024), 16, ao[i] | acut, 0, 0, 0);
        else
            __builtin_amdgcn_raw_ptr_buffer_load_lds(br, (__attribute__((address_space(3))) void *)(lb + (wave * WL + i - XL) * 1024), 16, bo[i - XL], 0, 0, 0);
    };
#pragma unroll
    for (int s = 0; s < NS; s++) {
        next_stage();
        static_for<L>([&](auto I) { request(I, s); });
    }

    f32x16_t acc[TC][TP];
#pragma unroll
    for (int i = 0; i < TC; i++)
#pragma unroll
        for (int j = 0; j < TP; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0.f;

    unsigned fa0[TP], fb0[TC];
#pragma unroll
    for (int j = 0; j < TP; j++) fa0[j] = lds_addr(lds) + TA::frag(wp * TP + j, lane);
#pragma unroll
    for (int i = 0; i < TC; i++) fb0[i] = lds_addr(lds) + TA::BYTES + TB::frag(wc * TC + i, lane);

    FA fa[2][TP];
    FB fb[2][TC];
    auto read_step = [&](auto Q, unsigned sb) {                // fragments of k-step Q (0, 1) of the stage at byte offset sb
        constexpr int q = decltype(Q)::value;
        if constexpr (!BX) {
            const unsigned w = xor_add(fb0[0], q << 5, sb);
            static_for<TC>([&](auto I) { constexpr int i = decltype(I)::value; fb[q][i].template read<i * 2048, 64>(w); });
        } else {
            static_for<TC>([&](auto I) { constexpr int i = decltype(I)::value; fb[q][i].template read<q *(BK / 2) * TB::RB, TB::RB>(fb0[i] + sb); });
        }
        if constexpr (!AX) {
            const unsigned x = xor_add(fa0[0], q << 5, sb);
            static_for<TP>([&](auto J) { constexpr int j = decltype(J)::value; fa[q][j].template read<j * 2048, 64>(x); });
        } else {
            static_for<TP>([&](auto J) { constexpr int j = decltype(J)::value; fa[q][j].template read<q *(BK / 2) * TA::RB, TA::RB>(fa0[j] + sb); });
        }
    };
    auto land = [&](auto Q) {
        constexpr int q = decltype(Q)::value;
        static_for<TC>([&](auto I) { fb[q][decltype(I)::value].land(); });
        static_for<TP>([&](auto J) { fa[q][decltype(J)::value].land(); });
    };
    auto multiply = [&](auto Q, auto &&between) {
        constexpr int q = decltype(Q)::value;
        static_for<TC * TP>([&](auto U) {
            constexpr int u = decltype(U)::value, i = u / TP, j = u % TP;
            Mma<T>::run(acc[i][j], fb[q][i].get(), fa[q][j].get());
            between(U);
        });
    };
    constexpr std::integral_constant<int, 0> Q0{};
    constexpr std::integral_constant<int, 1> Q1{};

    wait_vmcnt<(NS - 1) * L>();                                // the first stage has landed
    __builtin_amdgcn_s_barrier();
    read_step(Q0, 0u);

    unsigned sb = 0;
    int buf = 0;
    for (int s = s0; s < s1; s++) {
        const unsigned sbn = sb + STAGE == NS * STAGE ? 0u : sb + STAGE;
        read_step(Q1, sb);
        wait_lgkmcnt<(READS < 15 ? READS : 0)>();              // the first k-step's fragments are here
        land(Q0);
        multiply(Q0, [](auto) {});
        wait_lgkmcnt<0>();                                     // all of this stage is in registers
        land(Q1);
        wait_vmcnt<(NS - 2) * L>();                            // the next stage has landed
        __builtin_amdgcn_s_barrier();                          // ... for every wave, and nobody reads this one any more: it can be refilled
        read_step(Q0, sbn);
        next_stage();
        multiply(Q1, [&](auto U) {
            constexpr int u = decltype(U)::value;
            if constexpr (u < L) request(U, buf);
            if constexpr (u == TC * TP - 1 && L > TC * TP)
                static_for<(L > TC * TP ? L - TC * TP : 0)>([&](auto V) { request(std::integral_constant<int, TC * TP + decltype(V)::value>{}, buf); });
        });
        buf = buf + 1 == NS ? 0 : buf + 1;
        sb = sbn;
    }
    wait_lgkmcnt<0>();                                         // the fragments requested behind the last stage
    land(Q0);
    wait_vmcnt<0>();                                           // ... and its DMAs, zeros into dead slots
    __builtin_amdgcn_s_barrier();                              // the ring becomes the epilogue's strips

    // Epilogue: a wave takes 32 rows at a time through a strip of LDS of its own, so that a lane has 8 neighbouring columns of one row
    // (one call of dropout's generator) and a store writes whole lines.
    constexpr int LPR = TC * 4, RPS = 64 / LPR;
    float *strip = reinterpret_cast<float *>(lds) + wave * (32 * ERS);
    const int lr = lane & 31, lh = lane >> 5, erow = lane / LPR, ecol = (lane % LPR) * 8;
    const int n = c0 + wc * TC * 32 + ecol, nv = min(8, a.N - n);
    float bias8[8];
    uint32_t step = 0;
    if constexpr (KIND == GEMM_FORWARD) {
        load_bias8(a.epi.bias, n, nv, bias8);
        step = drop_step(a.epi.drop);
    }
    static_for<TP>([&](auto J) {
        constexpr int j = decltype(J)::value;
#pragma unroll
        for (int i = 0; i < TC; i++)
#pragma unroll
            for (int e = 0; e < 4; e++)
                *reinterpret_cast<float4 *>(strip + lr * ERS + i * 32 + 8 * e + 4 * lh) = make_float4(acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]);
        wave_lds_fence();
#pragma unroll 1
        for (int r = erow; r < 32; r += RPS) {
            const int m = p0 + (wp * TP + j) * 32 + r;
            if (m >= a.M || nv <= 0) continue;
            const float4 lo = *reinterpret_cast<const float4 *>(strip + r * ERS + ecol), hi = *reinterpret_cast<const float4 *>(strip + r * ERS + ecol + 4);
            float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            if (a.nsplit > 1) store8_any<float>(a.part + ((size_t)split * a.M + m) * a.N + n, v, nv);
            else if constexpr (KIND == GEMM_FORWARD) finish8<T>(a.epi, step, m, n, a.N, nv, v, bias8);
            else if (a.out_dt == SOL_F32) store8_any<float>(static_cast<float *>(a.out) + m * a.ldo + n, v, nv);
            else store8_any<T>(static_cast<T *>(a.out) + m * a.ldo + n, v, nv);
        }
        wave_lds_fence();
    });
#endif
}

template <typename T, GemmKind KIND, int WP, int WC, int TP, int TC, int NS, int PERCU> static sol_status launch_tile(GemmArgs a, hipStream_t st) {
    a.ntp = ceil_div(a.M, WP * TP * 32);
    a.ntc = ceil_div(a.N, WC * TC * 32);
    const int nk = ceil_div(a.K, 64 / (int)sizeof(T));
    a.nsplit = a.nsplit < 1 ? 1 : a.nsplit;
    a.steps = ceil_div(nk, a.nsplit);
    const long blocks = (long)ceil_div(a.ntp * a.ntc, 8) * 8 * a.nsplit;
    hipLaunchKernelGGL((linear_gemm_kernel<T, KIND, WP, WC, TP, TC, NS, PERCU>), dim3((unsigned)blocks), dim3(256), 0, st, a);
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

template <typename T, GemmKind KIND> static sol_status launch_kind(const GemmArgs &a, hipStream_t st) {
    const long big = (long)ceil_div(a.M, 256) * ceil_div(a.N, 128) * a.nsplit, mid = (long)ceil_div(a.M, 128) * ceil_div(a.N, 128) * a.nsplit;
    if (big >= 400) return launch_tile<T, KIND, 2, 2, 4, 2, 3, 2>(a, st);
    if (mid >= 200) return launch_tile<T, KIND, 2, 2, 2, 2, 4, 2>(a, st);
    return launch_tile<T, KIND, 2, 2, 1, 1, 5, 3>(a, st);
}

sol_status launch_linear_gemm(GemmArgs a, int dt, GemmKind kind, hipStream_t st) {
    if (dt == SOL_BF16) {
        switch (kind) {
            case GEMM_FORWARD: return launch_kind<bf16_t, GEMM_FORWARD>(a, st);
            case GEMM_DX: return launch_kind<bf16_t, GEMM_DX>(a, st);
            default: return launch_kind<bf16_t, GEMM_DW>(a, st);
        }
    }
    switch (kind) {
        case GEMM_FORWARD: return launch_kind<float, GEMM_FORWARD>(a, st);
        case GEMM_DX: return launch_kind<float, GEMM_DX>(a, st);
        default: return launch_kind<float, GEMM_DW>(a, st);
    }
}

}  // namespace sol
