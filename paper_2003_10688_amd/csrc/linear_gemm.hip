// The matrix products of the linear layer, forward and backward:  D[p][c] = sum_k A(p, k) B(c, k).
//
//   forward  z = x W^T     A = x  [m][in]   along k    B = W  [out][in]  along k
//   dx       = dz W        A = dz [m][out]  along k    B = W  [out][in]  across k
//   dW       = dz^T x      A = dz [m][out]  across k   B = x  [m][in]    across k
//
// Four waves share a tile of rows x columns; stages of 128 bytes of reduction per row (64 bf16, 32 fp32) travel memory -> LDS by DMA
// through a ring, each wave multiplies its quarter with 32x32 matrix instructions.
// An operand along k lies in LDS as rows of 128 bytes, read as 16-byte fragments; one across k lies as it is in memory, rows of
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

// All but the last N LDS reads have landed (they land in order; the counter has four bits, and waiting for more than needed is right too).
template <int N> __device__ __forceinline__ void wait_lds() { wait_lgkmcnt<(N < 15 ? N : 15)>(); }

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

constexpr int ROWB = 128;       // bytes of reduction of a stage: whole cache lines (with 64 every line came from L2 twice: 200 against 100 million requests)

// Where BR rows (or columns) of an operand lie in LDS and in memory, one stage of them.
template <typename T, bool ACROSS, int BR> struct Tile {
    static constexpr int ES = (int)sizeof(T), BK = ROWB / ES, RB = ACROSS ? BR * ES : ROWB;     // bytes of a row in LDS
    static constexpr int BYTES = BR * ROWB, SEGS = BYTES / 1024;                                // DMA instructions of 64 lanes x 16 bytes

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
            const int row = seg * 8 + (lane >> 3);
            return (unsigned)row * pitch + (unsigned)(((lane & 7) ^ swz<ROWB>(row)) << 4);
        }
    }
    // along k: whether what that instruction brings of the last stage lies behind `bytes` of it
    static __device__ __forceinline__ bool behind(int seg, int lane, int bytes) { return (((lane & 7) ^ swz<ROWB>(seg * 8 + (lane >> 3))) << 4) >= bytes; }
    // LDS offset of this lane's fragment of the first k-step for the 32-wide block `blk`
    static __device__ __forceinline__ unsigned frag(int blk, int lane) {
        const int lr = lane & 31, lh = lane >> 5;
        if constexpr (!ACROSS) {
            return (unsigned)((blk * 32 + lr) * ROWB + ((lh ^ swz<ROWB>(lr)) << 4));
        } else if constexpr (ES == 2) {
            const int s = lane & 15, k = 8 * lh + (s >> 2), slot = blk * 4 + ((lane >> 4) & 1) * 2 + ((s & 3) >> 1);
            return (unsigned)(k * RB + ((slot ^ permute(k)) << 4) + (s & 1) * 8);
        } else {
            const int k = 4 * lh, slot = blk * 8 + (lr >> 2);
            return (unsigned)(k * RB + ((slot ^ permute(k)) << 4) + (lr & 3) * 4);
        }
    }
};

// N blocks of 32 rows of an operand, one k-step, from LDS to registers.  base[]: Tile::frag of the blocks (along k: of the first).
template <typename T, bool ACROSS, int BR, int N> struct Frags {
    using TL = Tile<T, ACROSS, BR>;
    static constexpr int NB = ACROSS ? N : 1, READS = N * Frag<T, ACROSS>::READS;
    Frag<T, ACROSS> f[N];
    static __device__ __forceinline__ void bases(unsigned (&base)[NB], unsigned lds, int blk, int lane) {
#pragma unroll
        for (int i = 0; i < NB; i++) base[i] = lds + TL::frag(blk + i, lane);
    }
    template <int Q> __device__ __forceinline__ void read(const unsigned (&base)[NB], unsigned off) {      // k-step Q of the stage at byte offset off
        if constexpr (!ACROSS) {
            const unsigned at = xor_add(base[0], Q << 5, off);
            static_for<N>([&](auto I) { constexpr int i = decltype(I)::value; f[i].template read<i * 32 * ROWB, ROWB>(at); });
        } else {
            static_for<N>([&](auto I) { constexpr int i = decltype(I)::value; f[i].template read<Q *(TL::BK / 4) * TL::RB, TL::RB>(base[i] + off); });
        }
    }
    __device__ __forceinline__ void land() { static_for<N>([&](auto I) { f[decltype(I)::value].land(); }); }
};

// An operand's corner moves along the reduction as a scalar; what lies behind the tensor, or behind the part's last stage, is out of range of the resource and
// arrives as zeros.  Along k: rows from `rows` on.  Across k: rows of k from `left` on, and what lies behind row_bytes of the last one.
template <bool ACROSS, int BK> struct Cursor;
template <int BK> struct Cursor<false, BK> {
    const unsigned char *p;
    unsigned num;
    int left;
    __device__ __forceinline__ void init(const void *base, unsigned pitch, int es, int first, int limit, int, int s0, int s1, int) {
        p = static_cast<const unsigned char *>(base) + (size_t)first * pitch + (size_t)s0 * ROWB;
        num = (unsigned)max(0, min(256, limit - first)) * pitch;       // a row ends in memory where the pitch ends, or its last stage is cut
        left = s1 - s0;
    }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t next() {
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(p), 0, left > 0 ? (int)num : 0, 0x00020000);
        p += ROWB;
        --left;
        return r;
    }
};
template <int BK> struct Cursor<true, BK> {
    const unsigned char *p;
    unsigned pitch, lack;
    int left;
    __device__ __forceinline__ void init(const void *base, unsigned pitch_, int es, int first, int, int row_bytes, int s0, int s1, int K) {
        pitch = pitch_;
        p = static_cast<const unsigned char *>(base) + (size_t)first * es + (size_t)s0 * BK * pitch;
        const int row = row_bytes - first * es;
        lack = pitch - (unsigned)row;
        left = row > 0 ? min(K, s1 * BK) - s0 * BK : 0;
    }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t next() {
        const int rows = min(left, BK);
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(p), 0, rows > 0 ? (int)((unsigned)rows * pitch - lack) : 0, 0x00020000);
        p += (size_t)BK * pitch;
        left -= BK;
        return r;
    }
};

// Tile order.  Workgroups go to the eight XCDs in turn; each XCD takes a contiguous run of a sequence that walks the columns of eight rows of
// tiles, so that what runs on it at one time is a block of about eight by eight tiles and shares its operands in that L2.
__device__ __forceinline__ bool pick_tile(const GemmArgs &a, int &split, int &tp, int &tc) {
    const int ntiles = a.ntp * a.ntc, per = (ntiles + 7) >> 3;
    split = (int)blockIdx.x / (per * 8);
    const int bid = (int)blockIdx.x - split * per * 8, t = (bid & 7) * per + (bid >> 3);
    if (t >= ntiles) return false;
    const int g = t / (8 * a.ntc), in = t - g * 8 * a.ntc, rows = min(8, a.ntp - g * 8);
    // divisions run on the vector units: back to scalars, or every resource derived from them would be taken for different ones per lane
    tp = __builtin_amdgcn_readfirstlane(g * 8 + in % rows);
    tc = __builtin_amdgcn_readfirstlane(in / rows);
    split = __builtin_amdgcn_readfirstlane(split);
    return true;
}

// Results of 32 rows x 32 * TC columns of a wave.  They go through a strip of LDS of its own, so that a lane has 8 neighbouring columns of one row
// (one call of dropout's generator) and a store writes whole lines.
template <typename T, GemmKind KIND, int TC> struct Writer {
    static constexpr int ERS = TC * 32 + 4, LPR = TC * 4, RPS = 64 / LPR;       // floats of a strip's row; lanes per row, rows per pass
    static constexpr int BYTES = 32 * ERS * 4;
    float *strip;
    int lane, split, n, nv;
    float bias8[8];
    uint32_t step;
    __device__ __forceinline__ void init(const GemmArgs &a, unsigned char *lds, int wave, int lane_, int split_, int c0) {
        strip = reinterpret_cast<float *>(lds + wave * BYTES);
        lane = lane_; split = split_;
        n = c0 + (lane % LPR) * 8;
        nv = min(8, a.N - n);
        if constexpr (KIND == GEMM_FORWARD) {
            load_bias8(a.epi.bias, n, nv, bias8);
            step = drop_step(a.epi.drop);
        }
    }
    template <typename F> __device__ __forceinline__ void write(const GemmArgs &a, int m0, F &&block) {      // block(i): accumulators of column block i
        const int lr = lane & 31, lh = lane >> 5, ecol = (lane % LPR) * 8;
        static_for<TC>([&](auto I) {
            const f32x16_t &v = block(I);
#pragma unroll
            for (int e = 0; e < 4; e++)
                *reinterpret_cast<float4 *>(strip + lr * ERS + decltype(I)::value * 32 + 8 * e + 4 * lh) = make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
        });
        wave_lds_fence();
#pragma unroll 1
        for (int r = lane / LPR; r < 32; r += RPS) {
            const int m = m0 + r;
            if (m >= a.M || nv <= 0) continue;
            const float4 lo = *reinterpret_cast<const float4 *>(strip + r * ERS + ecol), hi = *reinterpret_cast<const float4 *>(strip + r * ERS + ecol + 4);
            float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            if (a.nsplit > 1) store8_any<float>(a.part + ((size_t)split * a.M + m) * a.N + n, v, nv);
            else if constexpr (KIND == GEMM_FORWARD) finish8<T>(a.epi, step, m, n, a.N, nv, v, bias8);
            else if (a.out_dt == SOL_F32) store8_any<float>(static_cast<float *>(a.out) + m * a.ldo + n, v, nv);
            else store8_any<T>(static_cast<T *>(a.out) + m * a.ldo + n, v, nv);
        }
        wave_lds_fence();
    }
};

// ---- tiles of 64 x 64 to 128 x 128: a ring of NS whole stages --------------------------------------------------------------------
// KIND: GEMM_FORWARD (A, B along k), GEMM_DX (B across), GEMM_DW (both across).  WP x WC = 4 waves of TP x TC blocks of 32 x 32.
template <typename T, GemmKind KIND, int WP, int WC, int TP, int TC, int NS, int PERCU>
__global__ void __launch_bounds__(256, PERCU) linear_tile_kernel(const GemmArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool AX = KIND == GEMM_DW, BX = KIND != GEMM_FORWARD;
    constexpr int NW = 4, ES = (int)sizeof(T), BP = WP * TP * 32, BC = WC * TC * 32, BK = ROWB / ES;
    using TA = Tile<T, AX, BP>;
    using TB = Tile<T, BX, BC>;
    using FA = Frags<T, AX, BP, TP>;
    using FB = Frags<T, BX, BC, TC>;
    using W = Writer<T, KIND, TC>;
    constexpr int STAGE = TA::BYTES + TB::BYTES, XL = TA::SEGS / NW, WL = TB::SEGS / NW, L = XL + WL;
    constexpr int READS = FA::READS + FB::READS;               // LDS instructions of a k-step
    static_assert(WP * WC == NW && TA::SEGS % (2 * NW) == 0 && TB::SEGS % NW == 0, "waves");
    static_assert(NW * W::BYTES <= NS * STAGE && NS >= 2 && (NS - 1) * L < 64, "strips in the ring; vmcnt");
    __shared__ __align__(1024) unsigned char lds[NS * STAGE];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wc = wave / WP;
    int split, tp, tc;
    if (!pick_tile(a, split, tp, tc)) return;
    const int p0 = tp * BP, c0 = tc * BC;
    const int nk = (a.K + BK - 1) / BK, s0 = split * a.steps, s1 = min(nk, s0 + a.steps);   // this part's stages

    const unsigned apitch = (unsigned)(a.lda * ES), bpitch = (unsigned)(a.ldb * ES);
    Cursor<AX, BK> ca;
    Cursor<BX, BK> cb;
    ca.init(a.a, apitch, ES, p0, a.M, a.a_row, s0, s1, a.K);
    cb.init(a.b, bpitch, ES, c0, a.N, a.b_row, s0, s1, a.K);
    unsigned ao[XL], bo[WL], cut[2] = {0u, 0u};                // cut: what lies behind K in the last stage (odd and even instructions)
#pragma unroll
    for (int i = 0; i < XL; i++) ao[i] = TA::offset(wave * XL + i, lane, apitch);
#pragma unroll
    for (int i = 0; i < WL; i++) bo[i] = TB::offset(wave * WL + i, lane, bpitch);
    if constexpr (!AX) {
#pragma unroll
        for (int i = 0; i < 2; i++) cut[i] = a.a_cut && TA::behind(wave * XL + i, lane, a.K * ES - (nk - 1) * ROWB) ? 0xffffffffu : 0u;
    }
    int at = s0;                                               // the next stage to request
    __amdgpu_buffer_rsrc_t ar, br;
    bool last = false;
    auto next_stage = [&]() {
        ar = ca.next();
        br = cb.next();
        last = at == nk - 1;
        ++at;
    };
    auto request = [&](auto I, unsigned off) {                 // the I-th DMA of this wave for that stage
        constexpr int i = decltype(I)::value;
        unsigned char *la = lds + off, *lb = la + TA::BYTES;
        if constexpr (i < XL)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ar, (__attribute__((address_space(3))) void *)(la + (wave * XL + i) * 1024), 16, !AX ? ao[i] | (last ? cut[i & 1] : 0u) : ao[i], 0, 0, 0);
        else
            __builtin_amdgcn_raw_ptr_buffer_load_lds(br, (__attribute__((address_space(3))) void *)(lb + (wave * WL + i - XL) * 1024), 16, bo[i - XL], 0, 0, 0);
    };
#pragma unroll
    for (int s = 0; s < NS; s++) {
        next_stage();
        static_for<L>([&](auto I) { request(I, (unsigned)(s * STAGE)); });
    }

    f32x16_t acc[TC][TP];
#pragma unroll
    for (int i = 0; i < TC; i++)
#pragma unroll
        for (int j = 0; j < TP; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0.f;

    unsigned abase[FA::NB], bbase[FB::NB];
    FA::bases(abase, lds_addr(lds), wp * TP, lane);
    FB::bases(bbase, lds_addr(lds) + TA::BYTES, wc * TC, lane);
    FA fa[2];
    FB fb[2];
    auto multiply = [&](auto S, auto &&between) {
        constexpr int set = decltype(S)::value;
        static_for<TC * TP>([&](auto U) {
            constexpr int u = decltype(U)::value, i = u / TP, j = u % TP;
            Mma<T>::run(acc[i][j], fb[set].f[i].get(), fa[set].f[j].get());
            between(U);
        });
        __builtin_amdgcn_sched_barrier(0);
    };

    wait_vmcnt<(NS - 1) * L>();                                // the first stage has landed
    __builtin_amdgcn_s_barrier();
    fb[0].template read<0>(bbase, 0u);
    fa[0].template read<0>(abase, 0u);
    unsigned sb = 0;
    for (int s = s0; s < s1; s++) {
        const unsigned sbn = sb + STAGE == NS * STAGE ? 0u : sb + STAGE;
        static_for<3>([&](auto Q) {                            // k-steps 0 .. 2, the next one's fragments on their way
            constexpr int q = decltype(Q)::value, set = q & 1;
            fb[set ^ 1].template read<q + 1>(bbase, sb);
            fa[set ^ 1].template read<q + 1>(abase, sb);
            wait_lds<READS>();
            fb[set].land();
            fa[set].land();
            multiply(std::integral_constant<int, set>{}, [](auto) {});
        });
        wait_lgkmcnt<0>();                                     // all of this stage is in registers
        fb[1].land();
        fa[1].land();
        wait_vmcnt<(NS - 2) * L>();                            // the next stage has landed
        __builtin_amdgcn_s_barrier();                          // ... for every wave, and nobody reads this one any more: it can be refilled
        fb[0].template read<0>(bbase, sbn);
        fa[0].template read<0>(abase, sbn);
        next_stage();
        multiply(std::integral_constant<int, 1>{}, [&](auto U) {
            constexpr int u = decltype(U)::value, per = (L + TC * TP - 1) / (TC * TP);
            static_for<per>([&](auto V) {
                constexpr int i = u * per + decltype(V)::value;
                if constexpr (i < L) request(std::integral_constant<int, i>{}, sb);
            });
        });
        sb = sbn;
    }
    wait_lgkmcnt<0>();                                         // the fragments requested behind the last stage
    fb[0].land();
    fa[0].land();
    wait_vmcnt<0>();                                           // ... and its DMAs, zeros into dead slots
    __builtin_amdgcn_s_barrier();                              // the ring becomes the strips

    W w;
    w.init(a, lds, wave, lane, split, c0 + wc * TC * 32);
    static_for<TP>([&](auto J) {
        constexpr int j = decltype(J)::value;
        w.write(a, p0 + (wp * TP + j) * 32, [&](auto I) -> const f32x16_t & { return acc[decltype(I)::value][j]; });
    });
#endif
}

// ---- tiles of 256 x 128 ----------------------------------------------------------------------------------------------------------
// Two workgroups per CU leave 80 KB of LDS each, and a stage of whole lines has 48.  So the ring counts not stages but units of 16 KB, 128 rows or columns each,
// five of them: a stage is B, A0 (rows 0 .. 127) and A1 (rows 128 .. 255).  A wave takes its fragments of B into registers once and multiplies A0, then A1, with
// them; when A0 is done its slot and B's are refilled, and when A1 is done its own.  Every unit is requested one stage (32 matrix instructions per wave) before it is needed.
template <typename T, GemmKind KIND>
__global__ void __launch_bounds__(256, 2) linear_big_kernel(const GemmArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool AX = KIND == GEMM_DW, BX = KIND != GEMM_FORWARD;
    constexpr int NW = 4, ES = (int)sizeof(T), BK = ROWB / ES, UNIT = 16384, UL = UNIT / 1024 / NW;      // UL: DMA instructions of a wave per unit
    using TA = Tile<T, AX, 128>;
    using TB = Tile<T, BX, 128>;
    using FA = Frags<T, AX, 128, 2>;
    using FB = Frags<T, BX, 128, 2>;
    using W = Writer<T, KIND, 2>;
    static_assert(NW * W::BYTES <= 5 * UNIT && UL == 4, "strips in the ring; requests per unit");
    __shared__ __align__(1024) unsigned char lds[5 * UNIT];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave & 1, wc = wave >> 1;
    int split, tp, tc;
    if (!pick_tile(a, split, tp, tc)) return;
    const int p0 = tp * 256, c0 = tc * 128;
    const int nk = (a.K + BK - 1) / BK, s0 = split * a.steps, s1 = min(nk, s0 + a.steps);   // this part's stages

    const unsigned apitch = (unsigned)(a.lda * ES), bpitch = (unsigned)(a.ldb * ES);
    Cursor<AX, BK> ca[2];
    Cursor<BX, BK> cb;
    ca[0].init(a.a, apitch, ES, p0, a.M, a.a_row, s0, s1, a.K);
    ca[1].init(a.a, apitch, ES, p0 + 128, a.M, a.a_row, s0, s1, a.K);
    cb.init(a.b, bpitch, ES, c0, a.N, a.b_row, s0, s1, a.K);
    unsigned ao[UL], bo[UL], cut[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < UL; i++) {
        ao[i] = TA::offset(wave * UL + i, lane, apitch);
        bo[i] = TB::offset(wave * UL + i, lane, bpitch);
    }
    if constexpr (!AX) {
#pragma unroll
        for (int i = 0; i < 2; i++) cut[i] = a.a_cut && TA::behind(wave * UL + i, lane, a.K * ES - (nk - 1) * ROWB) ? 0xffffffffu : 0u;
    }
    auto request_a = [&](const __amdgpu_buffer_rsrc_t &r, auto I, unsigned off, bool last) {
        constexpr int i = decltype(I)::value;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)(lds + off + (wave * UL + i) * 1024), 16, !AX ? ao[i] | (last ? cut[i & 1] : 0u) : ao[i], 0, 0, 0);
    };
    auto request_b = [&](const __amdgpu_buffer_rsrc_t &r, auto I, unsigned off) {
        constexpr int i = decltype(I)::value;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (__attribute__((address_space(3))) void *)(lds + off + (wave * UL + i) * 1024), 16, bo[i], 0, 0, 0);
    };

    unsigned o0 = 0, o1 = UNIT, o2 = 2 * UNIT, o3 = 3 * UNIT, o4 = 4 * UNIT;      // slots of this stage's B, A0, A1 and of the next one's B, A0
    __amdgpu_buffer_rsrc_t r0;                                  // of the A0 whose requests are spread over two halves
    {
        const __amdgpu_buffer_rsrc_t rb = cb.next(), r1 = ca[1].next(), rn = cb.next();
        r0 = ca[0].next();
        static_for<UL>([&](auto I) { request_b(rb, I, o0); });
        static_for<UL>([&](auto I) { request_a(r0, I, o1, s0 == nk - 1); });
        static_for<UL>([&](auto I) { request_a(r1, I, o2, s0 == nk - 1); });
        static_for<UL>([&](auto I) { request_b(rn, I, o3); });
        r0 = ca[0].next();
        static_for<UL / 2>([&](auto I) { request_a(r0, I, o4, s0 + 1 == nk - 1); });
    }

    f32x16_t acc[2][4];
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0.f;

    unsigned abase[FA::NB], bbase[FB::NB];
    FA::bases(abase, lds_addr(lds), wp * 2, lane);
    FB::bases(bbase, lds_addr(lds), wc * 2, lane);
    FA fa[4];                                                   // of the four k-steps of a half: two are on their way while one is multiplied
    FB fb[4];
    auto multiply = [&](auto H, auto Q, auto &&between) {       // four products of half H, k-step Q
        constexpr int h = decltype(H)::value, q = decltype(Q)::value;
        static_for<4>([&](auto U) {
            constexpr int u = decltype(U)::value, i = u / 2, j = u % 2;
            Mma<T>::run(acc[i][h * 2 + j], fb[q].f[i].get(), fa[q].f[j].get());
            between(U);
        });
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr std::integral_constant<int, 0> C0{};
    constexpr std::integral_constant<int, 1> C1{};
    constexpr std::integral_constant<int, 2> C2{};
    constexpr std::integral_constant<int, 3> C3{};

    wait_vmcnt<2 * UL + UL / 2>();                              // B and A0 of the first stage have landed
    __builtin_amdgcn_s_barrier();
    static_for<4>([&](auto Q) { fb[decltype(Q)::value].template read<decltype(Q)::value>(bbase, o0); });
    fa[0].template read<0>(abase, o1);
    fa[1].template read<1>(abase, o1);
    wait_lgkmcnt<0>();
    static_for<4>([&](auto Q) { fb[decltype(Q)::value].land(); });
    fa[0].land();
    fa[1].land();

    // The counts of the waits: LDS reads and DMAs land in the order in which they were issued, and each wait names how many were issued behind what it waits for.
    for (int s = s0; s < s1; s++) {
        // ---- A0 times B; the second half of the next stage's A0 is requested
        const bool next_last = s + 1 == nk - 1, third_last = s + 2 == nk - 1;
        fa[2].template read<2>(abase, o1);
        wait_lds<2 * FA::READS + 2 * FB::READS>();
        fa[0].land();
        fb[1].land();
        multiply(C0, C0, [&](auto U) { if constexpr (U == 3) request_a(r0, C2, o4, next_last); });
        fa[3].template read<3>(abase, o1);
        wait_lds<2 * FA::READS + FB::READS>();
        fa[1].land();
        fb[2].land();
        multiply(C0, C1, [&](auto U) { if constexpr (U == 3) request_a(r0, C3, o4, next_last); });
        wait_lgkmcnt<0>();                                      // all of A0 and B is in registers
        fa[2].land();
        fa[3].land();
        fb[3].land();
        wait_vmcnt<UL>();                                       // A1 and the next stage's B have landed
        __builtin_amdgcn_s_barrier();                           // ... for every wave, and nobody reads A0 and B any more: A1 and B of later stages take their slots
        fa[0].template read<0>(abase, o2);
        const __amdgpu_buffer_rsrc_t r1 = ca[1].next(), rb = cb.next();
        multiply(C0, C2, [&](auto U) { if constexpr (U & 1) request_a(r1, std::integral_constant<int, U / 2>{}, o0, next_last); });
        fa[1].template read<1>(abase, o2);
        multiply(C0, C3, [&](auto U) { if constexpr (U & 1) request_a(r1, std::integral_constant<int, 2 + U / 2>{}, o0, next_last); });
        // ---- A1 times B; behind each k-step's last products its fragments of B make room for the next stage's
        fa[2].template read<2>(abase, o2);
        wait_lds<2 * FA::READS>();
        fa[0].land();
        multiply(C1, C0, [&](auto U) { if constexpr (U & 1) request_b(rb, std::integral_constant<int, U / 2>{}, o1); });
        fb[0].template read<0>(bbase, o3);
        fa[3].template read<3>(abase, o2);
        wait_lds<2 * FA::READS + FB::READS>();
        fa[1].land();
        multiply(C1, C1, [&](auto U) { if constexpr (U & 1) request_b(rb, std::integral_constant<int, 2 + U / 2>{}, o1); });
        fb[1].template read<1>(bbase, o3);
        wait_lds<FB::READS>();                                  // all of A1 is in registers
        fa[2].land();
        fa[3].land();
        fb[0].land();
        wait_vmcnt<2 * UL>();                                   // the next stage's A0 has landed
        __builtin_amdgcn_s_barrier();
        fa[0].template read<0>(abase, o4);
        r0 = ca[0].next();
        multiply(C1, C2, [&](auto U) { if constexpr (U == 3) request_a(r0, C0, o2, third_last); });
        fb[2].template read<2>(bbase, o3);
        fa[1].template read<1>(abase, o4);
        multiply(C1, C3, [&](auto U) { if constexpr (U == 3) request_a(r0, C1, o2, third_last); });
        fb[3].template read<3>(bbase, o3);
        const unsigned t0 = o0, t1 = o1, t2 = o2;
        o0 = o3; o1 = o4; o2 = t0; o3 = t1; o4 = t2;
    }
    wait_lgkmcnt<0>();                                          // the fragments requested behind the last stage
    fa[0].land();
    fa[1].land();
    static_for<4>([&](auto Q) { fb[decltype(Q)::value].land(); });
    wait_vmcnt<0>();                                            // ... and its DMAs, zeros into dead slots
    __builtin_amdgcn_s_barrier();                               // the ring becomes the strips

    W w;
    w.init(a, lds, wave, lane, split, c0 + wc * 64);
    static_for<4>([&](auto J) {
        constexpr int j = decltype(J)::value;
        w.write(a, p0 + (j >> 1) * 128 + wp * 64 + (j & 1) * 32, [&](auto I) -> const f32x16_t & { return acc[decltype(I)::value][j]; });
    });
#endif
}

// ---- tiles of 256 x 256 ----------------------------------------------------------------------------------------------------------
// One workgroup of eight waves per CU: a row or column fetched once serves 256 of the other operand, 32 bytes a clock at the full rate of the matrix units, where the path
// from L2 to LDS gives 58 (with two workgroups of 256 x 128 it was 48, and their waves stood behind their own requests).
// A stage is four units of 16 KB: B0, B1 (columns 0 .. 127, 128 .. 255), A0, A1 (rows).  A wave has 64 rows of each half of A and 64 columns: it takes its fragments of B into
// registers once, multiplies A0, then A1, with them, and behind each k-step's last products reads the next stage's over them.  The ring has ten units; A0, A1 of
// stage s + 2 and B0 of s + 3 take the places of B0, B1 and A0 of stage s, and B1 of s + 3 that of A1, so every unit is requested one and a half stages (48 matrix instructions of a wave)
// before it is needed.
// The two waves of a SIMD issue one instruction each at a time, and everything that is not a product has to fit beside the products: resources and lane offsets are
// constants of the loop (a scalar offset moves along the reduction, and the range check includes it), and the loop is unrolled over the five stages after which the ring repeats.
template <int OFF> __device__ __forceinline__ unsigned add_const(unsigned v) {     // opaque: or sixty sums would be kept in registers across the loop
    unsigned d;
    asm volatile("v_add_u32_e32 %0, %1, %2" : "=v"(d) : "n"(OFF), "v"(v));
    return d;
}

// Fragments of one k-step of a unit at a constant place.  at[]: along k, the first block's place for each of the four k-steps; across, each block's for the first.
template <typename T, bool ACROSS> struct UnitFrags {
    using TL = Tile<T, ACROSS, 128>;
    static constexpr int NB = ACROSS ? 2 : 4, READS = 2 * Frag<T, ACROSS>::READS;
    Frag<T, ACROSS> f[2];
    static __device__ __forceinline__ void places(unsigned (&at)[NB], unsigned lds, int blk, int lane) {
#pragma unroll
        for (int i = 0; i < NB; i++) at[i] = ACROSS ? lds + TL::frag(blk + i, lane) : lds + (TL::frag(blk, lane) ^ (unsigned)(i << 5));
    }
    template <int Q, int OFF> __device__ __forceinline__ void read(const unsigned (&at)[NB]) {
        static_for<2>([&](auto I) {
            constexpr int i = decltype(I)::value, off = ACROSS ? Q *(TL::BK / 4) * TL::RB : i * 32 * ROWB, room = 65536 - (ACROSS ? 4 * TL::RB : 0);
            if constexpr (OFF + off < room) f[i].template read<OFF + off, TL::RB>(at[ACROSS ? i : Q]);
            else f[i].template read<off, TL::RB>(add_const<OFF>(at[ACROSS ? i : Q]));
        });
    }
    __device__ __forceinline__ void land() { f[0].land(); f[1].land(); }
};

// Bytes from the corner of a unit (its first row, or column, is `first` of `limit`) to the end of what may be read
__device__ __forceinline__ unsigned unit_bytes(bool across, int es, int first, int limit, int K, unsigned pitch, int row_bytes) {
    if (across) return row_bytes > first * es ? (unsigned)(K - 1) * pitch + (unsigned)(row_bytes - first * es) : 0u;
    const int rows = min(128, limit - first);
    return rows > 0 ? (unsigned)(rows - 1) * pitch + (unsigned)row_bytes : 0u;
}

template <typename T, GemmKind KIND>
__global__ void __launch_bounds__(512, 2) linear_huge_kernel(const GemmArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool AX = KIND == GEMM_DW, BX = KIND != GEMM_FORWARD;
    constexpr int NW = 8, ES = (int)sizeof(T), BK = ROWB / ES, UNIT = 16384, UL = UNIT / 1024 / NW, NU = 10;
    using TA = Tile<T, AX, 128>;
    using TB = Tile<T, BX, 128>;
    using FA = UnitFrags<T, AX>;
    using FB = UnitFrags<T, BX>;
    using W = Writer<T, KIND, 2>;
    static_assert(NW * W::BYTES <= NU * UNIT && UL == 2, "strips in the ring; requests per unit");
    __shared__ __align__(1024) unsigned char lds[NU * UNIT];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave & 1, wc = wave >> 1;
    int split, tp, tc;
    if (!pick_tile(a, split, tp, tc)) return;
    const int p0 = tp * 256, c0 = tc * 256, nk = (a.K + BK - 1) / BK;

    const unsigned apitch = (unsigned)(a.lda * ES), bpitch = (unsigned)(a.ldb * ES), astep = AX ? BK * apitch : ROWB, bstep = BX ? BK * bpitch : ROWB;
    __amdgpu_buffer_rsrc_t ra[2], rb[2];
#pragma unroll
    for (int h = 0; h < 2; h++) {
        const int p = p0 + h * 128, c = c0 + h * 128;
        ra[h] = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(static_cast<const unsigned char *>(a.a) + (size_t)p * (AX ? ES : apitch)), 0,
                                                  (int)unit_bytes(AX, ES, p, a.M, a.K, apitch, a.a_row), 0x00020000);
        rb[h] = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(static_cast<const unsigned char *>(a.b) + (size_t)c * (BX ? ES : bpitch)), 0,
                                                  (int)unit_bytes(BX, ES, c, a.N, a.K, bpitch, a.b_row), 0x00020000);
    }
    unsigned ao[UL], bo[UL];
#pragma unroll
    for (int i = 0; i < UL; i++) {
        ao[i] = TA::offset(wave * UL + i, lane, apitch);
        bo[i] = TB::offset(wave * UL + i, lane, bpitch);
    }
    // A along k whose rows do not end with zeros: from the last stage on, the slots behind K are out of range
    auto cut_last = [&](int stage) {
        if constexpr (!AX) {
            if (stage == nk - 1 && a.a_cut) {
#pragma unroll
                for (int i = 0; i < UL; i++) ao[i] |= TA::behind(wave * UL + i, lane, a.K * ES - (nk - 1) * ROWB) ? 0xffffffffu : 0u;
            }
        }
    };
    unsigned char *const mine = lds + wave * UL * 1024;         // where this wave's part of a unit goes
    auto request_a = [&](int h, auto I, int unit, unsigned soff) {
        constexpr int i = decltype(I)::value;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ra[h], (__attribute__((address_space(3))) void *)(mine + unit * UNIT + i * 1024), 16, ao[i], soff, 0, 0);
    };
    auto request_b = [&](int h, auto I, int unit, unsigned soff) {
        constexpr int i = decltype(I)::value;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rb[h], (__attribute__((address_space(3))) void *)(mine + unit * UNIT + i * 1024), 16, bo[i], soff, 0, 0);
    };
#pragma unroll
    for (int u = 0; u < NU - 1; u++) {                          // unit u: stage u / 4, B0, B1, A0, A1 in turn
        if (u % 4 == 2) cut_last(u / 4);
        static_for<UL>([&](auto I) {
            if (u % 4 < 2) request_b(u % 4, I, u, (unsigned)(u / 4) * bstep);
            else request_a(u % 4 - 2, I, u, (unsigned)(u / 4) * astep);
        });
    }

    f32x16_t acc[2][4];
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int e = 0; e < 16; e++) acc[i][j][e] = 0.f;

    unsigned aat[FA::NB], bat[FB::NB];
    FA::places(aat, lds_addr(lds), wp * 2, lane);
    FB::places(bat, lds_addr(lds) + (wc >> 1) * UNIT, (wc & 1) * 2, lane);       // B1 lies behind B0, except where the ring's end is between them: never, units go in twos
    FA fa[4];                                                   // of the four k-steps of a half: two are on their way while one is multiplied
    FB fb[4];
    auto multiply = [&](auto H, auto Q, auto &&request) {       // four products of half H, k-step Q, and a request among them
        constexpr int h = decltype(H)::value, q = decltype(Q)::value;
        static_for<4>([&](auto U) {
            constexpr int u = decltype(U)::value, i = u / 2, j = u % 2;
            Mma<T>::run(acc[i][h * 2 + j], fb[q].f[i].get(), fa[q].f[j].get());
            if constexpr (u == 1) request();
        });
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr std::integral_constant<int, 0> C0{};
    constexpr std::integral_constant<int, 1> C1{};
    constexpr std::integral_constant<int, 2> C2{};
    constexpr std::integral_constant<int, 3> C3{};

    wait_vmcnt<6 * UL>();                                       // B and A0 of the first stage have landed
    __builtin_amdgcn_s_barrier();
    static_for<4>([&](auto Q) { fb[decltype(Q)::value].template read<decltype(Q)::value, 0>(bat); });
    fa[0].template read<0, 2 * UNIT>(aat);
    fa[1].template read<1, 2 * UNIT>(aat);
    wait_lgkmcnt<0>();
    static_for<4>([&](auto Q) { fb[decltype(Q)::value].land(); });
    fa[0].land();
    fa[1].land();

    // The counts of the waits: LDS reads and DMAs land in the order in which they were issued, and each wait names how many were issued behind what it waits for.
    // One request per k-step and wave: a request holds its wave while the queue is full, and two at a time from eight waves fill it.
    unsigned asoff = 2 * astep, bsoff = 2 * bstep;              // of stage s + 2
    auto stage = [&](auto P, int s) {
        constexpr int p = decltype(P)::value;
        constexpr auto at = [](int k) { return (p * 4 + k) % NU; };      // unit k from this stage's B0 on
        constexpr int A0 = at(2) * UNIT, A1 = at(3) * UNIT, BN = at(4) * UNIT, AN = at(6) * UNIT;
        // ---- A0 times B
        fa[2].template read<2, A0>(aat);
        wait_lds<2 * FA::READS + 2 * FB::READS>();
        fa[0].land();
        fb[1].land();
        multiply(C0, C0, [&] { request_b(1, C0, at(9), bsoff); });
        fa[3].template read<3, A0>(aat);
        wait_lds<2 * FA::READS + FB::READS>();
        fa[1].land();
        fb[2].land();
        multiply(C0, C1, [&] { request_b(1, C1, at(9), bsoff); });
        wait_lgkmcnt<0>();                                      // all of A0 and B is in registers
        fa[2].land();
        fa[3].land();
        fb[3].land();
        wait_vmcnt<4 * UL>();                                   // A1 and the next stage's B have landed
        __builtin_amdgcn_s_barrier();                           // ... for every wave, and nobody reads A0 and B any more: units of later stages take their slots
        fa[0].template read<0, A1>(aat);
        cut_last(s + 2);
        multiply(C0, C2, [&] { request_a(0, C0, at(0), asoff); });
        fa[1].template read<1, A1>(aat);
        multiply(C0, C3, [&] { request_a(0, C1, at(0), asoff); });
        // ---- A1 times B; behind each k-step's last products its fragments of B make room for the next stage's
        fa[2].template read<2, A1>(aat);
        wait_lds<2 * FA::READS>();
        fa[0].land();
        multiply(C1, C0, [&] { request_a(1, C0, at(1), asoff); });
        fb[0].template read<0, BN>(bat);
        fa[3].template read<3, A1>(aat);
        wait_lds<2 * FA::READS + FB::READS>();
        fa[1].land();
        multiply(C1, C1, [&] { request_a(1, C1, at(1), asoff); });
        fb[1].template read<1, BN>(bat);
        wait_lds<FB::READS>();                                  // all of A1 is in registers
        fa[2].land();
        fa[3].land();
        fb[0].land();
        wait_vmcnt<5 * UL>();                                   // the next stage's A0 has landed
        __builtin_amdgcn_s_barrier();
        fa[0].template read<0, AN>(aat);
        asoff += astep;
        bsoff += bstep;
        multiply(C1, C2, [&] { request_b(0, C0, at(2), bsoff); });
        fb[2].template read<2, BN>(bat);
        fa[1].template read<1, AN>(aat);
        multiply(C1, C3, [&] { request_b(0, C1, at(2), bsoff); });
        fb[3].template read<3, BN>(bat);
    };
    for (int s = 0;;) {
        stage(C0, s);
        if (++s >= nk) break;
        stage(C1, s);
        if (++s >= nk) break;
        stage(C2, s);
        if (++s >= nk) break;
        stage(C3, s);
        if (++s >= nk) break;
        stage(std::integral_constant<int, 4>{}, s);
        if (++s >= nk) break;
    }
    wait_lgkmcnt<0>();                                          // the fragments requested behind the last stage
    fa[0].land();
    fa[1].land();
    static_for<4>([&](auto Q) { fb[decltype(Q)::value].land(); });
    wait_vmcnt<0>();                                            // ... and its DMAs into dead slots
    __builtin_amdgcn_s_barrier();                               // the ring becomes the strips

    W w;
    w.init(a, lds, wave, lane, split, c0 + wc * 64);
    static_for<4>([&](auto J) {
        constexpr int j = decltype(J)::value;
        w.write(a, p0 + (j >> 1) * 128 + wp * 64 + (j & 1) * 32, [&](auto I) -> const f32x16_t & { return acc[decltype(I)::value][j]; });
    });
#endif
}

static long tiles_of(GemmArgs &a, int dt, int bp, int bc) {     // fills in the tile counts; workgroups of the launch
    a.ntp = ceil_div(a.M, bp);
    a.ntc = ceil_div(a.N, bc);
    a.nsplit = a.nsplit < 1 ? 1 : a.nsplit;
    a.steps = ceil_div(ceil_div(a.K, ROWB / (int)dtype_size(dt)), a.nsplit);
    return (long)ceil_div(a.ntp * a.ntc, 8) * 8 * a.nsplit;
}

template <typename T, GemmKind KIND, int WP, int WC, int TP, int TC, int NS, int PERCU> static sol_status launch_tile(GemmArgs a, int dt, hipStream_t st) {
    const long blocks = tiles_of(a, dt, WP * TP * 32, WC * TC * 32);
    hipLaunchKernelGGL((linear_tile_kernel<T, KIND, WP, WC, TP, TC, NS, PERCU>), dim3((unsigned)blocks), dim3(256), 0, st, a);
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

template <typename T, GemmKind KIND> static sol_status launch_kind(GemmArgs a, int dt, hipStream_t st) {
    const long big = (long)ceil_div(a.M, 256) * ceil_div(a.N, 128) * a.nsplit, mid = (long)ceil_div(a.M, 128) * ceil_div(a.N, 128) * a.nsplit;
    const long huge = (long)ceil_div(a.M, 256) * ceil_div(a.N, 256) * a.nsplit;
    const double abytes = KIND == GEMM_DW ? ((double)a.K + 256) * a.lda * sizeof(T) : 256.0 * a.lda * sizeof(T);
    const double bbytes = KIND != GEMM_FORWARD ? ((double)a.K + 256) * a.ldb * sizeof(T) : 256.0 * a.ldb * sizeof(T);
    if (huge >= 200 && a.nsplit <= 1 && abytes < 4294967296.0 && bbytes < 4294967296.0) {       // 32-bit offsets along the reduction
        const long blocks = tiles_of(a, dt, 256, 256);
        hipLaunchKernelGGL((linear_huge_kernel<T, KIND>), dim3((unsigned)blocks), dim3(512), 0, st, a);
        SOL_HIP(hipGetLastError());
        return SOL_OK;
    }
    if (big >= 400) {
        const long blocks = tiles_of(a, dt, 256, 128);
        hipLaunchKernelGGL((linear_big_kernel<T, KIND>), dim3((unsigned)blocks), dim3(256), 0, st, a);
        SOL_HIP(hipGetLastError());
        return SOL_OK;
    }
    if (mid >= 200) return launch_tile<T, KIND, 2, 2, 2, 2, 2, 2>(a, dt, st);
    return launch_tile<T, KIND, 2, 2, 1, 1, 3, 3>(a, dt, st);
}

sol_status launch_linear_gemm(GemmArgs a, int dt, GemmKind kind, hipStream_t st) {
    if (dt == SOL_BF16) {
        switch (kind) {
            case GEMM_FORWARD: return launch_kind<bf16_t, GEMM_FORWARD>(a, dt, st);
            case GEMM_DX: return launch_kind<bf16_t, GEMM_DX>(a, dt, st);
            default: return launch_kind<bf16_t, GEMM_DW>(a, dt, st);
        }
    }
    switch (kind) {
        case GEMM_FORWARD: return launch_kind<float, GEMM_FORWARD>(a, dt, st);
        case GEMM_DX: return launch_kind<float, GEMM_DX>(a, dt, st);
        default: return launch_kind<float, GEMM_DW>(a, dt, st);
    }
}

}  // namespace sol
