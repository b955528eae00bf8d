// The matrix products of the linear layer, forward and backward:  D[p][c] = sum_k A(p, k) B(c, k).
//
//   forward  z = x W^T     A = x  [m][in]   along k    B = W  [out][in]  along k
//   dx       = dz W        A = dz [m][out]  along k    B = W  [out][in]  across k
//   dW       = dz^T x      A = dz [m][out]  across k   B = x  [m][in]    across k
//
// The waves of a workgroup share a tile of rows x columns; stages of 128 bytes of reduction per row (64 bf16, 32 fp32) travel memory -> LDS by DMA through a
// ring, and each wave multiplies its part with 16x16 matrix instructions.
// An operand along k lies in LDS as rows of 128 bytes, read as 16-byte fragments; one across k lies as it is in memory, rows of columns, and is transposed on the
// way to registers (ds_read_b64_tr_b16 for bf16, four 4-byte reads for fp32), so no transposed copy of W, dz or x is ever made.  Slots are permuted on the global
// side of the DMA so that neither kind of read meets a bank twice.
//
// Why 16x16x32 and not 32x32x16: large products run at the card's power limit, not at its clock, and on values as they occur a loop of nothing but 16x16x32
// instructions sustains 2.00 PFLOP/s where 32x32x16 sustains 1.76 (on zeros both reach 2.4): an accumulator is read and written half as often.
#include "linear_ops.h"

namespace sol {

using namespace lds_pipe;

typedef unsigned u32x2_t __attribute__((ext_vector_type(2)));

// All but the last N LDS reads have landed (they land in order; the counter has four bits, and waiting for more than needed is right too).
template <int N> __device__ __forceinline__ void wait_lds() { wait_lgkmcnt<(N < 15 ? N : 15)>(); }

// One fragment: 64 bytes of reduction of 16 rows or columns, 16 bytes per lane: row lane % 16, elements from 16 bytes' worth times lane / 16 on.  bf16 across k arrives in two halves.
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

    // Permutation of the 16-byte slots of a row across k.  32 lanes of a transposing read take 32 bytes of each of rows k .. k + 3 and k + 8 .. k + 11, those of a 4-byte read
    // 64 bytes of rows k and k + 4 (of 64 lanes: k + 8, k + 12 too).
    static __device__ __forceinline__ int permute(int k) {
        if constexpr (ES == 2) return (RB >= 256 ? (k & 3) << 2 : (k >> 1 & 1) << 2) | (k >> 3 & 1) << 1;
        else return (k >> 2 & 3) << 2;
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
    // LDS offset of this lane's fragment of the first 64 bytes of k for the block of 16 rows `blk`.  Along k the blocks are 2048 bytes apart and the second 64 bytes are at this ^ 64; across,
    // they are BK / 2 rows further.
    static __device__ __forceinline__ unsigned frag(int blk, int lane) {
        const int r = lane & 15, g = lane >> 4;
        if constexpr (!ACROSS) {
            return (unsigned)((blk * 16 + r) * ROWB + ((g ^ swz<ROWB>(r)) << 4));
        } else if constexpr (ES == 2) {
            const int k = 8 * g + (r >> 2), slot = blk * 2 + ((r & 3) >> 1);
            return (unsigned)(k * RB + ((slot ^ permute(k)) << 4) + (r & 1) * 8);
        } else {
            const int k = 4 * g, slot = blk * 4 + (r >> 2);
            return (unsigned)(k * RB + ((slot ^ permute(k)) << 4) + (r & 3) * 4);
        }
    }
};

template <int OFF> __device__ __forceinline__ unsigned add_const(unsigned v) {     // opaque: or dozens of sums would be kept in registers across the loop
    unsigned d;
    asm volatile("v_add_u32_e32 %0, %1, %2" : "=v"(d) : "n"(OFF), "v"(v));
    return d;
}
template <int OFF> __device__ __forceinline__ unsigned s_add_const(unsigned v) {   // likewise for scalars
    unsigned d;
    asm volatile("s_add_i32 %0, %1, %2" : "=s"(d) : "s"(v), "n"(OFF) : "scc");
    return d;
}

// Where a wave's N blocks of 16 rows lie in a tile's part of LDS: along k, the first block for either half of the stage; across, every block.
template <typename T, bool ACROSS, int BR, int N> struct Places {
    using TL = Tile<T, ACROSS, BR>;
    using F = Frag<T, ACROSS>;
    unsigned at[ACROSS ? N : 2];
    __device__ __forceinline__ void init(unsigned lds, int blk, int lane) {
        if constexpr (ACROSS) {
#pragma unroll
            for (int i = 0; i < N; i++) at[i] = lds + TL::frag(blk + i, lane);
        } else {
            at[0] = lds + TL::frag(blk, lane);
            at[1] = lds + (TL::frag(blk, lane) ^ 64u);
        }
    }
    // fragment of block I, half K of the stage, at byte offset OFF (a constant) + off
    template <int I, int K, int OFF> __device__ __forceinline__ void read(F &f, unsigned off) const {
        constexpr int in = ACROSS ? K *(TL::BK / 2) * TL::RB : I * 16 * ROWB, room = 65536 - (ACROSS ? 4 * TL::RB : 0);
        const unsigned base = at[ACROSS ? I : K] + off;
        if constexpr (OFF + in < room) f.template read<OFF + in, TL::RB>(base);
        else f.template read<in, TL::RB>(add_const<OFF>(base));
    }
};

// Tile order.  Workgroups go to the eight XCDs in turn; each XCD takes a contiguous run of a sequence that walks the columns of eight rows of
// tiles, so that what runs on it at one time is a block of about eight by four tiles and shares its operands in that L2.
__device__ __forceinline__ bool pick_tile(const GemmArgs &a, int block, int &split, int &tp, int &tc) {
    const int ntiles = a.ntp * a.ntc, per = (ntiles + 7) >> 3;
    split = block / (per * 8);
    const int bid = block - split * per * 8, t = (bid & 7) * per + (bid >> 3);
    if (t >= ntiles) return false;
    const int g = t / (8 * a.ntc), in = t - g * 8 * a.ntc, rows = min(8, a.ntp - g * 8);
    // divisions run on the vector units: back to scalars, or every resource derived from them would be taken for different ones per lane
    tp = __builtin_amdgcn_readfirstlane(g * 8 + in % rows);
    tc = __builtin_amdgcn_readfirstlane(in / rows);
    split = __builtin_amdgcn_readfirstlane(split);
    return true;
}

// Results of a wave, RP blocks of 16 rows by RC (even) of 16 columns, from accumulators to memory.  A lane has 4 neighbouring columns of one row of each block; an exchange
// between rows of 16 lanes over two blocks leaves it with 8 neighbouring columns (one call of dropout's generator), and a store with 64 contiguous bytes of 16 rows.
__device__ __forceinline__ void rows8(const f32x4_t &x, const f32x4_t &y, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; e++) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x[e]), __float_as_uint(y[e]), false, false);
        v[e] = __uint_as_float(r[0]);
        v[4 + e] = __uint_as_float(r[1]);
    }
}
template <typename T, GemmKind KIND, int RP, int RC>
__device__ __forceinline__ void write_results(const GemmArgs &a, int split, const f32x4_t (&acc)[RP][RC], int p0, int c0, int lane) {
    static_assert(RP % 2 == 0 && (RC == 2 || RC % 4 == 0), "two or four blocks at a time");
    const int lrow = lane & 15, lcol = (lane >> 4 & 1) * 16 + (lane >> 5) * 8;
    if constexpr (KIND == GEMM_FORWARD) {
        constexpr bool BESIDE = RC >= 4;                        // 16 rows x 64 columns at a time, or 32 x 32
        const uint32_t step = drop_step(a.epi.drop);
#pragma unroll 1
        for (int u = 0; u < RP * RC / 4; u++) {                 // one copy of the epilogue's code
            f32x4_t b[2][2];
            static_for<RP * RC / 4>([&](auto U) {
                constexpr int w = decltype(U)::value, j = BESIDE ? w / (RC / 4) : w % (RP / 2) * 2, i = BESIDE ? w % (RC / 4) * 4 : w / (RP / 2) * 2;
                if (u == w) {
                    b[0][0] = acc[j][i]; b[0][1] = acc[j][i + 1];
                    if constexpr (BESIDE) { b[1][0] = acc[j][i + 2]; b[1][1] = acc[j][i + 3]; }
                    else { b[1][0] = acc[j + 1][i]; b[1][1] = acc[j + 1][i + 1]; }
                }
            });
            const int m = p0 + (BESIDE ? u / (RC / 4) * 16 : u % (RP / 2) * 32) + lrow, n = c0 + (BESIDE ? u % (RC / 4) * 64 : u / (RP / 2) * 32) + lcol;
            float v[2][8];
            rows8(b[0][0], b[0][1], v[0]);
            rows8(b[1][0], b[1][1], v[1]);
            finish_two<T, BESIDE>(a.epi, step, m, n, a.M, a.N, v);
        }
    } else {
        static_for<RP * RC / 2>([&](auto U) {                   // the columns of a row one behind the other
            constexpr int j = decltype(U)::value / (RC / 2), i = decltype(U)::value % (RC / 2) * 2;
            const int m = p0 + j * 16 + lrow, n = c0 + i * 16 + lcol, nv = min(8, a.N - n);
            float v[8];
            rows8(acc[j][i], acc[j][i + 1], v);
            if (m >= a.M || nv <= 0) return;
            if (a.plan.split > 1) store8_any<float>(a.part + ((size_t)split * a.M + m) * a.N + n, v, nv);
            else if (a.out_dt == SOL_F32) store8_any<float>(static_cast<float *>(a.out) + (size_t)m * a.ldo + n, v, nv);
            else store8_any<T>(static_cast<T *>(a.out) + (size_t)m * a.ldo + n, v, nv);
        });
    }
}

// ---- tiles of 64 x 64 to 128 x 128: a ring of NS whole stages --------------------------------------------------------------------
// Products whose tiles of 256 x 256 would leave CUs idle.  A stage's first half is multiplied while the second is read from LDS, and the other way round; a slot is requested again as soon as
// every wave has read it.  One workgroup on a CU is bound by the way of the data (0.2 us a stage of 64 x 64 tiles, 0.39 of 128 x 128 where the products need 0.06 and 0.23), several by
// the matrix units: 2048 x 2048, 8192 bf16 66 us (1.05 PFLOP/s); 1021 x 2304, 1536 16 us; fp32, where the products are sixteen times as long, reaches 122 to 145 of 150 TFLOP/s (4096 x 4096, 4096 950 us).
// An operand's corner moves along the reduction as a scalar; what lies behind the tensor, or behind the part's last stage, is out of range of the resource and
// arrives as zeros.  Along k: rows from `limit` on.  Across k: rows of k from `left` on, and what lies behind row_bytes of the last one.
template <bool ACROSS, int BK> struct Cursor;
template <int BK> struct Cursor<false, BK> {
    const unsigned char *p;
    unsigned num;
    int left;
    __device__ __forceinline__ void init(const void *base, unsigned pitch, int es, int first, int limit, int row_bytes, int s0, int s1, int) {
        p = static_cast<const unsigned char *>(base) + (size_t)first * pitch + (size_t)s0 * ROWB;
        const int rows = min(128, limit - first);
        num = rows > 0 ? (unsigned)(rows - 1) * pitch + (unsigned)row_bytes - (unsigned)s0 * ROWB : 0u;
        left = s1 - s0;
    }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t next() {
        const __amdgpu_buffer_rsrc_t r = __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char *>(p), 0, left > 0 ? (int)num : 0, 0x00020000);
        p += ROWB;
        num -= ROWB;
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

// KIND: GEMM_FORWARD (A, B along k), GEMM_DX (B across), GEMM_DW (both across).  WP x WC waves of RP x RC blocks of 16 x 16, a ring of NS stages.
constexpr int ring_bytes(int WP, int WC, int RP, int RC, int NS) { return NS * (WP * RP + WC * RC) * 16 * ROWB; }
template <typename T, GemmKind KIND, int WP, int WC, int RP, int RC, int NS>
__device__ __forceinline__ void linear_tile(const GemmArgs &a, int block, unsigned char *lds) {
#if defined(__HIP_DEVICE_COMPILE__)
    constexpr bool AX = KIND == GEMM_DW, BX = KIND != GEMM_FORWARD;
    constexpr int NW = WP * WC, ES = (int)sizeof(T), BP = WP * RP * 16, BC = WC * RC * 16, BK = ROWB / ES;
    using TA = Tile<T, AX, BP>;
    using TB = Tile<T, BX, BC>;
    constexpr int STAGE = TA::BYTES + TB::BYTES, XL = TA::SEGS / NW, WL = TB::SEGS / NW, L = XL + WL;
    constexpr int READS = RP * Frag<T, AX>::READS + RC * Frag<T, BX>::READS;       // LDS instructions of half a stage
    static_assert(TA::SEGS % (2 * NW) == 0 && TB::SEGS % NW == 0 && BP <= 128, "waves; rows that a cursor covers");
    static_assert(NS >= 2 && (NS - 1) * L < 64 && NS * STAGE == ring_bytes(WP, WC, RP, RC, NS), "vmcnt; LDS");

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave % WP, wc = wave / WP;
    int split, tp, tc;
    if (!pick_tile(a, block, split, tp, tc)) return;
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

    f32x4_t acc[RP][RC];
#pragma unroll
    for (int j = 0; j < RP; j++)
#pragma unroll
        for (int i = 0; i < RC; i++) acc[j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    Places<T, AX, BP, RP> pa;
    Places<T, BX, BC, RC> pb;
    pa.init(lds_addr(lds), wp * RP, lane);
    pb.init(lds_addr(lds) + TA::BYTES, wc * RC, lane);
    Frag<T, AX> fa[2][RP];
    Frag<T, BX> fb[2][RC];
    auto read_half = [&](auto K, unsigned off) {
        constexpr int k = decltype(K)::value;
        static_for<RC>([&](auto I) { pb.template read<decltype(I)::value, k, 0>(fb[k][decltype(I)::value], off); });
        static_for<RP>([&](auto J) { pa.template read<decltype(J)::value, k, 0>(fa[k][decltype(J)::value], off); });
    };
    auto land = [&](auto K) {
        constexpr int k = decltype(K)::value;
        static_for<RC>([&](auto I) { fb[k][decltype(I)::value].land(); });
        static_for<RP>([&](auto J) { fa[k][decltype(J)::value].land(); });
    };
    auto multiply = [&](auto K, auto &&between) {
        constexpr int k = decltype(K)::value;
        static_for<RP * RC>([&](auto U) {
            constexpr int u = decltype(U)::value, j = u / RC, i = u % RC;
            Mma16<T>::run(acc[j][i], fb[k][i].get(), fa[k][j].get());
            between(U);
        });
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr std::integral_constant<int, 0> K0{};
    constexpr std::integral_constant<int, 1> K1{};

    wait_vmcnt<(NS - 1) * L>();                                // the first stage has landed
    __builtin_amdgcn_s_barrier();
    read_half(K0, 0u);
    unsigned sb = 0;
    for (int s = s0; s < s1; s++) {
        const unsigned sbn = sb + STAGE == NS * STAGE ? 0u : sb + STAGE;
        read_half(K1, sb);
        wait_lds<READS>();
        land(K0);
        multiply(K0, [](auto) {});
        wait_lgkmcnt<0>();                                     // all of this stage is in registers
        land(K1);
        wait_vmcnt<(NS - 2) * L>();                            // the next stage has landed
        __builtin_amdgcn_s_barrier();                          // ... for every wave, and nobody reads this one any more: it can be refilled
        read_half(K0, sbn);
        next_stage();
        multiply(K1, [&](auto U) {
            constexpr int u = decltype(U)::value, per = (L + RP * RC - 1) / (RP * RC);
            static_for<per>([&](auto V) {
                constexpr int i = u * per + decltype(V)::value;
                if constexpr (i < L) request(std::integral_constant<int, i>{}, sb);
            });
        });
        sb = sbn;
    }
    wait_lgkmcnt<0>();                                         // the fragments requested behind the last stage
    land(K0);
    wait_vmcnt<0>();                                           // ... and its DMAs, zeros into dead slots
    write_results<T, KIND, RP, RC>(a, split, acc, p0 + wp * RP * 16, c0 + wc * RC * 16, lane);
#endif
}

template <typename T, GemmKind KIND, int WP, int WC, int RP, int RC, int NS, int PERCU>
__global__ void __launch_bounds__(WP * WC * 64, PERCU * WP * WC / 4) linear_tile_kernel(const GemmArgs a) {
    static_assert(ring_bytes(WP, WC, RP, RC, NS) <= 160 * 1024 / PERCU, "LDS");
    __shared__ __align__(1024) unsigned char lds[ring_bytes(WP, WC, RP, RC, NS)];
    linear_tile<T, KIND, WP, WC, RP, RC, NS>(a, (int)blockIdx.x, lds);
}

// dx and dW of a small layer in one launch, and the column sums that are db: workgroups below `first` have tiles of dx, below `second` of dW, the others sum.
template <typename T> __global__ void __launch_bounds__(256, 3) linear_pair_kernel(const GemmArgs dx, const GemmArgs dw, int first, int second, const SumJob sum) {
    __shared__ __align__(1024) unsigned char lds[ring_bytes(2, 2, 2, 2, 3)];
    const int b = (int)blockIdx.x;
    if (b < first) linear_tile<T, GEMM_DX, 2, 2, 2, 2, 3>(dx, b, lds);
    else if (b < second) linear_tile<T, GEMM_DW, 2, 2, 2, 2, 3>(dw, b - first, lds);
    else sum_parts(sum, b - second, (int)gridDim.x - second, reinterpret_cast<float *>(lds));
}

// ---- tiles of 256 x 256 ----------------------------------------------------------------------------------------------------------
// One workgroup of eight waves per CU: a row or column fetched once serves 256 of the other operand, 32 bytes a clock at the full rate of the matrix units, where the path
// from L2 to LDS gives 58.  A stage is four units of 16 KB: B0, B1 (columns 0 .. 127, 128 .. 255), A0, A1 (rows).  A wave has 64 rows of each half of A and 64 columns: it takes
// its fragments of B into registers once, multiplies A0, then A1, with them, and reads the next stage's over them behind the last products that need them.  The ring has ten
// units; A0, A1 of stage s + 2 and B0 of s + 3 take the places of B0, B1 and A0 of stage s, and B1 of s + 3 that of A1, so every unit is requested one and a half stages (96 matrix
// instructions of a wave) before it is needed.
// The two waves of a SIMD issue one instruction each at a time, and everything that is not a product has to fit beside the products: resources and lane offsets are
// constants of the loop (a scalar offset moves along the reduction; the range check includes it, also where a unit behind the last stage is requested), and the loop is unrolled over the five stages after which the ring repeats.
// What bounds it: the card's power limit, and the starts and ends of tiles, which nothing overlaps.  8192 x 8192 x 8192 takes 775 us (1.42 PFLOP/s, a stage 2500 cycles of which
// the products need 2048); 8192 x 16384, 4096 860 us (1.28), 55 more with GELU, dropout and z
// stored (the epilogue is bound by its arithmetic, some 300 instructions for 8 elements; with the halves of a line stored apart, 32 rows x 32 columns at a time, half as much again
// went to memory, 803 for 536 MB, and it took 40 us more).
// Also measured on the former, us: two groups of waves that take turns at the matrix units 938; two workgroups a CU with tiles of 256 x 128 904; four waves of 128 x 128 with a
// ring of five half stages 747 for 743 on one card, but 3 % behind on the latter, 12 % on 2048 x 8192, 2048 and 11 % as dx; starts staggered over a CU's neighbours 778; one barrier
// a stage, 2 % slower.

// Bytes from the corner of a unit (its first row, or column, is `first` of `limit`) to the end of what may be read
__device__ __forceinline__ unsigned unit_bytes(bool across, int es, int first, int limit, int K, unsigned pitch, int row_bytes) {
    if (across) return row_bytes > first * es ? (unsigned)(K - 1) * pitch + (unsigned)(row_bytes - first * es) : 0u;
    const int rows = min(128, limit - first);
    return rows > 0 ? (unsigned)(rows - 1) * pitch + (unsigned)row_bytes : 0u;
}

template <GemmKind KIND>
__global__ void __launch_bounds__(512, 2) linear_huge_kernel(const GemmArgs a) {
#if defined(__HIP_DEVICE_COMPILE__)
    using T = bf16_t;
    constexpr bool AX = KIND == GEMM_DW, BX = KIND != GEMM_FORWARD;
    constexpr int NW = 8, ES = (int)sizeof(T), BK = ROWB / ES, UNIT = 16384, UL = UNIT / 1024 / NW, NU = 10;
    using TA = Tile<T, AX, 128>;
    using TB = Tile<T, BX, 128>;
    constexpr int RA = 2 * Frag<T, AX>::READS, RBK = 4 * Frag<T, BX>::READS;       // LDS instructions of a step's fragments of A, of half a stage's of B
    static_assert(UL == 2, "requests per unit");
    __shared__ __align__(1024) unsigned char lds[NU * UNIT];

    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), wp = wave & 1, wc = wave >> 1;
    int split, tp, tc;
    if (!pick_tile(a, (int)blockIdx.x, split, tp, tc)) return;
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
    const unsigned mine = lds_addr(lds) + wave * UL * 1024;     // where this wave's part of a unit goes
    auto request_a = [&](auto H, auto I, auto U, unsigned soff) {
        constexpr int h = decltype(H)::value, i = decltype(I)::value, at = decltype(U)::value * UNIT + i * 1024;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ra[h], (__attribute__((address_space(3))) void *)(size_t)s_add_const<at>(mine), 16, ao[i], soff, 0, 0);
    };
    auto request_b = [&](auto H, auto I, auto U, unsigned soff) {
        constexpr int h = decltype(H)::value, i = decltype(I)::value, at = decltype(U)::value * UNIT + i * 1024;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rb[h], (__attribute__((address_space(3))) void *)(size_t)s_add_const<at>(mine), 16, bo[i], soff, 0, 0);
    };
    static_for<NU - 1>([&](auto U) {                            // unit u: stage u / 4, B0, B1, A0, A1 in turn
        constexpr int u = decltype(U)::value;
        if constexpr (u % 4 == 2) cut_last(u / 4);
        static_for<UL>([&](auto I) {
            if constexpr (u % 4 < 2) request_b(std::integral_constant<int, u % 4>{}, I, U, (unsigned)(u / 4) * bstep);
            else request_a(std::integral_constant<int, u % 4 - 2>{}, I, U, (unsigned)(u / 4) * astep);
        });
    });

    f32x4_t acc[2][4][4];                                       // [half of A][block of rows][block of columns]
#pragma unroll
    for (int h = 0; h < 2; h++)
#pragma unroll
        for (int j = 0; j < 4; j++)
#pragma unroll
            for (int i = 0; i < 4; i++) acc[h][j][i] = f32x4_t{0.f, 0.f, 0.f, 0.f};

    Places<T, AX, 128, 4> pa;
    Places<T, BX, 128, 4> pb;
    pa.init(lds_addr(lds), wp * 4, lane);
    pb.init(lds_addr(lds) + (wc >> 1) * UNIT, (wc & 1) * 4, lane);       // B1 lies behind B0: units go in twos
    // A half stage of 64 rows is done in four steps of two blocks: step q has blocks q % 2 * 2 and + 1, half q / 2 of the stage's k.  Two steps' fragments are on their way while one is multiplied.
    Frag<T, AX> fa[4][2];
    Frag<T, BX> fb[2][4];
    auto read_a = [&](auto Q, auto OFF) {
        constexpr int q = decltype(Q)::value;
        static_for<2>([&](auto J) { pa.template read<(q & 1) * 2 + decltype(J)::value, q / 2, decltype(OFF)::value>(fa[q][decltype(J)::value], 0u); });
    };
    auto read_b = [&](auto K, auto OFF) {
        constexpr int k = decltype(K)::value;
        static_for<4>([&](auto I) { pb.template read<decltype(I)::value, k, decltype(OFF)::value>(fb[k][decltype(I)::value], 0u); });
    };
    auto land_a = [&](auto Q) { static_for<2>([&](auto J) { fa[decltype(Q)::value][decltype(J)::value].land(); }); };
    auto land_b = [&](auto K) { static_for<4>([&](auto I) { fb[decltype(K)::value][decltype(I)::value].land(); }); };
    auto multiply = [&](auto H, auto Q, auto &&request) {       // eight products of half H, step Q, and a request among them
        constexpr int h = decltype(H)::value, q = decltype(Q)::value;
        static_for<8>([&](auto U) {
            constexpr int u = decltype(U)::value, j = u / 4, i = u % 4;
            Mma16<T>::run(acc[h][(q & 1) * 2 + j][i], fb[q / 2][i].get(), fa[q][j].get());
            if constexpr (u == 3) request();
        });
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr std::integral_constant<int, 0> C0{};
    constexpr std::integral_constant<int, 1> C1{};
    constexpr std::integral_constant<int, 2> C2{};
    constexpr std::integral_constant<int, 3> C3{};
    constexpr std::integral_constant<int, 2 * UNIT> FIRST_A0{};

    wait_vmcnt<6 * UL>();                                       // B and A0 of the first stage have landed
    __builtin_amdgcn_s_barrier();
    read_b(C0, C0);
    read_b(C1, C0);
    read_a(C0, FIRST_A0);
    read_a(C1, FIRST_A0);
    wait_lgkmcnt<0>();
    land_b(C0);
    land_b(C1);
    land_a(C0);
    land_a(C1);

    // The counts of the waits: LDS reads and DMAs land in the order in which they were issued, and each wait names how many were issued behind what it waits for.
    // One request per step and wave: a request holds its wave while the queue is full, and two at a time from eight waves fill it.
    unsigned asoff = 2 * astep, bsoff = 2 * bstep;              // of stage s + 2
    auto stage = [&](auto P, int s) {
        constexpr int p = decltype(P)::value;
        constexpr auto at = [](int k) { return (p * 4 + k) % NU; };      // unit k from this stage's B0 on
        constexpr std::integral_constant<int, at(2) * UNIT> A0{};
        constexpr std::integral_constant<int, at(3) * UNIT> A1{};
        constexpr std::integral_constant<int, at(4) * UNIT> BN{};
        constexpr std::integral_constant<int, at(6) * UNIT> AN{};
        constexpr std::integral_constant<int, at(0)> U0{};
        constexpr std::integral_constant<int, at(1)> U1{};
        constexpr std::integral_constant<int, at(2)> U2{};
        constexpr std::integral_constant<int, at(9)> U9{};
        // ---- A0 times B
        read_a(C2, A0);
        wait_lds<2 * RA + RBK>();
        land_a(C0);
        land_b(C0);
        multiply(C0, C0, [&] { request_b(C1, C0, U9, bsoff); });
        read_a(C3, A0);
        wait_lds<2 * RA + RBK>();
        land_a(C1);
        multiply(C0, C1, [&] { request_b(C1, C1, U9, bsoff); });
        wait_lgkmcnt<0>();                                      // all of A0 and B is in registers
        land_a(C2);
        land_a(C3);
        land_b(C1);
        wait_vmcnt<4 * UL>();                                   // A1 and the next stage's B have landed
        __builtin_amdgcn_s_barrier();                           // ... for every wave, and nobody reads A0 and B any more: units of later stages take their slots
        read_a(C0, A1);
        cut_last(s + 2);
        multiply(C0, C2, [&] { request_a(C0, C0, U0, asoff); });
        read_a(C1, A1);
        multiply(C0, C3, [&] { request_a(C0, C1, U0, asoff); });
        // ---- A1 times B; behind the last products with half of B's fragments the next stage's take their registers
        read_a(C2, A1);
        wait_lds<2 * RA>();
        land_a(C0);
        multiply(C1, C0, [&] { request_a(C1, C0, U1, asoff); });
        read_a(C3, A1);
        wait_lds<2 * RA>();
        land_a(C1);
        multiply(C1, C1, [&] { request_a(C1, C1, U1, asoff); });
        read_b(C0, BN);
        wait_lds<RBK>();                                        // all of A1 is in registers
        land_a(C2);
        land_a(C3);
        wait_vmcnt<5 * UL>();                                   // the next stage's A0 has landed
        __builtin_amdgcn_s_barrier();
        read_a(C0, AN);
        asoff += astep;
        bsoff += bstep;
        multiply(C1, C2, [&] { request_b(C0, C0, U2, bsoff); });
        read_a(C1, AN);
        multiply(C1, C3, [&] { request_b(C0, C1, U2, bsoff); });
        read_b(C1, BN);
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
    land_a(C0);
    land_a(C1);
    land_b(C0);
    land_b(C1);
    wait_vmcnt<0>();                                            // ... and its DMAs into dead slots
#pragma unroll
    for (int h = 0; h < 2; h++) write_results<T, KIND, 4, 4>(a, 0, acc[h], p0 + h * 128 + wp * 64, c0 + wc * 64, lane);
#endif
}

// ---- which kernel ----------------------------------------------------------------------------------------------------------------
// Times of the kernels in us as fitted to 270 products of 16 .. 8192 rows, columns and steps on 256 CUs, `s` the 128-byte stages of the reduction.  They put the fastest kernel
// first, or one within 3 %, in 19 of 20.  They are there to be compared with one another: the epilogue is not in them, and long bf16 products, which run at the power limit, take 20 to 35 %
// longer (us, these times and measured: 256-tiles 4096 x 4096, 4096 74, 100; 8192 x 8192, 8192 560, 754; 8192 x 16384, 4096 589, 798; 128-tiles 2048 x 2048, 8192 53, 66; fp32 within 4 %:
// 4096 x 4096, 4096 974, 950).
//   bf16   64 x 64 tiles (three workgroups a CU): 0.36 + 0.22 s for up to 256 of them, 0.69 + 0.166 s for every 256 beyond
//          128 x 128 tiles: 3.3 + 0.39 s for up to 256 (one workgroup a CU, a ring of four stages), 3.3 + 0.76 s for every 512 beyond (two a CU, rings of two)
//          256 x 256 tiles: 7.0 + 1.04 s for every 256
//   fp32   64 x 64 tiles: 0.87 + 0.55 s for every 256; 128 x 128 tiles: 2.85 + 1.88 s for every 256; 256 x 256 tiles were never better by more than 3 %
// For instance 2048 x 2048 with a reduction of 8192 in bf16: 256 tiles of 128 x 128 take 66 us, 1024 of 64 x 64 83 (88 by the formula).
// A reduction in p parts makes p times as many tiles of 1 / p of the stages, and costs one more launch and the parts' way to memory and back; up to
// 1024 tiles, 64 MB of parts.
static double tile_time(long tiles, double s, int tile, int dt) {
    const double rounds = (double)((tiles + 255) / 256);
    if (dt == SOL_F32) return tile == 64 ? rounds * (0.87 + 0.55 * s) : rounds * (2.85 + 1.88 * s);
    if (tile == 64) return rounds <= 1 ? 0.36 + 0.22 * s : rounds * (0.69 + 0.166 * s);
    if (tile == 128) return rounds <= 1 ? 3.3 + 0.39 * s : (double)((tiles + 511) / 512) * (3.3 + 0.76 * s);
    return rounds * (7.0 + 1.04 * s);
}

static double parts_time(long p, int M, int N) { return p > 1 ? 4.0 + 2e-6 * p * M * N : 0.0; }

GemmPlan plan_gemm(int M, int N, int K, int dt, bool may_split) {
    const long stages = ceil_div(K, ROWB / (int)dtype_size(dt));
    GemmPlan best{64, 1, 0.0};
    for (int tile = 64; tile <= (dt == SOL_BF16 ? 256 : 128); tile *= 2) {
        const long tiles = (long)ceil_div(M, tile) * ceil_div(N, tile), most = may_split && tile < 256 ? min(min(16l, stages / 2), 1024 / tiles) : 1;
        for (long p = 1; p <= max(1l, most); p++) {
            const double t = tile_time(tiles * p, (double)((stages + p - 1) / p), tile, dt) + parts_time(p, M, N);
            if (best.us == 0.0 || t < best.us) best = GemmPlan{tile, (int)p, t};
        }
    }
    return best;
}

// dx and dW in one launch of 64 x 64 tiles: the CUs are full where either alone would leave some idle, and a launch (3 us) is saved.  The time is that of as many tiles of the
// average number of stages, or of the longest one.  Whole backward passes, us, with the plans that are best one by one (in one launch only where both have tiles of 64) and so:
// 946 rows, 1398 -> 882, fp32 79, 66; 97, 3439 -> 1060, bf16 22.1, 15.9; 2115, 2187 -> 274, fp32 110, 91; 91, 2665 -> 1001, fp32 27.9, 32.4; over 119 drawn ones 0.7 % less.
bool plan_pair(int m, int in_f, int out_f, int dt, const GemmPlan &dx, const GemmPlan &dw, GemmPlan *px, GemmPlan *pw) {
    const double per = ROWB / (double)dtype_size(dt), sx = ceil(out_f / per), sw = ceil(m / per);
    const long tx = (long)ceil_div(m, 64) * ceil_div(in_f, 64), tw = (long)ceil_div(out_f, 64) * ceil_div(in_f, 64);
    const double alone = dx.us + dw.us + 3.0;
    double best = alone;
    for (int a = 1; a <= 16 && a * tx <= 1024 && (a == 1 || 2 * a <= sx); a++) {
        for (int b = 1; b <= 16 && b * tw <= 1024 && (b == 1 || 2 * b <= sw); b++) {
            const long tiles = a * tx + b * tw;
            const double launch = a > 1 && b > 1 ? 5.0 : a > 1 || b > 1 ? 1.0 : 0.0;      // one launch sums both; 3 us fit it here
            const double longest = ceil(sx / a) > ceil(sw / b) ? ceil(sx / a) : ceil(sw / b), all = tile_time(tiles, (tx * sx + tw * sw) / tiles, 64, dt), one = tile_time(1, longest, 64, dt);
            const double t = (all > one ? all : one) + parts_time(a, m, in_f) + parts_time(b, out_f, in_f) - launch;
            if (t < best) {
                best = t;
                *px = GemmPlan{64, a, t};
                *pw = GemmPlan{64, b, t};
            }
        }
    }
    return best < alone;
}

static long tiles_of(GemmArgs &a, int dt, int tile) {     // fills in the tile counts; workgroups of the launch
    a.ntp = ceil_div(a.M, tile);
    a.ntc = ceil_div(a.N, tile);
    a.steps = ceil_div(ceil_div(a.K, ROWB / (int)dtype_size(dt)), a.plan.split);
    return (long)ceil_div(a.ntp * a.ntc, 8) * 8 * a.plan.split;
}

template <typename T, GemmKind KIND, int WP, int WC, int RP, int RC, int NS, int PERCU> static void launch_tile(const GemmArgs &a, long blocks, hipStream_t st) {
    hipLaunchKernelGGL((linear_tile_kernel<T, KIND, WP, WC, RP, RC, NS, PERCU>), dim3((unsigned)blocks), dim3(WP * WC * 64), 0, st, a);
}

static thread_local int t_tile[3];             // see sol_debug_linear_tile
int &linear_tile_of_thread(GemmKind kind) { return t_tile[kind]; }

template <typename T, GemmKind KIND> static sol_status launch_kind(GemmArgs a, int dt, hipStream_t st) {
    int tile = a.plan.tile;
    if (tile == 256) {                       // its offsets along a reduction over rows have 32 bits, requests of whole tiles behind the last row included
        const double rows = a.K + 512.0, abytes = (KIND == GEMM_DW ? rows : 256.0) * a.lda * sizeof(T), bbytes = (KIND != GEMM_FORWARD ? rows : 256.0) * a.ldb * sizeof(T);
        if (abytes >= 4294967296.0 || bbytes >= 4294967296.0) tile = 128;
    }
    t_tile[KIND] = tile;
    const long blocks = tiles_of(a, dt, tile);
    if constexpr (sizeof(T) == 2 && KIND == GEMM_FORWARD) {
        // One workgroup a CU or fewer: a longer ring in the place of neighbours (3123 x 128, 7488: 31.0 -> 25.8 us; 469 x 384, 6080: 25.6 -> 21.2).  With 270 .. 350 tiles it loses
        // 2 to 3 %, and the products of the backward pass gain 4 % on average.
        if (tile == 64 && blocks <= 256) {
            launch_tile<T, KIND, 2, 2, 2, 2, 5, 2>(a, blocks, st);
            SOL_HIP(hipGetLastError());
            return SOL_OK;
        }
    }
    if (tile == 64) launch_tile<T, KIND, 2, 2, 2, 2, 3, 3>(a, blocks, st);
    else if constexpr (sizeof(T) == 2) {
        if (tile == 256) hipLaunchKernelGGL((linear_huge_kernel<KIND>), dim3((unsigned)blocks), dim3(512), 0, st, a);
        else {
            // eight waves of 32 x 64, or of 64 x 32 for dx, whose fragments of W take twice the LDS instructions (2470 x 2240, 3200: dx 39.6 against 43 us; dW 19.9, 20.3; forward 43, 43)
            constexpr int WP = KIND == GEMM_DX ? 2 : 4, WC = 8 / WP, RP = 8 / WP, RC = 8 / WC;
            if (blocks <= 256) launch_tile<T, KIND, WP, WC, RP, RC, 4, 1>(a, blocks, st);
            else launch_tile<T, KIND, WP, WC, RP, RC, 2, 2>(a, blocks, st);
        }
    } else launch_tile<T, KIND, 2, 4, 4, 2, 2, 2>(a, blocks, st);
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

sol_status launch_linear_gemm(const GemmArgs &a, int dt, GemmKind kind, hipStream_t st) {
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

sol_status launch_linear_pair(GemmArgs dx, GemmArgs dw, const SumJob &sum, int dt, hipStream_t st) {
    t_tile[GEMM_DX] = t_tile[GEMM_DW] = 64;
    const long first = tiles_of(dx, dt, 64), second = first + tiles_of(dw, dt, 64);
    const dim3 grid((unsigned)(second + (sum.n > 0 ? sum_blocks(sum) : 0)));
    if (dt == SOL_BF16) hipLaunchKernelGGL(linear_pair_kernel<bf16_t>, grid, dim3(256), 0, st, dx, dw, (int)first, (int)second, sum);
    else hipLaunchKernelGGL(linear_pair_kernel<float>, grid, dim3(256), 0, st, dx, dw, (int)first, (int)second, sum);
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

}  // namespace sol
