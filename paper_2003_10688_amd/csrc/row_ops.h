// What the kernels over rows of features share: sums over a wave and over groups of its lanes, loads and stores of pieces and ends of rows, checks of the arguments (internal).
// Times in the comments of these kernels are a kernel's own, called again on the same inputs, of which the last cache (256 MB) holds a part or all, where they name nothing else: 6 TB/s and more are
// its doing.  With inputs that it does not hold, copies of 256 MB to 1 GB reach 5.05 to 5.40 TB/s.
#pragma once
#include <utility>

#include "linear_ops.h"

namespace sol {

#define SOL_TRY(call)                          \
    do {                                       \
        const sol_status s_ = (call);          \
        if (s_ != SOL_OK) return s_;           \
    } while (0)

template <int CTRL, int ROWS> __device__ __forceinline__ float dpp_from(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), CTRL, ROWS, 0xf, false));
}
// The sum over a wave's 64 lanes, in all of them: neighbours, quads, halves of rows of 16, rows, and then rows through the last lane.  Six additions without LDS.
__device__ __forceinline__ float wave_sum(float v) {
    v += dpp_from<0xB1, 0xf>(v);         // lane ^ 1
    v += dpp_from<0x4E, 0xf>(v);         // lane ^ 2
    v += dpp_from<0x141, 0xf>(v);        // the other half of 8
    v += dpp_from<0x140, 0xf>(v);        // the other half of 16
    v += dpp_from<0x142, 0xa>(v);        // rows 1 and 3: + the row in front
    v += dpp_from<0x143, 0xc>(v);        // rows 2 and 3: + the first two
    return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// Stores 4 neighbouring elements of a row, of which nv exist, at any element's address
typedef __attribute__((ext_vector_type(2), aligned(2))) uint32_t u32x2_any;
template <typename T> __device__ __forceinline__ void store4_any(T *p, const float v[4], int nv) {
    if (nv >= 4) {
        if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2_any *>(p) = u32x2_any{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
        else *reinterpret_cast<u32x4_any *>(p) = lds_pipe::u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (e < nv) Elem<T>::store(p + e, v[e]);
    }
}

// W = 4 or 8 neighbouring elements, of which nv exist, as they lie in memory, so that loads under way take no more registers than that
template <typename T, int W> struct RawPiece {
    uint32_t w[W * sizeof(T) / 4] = {};
    // REPEAT: places behind the nv elements hold the last of them instead of 0
    template <bool REPEAT = false> __device__ __forceinline__ void load(const T *p, int nv) {
        if (nv >= W) {
            if constexpr (sizeof(w) == 8) {
                const u32x2_any v = *reinterpret_cast<const u32x2_any *>(p);
                w[0] = v.x; w[1] = v.y;
            } else {
#pragma unroll
                for (int i = 0; i < (int)sizeof(w) / 16; i++) {
                    const lds_pipe::u32x4_t v = reinterpret_cast<const u32x4_any *>(p)[i];
#pragma unroll
                    for (int e = 0; e < 4; e++) w[4 * i + e] = v[e];
                }
            }
        } else {
            float v[W];
#pragma unroll
            for (int e = 0; e < W; e++) v[e] = nv > 0 ? Elem<T>::load(p + min(e, nv - 1)) : 0.f;
#pragma unroll
            for (int e = 1; e < W; e++) v[e] = REPEAT || e < nv ? v[e] : 0.f;
            if constexpr (sizeof(T) == 2) {
#pragma unroll
                for (int e = 0; e < W / 2; e++) w[e] = __float_as_uint(v[2 * e]) >> 16 | (__float_as_uint(v[2 * e + 1]) & 0xffff0000u);
            } else {
#pragma unroll
                for (int e = 0; e < W; e++) w[e] = __float_as_uint(v[e]);
            }
        }
    }
    __device__ __forceinline__ float get(int e) const {
        if constexpr (sizeof(T) == 2) return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
        else return __uint_as_float(w[e]);
    }
};
template <typename T, int W> __device__ __forceinline__ void store_piece(T *p, const float *v, int nv) {
    if constexpr (W == 4) store4_any<T>(p, v, nv);
    else store8_any<T>(p, v, nv);
}
// The same for a whole piece, past the caches: results as large as the last cache would push out what is still to be read, and little of them would be left for their reader.
// (The choice has to be the kernel's, at compile time: behind a branch the compiler makes one ordinary store of both.)
constexpr size_t STREAM_BYTES = (size_t)256 << 20;
template <typename T, int W> __device__ __forceinline__ void stream_piece(T *p, const float *v) {
    uint32_t w[W * sizeof(T) / 4];
#pragma unroll
    for (int i = 0; i < (int)(sizeof(w) / 4); i++) w[i] = sizeof(T) == 4 ? __float_as_uint(v[i]) : pack_bf16x2(v[2 * i], v[2 * i + 1]);
    if constexpr (sizeof(w) == 8) __builtin_nontemporal_store(u32x2_any{w[0], w[1]}, reinterpret_cast<u32x2_any *>(p));
    else {
#pragma unroll
        for (int i = 0; i < (int)(sizeof(w) / 16); i++) __builtin_nontemporal_store(lds_pipe::u32x4_t{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]}, reinterpret_cast<u32x4_any *>(p) + i);
    }
}

// W neighbouring columns of a row for one thread.  The last thread of a row whose length is no multiple of W takes the row's last W columns, of which it leaves the first `skip` to the
// thread in front: a load of one piece like the others', which is waited for where it is used and not where it is asked for, as pieces put together of elements are.
// Only rows shorter than W end early.
template <int W> struct Span {
    int c, skip, end;               // columns c + skip .. c + end - 1 are this thread's; skip = W: none
    __device__ __forceinline__ Span(int at, int cols) : c(at), skip(0), end(W) {
        if (at >= cols) { c = 0; skip = W; }
        else if (cols < W) end = cols;
        else if (at + W > cols) { c = cols - W; skip = at - c; }
    }
    __device__ __forceinline__ bool some() const { return skip < W; }
    __device__ __forceinline__ bool has(int e) const { return e >= skip && e < end; }
    // WHOLE: the row's length is a multiple of W
    template <bool WHOLE, bool REPEAT = false, typename T> __device__ __forceinline__ void load(const T *row, RawPiece<T, W> &r) const {
        if (!some()) return;
        if (WHOLE || end == W) r.load(row + c, W);
        else r.template load<REPEAT>(row + c, end);
    }
    template <bool WHOLE, bool STREAM = false, typename T> __device__ __forceinline__ void store(T *row, const float *v) const {
        if (!some()) return;
        if (WHOLE || (skip == 0 && end == W)) {
            if constexpr (STREAM) stream_piece<T, W>(row + c, v);
            else store_piece<T, W>(row + c, v, W);
        } else {
#pragma unroll
            for (int e = 0; e < W; e++)
                if (has(e)) Elem<T>::store(row + c + e, v[e]);
        }
    }
};

// COUNT of them, `apart` columns from one to the next
template <int W, int COUNT> struct Spans {
    Span<W> of[COUNT];
    template <int... K> __device__ __forceinline__ Spans(int at, int apart, int cols, std::integer_sequence<int, K...>) : of{Span<W>(at + K * apart, cols)...} {}
    __device__ __forceinline__ Spans(int at, int apart, int cols) : Spans(at, apart, cols, std::make_integer_sequence<int, COUNT>()) {}
    __device__ __forceinline__ const Span<W> &operator[](int k) const { return of[k]; }
};

// The sum over groups of LANES lanes (8, 16, 32 or the wave's 64), in all of a group's lanes
template <int LANES> __device__ __forceinline__ float group_sum(float v) {
    if constexpr (LANES >= 64) return wave_sum(v);
    v += dpp_from<0xB1, 0xf>(v);
    v += dpp_from<0x4E, 0xf>(v);
    v += dpp_from<0x141, 0xf>(v);
    if constexpr (LANES >= 16) v += dpp_from<0x140, 0xf>(v);
    if constexpr (LANES >= 32) v += __uint_as_float((uint32_t)__builtin_amdgcn_ds_swizzle((int)__float_as_uint(v), 0x401f));      // lane ^ 16
    return v;
}

constexpr int MAX_COLS = 1 << 20, MAX_ROW_PITCH = 1 << 21;

inline sol_status check_row_pitch(const char *what, int cols, int *ld) {
    if (*ld == 0) *ld = cols;
    SOL_REQUIRE(*ld >= cols, SOL_ERR_SHAPE, "pitch %d of %s is less than its %d columns", *ld, what, cols);
    SOL_REQUIRE(*ld <= MAX_ROW_PITCH, SOL_ERR_UNSUPPORTED, "pitch %d of %s is more than 2^21", *ld, what);
    return SOL_OK;
}
inline sol_status check_scratch(const void *workspace, size_t have, size_t need) {
    SOL_REQUIRE(have >= need, SOL_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", have, need);
    SOL_REQUIRE(workspace || need == 0, SOL_ERR_NULL, "workspace is NULL");
    SOL_REQUIRE(aligned16(workspace), SOL_ERR_ALIGN, "workspace must be 16-byte aligned");
    return SOL_OK;
}

}  // namespace sol
