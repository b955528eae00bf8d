// What the kernels over rows of features share: sums over a wave and a workgroup, checks of the arguments (internal).
#pragma once
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
