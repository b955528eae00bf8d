// C entry points of the linear layer with its epilogue, its backward pass, and dropout: checks of the arguments, plans, workspaces.
#include <math.h>

#include "linear_ops.h"

namespace sol {
namespace {

#define SOL_TRY(call) \
    do { \
        const sol_status s_ = (call); \
        if (s_ != SOL_OK) return s_; \
    } while (0)

constexpr int MAX_FEATURES = 1 << 20, MAX_PITCH = 1 << 21;

sol_status check_drop(const sol_dropout_desc *d, DropArgs *out) {
    *out = DropArgs{0, 0, 0, nullptr, 0, 1.f};
    if (!d) return SOL_OK;
    SOL_REQUIRE(d->p >= 0.f && d->p <= 1.f, SOL_ERR_SHAPE, "dropout probability %g is not in 0 .. 1", (double)d->p);       // refuses a NaN too
    SOL_REQUIRE((reinterpret_cast<uintptr_t>(d->step) & 3u) == 0, SOL_ERR_ALIGN, "dropout's step word must be 4-byte aligned");
    const int t = (int)lrint((double)d->p * 65536.0);
    *out = DropArgs{(uint32_t)d->seed, (uint32_t)(d->seed >> 32), d->call, d->step, (uint32_t)t, t < 65536 ? (float)(65536.0 / (65536 - t)) : 0.f};
    return SOL_OK;
}

sol_status check_pitch(const char *what, int rows, int cols, int *ld) {
    if (*ld == 0) *ld = cols;
    SOL_REQUIRE(*ld >= cols, SOL_ERR_SHAPE, "pitch %d of %s is less than its %d columns", *ld, what, cols);
    SOL_REQUIRE(*ld <= MAX_PITCH, SOL_ERR_UNSUPPORTED, "pitch %d of %s is more than 2^21", *ld, what);
    SOL_REQUIRE((double)rows * *ld < 2147483648.0, SOL_ERR_UNSUPPORTED, "%s spans 2^31 elements or more", what);
    return SOL_OK;
}

int pack_pitch(int n, int dt) { return (int)round_up((size_t)n, dt == SOL_BF16 ? 64 : 32); }
// rows that DMA can take as they are: they start and end at multiples of 16 bytes
bool rows_aligned(int ld, int cols, int dt) { return (ld * dtype_size(dt)) % 16 == 0 && (cols * dtype_size(dt)) % 16 == 0; }

// *l: the description with every pitch filled in
sol_status check_linear(const sol_linear_desc *ld, sol_linear_desc *l) {
    SOL_REQUIRE(ld, SOL_ERR_NULL, "linear descriptor is NULL");
    *l = *ld;
    SOL_REQUIRE(l->dtype == SOL_F32 || l->dtype == SOL_BF16, SOL_ERR_DTYPE, "linear: unknown dtype %d", l->dtype);
    SOL_REQUIRE(l->m >= 0 && l->in_f > 0 && l->out_f > 0, SOL_ERR_SHAPE, "bad linear shape m=%d in=%d out=%d", l->m, l->in_f, l->out_f);
    SOL_REQUIRE(l->in_f <= MAX_FEATURES && l->out_f <= MAX_FEATURES, SOL_ERR_UNSUPPORTED, "more than 2^20 features: in=%d out=%d", l->in_f, l->out_f);
    SOL_REQUIRE((double)l->in_f * l->out_f < 1073741824.0, SOL_ERR_UNSUPPORTED, "weight too large");
    SOL_REQUIRE(l->act >= SOL_ACT_NONE && l->act <= SOL_ACT_SILU, SOL_ERR_SHAPE, "bad activation %d", l->act);
    SOL_TRY(check_pitch("x", l->m, l->in_f, &l->ldx));
    SOL_TRY(check_pitch("y", l->m, l->out_f, &l->ldy));
    SOL_TRY(check_pitch("residual", l->m, l->out_f, &l->ldr));
    // The copy of x to aligned rows counts its groups of 8 elements, and the step of its grid (2^21 threads at most) beyond the last of them, in 32 bits.  A few features
    // make much more of a copy than of x: the element count of x does not bound it.
    if (!rows_aligned(l->ldx, l->in_f, l->dtype))
        SOL_REQUIRE((size_t)l->m * (pack_pitch(l->in_f, l->dtype) / 8) <= MAX_PAD_GROUPS, SOL_ERR_UNSUPPORTED, "%d rows of x to be copied to rows of %d elements: more than 2^35 - 2^24",
                    l->m, pack_pitch(l->in_f, l->dtype));
    return SOL_OK;
}

bool cut_needed(int k, int dt) { return (k * dtype_size(dt)) % 128 != 0; }

struct ForwardPlan {
    size_t bytes;
    bool pad;
};
ForwardPlan forward_plan(const sol_linear_desc &l) {
    ForwardPlan p{};
    p.pad = !rows_aligned(l.ldx, l.in_f, l.dtype);
    if (p.pad) p.bytes = (size_t)l.m * pack_pitch(l.in_f, l.dtype) * dtype_size(l.dtype);
    return p;
}

struct BackwardPlan {
    size_t dz, part, xpad, dw_sums, dx_sums, bytes;     // offsets
    bool pad, pair;
    GemmPlan dw, dx, pair_dw, pair_dx;      // one by one; in one launch (pair)
};
BackwardPlan backward_plan(const sol_linear_desc &l) {
    BackwardPlan p{};
    const size_t es = dtype_size(l.dtype);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at = round_up(at + bytes, 256); return here; };
    p.dz = take((size_t)l.m * pack_pitch(l.out_f, l.dtype) * es);
    p.part = take((size_t)linear_dz_chunks(l.m, l.out_f) * l.out_f * 4);
    p.pad = !rows_aligned(l.ldx, l.in_f, l.dtype);
    p.xpad = take(p.pad ? (size_t)l.m * pack_pitch(l.in_f, l.dtype) * es : 0);
    p.dw = plan_gemm(l.out_f, l.in_f, l.m, l.dtype, true);
    p.dx = plan_gemm(l.m, l.in_f, l.out_f, l.dtype, true);
    p.pair = plan_pair(l.m, l.in_f, l.out_f, l.dtype, p.dx, p.dw, &p.pair_dx, &p.pair_dw);
    const int wparts = p.pair ? max(p.dw.split, p.pair_dw.split) : p.dw.split, xparts = p.pair ? max(p.dx.split, p.pair_dx.split) : p.dx.split;
    p.dw_sums = take(wparts > 1 ? (size_t)wparts * l.out_f * l.in_f * 4 : 0);
    p.dx_sums = take(xparts > 1 ? (size_t)xparts * l.m * l.in_f * 4 : 0);
    p.bytes = at;
    return p;
}

sol_status check_workspace(const void *workspace, size_t have, size_t need) {
    SOL_REQUIRE(have >= need, SOL_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", have, need);
    SOL_REQUIRE(workspace || need == 0, SOL_ERR_NULL, "workspace is NULL");
    SOL_REQUIRE(aligned16(workspace), SOL_ERR_ALIGN, "workspace must be 16-byte aligned");
    return SOL_OK;
}

int row_bytes(int cols, int dt) { return cols * (int)dtype_size(dt); }

}  // namespace
}  // namespace sol

using namespace sol;

extern "C" {

size_t sol_linear_fused_workspace_bytes(const sol_linear_desc *ld) {
    sol_linear_desc l;
    return check_linear(ld, &l) == SOL_OK && l.m > 0 ? forward_plan(l).bytes : 0;
}

size_t sol_linear_backward_workspace_bytes(const sol_linear_desc *ld) {
    sol_linear_desc l;
    return check_linear(ld, &l) == SOL_OK && l.m > 0 ? backward_plan(l).bytes : 0;
}

sol_status sol_linear_fused(const sol_linear_desc *ld, const void *x, const void *w_packed, const float *bias, const sol_dropout_desc *drop, const void *residual, void *y,
                            void *preact, void *workspace, size_t workspace_bytes, void *stream) {
    sol_linear_desc l;
    DropArgs d;
    SOL_TRY(check_linear(ld, &l));
    SOL_TRY(check_drop(drop, &d));
    if (l.m == 0) return SOL_OK;
    SOL_REQUIRE(x && w_packed && y, SOL_ERR_NULL, "x, w_packed and y must not be NULL");
    SOL_REQUIRE(aligned16(x) && aligned16(w_packed) && aligned16(bias) && aligned16(residual) && aligned16(y) && aligned16(preact), SOL_ERR_ALIGN,
                "device pointers must be 16-byte aligned");
    SOL_REQUIRE(y != x && y != w_packed && preact != x && preact != w_packed && (!preact || (preact != y && preact != residual)), SOL_ERR_UNSUPPORTED,
                "linear: outputs must not alias inputs or each other");
    SOL_REQUIRE(y != residual || l.ldy == l.ldr, SOL_ERR_UNSUPPORTED, "linear: y in the residual's place needs its pitch");
    const ForwardPlan p = forward_plan(l);
    SOL_TRY(check_workspace(workspace, workspace_bytes, p.bytes));
    hipStream_t st = (hipStream_t)stream;
    const int kp = pack_pitch(l.in_f, l.dtype);

    GemmArgs a{};
    a.a = x; a.lda = l.ldx; a.a_row = row_bytes(l.in_f, l.dtype); a.a_cut = cut_needed(l.in_f, l.dtype);
    if (p.pad) {
        SOL_TRY(launch_pad_rows(PadRows{x, workspace, l.ldx, kp, l.m, l.in_f}, l.dtype, st));
        a.a = workspace; a.lda = kp; a.a_row = row_bytes(kp, l.dtype); a.a_cut = 0;
    }
    a.b = w_packed; a.ldb = kp; a.b_row = row_bytes(kp, l.dtype);
    a.M = l.m; a.N = l.out_f; a.K = l.in_f; a.plan = plan_gemm(l.m, l.out_f, l.in_f, l.dtype, false);
    a.epi = LinearEpi{bias, residual, y, preact, l.ldr, l.ldy, l.act, d};
    const double us = linear_rows_time(a, l.dtype);
    if (us >= 0.0 && us < a.plan.us) return launch_linear_rows(a, l.dtype, st);
    return launch_linear_gemm(a, l.dtype, GEMM_FORWARD, st);
}

sol_status sol_linear_backward(const sol_linear_desc *ld, const void *dy, const void *x, const void *w_packed, const void *preact, const sol_dropout_desc *drop, void *dx, void *dw,
                               int dw_dtype, float *db, void *workspace, size_t workspace_bytes, void *stream) {
    sol_linear_desc l;
    DropArgs d;
    SOL_TRY(check_linear(ld, &l));
    SOL_TRY(check_drop(drop, &d));
    SOL_REQUIRE(!dw || dw_dtype == l.dtype || dw_dtype == SOL_F32, SOL_ERR_DTYPE, "dw is of the layer's dtype or fp32, not %d", dw_dtype);
    SOL_REQUIRE(aligned16(dy) && aligned16(x) && aligned16(w_packed) && aligned16(preact) && aligned16(dx) && aligned16(dw) && aligned16(db), SOL_ERR_ALIGN,
                "device pointers must be 16-byte aligned");
    hipStream_t st = (hipStream_t)stream;
    SumJobs sums{};
    if (l.m == 0) {
        if (dw) sums.add(nullptr, 0, (long)l.out_f * l.in_f, dw, dw_dtype);
        if (db) sums.add(nullptr, 0, l.out_f, db, SOL_F32);
        return launch_sums(sums, st);
    }
    SOL_REQUIRE(dy && (x || !dw) && (w_packed || !dx), SOL_ERR_NULL, "dy, x (for dw) and w_packed (for dx) must not be NULL");
    SOL_REQUIRE(preact || l.act == SOL_ACT_NONE, SOL_ERR_NULL, "preact must not be NULL with an activation");
    const void *const outs[3] = {dx, dw, db}, *const ins[4] = {dy, x, w_packed, preact};
    for (int i = 0; i < 3; i++) {
        for (const void *in : ins) SOL_REQUIRE(!outs[i] || outs[i] != in, SOL_ERR_UNSUPPORTED, "linear backward: outputs must not alias inputs");
        for (int j = 0; j < i; j++) SOL_REQUIRE(!outs[i] || outs[i] != outs[j], SOL_ERR_UNSUPPORTED, "linear backward: outputs must not alias each other");
    }
    const BackwardPlan p = backward_plan(l);
    SOL_TRY(check_workspace(workspace, workspace_bytes, p.bytes));
    unsigned char *ws = static_cast<unsigned char *>(workspace);

    // dz is dy itself where neither an activation nor dropout lies between them
    const bool own_dz = (dx || dw) && (l.act != SOL_ACT_NONE || d.t || !rows_aligned(l.ldy, l.out_f, l.dtype));
    const long ldz = own_dz ? pack_pitch(l.out_f, l.dtype) : l.ldy;
    const void *dz = own_dz ? ws + p.dz : dy;
    const int dz_row = row_bytes(own_dz ? (int)ldz : l.out_f, l.dtype);
    const int kp = pack_pitch(l.in_f, l.dtype);
    const PadRows pad = dw && p.pad ? PadRows{x, ws + p.xpad, l.ldx, kp, l.m, l.in_f} : PadRows{nullptr, nullptr, 0, 8, 0, 0};
    SumJob columns{};
    if (own_dz || db) {
        const int chunks = linear_dz_chunks(l.m, l.out_f);
        float *part = !db ? nullptr : chunks == 1 ? db : reinterpret_cast<float *>(ws + p.part);
        SOL_TRY(launch_linear_dz(dy, l.ldy, preact, own_dz ? ws + p.dz : nullptr, ldz, l.m, l.out_f, l.act, d, l.dtype, part, pad, st));
        if (db && chunks > 1) columns = SumJob{part, chunks, l.out_f, db, SOL_F32};
    } else if (pad.x) {
        SOL_TRY(launch_pad_rows(pad, l.dtype, st));
    }
    const bool pair = p.pair && dx && dw;
    GemmArgs ax{}, aw{};
    if (dx) {
        ax.a = dz; ax.lda = ldz; ax.a_row = dz_row; ax.a_cut = !own_dz && cut_needed(l.out_f, l.dtype);
        ax.b = w_packed; ax.ldb = kp; ax.b_row = row_bytes(kp, l.dtype);
        ax.M = l.m; ax.N = l.in_f; ax.K = l.out_f; ax.plan = pair ? p.pair_dx : p.dx;
        ax.part = reinterpret_cast<float *>(ws + p.dx_sums);
        ax.out = dx; ax.ldo = l.in_f; ax.out_dt = l.dtype;
        if (ax.plan.split > 1) sums.add(ax.part, ax.plan.split, (long)l.m * l.in_f, dx, l.dtype);
    }
    if (dw) {
        aw.a = dz; aw.lda = ldz; aw.a_row = dz_row;
        aw.b = x; aw.ldb = l.ldx; aw.b_row = row_bytes(l.in_f, l.dtype);
        if (p.pad) {
            aw.b = ws + p.xpad; aw.ldb = kp; aw.b_row = row_bytes(kp, l.dtype);
        }
        aw.M = l.out_f; aw.N = l.in_f; aw.K = l.m; aw.plan = pair ? p.pair_dw : p.dw;
        aw.part = reinterpret_cast<float *>(ws + p.dw_sums);
        aw.out = dw; aw.ldo = l.in_f; aw.out_dt = dw_dtype;
        if (aw.plan.split > 1) sums.add(aw.part, aw.plan.split, (long)l.out_f * l.in_f, dw, dw_dtype);
    }
    if (pair) {
        SOL_TRY(launch_linear_pair(ax, aw, columns, l.dtype, st));
    } else {
        if (dx) SOL_TRY(launch_linear_gemm(ax, l.dtype, GEMM_DX, st));
        if (dw) SOL_TRY(launch_linear_gemm(aw, l.dtype, GEMM_DW, st));
        if (columns.n > 0) sums.add(columns.part, columns.nsplit, columns.n, columns.out, columns.out_dt);
    }
    return launch_sums(sums, st);
}

int sol_debug_linear_tile(int product) { return product >= GEMM_FORWARD && product <= GEMM_DW ? linear_tile_of_thread((GemmKind)product) : 0; }

sol_status sol_dropout(int rows, int cols, sol_dtype dt, const void *x, const sol_dropout_desc *drop, const void *residual, void *y, void *stream) {
    SOL_REQUIRE(dt == SOL_F32 || dt == SOL_BF16, SOL_ERR_DTYPE, "dropout: unknown dtype %d", (int)dt);
    SOL_REQUIRE(rows >= 0 && cols > 0, SOL_ERR_SHAPE, "bad dropout shape [%d,%d]", rows, cols);
    SOL_REQUIRE((double)rows * cols < 2147483648.0, SOL_ERR_UNSUPPORTED, "dropout: 2^31 elements or more");
    SOL_REQUIRE(drop, SOL_ERR_NULL, "dropout descriptor is NULL");
    DropArgs d;
    SOL_TRY(check_drop(drop, &d));
    if (rows == 0) return SOL_OK;
    SOL_REQUIRE(x && y, SOL_ERR_NULL, "x and y must not be NULL");
    SOL_REQUIRE(aligned16(x) && aligned16(residual) && aligned16(y), SOL_ERR_ALIGN, "device pointers must be 16-byte aligned");
    return launch_dropout(x, residual, y, rows, cols, dt, d, (hipStream_t)stream);
}

}  // extern "C"
