// Embedding and the gradient of its table.
//   forward   y[i] = scale * table[tokens[i]];  a padding token: zeros;  any other token outside the table: NaN
//   backward  dtable[v] = scale * sum of the dy[i] with tokens[i] = v, in the order of i
#include <float.h>

#include "row_ops.h"

namespace sol {
namespace {

// Lanes that a row takes: up to a wave's 64, 8 columns each; wider rows are cut into slabs of 512 columns.
int row_lanes_log2(int cols) {
    const int groups = ceil_div(cols, 8);
    int l = 3;
    while (l < 6 && (1 << l) < groups) l++;
    return l;
}
int row_slabs(int cols) { return ceil_div(cols, 512); }

struct EmbedArgs {
    const void *tokens, *table;
    void *y;
    long ldt, ldy;
    int n, vocab, cols, pad, lanes_log2;
    float scale;
};
template <typename T, typename I> __global__ void __launch_bounds__(256) embed_kernel(const EmbedArgs a) {
    const int lane = threadIdx.x & ((1 << a.lanes_log2) - 1), slot = threadIdx.x >> a.lanes_log2;
    const int c = ((int)blockIdx.y * 64 + lane) * 8, nv = min(8, a.cols - c);
    if (nv <= 0) return;
    for (long i = (long)blockIdx.x * (256 >> a.lanes_log2) + slot; i < a.n; i += (long)gridDim.x * (256 >> a.lanes_log2)) {
        const I tok = static_cast<const I *>(a.tokens)[i];
        float v[8];
        if (tok != (I)a.pad && tok >= 0 && tok < (I)a.vocab) {
            load8_any<T>(static_cast<const T *>(a.table) + (long)tok * a.ldt + c, v, nv);
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] *= a.scale;
        } else {
            const float none = tok == (I)a.pad ? 0.f : __uint_as_float(0x7fc00000u);
#pragma unroll
            for (int e = 0; e < 8; e++) v[e] = none;
        }
        store8_any<T>(static_cast<T *>(a.y) + i * a.ldy + c, v, nv);
    }
}

// ---- the gradient's first half: positions sorted by token --------------------------------------------------------------------
// Every workgroup owns a range of the table's rows and reads all tokens, twice: once to count those of its rows and those in front of them, once to write the positions of
// its rows' tokens, in order, behind each other.  So it takes one launch, without a word between the workgroups.  The tokens are read from L2.
constexpr int INDEX_THREADS = 1024, INDEX_EACH = 16, INDEX_TILE = INDEX_THREADS * INDEX_EACH, INDEX_ROWS = 8192, INDEX_GROUPS = 256;
constexpr int RUN = 64;         // longer runs of one token are summed in parts of the sorted order, RUN positions each

struct IndexArgs {
    const void *tokens;
    int n, vocab, pad, rows;    // rows: of the table, per workgroup
    int *start, *order, *sorted;    // [vocab + 1], [n], [n]
};

// 16 neighbouring tokens; -1 where there is none or it has no row
template <typename I> __device__ __forceinline__ void load_tokens(const IndexArgs &a, int at, int t[INDEX_EACH]) {
    const I *p = static_cast<const I *>(a.tokens) + at;
    constexpr int PER = 16 / sizeof(I);
    if (at + INDEX_EACH <= a.n) {
        uint4 raw[INDEX_EACH / PER];
#pragma unroll
        for (int q = 0; q < INDEX_EACH / PER; q++) raw[q] = reinterpret_cast<const uint4 *>(p)[q];
#pragma unroll
        for (int j = 0; j < INDEX_EACH; j++) {
            const I tok = reinterpret_cast<const I *>(raw)[j];
            t[j] = tok != (I)a.pad && tok >= 0 && tok < (I)a.vocab ? (int)tok : -1;
        }
    } else {
#pragma unroll
        for (int j = 0; j < INDEX_EACH; j++) {
            const I tok = at + j < a.n ? p[j] : (I)-1;
            t[j] = tok != (I)a.pad && tok >= 0 && tok < (I)a.vocab ? (int)tok : -1;
        }
    }
}

__device__ __forceinline__ int wave_scan(int v) {       // sum over the lanes up to this one
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(v, d);
        v += lane >= d ? o : 0;
    }
    return v;
}
// Sum over the threads in front of this one; *total: over all.  One set of slots: a barrier in front and one behind the writing.
__device__ __forceinline__ int block_scan(int v, int *slots, int *total) {
    const int inc = wave_scan(v), w = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 63) slots[w] = inc;
    __syncthreads();
    int before = 0, all = 0;
#pragma unroll
    for (int q = 0; q < INDEX_THREADS / 64; q++) {
        const int s = slots[q];
        before += q < w ? s : 0;
        all += s;
    }
    *total = all;
    return before + inc - v;
}

template <typename I> __global__ void __launch_bounds__(INDEX_THREADS) embed_index_kernel(const IndexArgs a) {
    __shared__ uint32_t next[INDEX_ROWS];               // counts, then where the next position of each row goes
    __shared__ uint32_t list[INDEX_TILE];               // a tile's tokens of this range: row << 14 | place in the tile
    __shared__ int slots[INDEX_THREADS / 64];
    const int lo = (int)blockIdx.x * a.rows, hi = min(a.vocab, lo + a.rows), mine = hi - lo;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int r = threadIdx.x; r < a.rows; r += INDEX_THREADS) next[r] = 0;
    __syncthreads();
    int t[INDEX_EACH], less = 0;
    for (int base = 0; base < a.n; base += INDEX_TILE) {
        const int at = base + threadIdx.x * INDEX_EACH;
        if (at >= a.n) continue;
        load_tokens<I>(a, at, t);
#pragma unroll
        for (int j = 0; j < INDEX_EACH; j++) {
            less += t[j] >= 0 && t[j] < lo ? 1 : 0;
            if (t[j] >= lo && t[j] < hi) atomicAdd(&next[t[j] - lo], 1u);
        }
    }
    int before;
    block_scan(less, slots, &before);                   // its barriers are behind the counts too
    const int each = (a.rows + INDEX_THREADS - 1) / INDEX_THREADS, r0 = threadIdx.x * each, r1 = min(mine, r0 + each);
    int sum = 0, here;
    for (int r = r0; r < r1; r++) sum += (int)next[r];
    int at = before + block_scan(sum, slots, &here);
    for (int r = r0; r < r1; r++) {
        const int k = (int)next[r];
        next[r] = (uint32_t)at;
        a.start[lo + r] = at;
        at += k;
    }
    if (hi == a.vocab && threadIdx.x == 0) a.start[a.vocab] = before + here;
    if (here == 0) return;
    for (int base = 0; base < a.n; base += INDEX_TILE) {
        const int at0 = base + threadIdx.x * INDEX_EACH;
        int found = 0;
        if (at0 < a.n) {
            load_tokens<I>(a, at0, t);
#pragma unroll
            for (int j = 0; j < INDEX_EACH; j++) found += t[j] >= lo && t[j] < hi ? 1 : 0;
        }
        int total;
        int to = block_scan(found, slots, &total);      // its first barrier: next[] is there, and the list's last readers are through
        if (found) {
#pragma unroll
            for (int j = 0; j < INDEX_EACH; j++)
                if (t[j] >= lo && t[j] < hi) list[to++] = (uint32_t)(t[j] - lo) << 14 | (uint32_t)(threadIdx.x * INDEX_EACH + j);
        }
        __syncthreads();
        // each wave takes the rows of one residue, 64 entries at a time; equal rows among them by one ballot per different row
        for (int i = 0; i < total; i += 64) {
            const uint32_t e = i + lane < total ? list[i + lane] : 0xffffffffu;
            const int row = (int)(e >> 14);
            const bool own = e != 0xffffffffu && (row & 15) == w;
            unsigned long long left = __ballot(own);
            while (left) {
                const int first = __ffsll((unsigned long long)left) - 1, r = __builtin_amdgcn_readlane(row, first);
                const unsigned long long same = __ballot(own && row == r);
                uint32_t dst = 0;
                if (lane == first) dst = atomicAdd(&next[r], (uint32_t)__popcll(same));
                dst = (uint32_t)__builtin_amdgcn_readlane((int)dst, first);
                if (own && row == r) {
                    dst += (uint32_t)__popcll(same & ((1ull << lane) - 1));
                    a.order[dst] = base + (int)(e & 16383u);
                    a.sorted[dst] = lo + r;
                }
                left &= ~same;
            }
        }
    }
}

// ---- its second half: sums over the sorted order ------------------------------------------------------------------------------
struct GatherArgs {
    const void *dy;
    void *out;
    const int *start, *order, *sorted;
    float *part;                // [windows][2][cols]: sums of the parts of long runs that a window of RUN positions holds, of the run that reaches in first, of the one that leaves it second
    long ldy;
    int n, vocab, cols, windows, accumulate, lanes_log2;
    float scale;
};

// acc += the rows order[b .. e), in that order; eight loads under way at a time
template <typename T> __device__ __forceinline__ void sum_rows(const GatherArgs &a, int b, int e, int c, int nv, float acc[8]) {
    const T *dy = static_cast<const T *>(a.dy) + c;
    for (; b + 8 <= e; b += 8) {
        float v[8][8];
#pragma unroll
        for (int u = 0; u < 8; u++) load8_any<T>(dy + (long)a.order[b + u] * a.ldy, v[u], nv);
#pragma unroll
        for (int u = 0; u < 8; u++)
#pragma unroll
            for (int k = 0; k < 8; k++) acc[k] += v[u][k];
    }
    for (; b < e; b++) {
        float v[8];
        load8_any<T>(dy + (long)a.order[b] * a.ldy, v, nv);
#pragma unroll
        for (int k = 0; k < 8; k++) acc[k] += v[k];
    }
}

template <typename TO> __device__ __forceinline__ void put_row(const GatherArgs &a, int v, int c, int nv, float acc[8]) {
    TO *out = static_cast<TO *>(a.out) + (size_t)v * a.cols + c;
    float old[8];
    if (a.accumulate) load8_any<TO>(out, old, nv);
#pragma unroll
    for (int k = 0; k < 8; k++) acc[k] = a.accumulate ? acc[k] * a.scale + old[k] : acc[k] * a.scale;
    store8_any<TO>(out, acc, nv);
}

// Items: the parts of long runs in each window, two a window, then the table's rows
template <typename T, typename TO> __global__ void __launch_bounds__(256) embed_gather_kernel(const GatherArgs a) {
    const int lane = threadIdx.x & ((1 << a.lanes_log2) - 1), slot = threadIdx.x >> a.lanes_log2;
    const long item = (long)blockIdx.x * (256 >> a.lanes_log2) + slot;
    const int c = ((int)blockIdx.y * 64 + lane) * 8, nv = min(8, a.cols - c);
    if (item >= (long)a.vocab + 2 * a.windows || nv <= 0) return;
    float acc[8];
#pragma unroll
    for (int k = 0; k < 8; k++) acc[k] = 0.f;
    if (item >= 2 * a.windows) {
        const int v = (int)(item - 2 * a.windows), b = a.start[v], e = a.start[v + 1];
        if (e - b > RUN || (a.accumulate && e == b)) return;
        sum_rows<T>(a, b, e, c, nv, acc);
        put_row<TO>(a, v, c, nv, acc);
        return;
    }
    const int win = (int)(item >> 1), used = a.start[a.vocab], w0 = win * RUN, w1 = min(used, w0 + RUN);
    if (w0 >= w1) return;
    const int first = a.sorted[w0], last = a.sorted[w1 - 1];
    if ((item & 1) && last == first) return;
    const int v = item & 1 ? last : first, b = a.start[v], e = a.start[v + 1];
    if (e - b <= RUN) return;
    sum_rows<T>(a, max(b, w0), min(e, w1), c, nv, acc);
    store8_any<float>(a.part + (size_t)item * a.cols + c, acc, nv);
}

// A long run ends behind the window that it starts in: at most one starts in each
template <typename TO> __global__ void __launch_bounds__(256) embed_join_kernel(const GatherArgs a) {
    const int lane = threadIdx.x & ((1 << a.lanes_log2) - 1), slot = threadIdx.x >> a.lanes_log2;
    const long win = (long)blockIdx.x * (256 >> a.lanes_log2) + slot;
    const int c = ((int)blockIdx.y * 64 + lane) * 8, nv = min(8, a.cols - c), used = a.start[a.vocab];
    if (win >= a.windows || nv <= 0 || win * RUN >= used) return;
    const int v = a.sorted[min(used, (int)win * RUN + RUN) - 1], b = a.start[v], e = a.start[v + 1];
    if (e - b <= RUN || b / RUN != win) return;
    float acc[8], p[8];
#pragma unroll
    for (int k = 0; k < 8; k++) acc[k] = 0.f;
    for (int w = (int)win; w * RUN < e; w++) {
        load8_any<float>(a.part + (size_t)(2 * w + (w == win && b % RUN ? 1 : 0)) * a.cols + c, p, nv);
#pragma unroll
        for (int k = 0; k < 8; k++) acc[k] += p[k];
    }
    put_row<TO>(a, v, c, nv, acc);
}

sol_status check_embed(const sol_embedding_desc *ed, sol_embedding_desc *d) {
    SOL_REQUIRE(ed, SOL_ERR_NULL, "embedding descriptor is NULL");
    *d = *ed;
    SOL_REQUIRE(d->dtype == SOL_F32 || d->dtype == SOL_BF16, SOL_ERR_DTYPE, "embedding: unknown dtype %d", d->dtype);
    SOL_REQUIRE(d->token_bits == 32 || d->token_bits == 64, SOL_ERR_DTYPE, "embedding: tokens of %d bits", d->token_bits);
    SOL_REQUIRE(d->tokens >= 0 && d->vocab > 0 && d->cols > 0, SOL_ERR_SHAPE, "bad embedding shape: %d tokens, table [%d,%d]", d->tokens, d->vocab, d->cols);
    SOL_REQUIRE(d->tokens <= 1 << 30 && d->vocab <= 1 << 24 && d->cols <= MAX_COLS, SOL_ERR_UNSUPPORTED, "more than 2^30 tokens, 2^24 rows or 2^20 columns: %d tokens, table [%d,%d]",
                d->tokens, d->vocab, d->cols);
    SOL_REQUIRE(d->scale >= -FLT_MAX && d->scale <= FLT_MAX, SOL_ERR_SHAPE, "embedding: scale %g", (double)d->scale);       // refuses a NaN too
    SOL_TRY(check_row_pitch("table", d->cols, &d->ldt));
    SOL_TRY(check_row_pitch("y", d->cols, &d->ldy));
    return SOL_OK;
}

struct EmbedPlan {
    size_t start, order, sorted, part, bytes;
    int windows;
};
EmbedPlan embed_plan(const sol_embedding_desc &d) {
    EmbedPlan p{};
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at = round_up(at + bytes, 256); return here; };
    p.windows = d.tokens > RUN ? ceil_div(d.tokens, RUN) : 0;       // no run is longer than the tokens are
    p.start = take(((size_t)d.vocab + 1) * 4);
    p.order = take((size_t)d.tokens * 4);
    p.sorted = take((size_t)d.tokens * 4);
    p.part = take((size_t)p.windows * 2 * d.cols * 4);
    p.bytes = at;
    return p;
}

template <typename T, typename TO> sol_status launch_gather(const GatherArgs &g, hipStream_t st) {
    const int per = 256 >> g.lanes_log2, slabs = row_slabs(g.cols);
    const long items = (long)g.vocab + 2 * g.windows;
    hipLaunchKernelGGL((embed_gather_kernel<T, TO>), dim3((unsigned)((items + per - 1) / per), (unsigned)slabs), dim3(256), 0, st, g);
    SOL_HIP(hipGetLastError());
    if (g.windows) {
        hipLaunchKernelGGL(embed_join_kernel<TO>, dim3((unsigned)ceil_div(g.windows, per), (unsigned)slabs), dim3(256), 0, st, g);
        SOL_HIP(hipGetLastError());
    }
    return SOL_OK;
}

}  // namespace
}  // namespace sol

using namespace sol;

extern "C" {

sol_status sol_embedding(const sol_embedding_desc *ed, const void *tokens, const void *table, void *y, void *stream) {
    sol_embedding_desc d;
    SOL_TRY(check_embed(ed, &d));
    if (d.tokens == 0) return SOL_OK;
    SOL_REQUIRE(tokens && table && y, SOL_ERR_NULL, "tokens, table and y must not be NULL");
    SOL_REQUIRE(aligned16(tokens) && aligned16(table) && aligned16(y), SOL_ERR_ALIGN, "device pointers must be 16-byte aligned");
    SOL_REQUIRE(y != table && y != tokens, SOL_ERR_UNSUPPORTED, "embedding: y must not alias the table or the tokens");
    hipStream_t st = (hipStream_t)stream;
    const EmbedArgs a{tokens, table, y, d.ldt, d.ldy, d.tokens, d.vocab, d.cols, d.pad, row_lanes_log2(d.cols), d.scale};
    const int per = 256 >> a.lanes_log2;
    const dim3 grid((unsigned)min(ceil_div(d.tokens, per), 1 << 16), (unsigned)row_slabs(d.cols));
    if (d.dtype == SOL_BF16) {
        if (d.token_bits == 64) hipLaunchKernelGGL((embed_kernel<bf16_t, int64_t>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((embed_kernel<bf16_t, int32_t>), grid, dim3(256), 0, st, a);
    } else {
        if (d.token_bits == 64) hipLaunchKernelGGL((embed_kernel<float, int64_t>), grid, dim3(256), 0, st, a);
        else hipLaunchKernelGGL((embed_kernel<float, int32_t>), grid, dim3(256), 0, st, a);
    }
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}

size_t sol_embedding_backward_workspace_bytes(const sol_embedding_desc *ed) {
    sol_embedding_desc d;
    return check_embed(ed, &d) == SOL_OK ? embed_plan(d).bytes : 0;
}

sol_status sol_embedding_backward(const sol_embedding_desc *ed, const void *tokens, const void *dy, void *dtable, int dtable_dtype, int accumulate, void *workspace, size_t workspace_bytes,
                                  void *stream) {
    sol_embedding_desc d;
    SOL_TRY(check_embed(ed, &d));
    SOL_REQUIRE(dtable_dtype == d.dtype || dtable_dtype == SOL_F32, SOL_ERR_DTYPE, "dtable is of the table's dtype or fp32, not %d", dtable_dtype);
    SOL_REQUIRE(dtable && (d.tokens == 0 || (tokens && dy)), SOL_ERR_NULL, "tokens, dy and dtable must not be NULL");
    SOL_REQUIRE(aligned16(tokens) && aligned16(dy) && aligned16(dtable), SOL_ERR_ALIGN, "device pointers must be 16-byte aligned");
    SOL_REQUIRE(dtable != dy && dtable != tokens, SOL_ERR_UNSUPPORTED, "embedding backward: dtable must not alias dy or the tokens");
    const EmbedPlan p = embed_plan(d);
    SOL_TRY(check_scratch(workspace, workspace_bytes, p.bytes));
    hipStream_t st = (hipStream_t)stream;
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    int *start = reinterpret_cast<int *>(ws + p.start), *order = reinterpret_cast<int *>(ws + p.order), *sorted = reinterpret_cast<int *>(ws + p.sorted);
    const int rows = min(INDEX_ROWS, max(1, ceil_div(d.vocab, INDEX_GROUPS)));
    const IndexArgs x{tokens, d.tokens, d.vocab, d.pad, rows, start, order, sorted};
    const dim3 grid((unsigned)ceil_div(d.vocab, rows));
    if (d.token_bits == 64) hipLaunchKernelGGL(embed_index_kernel<int64_t>, grid, dim3(INDEX_THREADS), 0, st, x);
    else hipLaunchKernelGGL(embed_index_kernel<int32_t>, grid, dim3(INDEX_THREADS), 0, st, x);
    SOL_HIP(hipGetLastError());
    const GatherArgs g{dy, dtable, start, order, sorted, reinterpret_cast<float *>(ws + p.part), d.ldy, d.tokens, d.vocab, d.cols, p.windows, accumulate ? 1 : 0, row_lanes_log2(d.cols), d.scale};
    if (d.dtype == SOL_F32) return launch_gather<float, float>(g, st);
    return dtable_dtype == SOL_F32 ? launch_gather<bf16_t, float>(g, st) : launch_gather<bf16_t, bf16_t>(g, st);
}

}  // extern "C"
