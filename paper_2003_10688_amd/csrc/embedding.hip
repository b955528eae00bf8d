// Embedding and the gradient of its table.
//   forward   y[i] = scale * table[tokens[i]];  a padding token: zeros;  any other token outside the table: NaN
//   backward  dtable[v] = scale * sum of the dy[i] with tokens[i] = v.  Rows of up to CROWD tokens (up to RUN of more than DIRECT in all) have them added in the order of i; longer ones in
//             stretches, which are summed by the waves that have them and then put together: an order that the tokens alone fix.
#include <float.h>

#include <type_traits>

#include "row_ops.h"

namespace sol {
namespace {

// Lanes that a row takes: 8 to a wave's 64, so many columns each
int row_lanes_log2(int cols, int each) {
    const int pieces = ceil_div(cols, each);
    int l = 3;
    while (l < 6 && (1 << l) < pieces) l++;
    return l;
}

struct EmbedArgs {
    const void *tokens, *table;
    void *y;
    long ldt, ldy;
    int n, vocab, cols, pad, lanes_log2;
    float scale;
};
// 16 bytes of a row for a lane: 2^lanes_log2 lanes, or slabs of 64, which vary fastest (see embed_sum_kernel); KEEP tokens of a lane under way at a time.  65536 tokens of 2048 bf16: one token 99 us,
// two 96, four 90 with ordinary stores, 54 to 57 with two to eight past the caches; 8 tokens of 4096 4.2, 4.5 and 5.2 us.
constexpr int KEEP = 2;
template <typename T, typename I, bool STREAM> __global__ void __launch_bounds__(256) embed_kernel(const EmbedArgs a) {
    constexpr int W = 16 / sizeof(T);
    const int lane = threadIdx.x & ((1 << a.lanes_log2) - 1), slot = threadIdx.x >> a.lanes_log2, per = 256 >> a.lanes_log2;
    const Span<W> sp(((int)blockIdx.x * 64 + lane) * W, a.cols);
    for (long i0 = (long)blockIdx.y * (per * KEEP) + slot; i0 < a.n; i0 += (long)gridDim.y * (per * KEEP)) {
        I tok[KEEP];
        RawPiece<T, W> raw[KEEP];
#pragma unroll
        for (int k = 0; k < KEEP; k++) tok[k] = static_cast<const I *>(a.tokens)[min(i0 + k * per, (long)a.n - 1)];
#pragma unroll
        for (int k = 0; k < KEEP; k++)
            if (tok[k] != (I)a.pad && tok[k] >= 0 && tok[k] < (I)a.vocab) sp.template load<false>(static_cast<const T *>(a.table) + (long)tok[k] * a.ldt, raw[k]);
#pragma unroll
        for (int k = 0; k < KEEP; k++) {
            if (i0 + k * per >= a.n) break;
            const bool row = tok[k] != (I)a.pad && tok[k] >= 0 && tok[k] < (I)a.vocab;
            const float none = tok[k] == (I)a.pad ? 0.f : __uint_as_float(0x7fc00000u);
            float v[W];
#pragma unroll
            for (int e = 0; e < W; e++) v[e] = row ? raw[k].get(e) * a.scale : none;
            sp.template store<false, STREAM>(static_cast<T *>(a.y) + (i0 + k * per) * a.ldy, v);
        }
    }
}

// ---- the gradient's first half: positions sorted by token --------------------------------------------------------------------
// The tokens' order is that of (v mod G, v / G) for G workgroups: each owns the rows of one residue, so that neighbouring rows, which frequent tokens often are, fall to different
// ones, and reads all tokens.  It counts those of each of its rows and those of the residues in front, keeps what is its own in a list, in order, and writes the positions
// of its rows' tokens behind each other.  So it takes one launch, without a word between the workgroups.  The tokens are read from L2, a second time where the list does not hold
// a workgroup's share.  65536 tokens of text 22 us (358 with neighbouring rows in one workgroup, which then has half of all tokens), 4096 9 us; every 16384 more take 4 us,
// 3 where tokens are spread evenly.  That is for tables of up to 2^18 rows, 1024 for each of 256 workgroups.  A longer table takes as many more workgroups, each of which looks at all tokens, one to a CU:
// 65536 tokens 33 to 36 us for 2^18 + 1 rows, 61 to 63 for 2^20, 211 to 217 for 2^22, 800 to 814 for 2^24 (the sums of 8 columns fp32 then take 52, 93, 255 and 1124).  Where all tokens are the same, one
// workgroup has them all: 4096 10 us, 16384 18, 65536 88, 262144 339, and the launch that joins the run's parts 4, 11, 38 and 143.
constexpr int INDEX_THREADS = 1024, INDEX_EACH = 16, INDEX_TILE = INDEX_THREADS * INDEX_EACH, INDEX_ROWS = 1024, INDEX_GROUPS = 256, INDEX_WAVES = INDEX_THREADS / 64;
constexpr int LIST_BITS = 22;   // of a position in a list's entry, the row's 10 above them
constexpr int RUN = 64;         // longer runs of one token are summed in parts of the sorted order, RUN positions each

struct IndexArgs {
    const void *tokens;
    int n, vocab, pad, rows, log2;  // 2^log2 workgroups, `rows` of the table each
    int *start, *order, *sorted;    // [places + 1], [n], [n]: a row's place is (v mod G) * rows + v / G
};

// A tile is PIECES pieces of 4 neighbouring tokens a thread: lanes next to each other read next to each other.  t: the tokens, where[j]: the lanes of the wave whose token j is this workgroup's own.
// Returns how many of this thread's belong to the residues in front.  What a token costs here is what the launch costs, since every workgroup looks at every token: six vector instructions, and as few
// scalar ones as can be, which all waves of a CU share one unit for.  PAD: the padding token is a row of the table.
constexpr int PIECES = INDEX_EACH / 4;
typedef unsigned long long lanes_t;
template <typename I, bool PAD> __device__ __forceinline__ uint32_t look_at_tokens(const IndexArgs &a, int base, uint32_t t[INDEX_EACH], lanes_t where[INDEX_EACH]) {
    const I *p = static_cast<const I *>(a.tokens);
    I raw[INDEX_EACH];
#pragma unroll
    for (int q = 0; q < PIECES; q++) {
        const int at = base + q * (INDEX_THREADS * 4) + (int)threadIdx.x * 4;
        if (at + 4 <= a.n) {
#pragma unroll
            for (int k = 0; k < (int)sizeof(I) / 4; k++) reinterpret_cast<lds_pipe::u32x4_t *>(raw + q * 4)[k] = reinterpret_cast<const u32x4_any *>(p + at)[k];
        } else {
#pragma unroll
            for (int j = 0; j < 4; j++) raw[q * 4 + j] = at + j < a.n ? p[at + j] : (I)-1;
        }
    }
    uint32_t less = 0;
    const uint32_t mine = blockIdx.x, mask = (1u << a.log2) - 1, vocab = (uint32_t)a.vocab;
#pragma unroll
    for (int j = 0; j < INDEX_EACH; j++) {
        typedef typename std::conditional<sizeof(I) == 8, uint64_t, uint32_t>::type U;
        t[j] = (uint32_t)raw[j];
        uint32_t res = (U)raw[j] < (U)vocab ? t[j] & mask : 0xffffffffu;       // a negative one is not below it
        if (PAD) res = raw[j] == (I)a.pad ? 0xffffffffu : res;
        where[j] = __ballot(res == mine);
        less += res < mine ? 1u : 0u;
    }
    return less;
}
__device__ __forceinline__ int place_in_tile(int j) { return (j >> 2) * (INDEX_THREADS * 4) + (int)threadIdx.x * 4 + (j & 3); }

// Sum over the lanes up to this one: rows of 16 by shifts, then the rows in front through their last lanes
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false);
    v += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false);
    return v;
}
// Two sums over the waves in front of this one of what each wave has; *total: over all.  One set of slots: a barrier in front and one behind the writing.
__device__ __forceinline__ uint2 sum_waves(uint2 v, uint2 *slots, uint2 *total) {
    const int w = threadIdx.x >> 6;
    __syncthreads();
    if ((threadIdx.x & 63) == 63) slots[w] = v;
    __syncthreads();
    uint2 before = make_uint2(0, 0), all = make_uint2(0, 0);
#pragma unroll
    for (int q = 0; q < INDEX_WAVES; q++) {
        const uint2 s = slots[q];
        before.x += q < w ? s.x : 0;
        before.y += q < w ? s.y : 0;
        all.x += s.x;
        all.y += s.y;
    }
    *total = all;
    return before;
}

struct IndexShared {
    uint32_t list[INDEX_TILE];                      // this residue's tokens, in order: row << LIST_BITS | position behind the list's base
    uint32_t count[INDEX_WAVES][INDEX_ROWS];        // of the rows in each wave's part of the list; then where each wave's next position of a row goes
    uint32_t next[INDEX_ROWS];                      // of all rows so far; then where the next position of each row goes
    uint2 slots[INDEX_WAVES];
};

// Appends a tile's tokens of this residue to the list, which has `have` entries, unless it would not hold them.  Returns how many there are then.
__device__ __forceinline__ int index_append(const IndexArgs &a, IndexShared &s, int behind, const uint32_t t[INDEX_EACH], const lanes_t where[INDEX_EACH], int have) {
    static_assert(PIECES == 4, "two counts in a word, two words");
    uint32_t found[2];                  // the pieces' counts, two in a word: a piece has 4096 tokens
#pragma unroll
    for (int k = 0; k < 2; k++) {
        int n[2] = {0, 0};
#pragma unroll
        for (int j = 0; j < 8; j++) n[j >> 2] += __popcll(where[8 * k + j]);
        found[k] = (uint32_t)n[0] | (uint32_t)n[1] << 16;
    }
    uint2 all;
    const uint2 before = sum_waves(make_uint2(found[0], found[1]), s.slots, &all);      // behind its first barrier the list's last readers are through
    const int many = (int)((all.x & 0xffff) + (all.x >> 16) + (all.y & 0xffff) + (all.y >> 16));
    if ((found[0] | found[1]) && have + many <= INDEX_TILE) {
        const uint32_t piece[PIECES] = {all.x & 0xffff, all.x >> 16, all.y & 0xffff, 0};
        const uint32_t wave[PIECES] = {before.x & 0xffff, before.x >> 16, before.y & 0xffff, before.y >> 16};
        uint32_t first = (uint32_t)have;
#pragma unroll
        for (int q = 0; q < PIECES; q++) {
            if (where[4 * q] | where[4 * q + 1] | where[4 * q + 2] | where[4 * q + 3]) {
                uint32_t to = first + wave[q];          // + those of the lanes in front
#pragma unroll
                for (int j = 0; j < 4; j++) to = __builtin_amdgcn_mbcnt_hi((uint32_t)(where[4 * q + j] >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)where[4 * q + j], to));
#pragma unroll
                for (int j = 0; j < 4; j++)
                    if (where[4 * q + j] >> (threadIdx.x & 63) & 1) s.list[to++] = (t[4 * q + j] >> a.log2) << LIST_BITS | (uint32_t)(behind + place_in_tile(4 * q + j));
            }
            first += piece[q];
        }
    }
    return have + many;
}

// The lanes whose row is this lane's, of those that have one
__device__ __forceinline__ lanes_t same_row(uint32_t row, bool has, int bits) {
    lanes_t same = __ballot(has);
    if (__ballot(has && row != (uint32_t)__builtin_amdgcn_readfirstlane((int)row)) == 0) return same;       // a frequent token's; lane 0 has one
    for (int b = 0; b < bits; b++) {
        const lanes_t one = __ballot(has && (row >> b & 1));
        same &= row >> b & 1 ? one : ~one;
    }
    return same;
}
// Each wave takes a part of the list, 64 entries at a time, in order; short lists have parts for a few waves only
__device__ __forceinline__ int part_length(int total) { return (total + INDEX_THREADS - 1) / INDEX_THREADS * 64; }
__device__ __forceinline__ int parts_of(int total) { return total ? (total + part_length(total) - 1) / part_length(total) : 0; }
template <typename F> __device__ __forceinline__ void index_part(const IndexShared &s, int total, int bits, F f) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, per = part_length(total), end = min(total, (w + 1) * per);
    for (int i = w * per; i < end; i += 64) {
        const bool has = i + lane < end;
        const uint32_t e = has ? s.list[i + lane] : 0u;
        f(w, e, has, same_row(e >> LIST_BITS, has, bits));
    }
}
// count[w][r]: how many entries of row r wave w's part has.  Ends with a barrier.
__device__ __forceinline__ void index_count(const IndexArgs &a, IndexShared &s, int total, int bits) {
    const int parts = parts_of(total);
    if ((int)threadIdx.x < a.rows)
        for (int w = 0; w < parts; w++) s.count[w][threadIdx.x] = 0;
    __syncthreads();
    index_part(s, total, bits, [&](int w, uint32_t e, bool has, lanes_t same) {
        if (has && (int)__ffsll(same) - 1 == (int)(threadIdx.x & 63)) s.count[w][e >> LIST_BITS] += (uint32_t)__popcll(same);
    });
    __syncthreads();
}
// Writes the positions of the list, whose counts are there, from next[] on, which moves behind them
__device__ __forceinline__ void index_place(const IndexArgs &a, IndexShared &s, int total, int bits, int base) {
    const int r = threadIdx.x, parts = parts_of(total);
    if (r < a.rows) {
        uint32_t at = s.next[r];
        for (int w = 0; w < parts; w++) {
            const uint32_t k = s.count[w][r];
            s.count[w][r] = at;
            at += k;
        }
        s.next[r] = at;
    }
    __syncthreads();
    index_part(s, total, bits, [&](int w, uint32_t e, bool has, lanes_t same) {
        const uint32_t row = e >> LIST_BITS, lane = threadIdx.x & 63;
        const uint32_t first = has ? s.count[w][row] : 0u;
        if (has) {
            const uint32_t dst = first + (uint32_t)__popcll(same & ((1ull << lane) - 1));
            a.order[dst] = base + (int)(e & ((1u << LIST_BITS) - 1));
            a.sorted[dst] = (int)blockIdx.x * a.rows + (int)row;
            if ((uint32_t)__ffsll(same) - 1 == lane) s.count[w][row] = first + (uint32_t)__popcll(same);
        }
    });
}

template <typename I, bool PAD> __global__ void __launch_bounds__(INDEX_THREADS) embed_index_kernel(const IndexArgs a) {
    __shared__ IndexShared s;
    const int r = (int)threadIdx.x, bits = 32 - __clz(a.rows - 1);      // 0 for one row
    s.next[r] = 0;
    uint32_t t[INDEX_EACH], less = 0;
    lanes_t where[INDEX_EACH];
    int have = 0;
    bool whole = a.n <= 1 << LIST_BITS;                 // the list has all of this residue, positions from the first token on
    auto add_counts = [&]() {
        index_count(a, s, have, bits);
        const int parts = parts_of(have);
        if (r < a.rows)
            for (int w = 0; w < parts; w++) s.next[r] += s.count[w][r];
    };
    for (int base = 0; base < a.n; base += INDEX_TILE) {
        less += look_at_tokens<I, PAD>(a, base, t, where);
        const int then = index_append(a, s, whole ? base : 0, t, where, have);
        if (then <= INDEX_TILE) {
            have = then;
            continue;
        }
        whole = false;
        add_counts();
        have = index_append(a, s, 0, t, where, 0);      // its barrier is behind the last reading of the list
    }
    __syncthreads();
    add_counts();
    uint2 all;
    const uint32_t count = s.next[r], up_to = wave_scan(count);      // next[r] is this thread's own
    const uint2 before = sum_waves(make_uint2((uint32_t)__builtin_amdgcn_readlane((int)up_to, 63), (uint32_t)__builtin_amdgcn_readlane((int)wave_scan(less), 63)), s.slots, &all);
    const uint32_t at = all.y + before.x + up_to - count;
    s.next[r] = at;
    if (r < a.rows) a.start[(int)blockIdx.x * a.rows + r] = (int)at;
    if (blockIdx.x == gridDim.x - 1 && r == 0) a.start[(int)gridDim.x * a.rows] = (int)(all.x + all.y);
    if (whole) {
        index_place(a, s, have, bits, 0);
        return;
    }
    for (int base = 0; base < a.n; base += INDEX_TILE) {
        look_at_tokens<I, PAD>(a, base, t, where);
        have = index_append(a, s, 0, t, where, 0);
        __syncthreads();
        index_count(a, s, have, bits);
        index_place(a, s, have, bits, base);
    }
}

// ---- its second half: sums over the sorted order ------------------------------------------------------------------------------
struct GatherArgs {
    const void *dy;
    void *out;
    const int *start, *order, *sorted;
    float *part;                // [windows][2][cols]: sums of the parts of long runs that a window of RUN positions holds, of the run that reaches in first, of the one that leaves it second
    long ldy;
    int vocab, cols, windows, accumulate;
    int rows, log2, places;         // as the index has them
    float scale;
    FastDiv by_rows;
};
__device__ __forceinline__ int row_of_place(const GatherArgs &a, int place) {
    uint32_t q, r;
    a.by_rows.divmod((uint32_t)place, q, r);
    return (int)(r << a.log2 | q);
}

// Items: the parts of long runs in each window, two a window, then the table's rows.  A part of a long run:
struct Part { int place, b, e; };
__device__ __forceinline__ bool window_part(const GatherArgs &a, int item, Part *q) {
    const int used = a.start[a.places], w0 = (item >> 1) * RUN, w1 = min(used, w0 + RUN);
    if (w0 >= w1) return false;
    const int first = a.sorted[w0], last = a.sorted[w1 - 1];
    if ((item & 1) && last == first) return false;
    const int p = item & 1 ? last : first, b = a.start[p], e = a.start[p + 1];
    if (e - b <= RUN) return false;
    *q = Part{p, max(b, w0), min(e, w1)};
    return true;
}
__device__ __forceinline__ int place_of_row(const GatherArgs &a, int v) { return (v & ((1 << a.log2) - 1)) * a.rows + (v >> a.log2); }

// acc += `many` rows (FLIGHT at most, all of them with FULL: no branch between the loads, which are then under way together); next() gives them one by one
template <int FLIGHT, bool FULL, typename T, int W, int PIECES, typename F>
__device__ __forceinline__ void add_rows(const T *dy, long ldy, const Spans<W, PIECES> &sp, int many, float (&acc)[PIECES][W], F next) {
    RawPiece<T, W> raw[FLIGHT][PIECES];
#pragma unroll
    for (int u = 0; u < FLIGHT; u++)
        if (FULL || u < many) {
            const T *p = dy + (long)next() * ldy;
#pragma unroll
            for (int i = 0; i < PIECES; i++) sp[i].template load<false>(p, raw[u][i]);
        }
#pragma unroll
    for (int u = 0; u < FLIGHT; u++)
        if (FULL || u < many) {
#pragma unroll
            for (int i = 0; i < PIECES; i++)
#pragma unroll
                for (int k = 0; k < W; k++) acc[i][k] += raw[u][i].get(k);
        }
}

// scale * acc into a row, or onto it
template <typename TO, int W, int PIECES, bool STREAM>
__device__ __forceinline__ void write_row(TO *out, const Spans<W, PIECES> &sp, float (&acc)[PIECES][W], float scale, int accumulate) {
#pragma unroll
    for (int i = 0; i < PIECES; i++) {
        RawPiece<TO, W> old;
        if (accumulate) sp[i].template load<false>(out, old);
#pragma unroll
        for (int k = 0; k < W; k++) acc[i][k] = accumulate ? acc[i][k] * scale + old.get(k) : acc[i][k] * scale;
        sp[i].template store<false, STREAM>(out, acc[i]);
    }
}

// A wave takes PIECES * 64 * W columns of a row, up to 1024.  Three round trips to memory: where its run is, the positions in it (a lane each), and FLIGHT of the gradient's rows at a time.
// Bound by memory where it is large: 65536 tokens of text, table 65536 x 2048, bf16 to fp32 125 us (6.3 TB/s, a part of the gradient from the last cache; 165 to 190 with results that go through
// the caches).  A row to a wave: the rows of frequent tokens are neighbours, and two rows a wave took 274 us in place of 224 for the whole gradient.
template <typename T, typename TO, int W, int PIECES, bool STREAM> __device__ __forceinline__ void sum_item(const GatherArgs &a, int item, int c0) {
    constexpr int FLIGHT = 64 / (W * PIECES);
    const int lane = threadIdx.x & 63;
    const bool window = item < 2 * a.windows;
    Part q;
    if (window) {
        if (!window_part(a, item, &q)) return;
    } else {
        const int p = place_of_row(a, item - 2 * a.windows);
        q = Part{p, a.start[p], a.start[p + 1]};
        if (q.e - q.b > RUN || (a.accumulate && q.e == q.b)) return;
    }
    const T *dy = static_cast<const T *>(a.dy);
    const Spans<W, PIECES> sp(c0, 64 * W, a.cols);
    const int many = q.e - q.b, order = lane < many ? a.order[q.b + lane] : 0;        // RUN of them at most
    float acc[PIECES][W];
#pragma unroll
    for (int i = 0; i < PIECES; i++)
#pragma unroll
        for (int k = 0; k < W; k++) acc[i][k] = 0.f;
    int j = 0;
    auto next = [&]() { return __builtin_amdgcn_readlane(order, j++); };
    while (j + FLIGHT <= many) add_rows<FLIGHT, true>(dy, a.ldy, sp, FLIGHT, acc, next);
    if (j < many) add_rows<FLIGHT, false>(dy, a.ldy, sp, many - j, acc, next);
    if (window) {
        float *part = a.part + (size_t)item * a.cols;
#pragma unroll
        for (int i = 0; i < PIECES; i++) sp[i].template store<false>(part, acc[i]);
        return;
    }
    write_row<TO, W, PIECES, STREAM>(static_cast<TO *>(a.out) + (size_t)(item - 2 * a.windows) * a.cols, sp, acc, a.scale, a.accumulate);
}
// Slabs of columns vary fastest: workgroups that run together then write whole rows, not the same part of every row, whose addresses would fall on a few of the memory's channels
// (326 us in place of 258 then; rows in the order of their places, 2 MB apart, 938).
template <typename T, typename TO, int W, int PIECES, bool STREAM> __global__ void __launch_bounds__(256) embed_sum_kernel(const GatherArgs a, int items) {
    const int c0 = (int)blockIdx.x * (PIECES * 64 * W) + (threadIdx.x & 63) * W;
    for (int item = (int)blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); item < items; item += (int)gridDim.y * 4) sum_item<T, TO, W, PIECES, STREAM>(a, item, c0);
}

// A long run ends behind the window that it starts in: at most one starts in each.  A workgroup joins its parts in a slab of columns, a wave a quarter of them, one behind the other.
template <typename TO, int W, int PIECES> __global__ void __launch_bounds__(256) embed_join_kernel(const GatherArgs a) {
    constexpr int FLIGHT = 64 / (W * PIECES);
    __shared__ float sums[3][PIECES * W][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, used = a.start[a.places];
    const Spans<W, PIECES> sp((int)blockIdx.x * (PIECES * 64 * W) + lane * W, 64 * W, a.cols);
    for (long win = blockIdx.y; win < a.windows && win * RUN < used; win += gridDim.y) {
        const int p = a.sorted[min(used, (int)win * RUN + RUN) - 1], b = a.start[p], e = a.start[p + 1];
        if (e - b <= RUN || b / RUN != win) continue;       // the same for all threads
        const int last = (e - 1) / RUN, per = (last - (int)win + 4) / 4, w0 = (int)win + wave * per, many = min(last + 1, w0 + per) - w0;
        float acc[PIECES][W];
#pragma unroll
        for (int i = 0; i < PIECES; i++)
#pragma unroll
            for (int k = 0; k < W; k++) acc[i][k] = 0.f;
        int w = w0;
        auto next = [&]() {                                 // the parts' rows
            const long row = 2 * (long)w + (w == (int)win && b % RUN ? 1 : 0);
            w++;
            return row;
        };
        while (w + FLIGHT <= w0 + many) add_rows<FLIGHT, true>(a.part, a.cols, sp, FLIGHT, acc, next);
        if (w < w0 + many) add_rows<FLIGHT, false>(a.part, a.cols, sp, w0 + many - w, acc, next);
        __syncthreads();                                    // the sums of a run in front are read
        if (wave > 0) {
#pragma unroll
            for (int i = 0; i < PIECES; i++)
#pragma unroll
                for (int k = 0; k < W; k++) sums[wave - 1][i * W + k][lane] = acc[i][k];
        }
        __syncthreads();
        if (wave > 0) continue;
#pragma unroll
        for (int i = 0; i < PIECES; i++)
#pragma unroll
            for (int k = 0; k < W; k++) acc[i][k] += sums[0][i * W + k][lane] + sums[1][i * W + k][lane] + sums[2][i * W + k][lane];
        write_row<TO, W, PIECES, false>(static_cast<TO *>(a.out) + (size_t)row_of_place(a, p) * a.cols, sp, acc, a.scale, a.accumulate);
    }
}

// ---- the gradient of few tokens, in one launch ----------------------------------------------------------------------------------
// A workgroup looks at all tokens, lists those of its `block` rows in order, and sums and writes its rows, a wave each, or all four where a row has more than CROWD tokens.  A wave's tokens are added
// one behind the other, so there can only be few; the rows without tokens, nearly all of them, are what the time goes into.  509 tokens, table 10007 x 201 fp32: 9 us, 20 in three launches; 512 equal tokens 18 and 36.
constexpr int DIRECT = 512, CROWD = 32;
struct DirectArgs {
    const void *tokens, *dy;
    void *out;
    long ldy;
    int n, vocab, cols, pad, block, accumulate;
    float scale;
};
template <typename T, typename TO, typename I, int W, int PIECES, bool STREAM> __global__ void __launch_bounds__(256) embed_direct_kernel(const DirectArgs a) {
    constexpr int FLIGHT = 64 / (W * PIECES);
    __shared__ uint32_t list[DIRECT];                   // row in the block << 16 | position
    __shared__ int counts[4];
    __shared__ float sums[3][PIECES * W][64];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Spans<W, PIECES> sp((int)blockIdx.x * (PIECES * 64 * W) + lane * W, 64 * W, a.cols);
    const T *dy = static_cast<const T *>(a.dy);
    int tok[2];
#pragma unroll
    for (int j = 0; j < 2; j++) {
        const int i = (int)threadIdx.x * 2 + j;
        const I t = i < a.n ? static_cast<const I *>(a.tokens)[i] : (I)-1;
        tok[j] = i < a.n && t != (I)a.pad && t >= 0 && t < (I)a.vocab ? (int)t : -1;
    }
    for (int v0 = (int)blockIdx.y * a.block; v0 < a.vocab; v0 += (int)gridDim.y * a.block) {
        const int v1 = min(a.vocab, v0 + a.block);
        const bool own0 = tok[0] >= v0 && tok[0] < v1, own1 = tok[1] >= v0 && tok[1] < v1;
        const lanes_t m0 = __ballot(own0), m1 = __ballot(own1);
        if (lane == 0) counts[w] = __popcll(m0) + __popcll(m1);
        __syncthreads();
        int at = 0, total = 0;
#pragma unroll
        for (int q = 0; q < 4; q++) {
            at += q < w ? counts[q] : 0;
            total += counts[q];
        }
        at = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m0 >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m0, (uint32_t)at));
        at = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m1 >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m1, (uint32_t)at));
        if (own0) list[at++] = (uint32_t)(tok[0] - v0) << 16 | threadIdx.x * 2;
        if (own1) list[at] = (uint32_t)(tok[1] - v0) << 16 | (threadIdx.x * 2 + 1);
        __syncthreads();
        // With a crowded list every wave looks at every row; one of more than CROWD tokens is summed by all four, 64 entries of the list in turn.  Else the waves take the rows in turn.
        const bool crowded = total > CROWD;
        uint32_t rows[DIRECT / 64];                     // the list's rows, 64 entries a lane each
#pragma unroll
        for (int c = 0; c < DIRECT / 64; c++) rows[c] = c * 64 + lane < total ? list[c * 64 + lane] >> 16 : 0xffffu;
        for (int r = crowded ? 0 : w; v0 + r < v1; r += crowded ? 1 : 4) {
            int many = 0;
#pragma unroll
            for (int c = 0; c < DIRECT / 64; c++)
                if (c * 64 < total) many += __popcll(__ballot((int)rows[c] == r));
            const bool shared = many > CROWD;
            if (crowded && !shared && (r & 3) != w) continue;
            float acc[PIECES][W];
#pragma unroll
            for (int i = 0; i < PIECES; i++)
#pragma unroll
                for (int k = 0; k < W; k++) acc[i][k] = 0.f;
            for (int c = many == 0 ? total : shared ? w * 64 : 0; c < total; c += shared ? 256 : 64) {
                const uint32_t e = c + lane < total ? list[c + lane] : 0xffffffffu;
                lanes_t left = __ballot((int)(e >> 16) == r);       // r < 2^15
                auto next = [&]() {
                    const int p = __builtin_amdgcn_readlane((int)(e & 0xffffu), __ffsll(left) - 1);
                    left &= left - 1;
                    return p;
                };
                while (__popcll(left) >= FLIGHT) add_rows<FLIGHT, true>(dy, a.ldy, sp, FLIGHT, acc, next);
                if (left) add_rows<FLIGHT, false>(dy, a.ldy, sp, __popcll(left), acc, next);
            }
            if (shared) {                               // the same for all four waves: the list says so
                __syncthreads();                        // the sums of a shared row in front are read
#pragma unroll
                for (int i = 0; i < PIECES; i++)
#pragma unroll
                    for (int k = 0; k < W; k++)
                        if (w > 0) sums[w - 1][i * W + k][lane] = acc[i][k];
                __syncthreads();
                if (w > 0) continue;
#pragma unroll
                for (int i = 0; i < PIECES; i++)
#pragma unroll
                    for (int k = 0; k < W; k++) acc[i][k] += sums[0][i * W + k][lane] + sums[1][i * W + k][lane] + sums[2][i * W + k][lane];
            } else if (a.accumulate && many == 0) continue;
            write_row<TO, W, PIECES, STREAM>(static_cast<TO *>(a.out) + (size_t)(v0 + r) * a.cols, sp, acc, a.scale, a.accumulate);
        }
        __syncthreads();                                // the list's readers are through
    }
}

template <typename T, typename TO, typename I, int PIECES> void launch_direct_of(const DirectArgs &a, hipStream_t st) {
    constexpr int W = sizeof(TO) == 4 ? 4 : 8;
    const dim3 grid((unsigned)ceil_div(a.cols, PIECES * 64 * W), (unsigned)min(ceil_div(a.vocab, a.block), 65535));
    if ((size_t)a.vocab * a.cols * sizeof(TO) >= STREAM_BYTES) hipLaunchKernelGGL((embed_direct_kernel<T, TO, I, W, PIECES, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((embed_direct_kernel<T, TO, I, W, PIECES, false>), grid, dim3(256), 0, st, a);
}
template <typename T, typename TO, typename I> sol_status launch_direct_of(DirectArgs a, hipStream_t st) {
    constexpr int W = sizeof(TO) == 4 ? 4 : 8;
    const int pieces = ceil_div(a.cols, 64 * W), slabs = pieces <= 1 ? 1 : ceil_div(pieces, 2);
    // rows enough for a workgroup to make up for its look at the tokens, workgroups enough to fill the GPU
    a.block = max(4, min(32, (int)((long)a.vocab * slabs / 1024) & ~3));
    if (pieces <= 1) launch_direct_of<T, TO, I, 1>(a, st);
    else launch_direct_of<T, TO, I, 2>(a, st);
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}
template <typename T, typename TO> sol_status launch_direct(const DirectArgs &a, int bits, hipStream_t st) {
    return bits == 64 ? launch_direct_of<T, TO, int64_t>(a, st) : launch_direct_of<T, TO, int32_t>(a, st);
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

sol_status check_tokens(const void *tokens, int bits) {
    SOL_REQUIRE((reinterpret_cast<uintptr_t>(tokens) & (bits / 8 - 1)) == 0, SOL_ERR_ALIGN, "tokens of %d bits must be aligned to them", bits);
    return SOL_OK;
}

template <typename T, typename I> sol_status launch_embed_of(const EmbedArgs &a, hipStream_t st) {
    const int per = (256 >> a.lanes_log2) * KEEP;
    const dim3 grid((unsigned)ceil_div(a.cols, 64 * 16 / (int)sizeof(T)), (unsigned)min(ceil_div(a.n, per), 65535));
    if ((size_t)a.n * a.cols * sizeof(T) >= STREAM_BYTES) hipLaunchKernelGGL((embed_kernel<T, I, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((embed_kernel<T, I, false>), grid, dim3(256), 0, st, a);
    SOL_HIP(hipGetLastError());
    return SOL_OK;
}
template <typename T> sol_status launch_embed(const EmbedArgs &a, int bits, hipStream_t st) {
    return bits == 64 ? launch_embed_of<T, int64_t>(a, st) : launch_embed_of<T, int32_t>(a, st);
}

struct EmbedPlan {
    size_t start, order, sorted, part, bytes;
    int windows, rows, log2, places;
};
EmbedPlan embed_plan(const sol_embedding_desc &d) {
    EmbedPlan p{};
    if (d.tokens <= DIRECT) return p;       // no scratch
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t here = at; at = round_up(at + bytes, 256); return here; };
    while ((1 << p.log2) < d.vocab && ((1 << p.log2) < INDEX_GROUPS || (size_t)INDEX_ROWS << p.log2 < (size_t)d.vocab)) p.log2++;
    p.rows = ceil_div(d.vocab, 1 << p.log2);
    p.places = p.rows << p.log2;
    p.windows = ceil_div(d.tokens, RUN);
    p.start = take(((size_t)p.places + 1) * 4);
    p.order = take((size_t)d.tokens * 4);
    p.sorted = take((size_t)d.tokens * 4);
    p.part = take((size_t)p.windows * 2 * d.cols * 4);
    p.bytes = at;
    return p;
}

template <typename T, typename TO, int PIECES> void launch_sums_of_rows(const GatherArgs &g, hipStream_t st) {
    constexpr int W = 16 / sizeof(TO);
    const int items = g.vocab + 2 * g.windows;
    const dim3 grid((unsigned)ceil_div(g.cols, PIECES * 64 * W), (unsigned)min(ceil_div(items, 4), 65535));
    if ((size_t)g.vocab * g.cols * sizeof(TO) >= STREAM_BYTES) hipLaunchKernelGGL((embed_sum_kernel<T, TO, W, PIECES, true>), grid, dim3(256), 0, st, g, items);
    else hipLaunchKernelGGL((embed_sum_kernel<T, TO, W, PIECES, false>), grid, dim3(256), 0, st, g, items);
}
// 1024 columns a wave where there are as many: see embed_sum_kernel
template <typename T, typename TO> sol_status launch_gather(const GatherArgs &g, hipStream_t st) {
    constexpr int W = 16 / sizeof(TO), PIECES = 16 / W;
    const int pieces = ceil_div(g.cols, 64 * W);
    if (pieces == 1) launch_sums_of_rows<T, TO, 1>(g, st);
    else if (pieces == 2 || PIECES == 2) launch_sums_of_rows<T, TO, 2>(g, st);
    else launch_sums_of_rows<T, TO, PIECES>(g, st);
    SOL_HIP(hipGetLastError());
    hipLaunchKernelGGL((embed_join_kernel<TO, W, PIECES / 2>), dim3((unsigned)ceil_div(g.cols, 512), (unsigned)min(g.windows, 65535)), dim3(256), 0, st, g);
    SOL_HIP(hipGetLastError());
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
    SOL_TRY(check_tokens(tokens, d.token_bits));
    SOL_REQUIRE(aligned16(table) && aligned16(y), SOL_ERR_ALIGN, "device pointers must be 16-byte aligned");
    SOL_REQUIRE(y != table && y != tokens, SOL_ERR_UNSUPPORTED, "embedding: y must not alias the table or the tokens");
    hipStream_t st = (hipStream_t)stream;
    const EmbedArgs a{tokens, table, y, d.ldt, d.ldy, d.tokens, d.vocab, d.cols, d.pad, row_lanes_log2(d.cols, 16 / (int)dtype_size(d.dtype)), d.scale};
    return d.dtype == SOL_BF16 ? launch_embed<bf16_t>(a, d.token_bits, st) : launch_embed<float>(a, d.token_bits, st);
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
    SOL_TRY(check_tokens(tokens, d.token_bits));
    SOL_REQUIRE(aligned16(dy) && aligned16(dtable), SOL_ERR_ALIGN, "device pointers must be 16-byte aligned");
    SOL_REQUIRE(dtable != dy && dtable != tokens, SOL_ERR_UNSUPPORTED, "embedding backward: dtable must not alias dy or the tokens");
    const EmbedPlan p = embed_plan(d);
    SOL_TRY(check_scratch(workspace, workspace_bytes, p.bytes));
    hipStream_t st = (hipStream_t)stream;
    if (d.tokens <= DIRECT) {
        const DirectArgs a{tokens, dy, dtable, d.ldy, d.tokens, d.vocab, d.cols, d.pad, 0, accumulate ? 1 : 0, d.scale};
        if (d.dtype == SOL_F32) return launch_direct<float, float>(a, d.token_bits, st);
        return dtable_dtype == SOL_F32 ? launch_direct<bf16_t, float>(a, d.token_bits, st) : launch_direct<bf16_t, bf16_t>(a, d.token_bits, st);
    }
    unsigned char *ws = static_cast<unsigned char *>(workspace);
    int *start = reinterpret_cast<int *>(ws + p.start), *order = reinterpret_cast<int *>(ws + p.order), *sorted = reinterpret_cast<int *>(ws + p.sorted);
    const IndexArgs x{tokens, d.tokens, d.vocab, d.pad, p.rows, p.log2, start, order, sorted};
    const dim3 grid(1u << p.log2);
    const bool pad = d.pad >= 0 && d.pad < d.vocab;
    if (d.token_bits == 64) {
        if (pad) hipLaunchKernelGGL((embed_index_kernel<int64_t, true>), grid, dim3(INDEX_THREADS), 0, st, x);
        else hipLaunchKernelGGL((embed_index_kernel<int64_t, false>), grid, dim3(INDEX_THREADS), 0, st, x);
    } else {
        if (pad) hipLaunchKernelGGL((embed_index_kernel<int32_t, true>), grid, dim3(INDEX_THREADS), 0, st, x);
        else hipLaunchKernelGGL((embed_index_kernel<int32_t, false>), grid, dim3(INDEX_THREADS), 0, st, x);
    }
    SOL_HIP(hipGetLastError());
    const GatherArgs g{dy, dtable, start, order, sorted, reinterpret_cast<float *>(ws + p.part), d.ldy, d.vocab, d.cols, p.windows, accumulate ? 1 : 0,
                 p.rows, p.log2, p.places, d.scale, FastDiv((uint32_t)p.rows)};
    if (d.dtype == SOL_F32) return launch_gather<float, float>(g, st);
    return dtable_dtype == SOL_F32 ? launch_gather<bf16_t, float>(g, st) : launch_gather<bf16_t, bf16_t>(g, st);
}

}  // extern "C"
