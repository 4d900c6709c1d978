// Attention of packed query rows over paged K/V: what the shared-prefix decode (ikv_prefix_*) and
// the sliding window (ikv_window_*) have in common.
//
// A unit is a set of query rows that read the same slots of one sequence: consecutive query tokens of
// a sequence (window), the members of a group over their prefix, or one sequence over its own slots
// behind it (prefix).  Row r of a unit is query head g * G + r % G of its token or member r / G, for
// each KV head g.  The slots that some row of a unit sees lie in at most two runs of 128-slot tiles:
// the sinks' and the window's.
//
// The tiles of all (unit, KV head) pairs are laid out one behind another and cut into equal shares, one
// for each CTA of the attention kernel, whatever the lengths are: a CTA takes the pairs, or parts of
// them, of its share in turn.  A part leaves an unnormalised output and its (max, sum) in the workspace
// for the merge kernel.  The plan kernel (one CTA) writes the units and where each share begins.
#pragma once
#include <atomic>

#include "ikv_internal.cuh"

namespace ikv {

constexpr int kRowsTile = 128;      // slots a tile
constexpr int kRowsMaxCtas = 512;

struct alignas(16) RowsUnit {                   // 64 bytes
    int32_t b;                      // the sequence whose block table is read
    int32_t m0;                     // window: first query token; prefix: first entry of the member list; -1: one
                                    // sequence's own slots
    int32_t n;                      // tokens or members
    int32_t S0;                     // slots below are numbers in b's slot space: S0 is its slot 0
    int32_t lo, hi;                 // every visible slot lies in [lo, hi)
    int32_t p0;                     // window: slot of the first query token (may be below S0)
    int32_t wlo, sh;                // some row sees the slots of [lo, sh) and of [wlo, hi), none sees others
    int32_t open;                   // nonzero: a copy of up to 64 slots that ends at hi or behind it may reach behind the
                                    // sequence's last slot, where anything may lie
    int32_t n_a, t_w, nt;           // tile i of nt: lo / 128 + i for i < n_a, t_w + i - n_a behind
    int32_t row0;                   // window: row of query token 0 in q and out
    int64_t cum;                    // cost of all earlier units, for all KV heads
};

// What a tile of a pair (unit, KV head) costs, and what the pair costs besides, for its first products, which
// nothing overlaps, and its output.  In the tensor-core kernel a tile took 1.0 to 1.4 us with one row tile and 1.4 to
// 1.6 with two, a pair besides 2.2 to 3.4 and 4.5 to 5.5.  (Shares of tiles alone: a window of 2k over 8k tokens
// 290 us a call instead of 223, the CTA with the shortest pairs 40% behind the others.)  A pair's constant is at the low
// end of what it took, and a part that continues a cut pair pays a start and an output that nothing counts: in three
// decode batches the last CTA, with the most short pairs, ends 31, 46 and 48% behind the mean.
struct RowsCost {
    int32_t tile, extra;
};
constexpr int kTileOne = 3, kExtraOne = 6, kTileTwo = 4, kExtraTwo = 12;

struct alignas(16) RowsHead {
    int64_t per;                    // cost of a CTA's share
    int32_t n_pre;                  // units of shared prefixes, in front of the others
    int32_t failed;                 // nonzero: a wait of the attention ran out, parts are missing
};
struct alignas(16) RowsStart {                  // where a CTA's share begins (at cost `at` of pair (unit, g)), and its cost
    int32_t unit, g, at, n;
};
// The score pass on the tensor cores: an item is a tile of a unit for up to 128 of its rows, and, with a utility
// row a KV head, one of those; item sub * nt + j of a unit is tile j of its sub-th such set.
struct alignas(16) RowsItems {                  // where a CTA's begin, and how many it has
    int32_t unit, sub, j, n;
};
struct alignas(16) RowsSeq {                    // prefix: what sequence b's rows are made from
    int32_t pre, entry;             // its group's unit that holds it (-1: none), its member number there
    int32_t own;                    // its unit of own slots (-1: none)
    int32_t len;                    // slots of its prefix
};

struct RowsArgs {
    const void *k, *v;
    PagedView pv;
    int32_t layer;
    const int32_t *len;             // [batch]
    const int32_t *pos;             // [rows][cap], -1 at dead slots, or null
    uint32_t *live;                 // with pos, on the tensor cores: [rows][live_words] workspace, bit j of a row: slot
                                    // j is live
    int32_t live_words;
    int32_t rows_per_seq, cap, batch, q_heads, group;
    float scale_log2;               // log2(e) / sqrt(d)
    const void *q;
    void *out;
    int64_t q_stride, out_stride;   // elements from a token's (sequence's) heads to the next
    int32_t unit_n, tile_n;         // most tokens or members of a unit, of a row tile of it
    // window
    int32_t window, sinks;          // window in [1, 2^30], sinks in [0, 2^30)
    const int32_t *row0, *count;
    int32_t max_count, seq_units;   // seq_units: units of max_count tokens
    // prefix
    int32_t prefix;                 // nonzero: a shared-prefix call
    int32_t n_groups;
    const int32_t *first, *member, *group_len;
    // workspace
    RowsHead *head;
    RowsStart *start;               // [ctas]
    RowsItems *items;               // [ctas] of the tensor-core score pass, or null
    int64_t *icum;                  // with items: items of all earlier units
    int32_t item_n, item_subs;      // members of an item, and how many times its tiles are gone through (1, or the KV
                                    // heads)
    RowsUnit *units;
    int32_t *owner;                 // prefix: [batch] first entry that names the sequence
    int32_t *vm;                    // prefix: [batch] the entries, -1 where one is left out
    int32_t *entry_group;           // prefix: [batch] the entries' groups
    int32_t *group_p, *group_lead, *group_unit;  // prefix: [n_groups] slots shared, first member, first unit
    RowsSeq *seq;                   // prefix: [batch]
    float2 *norm;                   // prefix: [batch][H] the maximum M that a row's weights go by (log2 domain)
                                    // and 1 over their sum.  (Not their log-sum-exp: at logits of 100 its
                                    // rounding alone costs a weight 3e-6 of its value)
    // partial results: slot s holds rows_cap rows, part_ml [s][row] (max, sum) in the log2 domain,
    // part_o [s][D / 4][row][4] (a thread stores a row, so that a warp's stores are one piece).  Window: slot 2 c + 1 of CTA c for a pair that it begins, 2 c for one that it
    // continues.  Prefix: pair number + CTA number, in regions of their own for the pairs of shared
    // prefixes and for those of own slots (own_ml, own_o; G rows a slot).
    int32_t rows_cap, ctas;
    int32_t small;                  // nonzero: a plan for one warp (at most 32 sequences, groups, units), in 32 bits
    float2 *part_ml, *own_ml;
    float *part_o, *own_o;
};

// Where the parts of pair (u, g) lie, CTA c's
__device__ __forceinline__ int64_t rows_slot(const RowsArgs &a, const RowsHead &h, const RowsUnit &u, int unit, int g,
                                             int c, bool begins) {
    if (!a.prefix) return 2 * (int64_t)c + (begins ? 1 : 0);
    return (int64_t)(u.m0 >= 0 ? unit : unit - h.n_pre) * a.pv.kv_heads + g + c;
}

// The tile of a unit
__device__ __forceinline__ int rows_tile(const RowsUnit &u, int i) { return i < u.n_a ? (u.lo >> 7) + i : u.t_w + i - u.n_a; }

__device__ __forceinline__ RowsUnit rows_unit(const RowsArgs &a, int unit) {
    RowsUnit u;
    const int4 *p = reinterpret_cast<const int4 *>(a.units + unit);
    int4 *q = reinterpret_cast<int4 *>(&u);
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = __ldcg(p + i);
    return u;
}

__device__ __forceinline__ RowsCost rows_cost(const RowsArgs &a, int n) { return n > a.tile_n ? RowsCost{kTileTwo, kExtraTwo} : RowsCost{kTileOne, kExtraOne}; }
__device__ __forceinline__ int64_t pair_cost(const RowsCost &c, int nt) { return c.extra + (int64_t)c.tile * nt; }
// The first tile of a pair that begins at its cost `at` or behind: a border there cuts in front of it
__device__ __forceinline__ int tile_at(const RowsCost &c, int64_t at) {
    return at <= c.extra ? 0 : (int)((uint32_t)(at - c.extra + c.tile - 1) / (uint32_t)c.tile);
}

// The parts of a share, in turn: while (left > 0) { part(); next(); }
struct RowsWalk {
    int32_t unit, g;                // the share goes on at cost `at` of pair (unit, g)
    int32_t at, left;
    __device__ __forceinline__ void begin(const int4 &s) {
        unit = s.x;
        g = s.y;
        at = s.z;
        left = s.w;
    }
    // the share's tiles of the pair: n (or none) from j0 on
    __device__ __forceinline__ int part(const RowsArgs &a, const RowsUnit &u, int &j0) const {
        const RowsCost c = rows_cost(a, u.n);
        j0 = tile_at(c, at);
        const int64_t end = (int64_t)at + left;
        return (end >= pair_cost(c, u.nt) ? u.nt : min(tile_at(c, end), u.nt)) - min(j0, u.nt);
    }
    __device__ __forceinline__ void next(const RowsArgs &a, const RowsUnit &u) {
        left = (int32_t)max(left - (pair_cost(rows_cost(a, u.n), u.nt) - at), (int64_t)0);
        at = 0;
        if (++g == a.pv.kv_heads) {
            g = 0;
            ++unit;
        }
    }
};
// What row r of a unit sees: slots s of [lo, hi] with s >= wlo or s < sh, live ones.  seq < 0: not a row.
struct RowsRow {
    int32_t seq;                    // its sequence
    int32_t lo, hi, wlo, sh;
    const int32_t *pos;             // its positions, by slot - S0, or null
    int64_t q, out;                 // its elements in q and out
};
template <int D>
__device__ __forceinline__ RowsRow rows_row(const RowsArgs &a, const RowsUnit &u, int g, int r) {
    RowsRow w;
    const int t = r / a.group, h = g * a.group + r % a.group;
    w.lo = u.lo;
    int64_t row;
    if (!a.prefix) {
        const int p = u.p0 + t;
        w.seq = t < u.n ? u.b : -1;
        w.hi = p;
        w.wlo = max(u.lo, p - a.window + 1);
        w.sh = u.S0 + a.sinks;
        row = (int64_t)u.row0 + u.m0 + t;
    } else {
        w.seq = t >= u.n ? -1 : u.m0 >= 0 ? __ldcg(a.vm + u.m0 + t) : u.b;
        w.hi = u.hi - 1;
        w.wlo = w.sh = u.lo;
        row = w.seq;
    }
    w.pos = a.pos && w.seq >= 0
                ? a.pos + ((int64_t)w.seq * a.rows_per_seq + (a.rows_per_seq == 1 ? 0 : g)) * a.cap
                : nullptr;
    w.q = row * a.q_stride + (int64_t)h * D;
    w.out = row * a.out_stride + (int64_t)h * D;
    return w;
}
__device__ __forceinline__ bool rows_sees(const RowsRow &w, int S0, int s) {
    return s >= w.lo && s <= w.hi && (s >= w.wlo || s < w.sh) && (!w.pos || __ldg(w.pos + (s - S0)) >= 0);
}

// cudaFuncSetAttribute(kernel, MaxDynamicSharedMemorySize, bytes), once a device (`done`: a bit each)
template <typename Kernel>
cudaError_t allow_smem(Kernel kernel, size_t bytes, std::atomic<uint64_t> &done) {
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (dev < 64 && (done.load(std::memory_order_relaxed) >> dev) & 1u) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == cudaSuccess && dev < 64) done.fetch_or(1ull << dev, std::memory_order_relaxed);
    return e;
}

cudaError_t launch_rows_plan(const RowsArgs &a, cudaStream_t st);
cudaError_t launch_rows_simt(const RowsArgs &a, int dtype, int head_dim, cudaStream_t st);
bool rows_tc_supported(const ikv_shape *s, const ikv_cache *c);
cudaError_t launch_rows_tc(const RowsArgs &a, int head_dim, cudaStream_t st);
cudaError_t read_clear_rows_tc_error(unsigned int *v);
cudaError_t launch_rows_merge(const RowsArgs &a, int dtype, int head_dim, cudaStream_t st);
int rows_simt_ctas_per_sm(int head_dim);
// the score pass on the tensor cores
cudaError_t launch_rows_score_tc(const RowsArgs &a, const struct RowsScoreArgs &s, int head_dim, cudaStream_t st);
cudaError_t read_clear_rows_score_error(unsigned int *v);
constexpr int kRowsSimt = 64;       // rows of a unit of the kernel without tensor cores

// prefix: scores and utilities from K once more, with the rows' maxima and sums known
struct RowsScoreArgs {
    float alpha;
    float *score, *ema;             // [rows][cap] or null
    int32_t max_len;
};
cudaError_t launch_rows_score(const RowsArgs &a, const RowsScoreArgs &s, int dtype, int head_dim, cudaStream_t st);

}  // namespace ikv
