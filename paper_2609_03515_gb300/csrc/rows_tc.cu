// Packed-row attention on the tensor cores: bf16, pages of a multiple of 8 slots (sm_103a).
//
// S = Q K^T and O += P V with the rows in the M dimension of 128 x 128 tcgen05 products, so that one tile
// of K and V serves up to 256 query rows: two row tiles, A and B, each with its scores and its output in
// tensor memory (S 128 columns, O D columns) and a warpgroup of its own whose thread r holds row r.  A
// thread turns its row of S into weights, 2^(S scale - m), and writes them as bf16 over S, from where the
// second product takes them as its A operand; nothing of S or P passes through shared memory.  While one
// warpgroup computes its weights, the tensor cores work for the other.
//
// A unit of at most 128 rows (decode) gives A and B every other tile of its slots instead; their outputs
// are joined at the end.
//
// The running maximum m only moves when a row's weights would grow past 2^8, so that O is seldom
// rescaled: weights and sum are relative to the same m, which cancels in O / l.  The sum takes the weights
// in 32 bits; rounding them to bf16 for the product costs at most 2^-8 of sum p |V|.
//
// A row that met a row of V which it does not see and which is not finite (0 * inf) is computed again behind the CTA's
// last part, where no warp waits for another any more: it may take as long as the row's slots do.
//
// Warps: 0-3 and 4-7 the two row tiles, 8 TMA, 9 MMA, 10-11 Q; 11 also finds the parts of the share, ahead of the
// others.  K and V tiles pass through a ring of 32 KB (D = 64: 16 KB) stages in the order K0 K1 V0 K2 V1 .., which
// is the order of the products.  Boxes of a tile that no row sees are fetched from behind the tensor's end, which
// fills zeros and reads nothing.  Every wait is bounded; on timeout the CTA sets the error word, drains what is in
// flight and returns.
//
// Measured: a causal prompt of 16384 tokens, 32 / 8 heads of 128, 1462 us (1.50 PFLOP/s), 869 steps of 256 rows by 128
// slots a CTA: 1.68 us a step with all that is besides, 1.36 at the rate that the library's large products reach.  Two
// prefixes of 8k for 16 sequences each: 31 of 49 us in here, 154 MB of K and V at 73% of the copy rate, the starts and
// outputs of 256 short pairs among them.
#include "rows_tc.cuh"

namespace ikv {

namespace {

constexpr int kThreads = 384;
constexpr float kSlack = 8.f;               // log2 of the largest weight before the maximum moves

// A part of the CTA's share, for all warps: n tiles from j0 on of pair (unit, g); n = 0 behind the last
struct alignas(16) Part {
    RowsUnit u;
    int32_t unit, g, j0, n;
};
constexpr int kParts = 4;                   // of them in shared memory, most of them ahead

template <int D>
struct Tc {
    static constexpr int kStage = kAtom * (D / 64);
    static constexpr int kStages = D == 128 ? 4 : 8;
    static constexpr int kOffRing = 2 * kStage;  // (Q of A and B in front)
    static constexpr int kOffOut = kOffRing + kStages * kStage;  // a warp: 32 channels of its 32 rows
    static constexpr int kOffEx = kOffOut + 8 * 2048;
    static constexpr int kOffPart = kOffEx + 2 * 128 * 8 + 128 * 4;
    static constexpr int kOffBar = kOffPart + kParts * sizeof(Part);
    static constexpr int kBars = 2 * kStages + 12 + 2 * kParts;
    static constexpr int kOffMisc = kOffBar + kBars * 8;
    static constexpr int kSmem = kOffMisc + 16 + 1024;  // (to align by 1024)
};

// bits of the slots a .. b of a tile that lie in its w-th 32
__device__ __forceinline__ uint32_t range_bits(int a, int b, int w) {
    const int lo = max(a - 32 * w, 0), hi = min(b - 32 * w, 31);
    return lo > hi ? 0u : (0xffffffffu >> (31 - (hi - lo))) << lo;
}
// tiles of a share's load stream: load x of a part of n tiles
__device__ __forceinline__ void load_of(int x, int n, int &tile, bool &is_v) {
    is_v = x == 2 * n - 1 || (x > 0 && !(x & 1));
    tile = x == 2 * n - 1 ? n - 1 : is_v ? (x - 2) / 2 : (x + 1) / 2;
}

// Whether a row that the CTA has stored holds NaN or infinities though its sum is a number.  (A whole pair's sums are
// not kept.)
template <int D>
__device__ __forceinline__ bool row_suspect(const RowsArgs &a, const RowsUnit &u, const RowsRow &row, bool whole, int64_t slot,
                                            int r) {
    const int lane = threadIdx.x & 31;
    bool bad = false;
#pragma unroll
    for (int e = 0; e < D / 32; ++e) {
        const int c = lane + 32 * e;
        const float x = whole ? __bfloat162float(static_cast<const __nv_bfloat16 *>(a.out)[row.out + c])
                              : __ldcg(rows_part_o<D>(a, u, slot, r) + (int64_t)(c / 4) * rows_part_step(a, u) + c % 4);
        bad |= !(fabsf(x) < INFINITY);
    }
    return __any_sync(0xffffffffu, bad) && (whole || !isnan(__ldcg(rows_part_ml(a, u, slot, r)).y));
}
// Whether among the part's tiles lies a row of V that is not finite and that the row does not see.  (In a box that was
// copied: elsewhere there need not be a page.  What was cleared of such a box counts too, and costs time alone.)
template <int D>
__device__ __forceinline__ bool row_misled(const RowsArgs &a, const TcMap &tm, const RowsUnit &u, const RowsRow &row, int g, int j0,
                                           int n) {
    const int lane = threadIdx.x & 31;
    for (int i = 4 * j0; i < 4 * (j0 + n); ++i) {
        const int s = rows_tile(u, i / 4) * kRowsTile + i % 4 * 32 + lane, s0 = s & -tm.rows_per_box, s1 = s0 + tm.rows_per_box;
        bool look = s >= u.lo && s0 < u.hi && (s1 > u.wlo || s0 < u.sh) && !rows_sees(row, u.S0, s);
        int64_t at = 0;
        if (look) {
            const int row8 = pool_row(a, u.b, g, s);
            look = row8 >= 0 && row8 < tm.pool_rows;
            at = ((int64_t)a.layer * tm.pool_rows + row8) * D;
        }
        unsigned all = __ballot_sync(0xffffffffu, look);
        while (all) {
            const int x = __ffs(all) - 1;
            all &= all - 1;
            const __nv_bfloat16 *v = static_cast<const __nv_bfloat16 *>(a.v) + __shfl_sync(0xffffffffu, at, x) + lane;
            bool bad = false;
#pragma unroll
            for (int e = 0; e < D / 32; ++e) bad |= !(fabsf(__bfloat162float(v[32 * e])) < INFINITY);
            if (__any_sync(0xffffffffu, bad)) return true;
        }
    }
    return false;
}
// The CTA's share once more, a warp of `warps` a row: the rows that have to be computed again
template <int D>
__device__ __noinline__ void redo_share(const RowsArgs &a, const TcMap &tm, int n_pre, int warp, int warps) {
    RowsHead h;
    h.n_pre = n_pre;
    RowsWalk w;
    w.begin(__ldcg(reinterpret_cast<const int4 *>(a.start + blockIdx.x)));
    while (w.left > 0) {
        const RowsUnit u = rows_unit(a, w.unit);
        int j0;
        const int n = w.part(a, u, j0);
        const bool begins = j0 == 0, whole = begins && n == u.nt && !a.prefix;
        const int64_t slot = whole || n <= 0 ? 0 : rows_slot(a, h, u, w.unit, w.g, blockIdx.x, begins);
        for (int r = warp; n > 0 && r < u.n * a.group; r += warps) {
            const RowsRow row = rows_row<D>(a, u, w.g, r);
            if (row.seq >= 0 && row_suspect<D>(a, u, row, whole, slot, r) && row_misled<D>(a, tm, u, row, w.g, j0, n))
                rows_redo<D, __nv_bfloat16>(a, w.unit, w.g, j0, n, whole, slot, r);
        }
        w.next(a, u);
    }
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
    rows_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                   const __grid_constant__ CUtensorMap tmK8, const __grid_constant__ CUtensorMap tmV8,
                   const __grid_constant__ RowsArgs a, const TcMap tm) {
    using C = Tc<D>;
    using T = __nv_bfloat16;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    unsigned char *sm = smem_raw + (base - raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t bar0 = base + C::kOffBar;
    auto kv_full = [&](int i) { return bar0 + 8u * i; };
    auto kv_empty = [&](int i) { return bar0 + 8u * (C::kStages + i); };
    const uint32_t bar1 = bar0 + 8u * (2 * C::kStages), q_empty = bar1, mma_done = bar1 + 8;
    auto q_full = [&](int x) { return bar1 + 16u + 8u * x; };
    auto s_full = [&](int x) { return bar1 + 32u + 8u * x; };
    auto p_full = [&](int x) { return bar1 + 48u + 8u * x; };
    auto o_full = [&](int x) { return bar1 + 64u + 8u * x; };
    auto part_full = [&](int i) { return bar1 + 80u + 8u * i; };
    auto part_empty = [&](int i) { return bar1 + 80u + 8u * (kParts + i); };
    const uint32_t joined = bar1 + 80u + 16u * kParts, stall_bar = joined + 8;  // (nothing arrives at the latter)
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(sm + C::kOffMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(sm + C::kOffMisc + 4);
    volatile int *redo_flag = abort_flag + 1;   // some row's output is not finite though its sum is
    if (warp == 8 && lane == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(kv_full(i), 1);
            mbar_init(kv_empty(i), 1);
        }
        mbar_init(q_empty, 1);
        for (int x = 0; x < 2; ++x) {
            mbar_init(q_full(x), 64);
            mbar_init(s_full(x), 1);
            mbar_init(p_full(x), 4);
            mbar_init(o_full(x), 1);
        }
        for (int i = 0; i < kParts; ++i) {
            mbar_init(part_full(i), 1);
            mbar_init(part_empty(i), 12);  // every warp
        }
        mbar_init(joined, 8);
        mbar_init(stall_bar, 1);
        mbar_init(mma_done, 1);
        *abort_flag = 0;
        *redo_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_slot))
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    const int tile_rows = 128 / a.group * a.group;  // rows of a row tile
    // the parts, which warp 11 finds ahead of the others; part number seg, until release()
    uint32_t seg = 0;
    const Part *const parts = reinterpret_cast<const Part *>(sm + C::kOffPart);
    auto part_at = [&] { return parts + seg % kParts; };
    auto part_wait = [&] { return warp_wait(part_full(seg % kParts), seg / kParts & 1, abort_flag) && part_at()->n > 0; };
    auto release = [&] {
        __syncwarp();
        if (lane == 0) mbar_arrive(part_empty(seg % kParts));
        ++seg;
    };

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 8) {
            // ---------------- K and V, a lane a box
            int J = 0;
            bool ok = true;
            const int boxes = kRowsTile / tm.rows_per_box;
            while (ok && part_wait()) {
                const Part p = *part_at();
                const RowsUnit &u = p.u;
                const int n = p.n, j0 = p.j0, ragged = u.open && (u.hi & (tm.rows_per_box - 1)) ? u.hi : 0x7fffffff;
                for (int x = 0; x < 2 * n && ok; ++x, ++J) {
                    int tile;
                    bool is_v;
                    load_of(x, n, tile, is_v);
                    const int t0 = rows_tile(u, j0 + tile) * kRowsTile, s0 = t0 + lane * tm.rows_per_box, s1 = s0 + tm.rows_per_box;
                    int row = tm.pool_rows;
                    if (lane < boxes && s0 < u.hi && (s1 > u.wlo || (s0 < u.sh && s1 > u.lo))) row = pool_row(a, u.b, p.g, s0);
                    // the box that the sequence ends in comes 8 rows at a time, and not those behind its end
                    // (V's box that the unit's slots begin in likewise, and not those in front)
                    const int last = t0 + kRowsTile > ragged ? (u.hi - t0) >> tm.box_shift : -1;
                    const int first = is_v && (u.lo & -kRowsTile) == t0 && (u.lo & (tm.rows_per_box - 1)) ? (u.lo - t0) >> tm.box_shift : -1;
                    const int st = J % C::kStages;
                    if (lane == 0) {
                        if (J >= C::kStages) ok = bar_wait(kv_empty(st), (J / C::kStages - 1) & 1, abort_flag);
                        if (ok) mbar_expect_tx(kv_full(st), C::kStage);
                    }
                    ok = __shfl_sync(0xffffffffu, ok, 0);
                    const uint32_t dst = base + C::kOffRing + st * C::kStage;
                    if (ok && lane < boxes && lane != last && lane != first)
                        tma_rows(dst + lane * tm.rows_per_box * (2 * D), is_v ? &tmV : &tmK, row, kv_full(st));
                    if (ok && (last >= 0 || first >= 0)) {
                        const int edge = lane < 8 ? last : lane < 16 && first != last ? first : -1;  // rows 8 (lane % 8) of it
                        const int from = __shfl_sync(0xffffffffu, row, max(edge, 0));
                        const int s = edge * tm.rows_per_box + 8 * (lane % 8);
                        const bool real = t0 + s < u.hi && t0 + s + 8 > u.lo && from < tm.pool_rows;
                        if (edge >= 0 && lane % 8 < tm.rows_per_box / 8)
                            tma_rows(dst + s * (2 * D), is_v ? &tmV8 : &tmK8, real ? from + 8 * (lane % 8) : tm.pool_rows, kv_full(st));
                    }
                    if (!ok) break;
                }
                release();
            }
            if (lane == 0)  // every copy has landed before the CTA ends
                for (int i = J - 1; i >= 0 && i >= J - C::kStages; --i) bar_drain(kv_full(i % C::kStages), (i / C::kStages) & 1);
            __syncwarp();
        } else if (warp == 9) {
            // ---------------- products
            // The warp stays converged and one lane issues: descriptors are then formed in uniform registers.
            // (A lane alone in a branch formed them in its own and took 125 cycles a product instead of 64.)
            constexpr uint32_t id_qk = idesc_bf16(false, 128, 128), id_pv = idesc_bf16(false, 128, D, true);
            const bool leader = elect_one();
            const uint64_t dq0 = sdesc(base, 16, 1024), dk0 = sdesc(base + C::kOffRing, 16, 16 * D),
                           dv0 = sdesc(base + C::kOffRing, kBlock, 16 * D);
            struct Stage {
                int i;
                uint32_t par;
            } at{0, 0};                    // the next load to be used
            auto take = [&] {
                const Stage s = at;
                if (++at.i == C::kStages) at = Stage{0, at.par ^ 1};
                return s;
            };
            uint32_t np[2] = {0, 0};       // weights taken
            bool ok = true;
            if (tm.stall) ok = __all_sync(0xffffffffu, bar_wait_long(stall_bar, 0, abort_flag, kStallNs));  // runs out
            while (ok && part_wait()) {
                const int n = __shfl_sync(0xffffffffu, part_at()->n, 0);
                const bool pair = __shfl_sync(0xffffffffu, part_at()->u.n * a.group > tile_rows, 0);
                // Slots behind a sequence's last, and those in front of a unit's first (of a page that begins earlier, of a
                // prefix that is read elsewhere), may hold anything, a pool that was never written, and 0 * NaN would have
                // every row of the part computed again: their rows of V, at most 7 at either end, become zeros.  (Those in
                // front cost two prefixes of 8k 0.8 us of 49, a small call 0.3 of 18.5.)
                const Part *p = part_at();
                const int hi = __shfl_sync(0xffffffffu, p->j0 + n == p->u.nt && p->u.open ? p->u.hi : 0, 0);
                const int lo = __shfl_sync(0xffffffffu, p->j0 == 0 && rows_tile(p->u, 0) == p->u.lo >> 7 ? p->u.lo : 0, 0);
                // rows of V behind or in front of slot `end`, in its group of 8
                auto clean = [&](Stage v, int end, bool behind) {
                    if (end % 8 == 0) return;
                    const int r0 = end % kRowsTile, r = r0 / 8 * 8 + lane / 4;
                    unsigned char *row = sm + C::kOffRing + v.i * C::kStage + (r >> 3) * (16 * D) + (r & 7) * 128;
                    if (behind == (r >= r0)) {
#pragma unroll
                        for (int i = 0; i < D / 32; ++i)  // 16-byte pieces lane % 4, + 4 ..
                            *reinterpret_cast<uint4 *>(row + (i >> 1) * kBlock + ((lane & 3) + 4 * (i & 1)) * 16) =
                                make_uint4(0, 0, 0, 0);
                    }
                    fence_async_smem();
                    __syncwarp();
                };
                auto there = [&](Stage s) { return warp_wait(kv_full(s.i), s.par, abort_flag); };
                // S of row tile x; (free: K's stage is done with then)
                auto qk = [&](int x, Stage k, bool free) {
                    fence_after_sync();
                    const uint64_t dq = dq0 + (pair ? x * (C::kStage >> 4) : 0), dk = dk0 + k.i * (C::kStage >> 4);
                    if (leader) {
#pragma unroll
                        for (int kk = 0; kk < D / 16; ++kk) {
                            const uint32_t c = (kk & 3) * 32;
                            mma_bf16(tmem + 128 * x, dq + (((kk >> 2) * kAtom + c) >> 4),
                                     dk + (((kk >> 2) * kBlock + c) >> 4), id_qk, kk > 0);
                        }
                        mma_commit(s_full(x));
                        if (free) mma_commit(kv_empty(k.i));
                    }
                    __syncwarp();
                };
                // O of row tile x
                auto pv = [&](int x, Stage v, bool first, bool free) {
                    if (!warp_wait(p_full(x), np[x] & 1, abort_flag)) return false;
                    ++np[x];
                    fence_after_sync();
                    const uint64_t dv = dv0 + v.i * (C::kStage >> 4);
                    if (leader) {
#pragma unroll
                        for (int kk = 0; kk < kRowsTile / 16; ++kk)  // V: channels contiguous, 64 of them 1 KB apart
                            mma_bf16_ts(tmem + 256 + 128 * x, tmem + 128 * x + 8 * kk, dv + kk * (32 * D >> 4), id_pv,
                                        !first || kk > 0);
                        mma_commit(o_full(x));
                        if (free) mma_commit(kv_empty(v.i));
                    }
                    __syncwarp();
                    return true;
                };
                auto q_done = [&] {
                    if (leader) mma_commit(q_empty);
                    __syncwarp();
                };
                // P of a tile lies over its S: S of the next is issued behind the product that takes P
                Stage k = take();
                ok = warp_wait(q_full(0), seg & 1, abort_flag) && there(k);
                if (!ok) break;
                qk(0, k, !pair);
                ok = warp_wait(q_full(1), seg & 1, abort_flag);
                if (!ok) break;
                if (pair) {
                    qk(1, k, true);
                    if (n == 1) q_done();
                    for (int j = 0; j < n; ++j) {
                        const bool more = j + 1 < n;
                        if (more) k = take();
                        const Stage v = take();
                        ok = (!more || there(k)) && there(v);
                        if (!ok) break;
                        if (j == 0) clean(v, lo, false);
                        if (!more) clean(v, hi, true);
                        ok = pv(0, v, j == 0, false);
                        if (!ok) break;
                        if (more) qk(0, k, false);
                        ok = pv(1, v, j == 0, true);
                        if (!ok) break;
                        if (more) qk(1, k, true);
                        if (j + 2 == n) q_done();
                    }
                } else {
                    if (n > 1) {
                        k = take();
                        if (!(ok = there(k))) break;
                        qk(1, k, true);
                    }
                    if (n <= 2) q_done();
                    for (int j = 0; j < n; ++j) {
                        const Stage v = take();
                        ok = there(v);
                        if (!ok) break;
                        if (j == 0) clean(v, lo, false);
                        if (j + 1 == n) clean(v, hi, true);
                        ok = pv(j & 1, v, j < 2, true);
                        if (!ok) break;
                        if (j + 2 < n) {
                            k = take();
                            if (!(ok = there(k))) break;
                            qk(j & 1, k, true);
                            if (j + 3 == n) q_done();
                        }
                    }
                }
                release();
            }
            if (leader) mma_commit(mma_done);  // also after an abort: no product may write TMEM when it is freed
            __syncwarp();
            bar_drain(mma_done, 0);
        } else {
            // ---------------- Q; warp 11 also finds the parts, three ahead
            RowsWalk w;
            w.begin(__ldcg(reinterpret_cast<const int4 *>(a.start + blockIdx.x)));
            uint32_t found = 0;
            bool ok = true, more = warp == 11;
            auto find = [&] {
                Part p;
                p.n = 0;
                while (w.left > 0 && p.n == 0) {
                    p.u = rows_unit(a, w.unit);
                    p.n = w.part(a, p.u, p.j0);
                    p.unit = w.unit;
                    p.g = w.g;
                    w.next(a, p.u);
                }
                more = p.n > 0;
                const uint32_t i = found % kParts;
                if (found >= kParts) ok = warp_wait(part_empty(i), found / kParts - 1 & 1, abort_flag);
                if (ok && lane == 0) {
                    const_cast<Part *>(parts)[i] = p;
                    mbar_arrive(part_full(i));
                }
                ++found;
            };
            if (more) find();
            // Every piece by an asynchronous copy, all of them in flight: four lanes a row, 16 rows an iteration.
            // A's rows are handed over first.
            constexpr int CH = D / 8;      // 16-byte pieces of a row
            constexpr int kAtOnce = 2;    // rows of a thread
            const int t = tid - 320, c = t & 3;
            while (ok && part_wait()) {
                const RowsUnit u = part_at()->u;
                const int rows = u.n * a.group;
                const bool many = a.prefix && u.m0 >= 0;
                const int64_t row0 = many ? 0 : a.prefix ? u.b : (int64_t)u.row0 + u.m0;
                const T *q = static_cast<const T *>(a.q) + (int64_t)part_at()->g * a.group * D + 8 * c;
                if (seg > 0) ok = warp_wait(q_empty, (seg - 1) & 1, abort_flag);
                for (int x = 0; x < 2 && ok; ++x) {
                    const int first = x * tile_rows, end = min(rows - first, tile_rows);
                    int tok = (first + t / 4) / a.group, h = (first + t / 4) % a.group;
                    for (int r0 = t / 4; r0 < end; r0 += 16 * kAtOnce) {
                        int who[kAtOnce], head[kAtOnce];  // (members are looked up ahead of the copies)
#pragma unroll
                        for (int k = 0; k < kAtOnce; ++k) {
                            who[k] = many && r0 + 16 * k < end ? a.vm[u.m0 + tok] : tok;
                            head[k] = h;
                            h += 16 % a.group;
                            tok += 16 / a.group;
                            if (h >= a.group) {
                                h -= a.group;
                                ++tok;
                            }
                        }
#pragma unroll
                        for (int k = 0; k < kAtOnce; ++k) {
                            const int r = r0 + 16 * k;
                            if (r >= end) break;
                            const bool real = who[k] >= 0;
                            const T *src = q + (row0 + (real ? who[k] : 0)) * a.q_stride + (int64_t)head[k] * D;
                            const uint32_t dst = base + x * C::kStage + r * 128;
#pragma unroll
                            for (int i = 0; i < CH / 4; ++i)
                                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                                                 dst + (i >> 1) * kAtom + ((((c + 4 * i) ^ r) & 7) << 4)),
                                             "l"(src + 32 * i), "r"(real ? 16 : 0)
                                             : "memory");
                        }
                    }
                    asm volatile("cp.async.commit_group;" ::: "memory");
                }
                // (while the copies are on their way)
                for (int i = seg == 0 ? 2 : 1; i > 0 && more && ok; --i) find();
                if (ok) {
                    asm volatile("cp.async.wait_group 1;" ::: "memory");
                    fence_async_smem();
                    mbar_arrive(q_full(0));
                    asm volatile("cp.async.wait_group 0;" ::: "memory");
                    fence_async_smem();
                    mbar_arrive(q_full(1));
                }
                release();
            }
            asm volatile("cp.async.wait_all;" ::: "memory");  // (after an abort some may be on their way)
        }
    } else {
        // ---------------- weights and outputs: thread r of a warpgroup holds row r of its row tile
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int X = warp >> 2, wq = warp & 3, row_in = wq * 32 + lane;
        const uint32_t lane_off = (uint32_t)(wq * 32) << 16;
        const uint32_t tS = tmem + 128 * X + lane_off, tO = tmem + 256 + lane_off;
        float2 *ex = reinterpret_cast<float2 *>(sm + C::kOffEx);  // [2][128] (m, l) of A's and B's rows
        float *found = reinterpret_cast<float *>(ex + 256);        // [128] B's probes
        const int n_pre = __ldcg(&a.head->n_pre);
        uint32_t ns = 0, np = 0, nj = 0;  // scores, weights and meetings so far
        bool ok = true;
        auto meet = [&] {  // A's and B's warps (a bounded wait, as every other: a warp may have given up)
            fence_before_sync();
            __syncwarp();
            if (lane == 0) mbar_arrive(joined);
            ok = warp_wait(joined, nj++ & 1, abort_flag) && ok;
            fence_after_sync();
        };
        while (part_wait()) {
            // (the part's fields are read from shared memory where they are needed: kept, they would push scores out of
            // the registers)
            const volatile Part *vp = part_at();
            int n, r, seq, hi, wlo, steps;
            bool pair, busy;
            {
                const Part *p = part_at();
                n = p->n;
                const int rows = p->u.n * a.group;
                pair = rows > tile_rows;
                r = pair ? X * tile_rows + row_in : row_in;
                const int mine = pair && X == 1 ? rows - tile_rows : min(rows, tile_rows);  // rows of this tile
                const RowsRow row = rows_row<D>(a, p->u, p->g, r);
                seq = row_in < mine ? row.seq : -1;
                hi = row.hi;
                wlo = row.wlo;
                busy = wq * 32 < mine;
                steps = pair ? n : X == 0 ? (n + 1) / 2 : n / 2;
            }
            float m = -INFINITY, l = 0.f;
            for (int s = 0; s < steps; ++s) {
                uint32_t see[4];
                bool masked;
                {
                    const int j = vp->j0 + (pair ? s : 2 * s + X), n_a = vp->u.n_a;
                    const int lo = vp->u.lo, t0 = (j < n_a ? (lo >> 7) + j : vp->u.t_w + j - n_a) * kRowsTile;
                    const int S0 = vp->u.S0, sh = a.prefix ? lo : S0 + a.sinks;
                    const bool full = seq < 0 || (t0 >= lo && t0 + 127 <= hi && (t0 >= wlo || t0 + 127 < sh));
                    masked = __any_sync(0xffffffffu, !full) || a.pos;
                    if (masked && busy) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            see[k] = seq < 0 ? 0u
                                             : range_bits(max(lo, wlo) - t0, hi - t0, k) |
                                                   range_bits(lo - t0, min(sh - 1, hi) - t0, k);
                        if (a.pos && seq >= 0) {  // the row's own live slots, by slot - S0
                            const int64_t rr = (int64_t)seq * a.rows_per_seq + (a.rows_per_seq == 1 ? 0 : vp->g);
                            const uint32_t *bits = a.live + rr * a.live_words;
                            const int x0 = (t0 - S0) >> 5, sh0 = (t0 - S0) & 31;
                            uint32_t lo_w = x0 >= 0 && x0 < a.live_words ? __ldcg(bits + x0) : 0u;
#pragma unroll
                            for (int x = 0; x < 4; ++x) {
                                const int k = x0 + x + 1;
                                const uint32_t hi_w = k >= 0 && k < a.live_words ? __ldcg(bits + k) : 0u;
                                see[x] &= __funnelshift_r(lo_w, hi_w, sh0);
                                lo_w = hi_w;
                            }
                        }
                    }
                }
                if (ok) ok = bar_wait(s_full(X), ns & 1, abort_flag);
                ok = __all_sync(0xffffffffu, ok);
                ++ns;
                if (ok && busy) {
                    fence_after_sync();
                    uint32_t v[128];
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_ld32(tS + 32 * c, v + 32 * c);
                    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_wait_ld(v + 32 * c);
                    if (masked) {
#pragma unroll
                        for (int k = 0; k < 128; ++k)
                            if (!((see[k >> 5] >> (k & 31)) & 1u)) v[k] = 0xff800000u;
                    }
#pragma unroll
                    for (int k = 0; k < 128; k += 2)
                        mx[(k >> 1) & 3] = fmaxf(fmaxf(mx[(k >> 1) & 3], __uint_as_float(v[k])), __uint_as_float(v[k + 1]));
                    const float top = __fmul_rn(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), a.scale_log2);
                    if (s == 0) {
                        m = top;
                    } else {
                        const bool move = seq >= 0 && top > m + kSlack;  // (rows that are none hold anything)
                        if (__any_sync(0xffffffffu, move)) {
                            const float f = move ? ex2(m - top) : 1.f;
                            ok = bar_wait(o_full(X), (np - 1) & 1, abort_flag);
                            ok = __all_sync(0xffffffffu, ok);
                            fence_after_sync();
                            if (ok) {
#pragma unroll
                                for (int k = 0; k < D; k += 32) {
                                    uint32_t o[32];
                                    tmem_ld32(tO + 128 * X + k, o);
                                    tmem_wait_ld(o);
#pragma unroll
                                    for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                    tmem_st32(tO + 128 * X + k, o);
                                }
                            }
                            l *= f;
                            if (move) m = top;
                        }
                    }
                    const float ref = m == -INFINITY ? 0.f : m;
                    const float2 sc2 = make_float2(a.scale_log2, a.scale_log2), ref2 = make_float2(-ref, -ref);
                    float2 sum[4] = {};
                    // (in place: the weights of slots 2 k and 2 k + 1 take register k)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
#pragma unroll
                        for (int k = 16 * c; k < 16 * c + 16; ++k) {
                            float2 x = fma2(make_float2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), sc2, ref2);
                            x.x = ex2(x.x);
                            x.y = ex2(x.y);
                            sum[k & 3] = add2(sum[k & 3], x);
                            const __nv_bfloat162 h = __floats2bfloat162_rn(x.x, x.y);
                            v[k] = *reinterpret_cast<const uint32_t *>(&h);
                        }
                        tmem_st16(tS + 16 * c, v + 16 * c);
                    }
                    const float2 s01 = add2(sum[0], sum[1]), s23 = add2(sum[2], sum[3]);
                    l += (s01.x + s01.y) + (s23.x + s23.y);
                    tmem_wait_st();
                }
                fence_before_sync();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full(X));
                ++np;
            }
            // where the results go (while the last product is under way)
            const Part *p = part_at();
            const bool begins = p->j0 == 0, whole = begins && n == p->u.nt && !a.prefix;
            RowsHead h;
            h.n_pre = n_pre;
            const int64_t slot = whole ? 0 : rows_slot(a, h, p->u, p->unit, p->g, blockIdx.x, begins);
            const int k0 = pair || X == 0 ? 0 : D / 2, step = rows_part_step(a, p->u);
            unsigned char *stage = sm + C::kOffOut + warp * 2048;
            T *to[4];  // of a whole pair: where this lane stores pieces of rows lane / 4 + 8 i
            float *part = rows_part_o<D>(a, p->u, slot, r) + (int64_t)(k0 / 4) * step;
            if (whole) {
                const int64_t mine = seq >= 0 ? rows_row<D>(a, p->u, p->g, r).out : -1;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int64_t at = __shfl_sync(0xffffffffu, mine, 8 * i + lane / 4);
                    to[i] = at >= 0 ? static_cast<T *>(a.out) + at + k0 + lane % 4 * 8 : nullptr;
                }
            }
            if (steps > 0) {
                if (ok) ok = bar_wait(o_full(X), (np - 1) & 1, abort_flag);
                ok = __all_sync(0xffffffffu, ok);
                fence_after_sync();
            }
            // One row tile: A and B join what they have of each row, half of the channels each
            float f0 = 1.f, f1 = 0.f;
            if (!pair) {
                ex[X * 128 + row_in] = make_float2(m, l);
                meet();
                if (n > 1) {
                    const float2 p0 = ex[row_in], p1 = ex[128 + row_in];
                    m = fmaxf(p0.x, p1.x);
                    const float ref = m == -INFINITY ? 0.f : m;
                    f0 = ex2(p0.x - ref);
                    f1 = ex2(p1.x - ref);
                    l = p0.y * f0 + p1.y * f1;
                } else {
                    const float2 p0 = ex[row_in];
                    m = p0.x;
                    l = p0.y;
                }
            }
            float probe = 0.f;  // NaN once a value is not finite
            if (ok && busy) {
                const float inv = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
                const float2 zero2 = make_float2(0.f, 0.f), inv2 = make_float2(inv, inv);
                float2 look = zero2;
                auto pair_of = [](const uint32_t *v, int i) {
                    return make_float2(__uint_as_float(v[2 * i]), __uint_as_float(v[2 * i + 1]));
                };
                // all of it on its way at once: beside running products a look into tensor memory takes some 1000 cycles
                constexpr int kHalf = D / 64;  // chunks of 32 channels of half a row
                const bool both = !pair && n > 1;
                const int chunks = pair ? 2 * kHalf : kHalf;
                const uint32_t from = tO + (pair ? 128 * X : 0) + k0, then = both ? tO + 128 + k0 : from + 32 * kHalf;
                uint32_t v[64 * kHalf];  // the row, or A's and B's parts of half of it
#pragma unroll
                for (int c = 0; c < kHalf; ++c) tmem_ld32(from + 32 * c, v + 32 * c);
#pragma unroll
                for (int c = 0; c < kHalf; ++c) tmem_ld32(then + 32 * c, v + 32 * (kHalf + c));
#pragma unroll
                for (int c = 0; c < 2 * kHalf; ++c) tmem_wait_ld(v + 32 * c);
                if (both) {
#pragma unroll
                    for (int i = 0; i < 16 * kHalf; ++i) {
                        const float2 z = fma2(pair_of(v + 32 * kHalf, i), make_float2(f1, f1), fma2(pair_of(v, i), make_float2(f0, f0), zero2));
                        v[2 * i] = __float_as_uint(z.x);
                        v[2 * i + 1] = __float_as_uint(z.y);
                    }
                }
#pragma unroll
                for (int c = 0; c < 2 * kHalf; ++c) {  // channels k0 + 32 c ..
                    if (c >= chunks) break;
#pragma unroll
                    for (int i = 0; i < 16; ++i) look = fma2(pair_of(v + 32 * c, i), zero2, look);
                    if (whole) {
                        // 32 channels of 32 rows at a time through shared memory: four lanes store 64 bytes of a row,
                        // where a lane a row would touch 32 lines with every store
                        __syncwarp();
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            uint32_t q[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float2 z = fma2(pair_of(v + 32 * c, 4 * i + e), inv2, zero2);
                                const __nv_bfloat162 b2 = __floats2bfloat162_rn(z.x, z.y);
                                q[e] = *reinterpret_cast<const uint32_t *>(&b2);
                            }
                            *reinterpret_cast<uint4 *>(stage + lane * 64 + (((i ^ (lane >> 1)) & 3) << 4)) =
                                make_uint4(q[0], q[1], q[2], q[3]);
                        }
                        __syncwarp();
                        uint4 x[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int rr = 8 * i + lane / 4;
                            x[i] = *reinterpret_cast<const uint4 *>(stage + rr * 64 + (((lane ^ (rr >> 1)) & 3) << 4));
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (to[i]) *reinterpret_cast<uint4 *>(to[i] + 32 * c) = x[i];
                    } else if (seq >= 0) {
                        float *d = part + (int64_t)(8 * c) * step;
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            *reinterpret_cast<uint4 *>(d + i * step) = make_uint4(v[32 * c + 4 * i], v[32 * c + 4 * i + 1], v[32 * c + 4 * i + 2], v[32 * c + 4 * i + 3]);
                    }
                }
                probe = look.x + look.y;
                if (seq >= 0 && !whole && (pair || X == 0)) rows_store_ml(a, p->u, slot, r, m, l);
            }
            if (!pair) {
                // both outputs have been read, and ex: B's findings go to A
                meet();
                if (X == 1) found[row_in] = probe;
                meet();
                if (X == 0) probe += found[row_in];
            }
            if (ok && busy && (pair || X == 0)) {
                // (perhaps for V rows that are not finite and that the row does not see)
                if (isnan(probe) && seq >= 0 && !isnan(l)) *redo_flag = 1;
            }
            release();
        }
        // every part of the share is stored: nothing waits for these warps but the end of the CTA
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (*redo_flag && !*abort_flag) redo_share<D>(a, tm, n_pre, warp, 8);
    }
    fence_before_sync();
    __syncthreads();
    if (tid == 0 && *abort_flag) a.head->failed = 1;  // (the merge and the scores have nothing to go by)
    if (warp == 9) {
        fence_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

template <int D>
cudaError_t launch_tc(const RowsArgs &a, cudaStream_t st) {
    TcMap t;
    CUtensorMap mk, mv, mk8, mv8;
    if (!layer_map(&mk8, a.k, a, D, &t, 8) || !layer_map(&mv8, a.v, a, D, &t, 8) || !layer_map(&mk, a.k, a, D, &t) ||
        !layer_map(&mv, a.v, a, D, &t))
        return cudaErrorInvalidValue;
    t.stall = g_stall_next.exchange(0);
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = allow_smem(rows_tc_kernel<D>, Tc<D>::kSmem, done);
    if (e != cudaSuccess) return e;
    return launch_k(rows_tc_kernel<D>, dim3(a.ctas), dim3(kThreads), Tc<D>::kSmem, st, mk, mv, mk8, mv8, a, t);
}

}  // namespace

// (A TMA coordinate is 32 bits, and one behind the last row has to be one too.  A pair of 2^18 tiles takes half a
// second, and the waits for one last a second at most.)
bool rows_tc_supported(const ikv_shape *s, const ikv_cache *c) {
    return s->dtype == IKV_BF16 && c->page_size % 8 == 0 && cap_of(c) <= 1 << 25 &&
           (uint64_t)c->num_pages * s->kv_heads * c->page_size < 0x7fffff00u;
}

cudaError_t launch_rows_tc(const RowsArgs &a, int head_dim, cudaStream_t st) {
    const cudaError_t e = head_dim == 64 ? launch_tc<64>(a, st) : launch_tc<128>(a, st);
    note_launch();
    return e;
}

cudaError_t read_clear_rows_tc_error(unsigned int *v) { return read_clear_timeout(v); }

}  // namespace ikv
