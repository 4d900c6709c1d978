// The plan of a packed-row attention: its units, and the share of each CTA (see rows.cuh).  One CTA;
// everything it reads is a few words a sequence, so its time is that of its chain of dependent loads and
// barriers: 2.5 us for one sequence's window, 5 us for 32 sequences with two shared prefixes.  Counts of units
// that fit in 32 bits are summed in them, and small tables stay in shared memory: either shortens the chain.
#include "rows.cuh"

namespace ikv {

__device__ unsigned int g_rows_error = 0;

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanCum = 1024;      // units whose offsets stay in shared memory for the search

constexpr int kPlanSmall = 512;     // sequences and groups whose tables stay there

struct Sums {
    int32_t n;                      // units
    int64_t cost, items;            // of the attention, of the score pass
    __device__ __forceinline__ Sums operator+(const Sums &o) const { return {n + o.n, cost + o.cost, items + o.items}; }
};
// the same in 32 bits, for plans that fit
struct Sums32 {
    int32_t n, cost, items;
    __device__ __forceinline__ Sums32 operator+(const Sums32 &o) const { return {n + o.n, cost + o.cost, items + o.items}; }
};

// Exclusive sums over the CTA's threads, on top of `carry`, which the totals are added to.
__device__ __forceinline__ Sums scan(Sums *sc, const Sums &x, Sums &carry) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    Sums a = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const Sums y{__shfl_up_sync(0xffffffffu, a.n, o), __shfl_up_sync(0xffffffffu, a.cost, o),
                     __shfl_up_sync(0xffffffffu, a.items, o)};
        if (lane >= o) a = a + y;
    }
    if (lane == 31) sc[warp] = a;
    __syncthreads();
    Sums before{0, 0, 0}, all{0, 0, 0};
    for (int w = 0; w < warps; ++w) {
        if (w == warp) before = all;
        all = all + sc[w];
    }
    __syncthreads();
    const Sums at = carry + before;
    carry = carry + all;
    return {at.n + a.n - x.n, at.cost + a.cost - x.cost, at.items + a.items - x.items};
}

__device__ __forceinline__ int clamp_start(const RowsArgs &a, int b) {
    return a.pv.start ? min(max(__ldg(a.pv.start + b), 0), a.cap) : 0;
}
__device__ __forceinline__ int clamp_len(const RowsArgs &a, int b, int S0) {
    return min(max(__ldg(a.len + b), 0), a.cap - S0);
}

// RowsUnit::open of a unit that ends at slot hi of a sequence that ends at `end`
__device__ __forceinline__ int32_t is_open(int hi, int end) { return ((hi + 63) & ~63) > end; }

// a run of slots [lo, hi) seen by every row of a unit
__device__ __forceinline__ void whole_run(RowsUnit &u, int lo, int hi) {
    u.lo = u.wlo = u.sh = lo;
    u.hi = hi;
    u.p0 = 0;
    u.open = u.n_a = 0;
    u.t_w = lo / kRowsTile;
    u.nt = hi > lo ? (hi - 1) / kRowsTile - u.t_w + 1 : 0;
    u.row0 = 0;
}

// Query tokens [t0, t0 + unit_n) of a sequence (window); nt = 0 where there are none
__device__ __forceinline__ RowsUnit window_unit(const RowsArgs &a, uint32_t i) {
    RowsUnit u{};
    const int b = (int)(i / (uint32_t)a.seq_units), t0 = (int)(i - (uint32_t)b * a.seq_units) * a.unit_n;
    const int c = a.count ? min(max(__ldg(a.count + b), 0), a.max_count) : a.max_count;
    u.S0 = clamp_start(a, b);
    const int len = clamp_len(a, b, u.S0);
    u.row0 = a.row0 ? __ldg(a.row0 + b) : b * a.max_count;
    if (t0 >= c) return u;
    u.b = b;
    u.m0 = t0;
    u.n = min(a.unit_n, c - t0);
    u.lo = u.S0;
    u.p0 = u.S0 + len - c + t0;
    u.hi = u.p0 + u.n;  // the last query's slot and those before
    if (u.hi > u.S0) {
        u.wlo = max(u.S0, u.p0 - a.window + 1);
        u.sh = min(u.S0 + a.sinks, u.hi);
        u.t_w = u.wlo / kRowsTile;
        u.open = is_open(u.hi, u.S0 + len);
        u.n_a = u.sh > u.S0 ? max(0, min((u.sh - 1) / kRowsTile + 1, u.t_w) - u.S0 / kRowsTile) : 0;
        u.nt = u.n_a + (u.hi - 1) / kRowsTile - u.t_w + 1;
    } else {  // no query sees a slot: a tile without one makes the zeros
        u.hi = u.wlo = u.sh = u.S0;
        u.t_w = u.S0 / kRowsTile;
        u.nt = 1;
    }
    return u;
}

__device__ __forceinline__ int64_t cost(const RowsArgs &a, const RowsUnit &u) {
    return u.nt > 0 ? pair_cost(rows_cost(a, u.n), u.nt) * a.pv.kv_heads : 0;
}

// tiles of the score pass: each for every `item_n` members, at least half of a unit's most (and, with a utility row a KV head, for each of those)
__device__ __forceinline__ int64_t items(const RowsArgs &a, const RowsUnit &u) {
    return a.items && u.nt > 0 ? (int64_t)u.nt * a.item_subs * (u.n > a.item_n ? 2 : 1) : 0;
}

__device__ __forceinline__ void store_unit(const RowsArgs &a, int at, const RowsUnit &u) {
    int4 *d = reinterpret_cast<int4 *>(a.units + at);
    const int4 *s = reinterpret_cast<const int4 *>(&u);
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = s[i];
}

// CTAs behind the first: the live slots of every utility row as bits, 1024 slots a warp at a time
__device__ __forceinline__ void live_bits(const RowsArgs &a) {
    const int lane = threadIdx.x & 31, warps = blockDim.x >> 5;
    const int chunks = (a.live_words + 31) / 32;
    const int64_t all = (int64_t)a.batch * a.rows_per_seq * chunks;
    for (int64_t i = (int64_t)(blockIdx.x - 1) * warps + (threadIdx.x >> 5); i < all; i += (int64_t)(gridDim.x - 1) * warps) {
        const int64_t row = i / chunks;
        const int w0 = (int)(i % chunks) * 32, b = (int)(row / a.rows_per_seq);
        const int len = clamp_len(a, b, clamp_start(a, b));
        if (w0 * 32 >= len) continue;
        const int32_t *pos = a.pos + row * a.cap + w0 * 32;
        const int n = min(len - w0 * 32, 1024);
        uint32_t mine = 0;
#pragma unroll 8
        for (int w = 0; w < 32; ++w) {
            const int j = 32 * w + lane;
            const uint32_t bits = __ballot_sync(0xffffffffu, j < n && __ldg(pos + j) >= 0);
            if (w == lane) mine = bits;
        }
        if (w0 + lane < a.live_words) a.live[row * a.live_words + w0 + lane] = mine;
    }
}

// Exclusive sums over a warp, on top of `carry`
__device__ __forceinline__ Sums32 warp_scan(const Sums32 &x, Sums32 &carry) {
    const int lane = threadIdx.x & 31;
    Sums32 s = x;
#pragma unroll 1
    for (int o = 1; o < 32; o <<= 1) {
        const Sums32 y{__shfl_up_sync(0xffffffffu, s.n, o), __shfl_up_sync(0xffffffffu, s.cost, o),
                       __shfl_up_sync(0xffffffffu, s.items, o)};
        if (lane >= o) s = s + y;
    }
    const Sums32 at{carry.n + s.n - x.n, carry.cost + s.cost - x.cost, carry.items + s.items - x.items};
    carry = carry + Sums32{__shfl_sync(0xffffffffu, s.n, 31), __shfl_sync(0xffffffffu, s.cost, 31),
                           __shfl_sync(0xffffffffu, s.items, 31)};
    return at;
}

// The prefix plan of at most 32 sequences and groups, each group one unit, by one warp without a barrier.  (Its time is
// that of the instructions on their way from memory, executed once each: it is kept short.)  tab: 64 words of shared memory.
template <typename Put>
__device__ __forceinline__ void small_plan(const RowsArgs &a, Put put, Sums32 &sum, int &n_pre, int32_t *tab) {
    constexpr unsigned kAll = 0xffffffffu;
    const int lane = threadIdx.x & 31;
    int f0 = 0x7fffffff, f1 = 0x7fffffff, glen = 0, S0 = 0, L = 0;
    if (lane < a.n_groups) {
        f0 = __ldg(a.first + lane);
        f1 = __ldg(a.first + lane + 1);
        glen = max(__ldg(a.group_len + lane), 0);
    }
    if (lane < a.batch) {
        S0 = clamp_start(a, lane);
        L = clamp_len(a, lane, S0);
    }
    int n_groups = a.n_groups;
    if (__any_sync(kAll, lane < n_groups && (f0 < 0 || f0 > f1))) n_groups = 0;  // the groups' entries would overlap
    const int raw = n_groups > 0 ? __shfl_sync(kAll, f1, n_groups - 1) : 0;
    const int entries = min(raw, a.batch), entry0 = n_groups > 0 ? __shfl_sync(kAll, f0, 0) : 0;
    bool wrong = (n_groups != a.n_groups || raw > a.batch) && lane == 0;
    // lane: entry
    const bool entry = lane >= entry0 && lane < entries;
    int b = entry ? __ldg(a.member + lane) : -1;
    const unsigned same = __match_any_sync(kAll, entry && b >= 0 && b < a.batch ? b : -1 - lane);
    if (entry && !(b >= 0 && b < a.batch && __ffs(same) - 1 == lane)) {  // it counts if it is the first that names it
        wrong = true;
        b = -1;
    }
    if (__any_sync(kAll, wrong) && lane == 0) atomicOr(&g_rows_error, 128u);
    if (entry) a.vm[lane] = b;
    int gi = 0;  // its group: the last that begins at or before it
#pragma unroll 1
    for (int o = 16; o > 0; o >>= 1) {
        const int f = __shfl_sync(kAll, f0, min(gi + o, 31));
        if (gi + o < n_groups && f <= lane) gi += o;
    }
    const bool counts = entry && b >= 0;
    const unsigned mates = __match_any_sync(kAll, counts ? gi : -1 - lane);
    const int my_len = __shfl_sync(kAll, L, max(b, 0)), my_S0 = __shfl_sync(kAll, S0, max(b, 0));
    int p = min((int)__reduce_min_sync(mates, (unsigned)my_len), __shfl_sync(kAll, glen, gi));
    if (!counts || __popc(mates) < 2) p = 0;  // (one alone: nothing to share)
    const int e0 = __shfl_sync(kAll, f0, gi), e1 = min(__shfl_sync(kAll, f1, gi), entries);
    RowsUnit u{};
    if (p > 0 && __ffs(mates) - 1 == lane) {  // the first member makes the group's unit
        u.b = b;
        u.m0 = e0;
        u.n = e1 - e0;
        u.S0 = my_S0;
        whole_run(u, u.S0, u.S0 + p);
        u.open = is_open(u.hi, u.S0 + my_len);
    }
    const Sums32 at = warp_scan({u.nt > 0 ? 1 : 0, (int)cost(a, u), (int)items(a, u)}, sum);
    const int unit0 = __shfl_sync(kAll, at.n, __ffs(mates) - 1);
    if (u.nt > 0) put(u, {at.n, at.cost, at.items});
    n_pre = sum.n;
    // lane: sequence
    tab[lane] = -1;
    __syncwarp();
    if (counts && p > 0) {
        tab[b] = unit0 | (lane - e0) << 16;
        tab[32 + b] = p;
    }
    __syncwarp();
    RowsSeq s{-1, 0, -1, 0};
    if (tab[lane] >= 0) {
        s.pre = tab[lane] & 0xffff;
        s.entry = tab[lane] >> 16;
        s.len = tab[32 + lane];
    }
    u = RowsUnit{};
    if (lane < a.batch) {
        u.b = lane;
        u.m0 = -1;
        u.n = 1;
        u.S0 = S0;
        whole_run(u, S0 + s.len, S0 + L);
        u.open = 1;
    }
    const Sums32 own = warp_scan({u.nt > 0 ? 1 : 0, (int)cost(a, u), (int)items(a, u)}, sum);
    if (u.nt > 0) {
        put(u, {own.n, own.cost, own.items});
        s.own = own.n;
    }
    if (lane < a.batch) *reinterpret_cast<int4 *>(a.seq + lane) = *reinterpret_cast<int4 *>(&s);
}

__global__ void __launch_bounds__(kPlanThreads) rows_plan_kernel(const RowsArgs a) {
    pdl_wait();
    if (blockIdx.x > 0) {
        live_bits(a);
        return;
    }
    __shared__ Sums sc[kPlanThreads / 32];
    __shared__ int64_t cums[kPlanCum], icums[kPlanCum];
    __shared__ int2 sizes[kPlanCum];  // tiles, cost of a pair
    __shared__ int32_t small_tab[6 * kPlanSmall];
    __shared__ int32_t bcast;
    __shared__ Sums bcast_sum;
    const int tid = threadIdx.x, nthr = blockDim.x;
    int n_pre = 0;
    Sums sum{0, 0, 0};
    auto put = [&](RowsUnit u, const Sums &at) {  // unit number at.n
        u.cum = at.cost;
        store_unit(a, at.n, u);
        if (a.icum) a.icum[at.n] = at.items;
        if (at.n < kPlanCum) {
            cums[at.n] = at.cost;
            icums[at.n] = at.items;
            sizes[at.n] = make_int2(u.nt, (int)pair_cost(rows_cost(a, u.n), u.nt));
        }
    };
    if (a.small) {
        if (tid < 32) {
            Sums32 x{0, 0, 0};
            if (a.prefix) {
                small_plan(a, put, x, n_pre, small_tab);
            } else {
                RowsUnit u{};
                if (tid < a.batch * a.seq_units) u = window_unit(a, tid);
                const Sums32 at = warp_scan({u.nt > 0 ? 1 : 0, (int)cost(a, u), 0}, x);
                if (u.nt > 0) put(u, {at.n, at.cost, 0});
            }
            if (tid == 0) {
                bcast = n_pre;
                bcast_sum = {x.n, x.cost, x.items};
            }
        }
        __syncthreads();
        n_pre = bcast;
        sum = bcast_sum;
    } else if (!a.prefix) {
        const uint32_t all = (uint32_t)a.batch * a.seq_units;  // (at most 2^30)
        for (uint32_t i0 = 0; i0 < all; i0 += nthr) {
            RowsUnit u{};
            if (i0 + tid < all) u = window_unit(a, i0 + tid);
            const Sums at = scan(sc, {u.nt > 0 ? 1 : 0, cost(a, u), 0}, sum);
            if (u.nt > 0) put(u, at);
        }
    } else {
        // (small batches keep the tables in shared memory: the chain of their look-ups is the time)
        int32_t *owner = a.owner, *vm = a.vm, *group = a.entry_group;
        int32_t *gp = a.group_p, *glead = a.group_lead, *gunit = a.group_unit;
        if (a.batch <= kPlanSmall && a.n_groups <= kPlanSmall) {
            owner = small_tab;
            vm = small_tab + kPlanSmall;
            group = small_tab + 2 * kPlanSmall;
            gp = small_tab + 3 * kPlanSmall;
            glead = small_tab + 4 * kPlanSmall;
            gunit = small_tab + 5 * kPlanSmall;
        }
        int n_groups = a.n_groups;
        int bad = 0;
        for (int i = tid; i < n_groups; i += nthr) {
            const int f = __ldg(a.first + i);
            if (f < 0 || f > __ldg(a.first + i + 1)) bad = 1;
        }
        for (int b = tid; b < a.batch; b += nthr) owner[b] = 0x7fffffff;
        if (__syncthreads_or(bad)) {  // the groups' entries would overlap
            if (tid == 0) atomicOr(&g_rows_error, 128u);
            n_groups = 0;
        }
        const int entries_raw = n_groups > 0 ? __ldg(a.first + n_groups) : 0;
        const int entries = min(entries_raw, a.batch), entry0 = n_groups > 0 ? min(__ldg(a.first), entries) : 0;
        if (tid == 0 && entries_raw > a.batch) atomicOr(&g_rows_error, 128u);
        // an entry counts if it is the first that names its sequence
        for (int e = entry0 + tid; e < entries; e += nthr) {
            const int b = __ldg(a.member + e);
            if (b >= 0 && b < a.batch) atomicMin(owner + b, e);
        }
        __syncthreads();
        for (int e = entry0 + tid; e < entries; e += nthr) {
            const int b = __ldg(a.member + e);
            const bool ok = b >= 0 && b < a.batch && owner[b] == e;
            vm[e] = ok ? b : -1;
            if (vm != a.vm) a.vm[e] = vm[e];
            if (!ok) atomicOr(&g_rows_error, 128u);
        }
        __syncthreads();
        // a warp a group: its first member, and the slots that all of its members have
        for (int i = tid >> 5; i < n_groups; i += nthr >> 5) {
            const int e0 = min(__ldg(a.first + i), entries), e1 = min(__ldg(a.first + i + 1), entries);
            const int lane = tid & 31;
            int p = max(__ldg(a.group_len + i), 0), lead = 0x7fffffff, n = 0;
            for (int e = e0 + lane; e < e1; e += 32) {
                const int b = vm[e];
                group[e] = i;
                if (b < 0) continue;
                p = min(p, clamp_len(a, b, clamp_start(a, b)));
                lead = min(lead, e);
                ++n;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) {
                p = min(p, __shfl_xor_sync(0xffffffffu, p, o));
                lead = min(lead, __shfl_xor_sync(0xffffffffu, lead, o));
                n += __shfl_xor_sync(0xffffffffu, n, o);
            }
            if (n > 0) p = min(p, a.cap - clamp_start(a, vm[lead]));
            if (n < 2) p = 0;  // nothing to share
            if (lane == 0) {
                gp[i] = p;
                glead[i] = p > 0 ? vm[lead] : -1;
            }
        }
        __syncthreads();
        for (int i0 = 0; i0 < n_groups; i0 += nthr) {
            const int i = i0 + tid;
            RowsUnit u{};
            int n = 0, e0 = 0, e1 = 0;
            if (i < n_groups && gp[i] > 0) {
                e0 = min(__ldg(a.first + i), entries);
                e1 = min(__ldg(a.first + i + 1), entries);
                n = (e1 - e0 + a.unit_n - 1) / a.unit_n;
                u.b = glead[i];
                u.S0 = clamp_start(a, u.b);
                u.n = min(a.unit_n, e1 - e0);
                whole_run(u, u.S0, u.S0 + gp[i]);
                u.open = is_open(u.hi, u.S0 + clamp_len(a, u.b, u.S0));
            }
            // (all but a group's last unit are full)
            const int most = u.n, rest = n > 0 ? e1 - e0 - (n - 1) * most : 0;
            RowsUnit last = u;
            last.n = rest;
            Sums at = scan(sc, {n, n > 0 ? (n - 1) * cost(a, u) + cost(a, last) : 0,
                                n > 0 ? (n - 1) * items(a, u) + items(a, last) : 0}, sum);
            if (i < n_groups) gunit[i] = at.n;
            for (int k = 0; k < n; ++k) {
                u.m0 = e0 + k * most;
                u.n = k == n - 1 ? rest : most;
                put(u, at);
                at = at + Sums{1, cost(a, u), items(a, u)};
            }
        }
        n_pre = sum.n;
        __syncthreads();
        for (int b0 = 0; b0 < a.batch; b0 += nthr) {
            const int b = b0 + tid;
            RowsUnit u{};
            RowsSeq s{-1, 0, -1, 0};
            if (b < a.batch) {
                const int e = owner[b];
                if (e < entries) {
                    const int i = group[e];
                    if (gp[i] > 0) {
                        const int k = e - __ldg(a.first + i);
                        s.pre = gunit[i] + k / a.unit_n;
                        s.entry = k % a.unit_n;
                        s.len = gp[i];
                    }
                }
                u.b = b;
                u.m0 = -1;
                u.n = 1;
                u.S0 = clamp_start(a, b);
                whole_run(u, u.S0 + s.len, u.S0 + clamp_len(a, b, u.S0));
                u.open = 1;
            }
            const Sums at = scan(sc, {u.nt > 0 ? 1 : 0, cost(a, u), items(a, u)}, sum);
            if (u.nt > 0) {
                put(u, at);
                s.own = at.n;
            }
            if (b < a.batch) *reinterpret_cast<int4 *>(a.seq + b) = *reinterpret_cast<int4 *>(&s);
        }
    }
    __syncthreads();
    auto share = [&](int64_t x) { return x >> 31 ? (x + a.ctas - 1) / a.ctas : (int64_t)(((uint32_t)x + a.ctas - 1) / (uint32_t)a.ctas); };
    // (a share has at least a tile's cost: none that lies in a pair's tiles is empty)
    const int64_t per = max(share(sum.cost), (int64_t)(a.unit_n > a.tile_n ? kTileTwo : kTileOne));
    if (tid == 0) {
        a.head->per = per;
        a.head->n_pre = n_pre;
        a.head->failed = 0;
    }
    auto size = [&](int i) {
        return i < kPlanCum ? sizes[i]
                            : make_int2(__ldcg(&a.units[i].nt), (int)pair_cost(rows_cost(a, __ldcg(&a.units[i].n)), __ldcg(&a.units[i].nt)));
    };
    auto divide = [](int64_t x, int y) { return x >> 31 ? (int32_t)(x / y) : (int32_t)((uint32_t)x / (uint32_t)y); };
    // the last unit that begins at or before x
    auto find = [&](const int64_t *small, auto big, int64_t x) {
        int lo = 0, hi = sum.n;
        if (hi <= kPlanCum) {  // (no look-ups in memory)
#pragma unroll 1
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (small[mid] <= x)
                    lo = mid;
                else
                    hi = mid;
            }
            return lo;
        }
#pragma unroll 1
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if ((mid < kPlanCum ? small[mid] : big(mid)) <= x)
                lo = mid;
            else
                hi = mid;
        }
        return lo;
    };
    for (int c = tid; c < a.ctas; c += nthr) {
        RowsStart s{};
        const int64_t x = (int64_t)c * per;
        if (x < sum.cost) {
            auto big = [&](int i) { return __ldcg(&a.units[i].cum); };
            s.unit = find(cums, big, x);
            const int each = size(s.unit).y;
            const int64_t r = x - (s.unit < kPlanCum ? cums[s.unit] : big(s.unit));
            s.g = divide(r, each);
            s.at = (int32_t)(r - (int64_t)s.g * each);
            s.n = (int32_t)min(per, sum.cost - x);
        }
        *reinterpret_cast<int4 *>(a.start + c) = *reinterpret_cast<int4 *>(&s);
        if (!a.items) continue;
        RowsItems t{0, 0, 0, 0};
        const int64_t many = share(sum.items), y = c * many;
        if (y < sum.items) {
            auto big = [&](int i) { return __ldcg(a.icum + i); };
            t.unit = find(icums, big, y);
            const int nt = size(t.unit).x;
            const int64_t r = y - (t.unit < kPlanCum ? icums[t.unit] : big(t.unit));
            t.sub = divide(r, nt);
            t.j = (int32_t)(r - (int64_t)t.sub * nt);
            t.n = (int32_t)min(many, sum.items - y);
        }
        *reinterpret_cast<int4 *>(a.items + c) = *reinterpret_cast<int4 *>(&t);
    }
}

}  // namespace

cudaError_t launch_rows_plan(const RowsArgs &a, cudaStream_t st) {
    const int64_t most = a.prefix ? (int64_t)(a.batch > a.n_groups ? a.batch : a.n_groups) : (int64_t)a.batch * a.seq_units;
    int threads = 256;  // (of which each finds where a share begins)
    while (threads < kPlanThreads && threads < most) threads *= 2;
    int ctas = 1;
    if (a.live) {
        const int64_t warps = (int64_t)a.batch * a.rows_per_seq * ((a.live_words + 31) / 32);
        const int64_t n = (warps + threads / 32 - 1) / (threads / 32);
        ctas += (int)(n < 4 * a.ctas ? n : 4 * a.ctas);
    }
    const cudaError_t e = launch_k(rows_plan_kernel, dim3(ctas), dim3(threads), 0, st, a);
    note_launch();
    return e;
}

cudaError_t read_clear_rows_error(unsigned int *v) {
    unsigned int z = 0;
    cudaError_t e = cudaMemcpyFromSymbol(v, g_rows_error, sizeof(*v));
    if (e == cudaSuccess && *v) e = cudaMemcpyToSymbol(g_rows_error, &z, sizeof(z));
    unsigned int tc = 0, sc = 0;
    if (e == cudaSuccess) e = read_clear_rows_tc_error(&tc);
    if (e == cudaSuccess) e = read_clear_rows_score_error(&sc);
    *v |= tc | sc;
    return e;
}

}  // namespace ikv
