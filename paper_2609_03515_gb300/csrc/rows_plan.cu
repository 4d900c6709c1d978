// The plan of a packed-row attention: its units, and the share of each CTA (see rows.cuh).  One CTA;
// everything it reads is a few words a sequence, so its time is that of its chain of dependent loads and
// barriers.
#include "rows.cuh"

namespace ikv {

__device__ unsigned int g_rows_error = 0;

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanCum = 1024;      // units whose offsets stay in shared memory for the search

constexpr int kPlanSmall = 1024;    // sequences and groups whose tables stay there

struct Scan {
    int64_t sum[kPlanThreads / 32];
    int32_t cnt[kPlanThreads / 32];
};

// Exclusive sums of (n, tiles) over the CTA's threads; the totals are added to the carries.
__device__ __forceinline__ void scan(Scan &sc, int n, int64_t tiles, int &n_carry, int64_t &t_carry, int &n_at,
                                     int64_t &t_at) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    int a = n;
    int64_t b = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, a, o);
        const int64_t y = __shfl_up_sync(0xffffffffu, b, o);
        if (lane >= o) {
            a += x;
            b += y;
        }
    }
    if (lane == 31) {
        sc.cnt[warp] = a;
        sc.sum[warp] = b;
    }
    __syncthreads();
    int na = 0, nall = 0;
    int64_t ta = 0, tall = 0;
    for (int w = 0; w < warps; ++w) {
        if (w == warp) {
            na = nall;
            ta = tall;
        }
        nall += sc.cnt[w];
        tall += sc.sum[w];
    }
    __syncthreads();
    n_at = n_carry + na + a - n;
    t_at = t_carry + ta + b - tiles;
    n_carry += nall;
    t_carry += tall;
}

__device__ __forceinline__ int clamp_start(const RowsArgs &a, int b) {
    return a.pv.start ? min(max(__ldg(a.pv.start + b), 0), a.cap) : 0;
}
__device__ __forceinline__ int clamp_len(const RowsArgs &a, int b, int S0) {
    return min(max(__ldg(a.len + b), 0), a.cap - S0);
}

// a run of slots [lo, hi) seen by every row of a unit
__device__ __forceinline__ void whole_run(RowsUnit &u, int lo, int hi) {
    u.lo = u.wlo = u.sh = lo;
    u.hi = hi;
    u.p0 = 0;
    u.t_a = u.n_a = 0;
    u.t_w = lo / kRowsTile;
    u.nt = hi > lo ? (hi - 1) / kRowsTile - u.t_w + 1 : 0;
    u.row0 = 0;
}

__device__ __forceinline__ int64_t cost(const RowsUnit &u, int kv_heads) {
    return u.nt > 0 ? (int64_t)(u.nt + kRowsExtra) * kv_heads : 0;
}

__device__ __forceinline__ void store_unit(const RowsArgs &a, int at, const RowsUnit &u) {
    int4 *d = reinterpret_cast<int4 *>(a.units + at);
    const int4 *s = reinterpret_cast<const int4 *>(&u);
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = s[i];
}

__global__ void __launch_bounds__(kPlanThreads) rows_plan_kernel(const RowsArgs a) {
    pdl_wait();
    __shared__ Scan sc;
    __shared__ int64_t cums[kPlanCum];
    __shared__ int32_t small_tab[6 * kPlanSmall];
    const int tid = threadIdx.x, nthr = blockDim.x, hk = a.pv.kv_heads;
    int units = 0, n_pre = 0;
    int64_t tiles = 0;  // (their cost)
    if (!a.prefix) {
        const int64_t all = (int64_t)a.batch * a.seq_units;
        for (int64_t i0 = 0; i0 < all; i0 += nthr) {
            const int64_t i = i0 + tid;
            RowsUnit u{};
            if (i < all) {
                const int b = (int)(i / a.seq_units), t0 = (int)(i % a.seq_units) * a.unit_n;
                const int c = a.count ? min(max(__ldg(a.count + b), 0), a.max_count) : a.max_count;
                if (t0 < c) {
                    u.b = b;
                    u.m0 = t0;
                    u.n = min(a.unit_n, c - t0);
                    u.S0 = clamp_start(a, b);
                    u.lo = u.S0;
                    u.row0 = a.row0 ? __ldg(a.row0 + b) : b * a.max_count;
                    u.p0 = u.S0 + clamp_len(a, b, u.S0) - c + t0;
                    u.hi = u.p0 + u.n;  // the last query's slot and those before
                    if (u.hi > u.S0) {
                        u.wlo = max(u.S0, u.p0 - a.window + 1);
                        u.sh = min(u.S0 + a.sinks, u.hi);
                        u.t_w = u.wlo / kRowsTile;
                        u.t_a = u.S0 / kRowsTile;
                        u.n_a = u.sh > u.S0 ? max(0, min((u.sh - 1) / kRowsTile + 1, u.t_w) - u.t_a) : 0;
                        u.nt = u.n_a + (u.hi - 1) / kRowsTile - u.t_w + 1;
                    } else {  // no query sees a slot: a tile without one makes the zeros
                        u.hi = u.wlo = u.sh = u.S0;
                        u.t_w = u.S0 / kRowsTile;
                        u.nt = 1;
                    }
                }
            }
            int at;
            scan(sc, u.nt > 0 ? 1 : 0, cost(u, hk), units, tiles, at, u.cum);
            if (u.nt > 0) {
                store_unit(a, at, u);
                if (at < kPlanCum) cums[at] = u.cum;
            }
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
                whole_run(u, u.S0, u.S0 + gp[i]);
            }
            int at;
            int64_t cum;
            scan(sc, n, n * cost(u, hk), units, tiles, at, cum);
            if (i < n_groups) gunit[i] = at;
            for (int k = 0; k < n; ++k) {
                u.m0 = e0 + k * a.unit_n;
                u.n = min(a.unit_n, e1 - u.m0);
                u.cum = cum + k * cost(u, hk);
                store_unit(a, at + k, u);
                if (at + k < kPlanCum) cums[at + k] = u.cum;
            }
        }
        n_pre = units;
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
            }
            int at;
            scan(sc, u.nt > 0 ? 1 : 0, cost(u, hk), units, tiles, at, u.cum);
            if (u.nt > 0) {
                store_unit(a, at, u);
                if (at < kPlanCum) cums[at] = u.cum;
                s.own = at;
            }
            if (b < a.batch) *reinterpret_cast<int4 *>(a.seq + b) = *reinterpret_cast<int4 *>(&s);
        }
    }
    __syncthreads();
    int64_t per = (tiles + a.ctas - 1) / a.ctas;
    if (per < 1) per = 1;
    if (tid == 0) {
        a.head->total = tiles;
        a.head->per = per;
        a.head->n_units = units;
        a.head->n_pre = n_pre;
    }
    for (int c = tid; c < a.ctas; c += nthr) {
        RowsStart s{0, 0, 0, 0};
        const int64_t x = (int64_t)c * per;
        if (x < tiles) {
            int lo = 0, hi = units;  // the last unit that begins at or before x
            while (hi - lo > 1) {
                const int mid = (lo + hi) / 2;
                if ((mid < kPlanCum ? cums[mid] : __ldcg(&a.units[mid].cum)) <= x)
                    lo = mid;
                else
                    hi = mid;
            }
            const int each = __ldcg(&a.units[lo].nt) + kRowsExtra;
            const int64_t r = x - (lo < kPlanCum ? cums[lo] : __ldcg(&a.units[lo].cum));
            s.unit = lo;
            s.g = (int32_t)(r / each);
            s.at = (int32_t)(r % each);
            s.n = (int32_t)min(per, tiles - x);
        }
        *reinterpret_cast<int4 *>(a.start + c) = *reinterpret_cast<int4 *>(&s);
    }
}

}  // namespace

cudaError_t launch_rows_plan(const RowsArgs &a, cudaStream_t st) {
    const int64_t most = a.prefix ? (int64_t)(a.batch > a.n_groups ? a.batch : a.n_groups) : (int64_t)a.batch * a.seq_units;
    int threads = 128;
    while (threads < kPlanThreads && threads < most) threads *= 2;
    const cudaError_t e = launch_k(rows_plan_kernel, dim3(1), dim3(threads), 0, st, a);
    note_launch();
    return e;
}

cudaError_t read_clear_rows_error(unsigned int *v) {
    unsigned int z = 0;
    cudaError_t e = cudaMemcpyFromSymbol(v, g_rows_error, sizeof(*v));
    if (e == cudaSuccess && *v) e = cudaMemcpyToSymbol(g_rows_error, &z, sizeof(z));
    unsigned int tc = 0;
    if (e == cudaSuccess) e = read_clear_rows_tc_error(&tc);
    *v |= tc;
    return e;
}

}  // namespace ikv
