// Pages that sequences share, take and give back.
//
// Page 0 is nobody's: a block table entry of 0 means "no page", so that every entry names a valid
// page whatever it is.  refs counts the entries that hold a page; a page with none is free.  Pages
// are handed out lowest first, in the order of the sequences and their slots, so that a run can
// be repeated.
#include "q4.cuh"

namespace ikv {

__device__ unsigned int g_pages_error = 0;  // bit 2: slots past the slot space; bit 6: too few free pages; bit 7: bad index

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kCopyThreads = 256;
constexpr int kRowThreads = 256;

// (within the slot space, whatever the array holds: table entries are found from it)
__device__ __forceinline__ int start_of(const PagesArgs &a, int b) { return a.start ? min(max(a.start[b], 0), a.cap) : 0; }
// slots that a sequence keeps in a compaction: no more than lie behind its start
__device__ __forceinline__ int kept_of(const PagesArgs &a, int b, int keep_len) { return min(keep_len, a.cap - start_of(a, b)); }

// Whether a block table entry names a page; one that is neither a page nor 0 is reported.
__device__ __forceinline__ bool holds_page(const PagesArgs &a, int entry) {
    if (entry > 0 && entry < a.num_pages) return true;
    if (entry != 0) atomicOr(&g_pages_error, 128u);
    return false;
}
// A page of the sequence's went, or others hold it too: it has to ask again before it writes.
__device__ __forceinline__ void forget_granted(const PagesArgs &a, int b) {
    if (a.writable) a.writable[b] = make_int2(0, 0);
}

// Exclusive prefix sum of x over the CTA (kPlanThreads threads), and the total.
__device__ __forceinline__ int block_scan(int x, int *total) {
    __shared__ int sums[32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int y = x;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int z = __shfl_up_sync(0xffffffffu, y, d);
        if (lane >= d) y += z;
    }
    __syncthreads();  // (the sums of a scan before)
    if (lane == 31) sums[warp] = y;
    __syncthreads();
    if (warp == 0) {
        int s = sums[lane];
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int z = __shfl_up_sync(0xffffffffu, s, d);
            if (lane >= d) s += z;
        }
        sums[lane] = s;
    }
    __syncthreads();
    *total = sums[31];
    return y - x + (warp ? sums[warp - 1] : 0);
}

// The lowest free pages, by one CTA.  A pass looks at kPlanThreads x kPass pages, a warp at
// 32 kPass behind one another; the first pass is loaded ahead of what says how many are wanted.
struct FreePages {
    static constexpr int kPass = 16;
    const int32_t *refs;
    int pages;
    int32_t r[kPass];
    __device__ __forceinline__ void load(int p0) {
#pragma unroll
        for (int u = 0; u < kPass; ++u) {
            const int p = p0 + (threadIdx.x >> 5) * 32 * kPass + 32 * u + (threadIdx.x & 31);
            r[u] = p > 0 && p < pages ? __ldcg(refs + p) : 1;
        }
    }
    // `want` of them into ids (which all threads may read then), after load(0); how many there are, at most `want`
    __device__ __forceinline__ int find(int want, int32_t *ids) {
        const int lane = threadIdx.x & 31, mine0 = (threadIdx.x >> 5) * 32 * kPass;
        int found = 0;
        for (int p0 = 0; p0 < pages && found < want; p0 += kPlanThreads * kPass) {
            if (p0 > 0) load(p0);
            uint32_t free[kPass];
            int mine = 0;
#pragma unroll
            for (int u = 0; u < kPass; ++u) {
                free[u] = __ballot_sync(0xffffffffu, r[u] == 0);
                mine += __popc(free[u]);
            }
            int n, at = block_scan(lane == 0 ? mine : 0, &n);
            at = found + __shfl_sync(0xffffffffu, at, 0);
#pragma unroll
            for (int u = 0; u < kPass; ++u) {
                const int to = at + __popc(free[u] & ((1u << lane) - 1));
                if ((free[u] >> lane & 1u) && to < want) ids[to] = p0 + mine0 + 32 * u + lane;
                at += __popc(free[u]);
            }
            found += n;
        }
        __syncthreads();
        return min(found, want);
    }
};

__global__ void __launch_bounds__(kRowThreads) release_kernel(const PagesArgs a, int extra) {
    pdl_wait();
    const int64_t i = (int64_t)blockIdx.x * kRowThreads + threadIdx.x;
    if (i >= (int64_t)a.batch * a.max_pages) return;
    const int e = a.table[i];
    if (!holds_page(a, e)) return;
    const int b = (int)(i / a.max_pages), lp = (int)(i % a.max_pages);
    const int64_t S = start_of(a, b), L = a.len[b], p0 = (int64_t)lp * a.page_size;
    if (L > 0 && p0 + a.page_size > S && p0 < S + L + extra) return;
    a.table[i] = 0;
    atomicSub(a.refs + e, 1);
    forget_granted(a, b);
}

template <typename T>
__device__ __forceinline__ void copy_words(T *dst, const T *src, int64_t n, int64_t at, int64_t step) {
    constexpr int U = 8;
    for (int64_t j0 = at; j0 < n; j0 += U * step) {
        T x[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j0 + u * step < n) x[u] = src[j0 + u * step];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (j0 + u * step < n) dst[j0 + u * step] = x[u];
    }
}

// CTAs (part, fork): part 0 the parent's table entries and counts, the others its rows of pos and vnorm,
// and of ema.  Apart, because one CTA after another of them waits for memory: 30 forks of 8k slots with
// release and writable 52.2 us, 53.9 when every CTA did a share of each.
__global__ void __launch_bounds__(kRowThreads) fork_kernel(const PagesArgs a, const int32_t *src, const int32_t *dst) {
    pdl_wait();
    const int i = blockIdx.y, s = src[i], d = dst[i];
    if (s < 0 || s >= a.batch || d < 0 || d >= a.batch || s == d) {
        if (blockIdx.x == 0 && threadIdx.x == 0) atomicOr(&g_pages_error, 128u);
        return;
    }
    if (blockIdx.x == 0) {
        constexpr int U = 4;
        const int32_t *from = a.table + (int64_t)s * a.max_pages;
        int32_t *to = a.table + (int64_t)d * a.max_pages;
        for (int p0 = threadIdx.x; p0 < a.max_pages; p0 += U * kRowThreads) {
            int e[U];
#pragma unroll
            for (int u = 0; u < U; ++u) e[u] = p0 + u * kRowThreads < a.max_pages ? from[p0 + u * kRowThreads] : 0;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const bool held = holds_page(a, e[u]);
                if (p0 + u * kRowThreads < a.max_pages) to[p0 + u * kRowThreads] = held ? e[u] : 0;
                if (held) atomicAdd(a.refs + e[u], 1);
            }
        }
        if (threadIdx.x == 0) {
            a.len[d] = a.len[s];
            forget_granted(a, s);
            forget_granted(a, d);
            if (a.next_pos) a.next_pos[d] = a.next_pos[s];
            if (a.start) a.start[d] = a.start[s];
        }
        return;
    }
    // half of the other CTAs take pos and vnorm, half ema
    const int parts = (gridDim.x - 1) / 2, part = (blockIdx.x - 1) % parts;
    const int64_t at = (int64_t)part * kRowThreads + threadIdx.x, step = (int64_t)parts * kRowThreads;
    const int64_t n = (int64_t)a.rows_per_seq * a.cap;
    if ((int)blockIdx.x > parts) {
        if (a.ema) copy_words(a.ema + d * n, a.ema + s * n, n, at, step);
        return;
    }
    if (a.pos) copy_words(a.pos + d * n, a.pos + s * n, n, at, step);
    if (a.vnorm) {
        const int64_t m = (int64_t)a.kv_heads * a.cap;
        for (int l = 0; l < a.layers; ++l)
            copy_words(a.vnorm + ((int64_t)l * a.batch + d) * m, a.vnorm + ((int64_t)l * a.batch + s) * m, m, at, step);
    }
}

// One CTA decides which pages of the slots to be written are missing or shared, takes free ones for
// them and lists the copies to make: {page, copy, first row, rows}.  Of the sequences of this call
// that would write a shared page which nobody else holds, the last keeps it.  A chain of round
// trips to memory, and FEW (kFewRequests at most: single tokens) has the fewest: lengths, entries,
// counts; the writers are counted in shared memory, and the free pages are looked for meanwhile.
constexpr int kFewRequests = 256;
template <bool FEW>
__global__ void __launch_bounds__(kPlanThreads)
writable_plan_kernel(const PagesArgs a, const PagesWs w, const int32_t *first, const int32_t *count, int max_count,
                     int span, int32_t *lacking) {
    pdl_wait();
    __shared__ int32_t shared_pages[FEW ? kFewRequests : 1], ids_s[FEW ? kFewRequests : 1];
    const int64_t R = (int64_t)a.batch * span;
    FreePages pages{a.refs, a.num_pages};
    pages.load(0);
    if (threadIdx.x == 0) w.total[2] = 0;  // rows of the longest copy
    // the slots that sequence b asks for: {first, count}, or {-, 0}
    auto asked = [&](int b) -> int2 {
        const int n = min(count ? count[b] : max_count, max_count), from = first ? first[b] : a.len[b];
        return make_int2(from, from < 0 ? 0 : max(n, 0));
    };
    // request i: page lp of sequence b
    auto page_of = [&](int64_t i, int *b, int *lp) -> bool {
        if (i >= R) return false;
        *b = FEW ? (int)i / span : (int)(i / span);
        const int x = (int)(i - (int64_t)*b * span), S = start_of(a, *b);
        const int2 w = asked(*b);
        if (w.y == 0) return false;
        if ((int64_t)S + w.x + w.y > a.cap) {
            if (x == 0) atomicOr(&g_pages_error, 4u);
            return false;
        }
        const int f = S + w.x, p = f / a.page_size + x;
        *lp = p;
        return p <= (f + w.y - 1) / a.page_size;
    };
    // its entry, or -1
    auto request = [&](int64_t i, int *b, int *lp) -> int {
        if (!page_of(i, b, lp)) return -1;
        const int p = *lp;
        const int e = a.table[(int64_t)*b * a.max_pages + p];
        if (e >= 0 && e < a.num_pages) return e;
        atomicOr(&g_pages_error, 128u);
        return -1;
    };
    auto assign = [&](int b, int lp, int e, int to, int rank) {
        a.table[(int64_t)b * a.max_pages + lp] = to;
        a.refs[to] = 1;
        // rows of the page that hold slots in use
        const int64_t S = start_of(a, b), p0 = (int64_t)lp * a.page_size;
        const int r0 = (int)min(max(S - p0, (int64_t)0), (int64_t)a.page_size);
        const int r1 = (int)min(max(S + a.len[b] - p0, (int64_t)0), (int64_t)a.page_size);
        const int rows = e > 0 ? max(r1 - r0, 0) : 0;
        *reinterpret_cast<int4 *>(w.jobs + 4 * (int64_t)rank) = make_int4(e, to, r0, rows);
        if (rows > 0) atomicMax(w.total + 2, rows);
    };
    auto report_total = [&](int total, int have) {
        if (threadIdx.x == 0) {
            w.total[0] = have == total ? total : 0;
            if (lacking) *lacking = total - have;
            if (have < total) atomicOr(&g_pages_error, 64u);
        }
    };
    int b = 0, lp = 0;
    if constexpr (FEW) {
        const int i = threadIdx.x, e = request(i, &b, &lp);
        const int r = e > 0 ? __ldcg(a.refs + e) : 0;
        if (i < kFewRequests) shared_pages[i] = r > 1 ? e : 0;
        __syncthreads();
        bool need = e == 0;
        if (r > 1) {  // requests are in the order of the sequences
            int writers = 0;
            bool later = false;
            for (int j = 0; j < (int)R; ++j)
                if (shared_pages[j] == e) {
                    ++writers;
                    later |= j > i;
                }
            need = writers < r || later;
        }
        int total;
        const int rank = block_scan(need ? 1 : 0, &total);
        const int have = pages.find(total, ids_s);
        report_total(total, have);
        if (have == total && need) {
            assign(b, lp, e, ids_s[rank], rank);
            if (e > 0) atomicSub(a.refs + e, 1);  // (every count is read)
        }
    } else {
        for (int64_t i = threadIdx.x; i < R; i += kPlanThreads) {
            const int e = request(i, &b, &lp);
            if (e > 0) {
                w.count[e] = 0;
                w.last[e] = -1;
            }
        }
        __syncthreads();
        for (int64_t i = threadIdx.x; i < R; i += kPlanThreads) {
            const int e = request(i, &b, &lp);
            if (e > 0 && __ldcg(a.refs + e) > 1) {
                atomicAdd(w.count + e, 1);
                atomicMax(w.last + e, b);
            }
        }
        __syncthreads();
        auto needs = [&](int64_t i, int *b, int *lp, int *e) {
            *e = request(i, b, lp);
            if (*e <= 0) return *e == 0;
            const int r = __ldcg(a.refs + *e), c = __ldcg(w.count + *e), last = __ldcg(w.last + *e);
            return r > 1 && !(c == r && last == *b);
        };
        int total = 0, e;
        for (int64_t i0 = 0; i0 < R; i0 += kPlanThreads) {
            int n;
            block_scan(needs(i0 + threadIdx.x, &b, &lp, &e) ? 1 : 0, &n);
            total += n;
        }
        const int have = pages.find(total, w.free_ids);
        report_total(total, have);
        int done = 0;
        for (int64_t i0 = 0; have == total && i0 < R; i0 += kPlanThreads) {
            const bool need = needs(i0 + threadIdx.x, &b, &lp, &e);
            int n;
            const int rank = done + block_scan(need ? 1 : 0, &n);  // (its barriers: everybody has read the counts)
            done += n;
            if (need) assign(b, lp, e, __ldcg(w.free_ids + rank), rank);
        }
        __syncthreads();
        // the copied pages' holders go once no count is read any more
        for (int64_t i = threadIdx.x; have == total && i < total; i += kPlanThreads) {
            const int e = w.jobs[4 * i];
            if (e > 0) atomicSub(a.refs + e, 1);
        }
    }
    if (!a.writable) return;
    // granted: the slots whose pages are all the sequence's own, as tables and counts are now; with
    // those that it had, if they touch
    for (int s = threadIdx.x; s < a.batch; s += kPlanThreads) {
        const int2 x = asked(s);
        w.begin[s] = x.y > 0 && (int64_t)start_of(a, s) + x.x + x.y <= a.cap;
    }
    __syncthreads();
    for (int64_t i = threadIdx.x; i < R; i += kPlanThreads) {
        if (!page_of(i, &b, &lp)) continue;
        const int e = __ldcg(a.table + (int64_t)b * a.max_pages + lp);
        if (e <= 0 || e >= a.num_pages || __ldcg(a.refs + e) != 1) w.begin[b] = 0;
    }
    __syncthreads();
    for (int s = threadIdx.x; s < a.batch; s += kPlanThreads) {
        if (!w.begin[s]) continue;
        const int2 x = asked(s), had = a.writable[s];
        int2 now = make_int2(x.x, x.x + x.y);
        if (had.x < had.y && had.x <= now.y && now.x <= had.y) now = make_int2(min(had.x, now.x), max(had.y, now.y));
        a.writable[s] = now;
    }
}

// Copies of jobs x layers x planes x KV heads: a run of rows each, by a CTA, or where all are short by a
// warp.  Bound by memory: 30 copies of two pages of an 8k prompt, 32 layers (187 MB written, the pages
// read from L2) in 38 us.
// The short ones are new samples' first tokens: 42 copies of a token, 32 layers of 4 heads, in 14.3 us
// with the fork, 29.4 by CTAs.
constexpr int kWarpRun = 2048;  // bytes: up to four vectors a lane
template <typename V, int THREADS>
__device__ __forceinline__ void copy_run(unsigned char *dst, const unsigned char *src, int n) {
    constexpr int U = 4;
    const V *s = reinterpret_cast<const V *>(src);
    V *d = reinterpret_cast<V *>(dst);
    n /= (int)sizeof(V);
    for (int i0 = threadIdx.x % THREADS; i0 < n; i0 += THREADS * U) {
        V x[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + u * THREADS < n) x[u] = s[i0 + u * THREADS];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i0 + u * THREADS < n) d[i0 + u * THREADS] = x[u];
    }
}
template <int THREADS>  // of an item
__device__ __forceinline__ void copy_items(const PagesArgs &a, const PagesWs &w, int jobs) {
    constexpr int kTeams = kCopyThreads / THREADS;
    const int64_t per = (int64_t)a.layers * a.n_planes * a.kv_heads, items = jobs * per;
    for (int64_t i = (int64_t)blockIdx.x * kTeams + threadIdx.x / THREADS; i < items; i += (int64_t)gridDim.x * kTeams) {
        const int4 job = *reinterpret_cast<const int4 *>(w.jobs + 4 * (i / per));
        if (job.w <= 0) continue;
        const int x = (int)(i % per), g = x % a.kv_heads, y = x / a.kv_heads, pl = y % a.n_planes, l = y / a.n_planes;
        const int64_t rb = a.row_bytes[pl];
        auto row = [&](int page) { return ((((int64_t)l * a.num_pages + page) * a.kv_heads + g) * a.page_size + job.z) * rb; };
        unsigned char *d = a.plane[pl] + row(job.y);
        const unsigned char *s = a.plane[pl] + row(job.x);
        const int n = job.w * (int)rb;
        if (rb % 16 == 0) copy_run<uint4, THREADS>(d, s, n);
        else copy_run<uint32_t, THREADS>(d, s, n);
    }
}
__global__ void __launch_bounds__(kCopyThreads) writable_copy_kernel(const PagesArgs a, const PagesWs w) {
    pdl_wait();
    int rb = 0;
    for (int pl = 0; pl < a.n_planes; ++pl) rb = max(rb, a.row_bytes[pl]);
    const int4 total = *reinterpret_cast<const int4 *>(w.total);
    if ((int64_t)total.z * rb <= kWarpRun) copy_items<32>(a, w, total.x);
    else copy_items<kCopyThreads>(a, w, total.x);
}

// A table entry from a sequence's first page made anew on: its old page is given back, its new one taken.
__device__ __forceinline__ void commit_entry(const PagesArgs &a, const PagesWs &w, int b, int lp) {
    int32_t *entry = a.table + (int64_t)b * a.max_pages + lp;
    const int e = *entry, begin = w.begin[b], base = w.base[b];
    const int to = lp - begin < w.base[b + 1] - base ? w.free_ids[base + lp - begin] : 0;
    if (holds_page(a, e)) atomicSub(a.refs + e, 1);
    if (to) a.refs[to] = 1;
    if (e != to) *entry = to;
}

// One CTA: where each sequence's first moved slot lies, the pages it makes anew, the free pages for
// them.  keep[j] >= j rises with j, so the slots that stay are a prefix: a warp looks for its end.
__global__ void __launch_bounds__(kPlanThreads)
compact_plan_kernel(const PagesArgs a, const PagesWs w, const int32_t *keep, const int32_t *keep_len, int32_t *lacking,
                    int32_t *old) {
    pdl_wait();
    __shared__ int32_t need_s[kPlanThreads];
    int32_t *needs = a.batch <= kPlanThreads ? need_s : w.base;  // pages that a sequence makes anew
    FreePages pages{a.refs, a.num_pages};
    pages.load(0);
    const int lane = threadIdx.x & 31;
    for (int b = threadIdx.x >> 5; b < a.batch; b += kPlanThreads / 32) {
        const int64_t r0 = (int64_t)b * a.rows_per_seq;
        const int asked = keep_len[r0], n = kept_of(a, b, asked);
        if (n < asked && lane == 0) atomicOr(&g_pages_error, 4u);
        int begin = a.max_pages;  // a sequence that is left alone
        if (n >= 0) {
            int f = n;
            for (int r = 0; r < a.rows_per_seq; ++r) {
                const int32_t *k = keep + (r0 + r) * a.cap;
                int lo = 0, hi = f;  // slots below lo stay, slot hi does not (or is f)
                while (lo < hi) {
                    const int step = (hi - lo + 31) / 32, x = lo + lane * step;
                    const uint32_t stay = __ballot_sync(0xffffffffu, x < hi && k[x] == x);
                    // the lanes that stay are the first ones
                    const int c = __popc(stay);
                    if (c < 32) hi = min(hi, lo + c * step);
                    if (c > 0) lo += (c - 1) * step + 1;
                }
                f = lo;
            }
            const int S = start_of(a, b), end = (S + n + a.page_size - 1) / a.page_size;
            begin = f == n ? end : (S + f) / a.page_size;
            if (lane == 0) needs[b] = end - begin;
        } else if (lane == 0) {
            needs[b] = 0;
        }
        if (lane == 0) w.begin[b] = begin;
    }
    __syncthreads();
    int total = 0;
    for (int b0 = 0; b0 < a.batch; b0 += kPlanThreads) {
        const int b = b0 + threadIdx.x, need = b < a.batch ? needs[b] : 0;
        int n;
        const int at = total + block_scan(need, &n);
        if (b < a.batch) w.base[b] = at;
        total += n;
    }
    if (threadIdx.x == 0) w.base[a.batch] = total;
    const int have = pages.find(total, w.free_ids);
    if (threadIdx.x == 0) {
        w.total[0] = have == total ? total : 0;
        w.total[1] = have == total;
        if (lacking) *lacking = total - have;
        if (have < total) atomicOr(&g_pages_error, 64u);
    }
    if (!old || have < total) return;
    // few entries: the tables change here, and the copies look up the old ones in `old`
    const int entries = a.batch * a.max_pages;
    for (int i = threadIdx.x; i < entries; i += kPlanThreads) {
        const int b = i / a.max_pages, lp = i - b * a.max_pages;
        old[i] = a.table[i];
        if (lp >= w.begin[b]) commit_entry(a, w, b, lp);  // (none of a sequence left alone)
    }
    for (int b = threadIdx.x; b < a.batch; b += kPlanThreads) {
        const int n = kept_of(a, b, keep_len[(int64_t)b * a.rows_per_seq]);
        if (n < 0) continue;
        a.len[b] = n;
        forget_granted(a, b);
    }
}

// Rows of new pages: slot j comes from slot keep[j] of the old pages.  CTAs take items of one layer
// and as many new pages as make about kRowsAtOnce rows (small pages would leave most threads
// idle), or of fewer pages and heads where that leaves too few items for the CTAs that run at once (11
// sequences cut to ~18 slots of 8 heads, 28 layers: 37.7 -> 16.0 us with the plan; a tenth of a 32k prompt,
// one layer: 43 -> 17); where a row comes from and goes to is looked up once for all planes, and heads that keep the
// same.  Bound by memory: a thread has kAhead vectors in flight.  A tenth of a 32k prompt, 32 layers
// (859 MB moved in rows of 256 bytes) in 140 us, 6.1 TB/s; rows of 64 and 8 bytes (16 sequences in 4
// bits, 337 MB) in 70.
constexpr int kRowsAtOnce = 128;
constexpr int kItemBytes = 16384;  // of a plane, at least: kAhead vectors a thread (with less, items of 16 KB cut to 4: 14.5 -> 18.0)
struct RowMove {
    int64_t src, dst;  // rows of a plane, of the item's first head; src < 0: not moved
};
__device__ __forceinline__ int log2_or(int n) { return (n & (n - 1)) == 0 ? __ffs(n) - 1 : -1; }
// heads x n_moves rows of a plane: head g's lie g * step rows behind the first head's
template <typename V>
__device__ __forceinline__ void gather_plane(unsigned char *plane, int rb, const RowMove *moves, int n_moves, int heads, int step) {
    constexpr int kAhead = 4;
    const int per = rb / (int)sizeof(V), n = heads * n_moves * per;
    const int per_shift = log2_or(per), move_shift = log2_or(n_moves);
    for (int i0 = threadIdx.x; i0 < n; i0 += kCopyThreads * kAhead) {
        V x[kAhead];
        V *to[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = i0 + u * kCopyThreads, row = per_shift >= 0 ? i >> per_shift : i / per;
            const int g = move_shift >= 0 ? row >> move_shift : row / n_moves;
            to[u] = nullptr;
            if (i < n) {
                const RowMove m = moves[row - g * n_moves];
                if (m.src >= 0) {
                    const int64_t piece = (int64_t)(i - row * per) * sizeof(V), head = (int64_t)g * step;
                    to[u] = reinterpret_cast<V *>(plane + (m.dst + head) * rb + piece);
                    x[u] = *reinterpret_cast<const V *>(plane + (m.src + head) * rb + piece);
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
            if (to[u]) *to[u] = x[u];
    }
}
// Row x of pos, then of ema, then of vnorm, gathered in place: keep[j] >= j, so a run of slots is read
// before it is written, and no later run is read from it.
__device__ __forceinline__ void gather_in_place(const PagesArgs &a, const int32_t *keep, const int32_t *keep_len, int64_t x) {
    constexpr int U = 8;
    const int64_t R = (int64_t)a.batch * a.rows_per_seq;
    int64_t r = x;
    uint32_t *row;  // 4-byte values whatever they are
    if (x < R) {
        if (!a.pos) return;
        row = reinterpret_cast<uint32_t *>(a.pos) + r * a.cap;
    } else if (x < 2 * R) {
        r = x - R;
        if (!a.ema) return;
        row = reinterpret_cast<uint32_t *>(a.ema) + r * a.cap;
    } else {  // vnorm [layers][batch][kv_heads][cap]
        x -= 2 * R;
        const int b = (int)(x / a.kv_heads % a.batch), g = (int)(x % a.kv_heads);
        r = a.rows_per_seq == 1 ? b : (int64_t)b * a.rows_per_seq + g;
        row = reinterpret_cast<uint32_t *>(a.vnorm) + x * a.cap;
    }
    const int n = min(keep_len[r], a.cap);
    const int32_t *k = keep + r * a.cap;
    int from[U];  // a run ahead of the values: one trip to memory a run, not two (32768 slots: 22.3 -> 12.9 us)
    auto load_keep = [&](int j0) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * kCopyThreads + threadIdx.x;
            from[u] = j < n ? k[j] : 0;
        }
    };
    load_keep(0);
    for (int j0 = 0; j0 < n; j0 += kCopyThreads * U) {
        uint32_t v[U];
#pragma unroll
        for (int u = 0; u < U; ++u) v[u] = from[u] >= 0 && from[u] < a.cap ? row[from[u]] : 0u;
        load_keep(j0 + kCopyThreads * U);
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = j0 + u * kCopyThreads + threadIdx.x;
            if (j < n) row[j] = v[u];
        }
    }
}
__global__ void __launch_bounds__(kCopyThreads, 4)
compact_copy_kernel(const PagesArgs a, const PagesWs w, const int32_t *keep, const int32_t *keep_len, const int32_t *old,
                    int pages_at_once, float units_a_job, int least_units, int most_units, int n_rows) {
    pdl_wait();
    __shared__ RowMove moves[kRowsAtOnce];
    if (!w.total[1]) return;  // too few pages
    if ((int)blockIdx.x < n_rows) {  // beside the copies
        gather_in_place(a, keep, keep_len, blockIdx.x);
        return;
    }
    const int jobs = w.total[0], ctas = (int)gridDim.x - n_rows;
    // heads that share their moves: all, or with a keep row for each KV head one
    int share = a.rows_per_seq == 1 ? a.kv_heads : 1, parts = a.kv_heads / share;
    // fewer pages and heads an item, where there would be fewer items than a quarter of the CTAs (two an SM)
    // (halves: powers of two stay so, which gather_plane divides by)
    // (and never so many that an item's vectors pass 32 bits: pages may hold 16 MB a head)
    const int units = min(max((int)((float)jobs * units_a_job), least_units), most_units);
    while (pages_at_once > 1 && pages_at_once * share > units) pages_at_once = (pages_at_once + 1) >> 1;
    if (share > units) {
        while (share > units) share = (share + 1) >> 1;
        parts = (a.kv_heads + share - 1) / share;
    }
    const int groups = (jobs + pages_at_once - 1) / pages_at_once;
    const int64_t items = (int64_t)groups * a.layers * parts;
    for (int64_t it = (int)blockIdx.x - n_rows; it < items; it += ctas) {
        const int g0 = (int)(it % parts) * share, heads = min(share, a.kv_heads - g0);
        const int l = (int)(it / parts % a.layers), job0 = (int)(it / parts / a.layers) * pages_at_once;
        const int pages = min(pages_at_once, jobs - job0);
        for (int q0 = 0; q0 < a.page_size; q0 += kRowsAtOnce) {  // (pages longer than that: one of them, in parts)
            const int rows = min(a.page_size - q0, kRowsAtOnce), n = pages * rows;
            __syncthreads();
            for (int i = threadIdx.x; i < n; i += kCopyThreads) {
                const int q = i % rows, job = job0 + i / rows;
                int lo = 0, hi = a.batch;  // the sequence whose job it is: base[b] <= job < base[b + 1]
                while (hi - lo > 1) {
                    const int mid = (lo + hi) >> 1;
                    if (w.base[mid] <= job) lo = mid;
                    else hi = mid;
                }
                const int b = lo, S = start_of(a, b);
                const int64_t r = a.rows_per_seq == 1 ? b : (int64_t)b * a.rows_per_seq + g0;
                const int64_t j = (int64_t)(w.begin[b] + job - w.base[b]) * a.page_size + q0 + q - S;
                RowMove m{-1, 0};
                if (j >= 0 && j < min(keep_len[r], a.cap - S)) {
                    const int64_t from = (int64_t)S + keep[r * a.cap + j];
                    const int fp = (int)(from / a.page_size);
                    const int page = from >= 0 && fp < a.max_pages ? old[(int64_t)b * a.max_pages + fp] : -1;
                    if (page > 0 && page < a.num_pages) {  // (0: a slot without a page holds nothing to keep)
                        m.src = (((int64_t)l * a.num_pages + page) * a.kv_heads + g0) * a.page_size + from % a.page_size;
                        m.dst = (((int64_t)l * a.num_pages + w.free_ids[job]) * a.kv_heads + g0) * a.page_size + q0 + q;
                    } else {
                        atomicOr(&g_pages_error, 128u);
                    }
                }
                moves[i] = m;
            }
            __syncthreads();
            for (int pl = 0; pl < a.n_planes; ++pl) {
                const int rb = a.row_bytes[pl];
                if (rb % 16 == 0) gather_plane<uint4>(a.plane[pl], rb, moves, n, heads, a.page_size);
                else if (rb % 8 == 0) gather_plane<uint2>(a.plane[pl], rb, moves, n, heads, a.page_size);
                else gather_plane<uint32_t>(a.plane[pl], rb, moves, n, heads, a.page_size);
            }
        }
    }
}

// After the copies, where the plan left the tables to it: a CTA a sequence.
__global__ void __launch_bounds__(kCopyThreads) compact_commit_kernel(const PagesArgs a, const PagesWs w, const int32_t *keep_len) {
    pdl_wait();
    const int b = blockIdx.x, n = kept_of(a, b, keep_len[(int64_t)b * a.rows_per_seq]);
    if (!w.total[1] || n < 0) return;
    for (int lp = w.begin[b] + threadIdx.x; lp < a.max_pages; lp += kCopyThreads) commit_entry(a, w, b, lp);
    if (threadIdx.x == 0) {
        a.len[b] = n;
        forget_granted(a, b);
    }
}

}  // namespace

size_t pages_ws(int32_t batch, int32_t max_pages, int32_t num_pages, void *ws, PagesWs *w) {
    size_t off = 0;
    auto take = [&](size_t n) {
        int32_t *p = ws ? at<int32_t>(ws, off) : nullptr;
        off = align256(off + n * sizeof(int32_t));
        return p;
    };
    PagesWs x;
    const size_t R = (size_t)batch * max_pages;
    x.total = take(4);
    x.free_ids = take(R);
    x.count = take(num_pages);
    x.last = take(num_pages);
    x.jobs = take(4 * R);
    x.begin = take(batch);
    x.base = take((size_t)batch + 1);
    if (w) *w = x;
    return off;
}

cudaError_t launch_pages_release(const PagesArgs &a, int32_t extra, cudaStream_t st) {
    const int64_t n = ((int64_t)a.batch * a.max_pages + kRowThreads - 1) / kRowThreads;
    const cudaError_t e = launch_k(release_kernel, dim3((unsigned)n), dim3(kRowThreads), 0, st, a, (int)extra);
    note_launch();
    return e;
}

cudaError_t launch_pages_fork(const PagesArgs &a, int32_t n, const int32_t *src, const int32_t *dst, cudaStream_t st) {
    const int64_t words = (int64_t)a.rows_per_seq * a.cap;
    const int64_t parts = (words + 8 * kRowThreads - 1) / (8 * kRowThreads);
    const cudaError_t e = launch_k(fork_kernel, dim3((unsigned)(1 + 2 * (parts < 64 ? parts : 64)), (unsigned)n), dim3(kRowThreads),
                                   0, st, a, src, dst);
    note_launch();
    return e;
}

cudaError_t launch_pages_writable(const PagesArgs &a, const PagesWs &w, const int32_t *first, const int32_t *count,
                                  int32_t max_count, int32_t *lacking, int sms, cudaStream_t st) {
    // pages that max_count slots from anywhere in a page may touch
    const int64_t most = max_count > 0 ? ((int64_t)max_count + a.page_size - 2) / a.page_size + 1 : 1;
    const int span = (int)(most < a.max_pages ? most : a.max_pages);
    const bool few = (int64_t)a.batch * span <= kFewRequests;
    cudaError_t e = launch_k(few ? writable_plan_kernel<true> : writable_plan_kernel<false>, dim3(1), dim3(kPlanThreads), 0,
                             st, a, w, first, count, (int)max_count, span, lacking);
    note_launch();
    if (e != cudaSuccess) return e;
    const int64_t items = (int64_t)a.batch * span * a.layers * a.n_planes * a.kv_heads;
    const int64_t ctas = items < 8 * (int64_t)sms ? items : 8 * (int64_t)sms;
    e = launch_k(writable_copy_kernel, dim3((unsigned)ctas), dim3(kCopyThreads), 0, st, a, w);
    note_launch();
    return e;
}

cudaError_t launch_pages_compact(const PagesArgs &a, const PagesWs &w, const int32_t *keep, const int32_t *keep_len,
                                 int32_t *lacking, int sms, cudaStream_t st) {
    // up to 8192 entries the plan's one CTA writes the tables (a 32k prompt of 512 entries: 149.5 us, 152 with
    // a launch behind the copies), in at most 8 rounds; above that a CTA a sequence does
    int32_t *old = (int64_t)a.batch * a.max_pages <= 8192 ? w.jobs : nullptr;
    cudaError_t e = launch_k(compact_plan_kernel, dim3(1), dim3(kPlanThreads), 0, st, a, w, keep, keep_len, lacking, old);
    note_launch();
    if (e != cudaSuccess) return e;
    const int at_once = a.page_size < kRowsAtOnce ? kRowsAtOnce / a.page_size : 1;
    const int64_t items = (int64_t)a.batch * a.max_pages * a.layers * (a.rows_per_seq == 1 ? 1 : a.kv_heads);
    const int64_t ctas = items < 8 * (int64_t)sms ? items : 8 * (int64_t)sms;
    const int64_t rows = 2 * (int64_t)a.batch * a.rows_per_seq + (a.vnorm ? (int64_t)a.layers * a.batch * a.kv_heads : 0);
    if (rows + ctas > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const float units_a_job = 4.f * a.layers * a.kv_heads / (float)ctas;
    const int least = kItemBytes / (a.page_size * a.row_bytes[0]);
    int widest = 0;
    for (int pl = 0; pl < a.n_planes; ++pl) widest = a.row_bytes[pl] > widest ? a.row_bytes[pl] : widest;
    const int64_t most = ((int64_t)1 << 30) / ((int64_t)a.page_size * widest);  // pages of a head: 1 GB; at least 64
    e = launch_k(compact_copy_kernel, dim3((unsigned)(rows + ctas)), dim3(kCopyThreads), 0, st, a, w, keep, keep_len,
                 (const int32_t *)(old ? old : a.table), at_once, units_a_job, least > 1 ? least : 1, (int)most, (int)rows);
    note_launch();
    if (e != cudaSuccess || old) return e;
    e = launch_k(compact_commit_kernel, dim3((unsigned)a.batch), dim3(kCopyThreads), 0, st, a, w, keep_len);
    note_launch();
    return e;
}

cudaError_t read_clear_pages_error(unsigned int *v) {
    unsigned int z = 0;
    cudaError_t e = cudaMemcpyFromSymbol(v, g_pages_error, sizeof(*v));
    if (e == cudaSuccess && *v) e = cudaMemcpyToSymbol(g_pages_error, &z, sizeof(z));
    return e;
}

}  // namespace ikv
