// The score pass of the shared-prefix decode on the tensor cores (bf16): K is read once more, with each row's
// maximum M and sum of weights W known from the merge,
//     score[b][j] = mean over the row's heads of 2^(q . k_j scale - M) / W.
// The scores' own products are the attention's bit for bit, so what W is off by is common to numerator and sum.
// Writing the logits instead costs 8 bytes a (row, slot), more than K from 32 rows on.
//
// S^T = K Q^T with the 128 slots of a tile in the M dimension: a thread holds a slot, and the query heads that
// it averages over are columns of its TMEM lane, so the sum over heads needs no exchange and has a fixed order.
// An item is a tile for up to 128 rows; averaging over all heads goes through the KV heads in turn with the sums
// of up to 64 members (16 at G = 4) in a thread's registers.
//
// Warps: 0-3 columns 0-63, 4-7 columns 64-127 of S^T; 8 TMA (K), 9 MMA, 10-11 Q.  K and Q pass through a ring of
// three stages, S^T through two halves of tensor memory.
//
// Measured: two prefixes of 8k for 16 sequences each, 32 / 8 heads of 128, mean over all 32: 23 us, of
// which K's 82 MB out of HBM take 12; 305 items are dealt to 152 CTAs by threes, so that 50 have none.
#include "rows_tc.cuh"

namespace ikv {
namespace {

constexpr int kThreads = 384;

template <int D>
struct Sc {
    static constexpr int kTile = kAtom * (D / 64);  // bytes of K, of Q
    static constexpr int kStages = 3;
    static constexpr int kOffNorm = kStages * 2 * kTile;  // (M, 1 / W) of a product's rows
    static constexpr int kNorms = 8;  // Q may be three products ahead of the products, and they two ahead of the weights
    static constexpr int kOffBar = kOffNorm + kNorms * 128 * 8;
    static constexpr int kBars = 3 * kStages + 6 + kNorms;
    static constexpr int kOffMisc = kOffBar + kBars * 8;
    static constexpr int kSmem = kOffMisc + 16 + 1024;
};

struct Item {
    RowsUnit u;
    int m0, n, t0, g0, gs;  // members, first slot, KV heads
};

// A CTA's items, in turn
struct Items {
    int unit, sub, j, left;
    __device__ __forceinline__ void begin(const RowsArgs &a) {
        const int4 s = __ldcg(reinterpret_cast<const int4 *>(a.items) + blockIdx.x);
        unit = s.x;
        sub = s.y;
        j = s.z;
        left = s.w;
    }
    __device__ __forceinline__ Item item(const RowsArgs &a) const {
        Item t;
        t.u = rows_unit(a, unit);
        t.m0 = sub / a.item_subs * a.item_n;
        t.n = min(a.item_n, t.u.n - t.m0);
        t.t0 = rows_tile(t.u, j) * kRowsTile;
        t.g0 = a.item_subs > 1 ? sub % a.item_subs : 0;
        t.gs = a.item_subs > 1 ? 1 : a.pv.kv_heads;
        return t;
    }
    __device__ __forceinline__ void next(const RowsArgs &a, const RowsUnit &u) {
        --left;
        if (++j < u.nt) return;
        j = 0;
        if (++sub < a.item_subs * ((u.n + a.item_n - 1) / a.item_n)) return;
        sub = 0;
        ++unit;
    }
};

__device__ __forceinline__ int member_of(const RowsArgs &a, const RowsUnit &u, int m) {
    return u.m0 >= 0 ? __ldcg(a.vm + u.m0 + m) : u.b;
}

template <int D, int G>
__global__ void __launch_bounds__(kThreads, 1)
    rows_score_tc_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ RowsArgs a, const TcMap tm,
                         const RowsScoreArgs sc) {
    using C = Sc<D>;
    using T = __nv_bfloat16;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t raw = smem_u32(smem_raw), base = (raw + 1023u) & ~1023u;
    unsigned char *sm = smem_raw + (base - raw);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t bar0 = base + C::kOffBar;
    auto k_full = [&](int i) { return bar0 + 8u * i; };
    auto q_full = [&](int i) { return bar0 + 8u * (C::kStages + i); };
    auto empty = [&](int i) { return bar0 + 8u * (2 * C::kStages + i); };  // K's and Q's stage
    const uint32_t bar1 = bar0 + 8u * (3 * C::kStages);
    auto s_full = [&](int x) { return bar1 + 8u * x; };
    auto s_empty = [&](int x) { return bar1 + 16u + 8u * x; };
    const uint32_t mma_done = bar1 + 32u;
    auto n_full = [&](int i) { return bar1 + 40u + 8u * i; };  // a product's norms
    const uint32_t stall_bar = n_full(C::kNorms);  // nothing arrives here
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(sm + C::kOffMisc);
    volatile int *abort_flag = reinterpret_cast<volatile int *>(sm + C::kOffMisc + 4);
    if (warp == 8 && lane == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            mbar_init(k_full(i), 1);
            mbar_init(q_full(i), 64);
            mbar_init(empty(i), 1);
        }
        for (int x = 0; x < 2; ++x) {
            mbar_init(s_full(x), 1);
            mbar_init(s_empty(x), 256);
        }
        for (int i = 0; i < C::kNorms; ++i) mbar_init(n_full(i), 64);
        mbar_init(mma_done, 1);
        mbar_init(stall_bar, 1);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 256;" ::"r"(smem_u32(tmem_slot))
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    fence_before_sync();
    __syncthreads();
    fence_after_sync();
    const uint32_t tmem = *tmem_slot;
    Items w;
    w.begin(a);
    if (__ldcg(&a.head->failed)) w.left = 0;  // no norms
    int J = 0;  // (item, KV head) products so far: stage J % kStages, half J % 2 of tensor memory
    if (warp == 8) {
        // ---------------- K
        bool ok = true;
        const int boxes = kRowsTile / tm.rows_per_box;
        for (; w.left > 0 && ok;) {
            const Item t = w.item(a);
            const int s0 = t.t0 + lane * tm.rows_per_box;
            const bool need = lane < boxes && s0 < t.u.hi && s0 + tm.rows_per_box > t.u.lo;
            int row = need ? pool_row(a, t.u.b, t.g0, s0) : tm.pool_rows;
            for (int g = 0; g < t.gs && ok; ++g, ++J) {
                const int st = J % C::kStages;
                if (lane == 0) {
                    if (J >= C::kStages) ok = bar_wait(empty(st), (J / C::kStages - 1) & 1, abort_flag);
                    if (ok) mbar_expect_tx(k_full(st), C::kTile);
                }
                ok = __shfl_sync(0xffffffffu, ok, 0);
                if (!ok) break;
                if (lane < boxes) tma_rows(base + st * 2 * C::kTile + lane * tm.rows_per_box * (2 * D), &tmK, row, k_full(st));
                if (need) row += a.pv.page_size;  // (the next KV head's)
            }
            w.next(a, t.u);
        }
        if (lane == 0)
            for (int i = J - 1; i >= 0 && i >= J - C::kStages; --i) bar_drain(k_full(i % C::kStages), (i / C::kStages) & 1);
        __syncwarp();
    } else if (warp == 9) {
        // ---------------- products
        const bool leader = elect_one();
        bool ok = true;
        const uint64_t dk0 = sdesc(base, 16, 16 * D), dq0 = sdesc(base + C::kTile, 16, 1024);
        for (; w.left > 0 && ok;) {
            const Item t = w.item(a);
            const int half = 64 / G;
            const int cols = __shfl_sync(0xffffffffu, t.n > half ? 64 + ((t.n - half) * G + 15) / 16 * 16 : (t.n * G + 15) / 16 * 16, 0), gs = __shfl_sync(0xffffffffu, t.gs, 0);
            const uint32_t id = idesc_bf16(false, 128, cols);
            for (int g = 0; g < gs && ok; ++g, ++J) {
                const int st = J % C::kStages, x = J & 1;
                ok = warp_wait(k_full(st), (J / C::kStages) & 1, abort_flag) &&
                     warp_wait(q_full(st), (J / C::kStages) & 1, abort_flag) &&
                     (J < 2 || warp_wait(s_empty(x), (J / 2 - 1) & 1, abort_flag));
                if (tm.stall && J == 1)  // runs out, within an item that averages over KV heads
                    ok = __all_sync(0xffffffffu, bar_wait_long(stall_bar, 0, abort_flag, kStallNs));
                if (!ok) break;
                fence_async_smem();  // (Q came by plain copies)
                fence_after_sync();
                const uint64_t dk = dk0 + st * (2 * C::kTile >> 4), dq = dq0 + st * (2 * C::kTile >> 4);
                if (leader) {
#pragma unroll
                    for (int kk = 0; kk < D / 16; ++kk) {
                        const uint32_t c = (kk & 3) * 32;
                        mma_bf16(tmem + 128 * x, dk + (((kk >> 2) * kBlock + c) >> 4), dq + (((kk >> 2) * kAtom + c) >> 4), id,
                                 kk > 0);
                    }
                    mma_commit(s_full(x));
                    mma_commit(empty(st));
                }
                __syncwarp();
            }
            w.next(a, t.u);
        }
        if (leader) mma_commit(mma_done);
        __syncwarp();
        bar_drain(mma_done, 0);
    } else if (warp >= 10) {
        // ---------------- Q, four lanes a row, and the rows' norms.  The copies report to the stage's barrier
        // themselves, so that the next stage's go out at once: waiting for each took 2 us a product.
        const int th = tid - 320, c = th & 3;
        constexpr int kHalf = 64 / G, kRows = 8;  // rows a thread: th / 4 + 16 i
        bool ok = true;
        for (; w.left > 0 && ok;) {
            const Item t = w.item(a);
            const int rows = t.n * G;
            int64_t row[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const int x = th / 4 + 16 * i, b = x < rows ? member_of(a, t.u, t.m0 + x / G) : -1;
                row[i] = b >= 0 ? (int64_t)b * a.q_heads + t.g0 * G + x % G : -1;
            }
            for (int g = 0; g < t.gs && ok; ++g, ++J) {
                const int st = J % C::kStages;
                if (J >= C::kStages) ok = bar_wait(empty(st), (J / C::kStages - 1) & 1, abort_flag);
                if (!ok) break;
                const uint32_t dst0 = base + st * 2 * C::kTile + C::kTile, norm = base + C::kOffNorm + J % C::kNorms * 128 * 8;
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const int x = th / 4 + 16 * i;
                    if (x >= rows) break;
                    const int r = x < kHalf * G ? x : x - kHalf * G + 64;  // its column of S^T
                    const bool real = row[i] >= 0;
                    const int64_t at = real ? row[i] + g * G : 0;
                    const T *src = static_cast<const T *>(a.q) + at * D + 8 * c;
#pragma unroll
                    for (int k = 0; k < D / 32; ++k)
                        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                                         dst0 + (k >> 1) * kAtom + r * 128 + ((((c + 4 * k) ^ r) & 7) << 4)),
                                     "l"(src + 32 * k), "r"(real ? 16 : 0)
                                     : "memory");
                    if (c == 0)
                        asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(norm + 8 * r), "l"(a.norm + at),
                                     "r"(real ? 8 : 0)
                                     : "memory");
                }
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(q_full(st)) : "memory");
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(n_full(J % C::kNorms)) : "memory");
            }
            w.next(a, t.u);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else {
        // ---------------- weights: a thread a slot, half of the columns
        constexpr int kMembers = 64 / G;  // of a thread's 64 columns; G = 7 uses 63
        constexpr int kBlockM = kMembers < 8 ? kMembers : 8;
        const int half = warp >> 2;
        const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
        const int rps = a.rows_per_seq;
        bool ok = true;
        for (; w.left > 0;) {
            const Item t = w.item(a);
            const int slot = t.t0 + (warp & 3) * 32 + lane, m1 = half * kMembers;
            const int mine = min(max(t.n - m1, 0), kMembers);  // members of this half
            // (looked up ahead, a lane a member, and so are their slots' liveness and old utilities below: between the
            // stores each would wait for memory by itself)
            int who[(kMembers + 31) / 32];
#pragma unroll
            for (int k = 0; k < (kMembers + 31) / 32; ++k)
                who[k] = lane + 32 * k < mine ? member_of(a, t.u, t.m0 + m1 + lane + 32 * k) : -1;
            const bool inside = ok && slot >= t.u.lo && slot < t.u.hi;
            const int j = slot - t.u.S0;
            const float inv = 1.f / (float)(rps == 1 ? a.q_heads : G);
            float sum[kMembers];
#pragma unroll
            for (int m = 0; m < kMembers; ++m) sum[m] = 0.f;
            for (int g = 0; g < t.gs; ++g, ++J) {
                const int x = J & 1;
                const bool out = rps > 1 || g == t.gs - 1;  // the sums are complete behind this product
                uint64_t dead = 0;
                if (out && a.live) {
#pragma unroll
                    for (int m = 0; m < kMembers; ++m) {
                        const int b = __shfl_sync(0xffffffffu, who[m / 32], m % 32);
                        if (inside && b >= 0 &&
                            !((__ldcg(a.live + ((int64_t)b * rps + (rps > 1 ? t.g0 + g : 0)) * a.live_words + (j >> 5)) >> (j & 31)) & 1u))
                            dead |= 1ull << m;
                        if (m % kBlockM == kBlockM - 1 && m + 1 >= mine) break;
                    }
                }
                // (not Q's stage, which may be full again by now)
                if (ok) ok = bar_wait(n_full(J % C::kNorms), (J / C::kNorms) & 1, abort_flag);
                if (ok) ok = bar_wait(s_full(x), (J / 2) & 1, abort_flag);
                ok = __all_sync(0xffffffffu, ok);
                fence_after_sync();
                const float2 *norm = reinterpret_cast<const float2 *>(sm + C::kOffNorm) + J % C::kNorms * 128 + 64 * half;
                if (ok && mine > 0) {
                    uint32_t v[64];
                    const uint32_t at = tmem + 128 * x + lane_off + 64 * half;
                    tmem_ld32(at, v);
                    if (mine * G > 32) tmem_ld32(at + 32, v + 32);
                    tmem_wait_ld(v);
                    if (mine * G > 32) tmem_wait_ld(v + 32);
                    // (a block of members at once, those that are not there too: a branch for each would put their
                    // look-ups and exponentials one behind another)
#pragma unroll
                    for (int m0 = 0; m0 < kMembers; m0 += kBlockM)
                        if (m0 < mine) {
#pragma unroll
                            for (int m = m0; m < m0 + kBlockM && m < kMembers; ++m) {
                                float w4 = 0.f;
#pragma unroll
                                for (int h = 0; h < G; ++h) {
                                    const float2 mw = norm[m * G + h];
                                    w4 = __fmaf_rn(ex2(__fmaf_rn(__uint_as_float(v[m * G + h]), a.scale_log2, -mw.x)), mw.y, w4);
                                }
                                sum[m] += w4;
                            }
                        }
                }
                fence_before_sync();
                mbar_arrive(s_empty(x));
                if (out && ok) {  // (after a wait that ran out the sums are not whole: score and ema stay as they are)
#pragma unroll
                    for (int m0 = 0; m0 < kMembers; m0 += kBlockM) {
                        if (m0 >= mine) continue;
                        int64_t at[kBlockM];
                        float old[kBlockM];
#pragma unroll
                        for (int k = 0; k < kBlockM; ++k) {
                            const int m = m0 + k < kMembers ? m0 + k : 0;
                            const int b = __shfl_sync(0xffffffffu, who[m / 32], m % 32);  // (-1 where m >= mine)
                            at[k] = m0 + k < kMembers && b >= 0 && inside
                                        ? ((int64_t)b * rps + (rps > 1 ? t.g0 + g : 0)) * a.cap + j
                                        : -1;
                            if (sc.ema && at[k] >= 0) old[k] = sc.ema[at[k]];
                        }
#pragma unroll
                        for (int k = 0; k < kBlockM; ++k) {
                            const int m = m0 + k < kMembers ? m0 + k : 0;
                            if (at[k] >= 0) {
                                const float s = (dead >> m) & 1ull ? 0.f : sum[m] * inv;
                                if (sc.score) sc.score[at[k]] = s;
                                if (sc.ema) sc.ema[at[k]] = sc.alpha * old[k] + (1.f - sc.alpha) * s;
                            }
                            if (m0 + k < kMembers) sum[m] = 0.f;
                        }
                    }
                }
            }
            w.next(a, t.u);
        }
    }
    fence_before_sync();
    __syncthreads();
    if (warp == 9) {
        fence_after_sync();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 256;" ::"r"(tmem) : "memory");
    }
}

template <int D, int G>
cudaError_t launch_dg(const RowsArgs &a, const RowsScoreArgs &s, cudaStream_t st) {
    TcMap t;
    CUtensorMap mk;
    if (!layer_map(&mk, a.k, a, D, &t)) return cudaErrorInvalidValue;
    t.stall = g_stall_next_score.exchange(0);
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = allow_smem(rows_score_tc_kernel<D, G>, Sc<D>::kSmem, done);
    if (e != cudaSuccess) return e;
    return launch_k(rows_score_tc_kernel<D, G>, dim3(a.ctas), dim3(kThreads), Sc<D>::kSmem, st, mk, a, t, s);
}
template <int D>
cudaError_t launch_d(const RowsArgs &a, const RowsScoreArgs &s, cudaStream_t st) {
    switch (a.group) {
        case 1: return launch_dg<D, 1>(a, s, st);
        case 2: return launch_dg<D, 2>(a, s, st);
        case 4: return launch_dg<D, 4>(a, s, st);
        case 7: return launch_dg<D, 7>(a, s, st);
        case 8: return launch_dg<D, 8>(a, s, st);
        default: return cudaErrorInvalidValue;
    }
}

}  // namespace

cudaError_t launch_rows_score_tc(const RowsArgs &a, const RowsScoreArgs &s, int head_dim, cudaStream_t st) {
    const cudaError_t e = head_dim == 64 ? launch_d<64>(a, s, st) : launch_d<128>(a, s, st);
    note_launch();
    return e;
}

cudaError_t read_clear_rows_score_error(unsigned int *v) { return read_clear_timeout(v); }

}  // namespace ikv
