// Merges the parts of packed-row attentions (rows.cuh): with (m_i, l_i, O_i) of each part of a row,
//     M = max m_i, out = (sum 2^(m_i - M) O_i) / (sum 2^(m_i - M) l_i).
// A CTA merges up to 8 rows of one pair.  Window: only the pairs that a share's border cuts have parts, and
// each border's CTA finds its own.  Prefix: every row has parts, of its group's pair and of its own.
// Latency is what it costs, 3 us for a few parts a row: the first parts' outputs are loaded before their weights are
// known, and every thread looks its row's weights up itself.
#include "rows_redo.cuh"

namespace ikv {
namespace {

constexpr int kMergeRows = 8;

__device__ __forceinline__ RowsHead rows_head(const RowsArgs &a) {
    RowsHead h;
    *reinterpret_cast<int4 *>(&h) = __ldcg(reinterpret_cast<const int4 *>(a.head));
    return h;
}
// (a division of 64 bits takes longer than a look-up in memory)
__device__ __forceinline__ int64_t divide(int64_t x, int64_t y) {
    return (x | y) >> 31 ? x / y : (int64_t)((uint32_t)x / (uint32_t)y);
}

// n parts that lie one behind another: (max, sum) of row r of part i at ml[i * sm + r], channels 4 c .. of it at
// o[i * so + c * step + 4 r]
struct Run {
    const float2 *ml;
    const float *o;
    int n, sm, so, step;
    __device__ __forceinline__ float2 sum(int i, int r) const { return __ldcg(ml + (int64_t)i * sm + r); }
    __device__ __forceinline__ float4 out(int i, int r, int c) const {
        return __ldcg(reinterpret_cast<const float4 *>(o + (int64_t)i * so + (c * step + 4 * r)));
    }
};

// The parts of x, then those of y, of up to 8 rows: a thread four channels of a row (2 D threads), kAhead parts at a
// time.  Every thread looks up its row's maxima and sums itself, so that they come with the outputs and nothing is
// exchanged.  done(r, M, 1 / W): row r's maximum and sum, out(r): its output.
template <int D, typename T, int kAhead, typename Done, typename Out>
__device__ __forceinline__ void merge_rows(const Run &x, const Run &y, int rows, Done done, Out out) {
    const int row = threadIdx.x % kMergeRows, chunk = threadIdx.x / kMergeRows, n = x.n + y.n;
    if (row >= rows) return;
    float M = -INFINITY, W = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i0 = 0; i0 < n; i0 += kAhead) {
        float2 s[kAhead];
        float4 v[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            s[i] = make_float2(-INFINITY, 0.f);
            v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i0 + i < n) {
                const bool in_x = i0 + i < x.n;
                const Run &z = in_x ? x : y;
                const int k = in_x ? i0 + i : i0 + i - x.n;
                s[i] = z.sum(k, row);
                v[i] = z.out(k, row, chunk);
            }
        }
        float top = M;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) top = fmaxf(top, s[i].x);
        const float ref = top == -INFINITY ? 0.f : top, f = exp2f(M - ref);
        M = top;
        W *= f;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] *= f;
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const float w = exp2f(s[i].x - ref);
            W += s[i].y * w;
            acc[0] += v[i].x * w;
            acc[1] += v[i].y * w;
            acc[2] += v[i].z * w;
            acc[3] += v[i].w * w;
        }
    }
    const float inv = W == 0.f ? 0.f : 1.f / W;  // (a NaN sum leaves NaN)
    if (inv == 0.f) acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
    store4(out(row) + 4 * chunk, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
    if (chunk == 0) done(row, M == -INFINITY ? 0.f : M, inv);
}

// Grid: (CTAs of the attention, row blocks).  CTA c: the pair that the border in front of share c cuts,
// if no earlier border cuts it.
// kAhead: parts in flight.  2 for prompts, whose pairs have rarely more and many rows (37 us after a prompt of 8k with
// 8, for want of resident CTAs, 20 with 2), 8 for few rows, split over many shares.  A call of 4 sequences with 4k slots,
// by tokens a sequence at 32 / 8 heads, 2 / 8 in flight: 1 token 24.9 / 23.9 us, 16 (64 rows) 31.5 / 30.6, 64 (256 rows,
// one unit) 54.2 / 52.8, 256 (four units) 81.8 / 88.9.
template <int D, typename T, int kAhead>
__global__ void __launch_bounds__(2 * D, (kAhead == 2 ? 1280 : 768) / (2 * D)) rows_merge_window_kernel(const RowsArgs a) {
    pdl_wait();
    const int c = blockIdx.x;
    RowsWalk w;
    w.begin(__ldcg(reinterpret_cast<const int4 *>(a.start + c)));
    if (w.left == 0 || w.at == 0) return;
    const RowsHead head = rows_head(a);
    if (head.failed) return;
    const int64_t per = head.per;
    const RowsUnit u = rows_unit(a, w.unit);
    const RowsCost cost = rows_cost(a, u.n);
    const int j = tile_at(cost, w.at);
    // no tile in front of the border or none behind it, or an earlier border cuts the pair too
    if (j == 0 || j >= u.nt || tile_at(cost, w.at - per) > 0) return;
    // parts: share c - 1's, and those up to the share that the last tile begins in
    const int n = 2 + (int)divide(cost.extra + (int64_t)(u.nt - 1) * cost.tile - w.at, per);
    const int rows = u.n * a.group;
    const int so = a.rows_cap * D;
    for (int r0 = blockIdx.y * kMergeRows; r0 < rows; r0 += gridDim.y * kMergeRows) {
        auto run = [&](int slot, int parts) {
            return Run{a.part_ml + (int64_t)slot * a.rows_cap + r0, a.part_o + (int64_t)slot * so + 4 * r0, parts,
                       2 * a.rows_cap, 2 * so, 4 * a.rows_cap};
        };
        merge_rows<D, T, kAhead>(run(2 * (c - 1) + 1, 1), run(2 * c, n - 1), min(kMergeRows, rows - r0), [](int, float, float) {},
                         [&](int r) { return static_cast<T *>(a.out) + rows_row<D>(a, u, w.g, r0 + r).out; });
    }
}

// A CTA a (sequence, KV head)
template <int D, typename T>
__global__ void __launch_bounds__(2 * D, 768 / (2 * D)) rows_merge_prefix_kernel(const RowsArgs a) {
    pdl_wait();
    const int hk = a.pv.kv_heads, b = blockIdx.x / hk, g = blockIdx.x % hk;
    const int4 s = __ldcg(reinterpret_cast<const int4 *>(a.seq) + b);
    const RowsHead head = rows_head(a);
    if (head.failed) return;
    RowsUnit pre, own;
    if (s.x >= 0) pre = rows_unit(a, s.x);
    if (s.z >= 0) own = rows_unit(a, s.z);
    int64_t slot_p = 0, slot_o = 0;
    int np = 0, no = 0;
    auto parts = [&](const RowsUnit &u, int64_t pair0, int64_t &slot) {  // of pair (u, g); slot: its first part's
        const RowsCost c = rows_cost(a, u.n);
        const int64_t x0 = u.cum + g * pair_cost(c, u.nt) + c.extra;
        const int64_t c0 = divide(x0, head.per);
        slot = pair0 + g + c0;
        return (int)(divide(x0 + (int64_t)(u.nt - 1) * c.tile, head.per) - c0) + 1;
    };
    if (s.x >= 0) np = parts(pre, (int64_t)s.x * hk, slot_p);
    if (s.z >= 0) no = parts(own, (int64_t)(s.z - head.n_pre) * hk, slot_o);
    const int rp = s.y * a.group, so = a.rows_cap * D, sw = a.group * D;  // rp: the pre part's rows
    const int64_t row0 = (int64_t)b * a.q_heads + g * a.group;
    merge_rows<D, T, 8>(
        Run{a.part_ml + slot_p * a.rows_cap + rp, a.part_o + slot_p * so + 4 * rp, np, a.rows_cap, so, 4 * a.rows_cap},
        Run{a.own_ml + slot_o * a.group, a.own_o + slot_o * sw, no, a.group, sw, 4 * a.group}, a.group,
        [&](int r, float ref, float inv) { a.norm[row0 + r] = make_float2(ref, inv); },
        [&](int r) { return static_cast<T *>(a.out) + (row0 + r) * D; });
}

template <int D, typename T>
cudaError_t launch_merge(const RowsArgs &a, cudaStream_t st) {
    if (a.prefix)
        return launch_k(rows_merge_prefix_kernel<D, T>, dim3((unsigned)(a.batch * a.pv.kv_heads)), dim3(2 * D), 0,
                        st, a);
    const int y = (a.rows_cap + kMergeRows - 1) / kMergeRows;
    return a.rows_cap > 64 ? launch_k(rows_merge_window_kernel<D, T, 2>, dim3(a.ctas, y), dim3(2 * D), 0, st, a)
                           : launch_k(rows_merge_window_kernel<D, T, 8>, dim3(a.ctas, y), dim3(2 * D), 0, st, a);
}

// Scores without tensor cores: K once more, a shared prefix's once a member, with each row's maximum M and sum of weights W,
//     score = mean over the row's heads of 2^(q . k scale - M) / W.
// A CTA: 32 slots of a sequence, a lane a slot, a warp every eighth KV head with all of its query heads.  Each lane
// reads its own row of K, whose lines the first-level cache holds until they are used up; no warp waits for another
// until the sums of the heads meet, in a fixed order.
constexpr int kScoreWarps = 8;
__device__ __forceinline__ float4 load_four(const float *p) { return __ldg(reinterpret_cast<const float4 *>(p)); }
__device__ __forceinline__ float4 load_four(const __nv_bfloat16 *p) {
    const uint2 x = __ldg(reinterpret_cast<const uint2 *>(p));
    return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16),
                       __uint_as_float(x.y & 0xffff0000u));
}
template <int D, typename T, int G>
__global__ void __launch_bounds__(kScoreWarps * 32) rows_score_kernel(const RowsArgs a, const RowsScoreArgs sc) {
    pdl_wait();
    __shared__ float part[kScoreWarps][33];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rps = a.rows_per_seq, hk = a.pv.kv_heads;
    for (int b = blockIdx.y; b < a.batch; b += gridDim.y) {
        const int S0 = a.pv.start ? min(max(__ldg(a.pv.start + b), 0), a.cap) : 0;
        const int L = min(max(__ldg(a.len + b), 0), a.cap - S0);
        const int4 s = __ldcg(reinterpret_cast<const int4 *>(a.seq) + b);
        int lead = b, lead_s0 = S0;
        if (s.x >= 0) {
            lead = __ldcg(&a.units[s.x].b);
            lead_s0 = __ldcg(&a.units[s.x].S0);
        }
        for (int j0 = blockIdx.x * 32; j0 < L; j0 += gridDim.x * 32) {
            const int j = j0 + lane;
            const bool inside = j < L, shared = j < s.w;
            auto put = [&](int row, float t) {
                const int64_t at = ((int64_t)b * rps + row) * a.cap + j;
                if (a.pos && __ldg(a.pos + at) < 0) t = 0.f;
                if (sc.score) sc.score[at] = t;
                if (sc.ema) sc.ema[at] = sc.alpha * sc.ema[at] + (1.f - sc.alpha) * t;
            };
            float sum = 0.f;
            for (int g = warp; g < hk; g += kScoreWarps) {
                const T *k = static_cast<const T *>(a.k) +
                             (inside ? a.pv.row_phys(shared ? lead : b, a.layer, g, (shared ? lead_s0 : S0) + j) : 0) * D;
                const int64_t row = (int64_t)b * a.q_heads + g * G;
                const T *q = static_cast<const T *>(a.q) + row * D;
                float2 z[G];
#pragma unroll
                for (int h = 0; h < G; ++h) z[h] = make_float2(0.f, 0.f);
#pragma unroll 8
                for (int c = 0; c < D; c += 4) {
                    const float4 x = load_four(k + c);
#pragma unroll
                    for (int h = 0; h < G; ++h) {
                        const float4 y = load_four(q + h * D + c);
                        z[h] = fma2(make_float2(x.x, x.y), make_float2(y.x, y.y), z[h]);
                        z[h] = fma2(make_float2(x.z, x.w), make_float2(y.z, y.w), z[h]);
                    }
                }
#pragma unroll
                for (int h = 0; h < G; ++h) {
                    const float2 mw = __ldcg(a.norm + row + h);
                    if (mw.y != 0.f) sum += exp2f(__fmaf_rn(z[h].x + z[h].y, a.scale_log2, -mw.x)) * mw.y;
                }
                if (rps > 1) {
                    if (inside) put(g, sum * (1.f / G));
                    sum = 0.f;
                }
            }
            if (rps == 1) {
                part[warp][lane] = sum;
                __syncthreads();
                if (warp == 0 && inside) {
                    float t = 0.f;
#pragma unroll
                    for (int w = 0; w < kScoreWarps; ++w) t += part[w][lane];
                    put(0, t / (float)a.q_heads);
                }
                __syncthreads();
            }
        }
    }
}

template <int D, typename T>
cudaError_t launch_score(const RowsArgs &a, const RowsScoreArgs &s, cudaStream_t st) {
    const int blocks = s.max_len > 32 ? (s.max_len + 31) / 32 : 1;
    const dim3 grid(blocks, a.batch < 65535 ? a.batch : 65535), block(kScoreWarps * 32);
    switch (a.group) {
        case 1: return launch_k(rows_score_kernel<D, T, 1>, grid, block, 0, st, a, s);
        case 2: return launch_k(rows_score_kernel<D, T, 2>, grid, block, 0, st, a, s);
        case 4: return launch_k(rows_score_kernel<D, T, 4>, grid, block, 0, st, a, s);
        case 7: return launch_k(rows_score_kernel<D, T, 7>, grid, block, 0, st, a, s);
        case 8: return launch_k(rows_score_kernel<D, T, 8>, grid, block, 0, st, a, s);
        default: return cudaErrorInvalidValue;
    }
}

}  // namespace

cudaError_t launch_rows_merge(const RowsArgs &a, int dtype, int head_dim, cudaStream_t st) {
    cudaError_t e;
    if (dtype == IKV_BF16)
        e = head_dim == 64 ? launch_merge<64, __nv_bfloat16>(a, st) : launch_merge<128, __nv_bfloat16>(a, st);
    else
        e = head_dim == 64 ? launch_merge<64, float>(a, st) : launch_merge<128, float>(a, st);
    note_launch();
    return e;
}

cudaError_t launch_rows_score(const RowsArgs &a, const RowsScoreArgs &s, int dtype, int head_dim, cudaStream_t st) {
    cudaError_t e;
    if (dtype == IKV_BF16)
        e = head_dim == 64 ? launch_score<64, __nv_bfloat16>(a, s, st) : launch_score<128, __nv_bfloat16>(a, s, st);
    else
        e = head_dim == 64 ? launch_score<64, float>(a, s, st) : launch_score<128, float>(a, s, st);
    note_launch();
    return e;
}

}  // namespace ikv
