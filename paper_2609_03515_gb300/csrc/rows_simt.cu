// Packed-row attention without tensor cores: fp32 caches, and bf16 ones in pages whose size is no multiple
// of 8.  One pass over the slots with a running maximum and sum (online softmax):
//     S = Q K^T, p_j = 2^(S_j - m'), l' = l 2^(m - m') + sum p, O' = O 2^(m - m') + p V, out = O / l
// in fp32 on the FMA units, 64 slots of K and V a step, copied asynchronously a step ahead.  m' is the maximum
// so far where a weight would pass 2^8, m otherwise.
//
// A CTA of 8 warps holds 64 rows (16 where a part has no more): a warp 8 (2) of them, lane x of it slots x and x + 32
// of S and channels 2 x, 2 x + 1 (+ 64) of O.  What a warp reads of Q and P is then the same for all lanes, and what it
// reads of K and V is used for 8 rows.  Half-warps of 4 rows read shared memory 1.5 times as often, warps of 16 rows 0.75
// times, but leave too few warps to cover the latencies.
//
// Measured: 8 fp32 prompts of 17 to 1021 tokens, window 256, 16 / 4 heads of 64: 287 us with warps of 8 rows, 294
// with half-warps of 4, 354 with 4 warps of 16.  That is 44% of the FMA units' rate, for twice the products that
// rows see (whole steps of 64 slots at both ends of a window).
#include "merge.cuh"
#include "rows.cuh"
#include "rows_redo.cuh"

namespace ikv {
namespace {

constexpr int kStep = 64;           // slots of K and V a step
constexpr int kSimtThreads = 256, kSimtWarps = 8;

template <int D, typename T>
__host__ __device__ constexpr int row_stride() { return D + 16 / (int)sizeof(T); }  // elements: 16 bytes of padding a row
template <int D, typename T>
constexpr size_t simt_smem() {
    return sizeof(float) * kRowsSimt * (D + 4) + 4 * sizeof(T) * kStep * row_stride<D, T>() +
           sizeof(float) * kRowsSimt * (kStep + 4);
}

__device__ __forceinline__ float4 load4(const float *p) { return *reinterpret_cast<const float4 *>(p); }
__device__ __forceinline__ float4 load4(const __nv_bfloat16 *p) {
    const uint2 x = *reinterpret_cast<const uint2 *>(p);
    return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16),
                       __uint_as_float(x.y & 0xffff0000u));
}
__device__ __forceinline__ void cp16(void *dst, const void *src, bool real) {
    const uint32_t d = static_cast<uint32_t>(__cvta_generic_to_shared(dst));
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(d), "l"(src), "r"(real ? 16 : 0) : "memory");
}

__device__ __forceinline__ float2 load2(const float *p) { return *reinterpret_cast<const float2 *>(p); }
__device__ __forceinline__ float2 load2(const __nv_bfloat16 *p) {
    const uint32_t x = *reinterpret_cast<const uint32_t *>(p);
    return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
}

// One part: tiles [j0, j0 + n) of pair (unit, g).  (whole: its rows' outputs are final)
template <int D, typename T, int RPT>
__device__ void simt_part(const RowsArgs &a, const RowsHead &head, const RowsUnit &u, int unit, int g, int j0, int n,
                          float *sQ, T *sK, T *sV, float *sP, int4 *sRow) {
    constexpr int RS = row_stride<D, T>(), NC = D / 64, CH = D * (int)sizeof(T) / 16, QS = D + 4, PS = kStep + 4;
    const int tid = threadIdx.x, lane = tid & 31, r0 = (tid >> 5) * RPT;
    const int rows = u.n * a.group;
    const int sh = a.prefix ? u.lo : u.S0 + a.sinks;
    // the slots that every row sees: [lo, all_hi], without [sh, all_wlo)
    const int all_hi = a.prefix ? u.hi - 1 : u.p0, all_wlo = a.prefix ? u.lo : max(u.lo, u.p0 + u.n - a.window);
    __syncthreads();  // (the last part's shared memory has been read)
    if (lane < RPT) {  // (sequence, last slot, first of the window) of each row, by the warp that reads it: a unit
                       // that sees no slot has no step, and no other barrier
        const int r = r0 + lane;
        const RowsRow w = rows_row<D>(a, u, g, r);
        sRow[r] = make_int4(r < rows ? w.seq : -1, w.hi, w.wlo, 0);
    }
    __syncwarp();
    const int steps = n * (kRowsTile / kStep);
    auto first_slot = [&](int i) { return rows_tile(u, j0 + i / 2) * kRowsTile + (i & 1) * kStep; };
    auto step_from = [&](int i) {  // the first from i on with a slot that some row sees
        for (; i < steps; ++i) {
            const int s = first_slot(i);
            if (s < u.hi && (s + kStep > u.wlo || (s < u.sh && s + kStep > u.lo))) break;
        }
        return i;
    };
    auto fetch = [&](int i, int buf) {
        T *k = sK + buf * kStep * RS, *v = sV + buf * kStep * RS;
        const int s0 = first_slot(i);
#pragma unroll 4
        for (int x = tid; x < kStep * CH; x += kSimtThreads) {
            const int r = x / CH, c = x % CH * (16 / (int)sizeof(T)), s = s0 + r;
            // (slots that no row sees are zeros)
            const bool real = s < u.hi && (s >= u.wlo || (s >= u.lo && s < u.sh));
            const int64_t e = real ? a.pv.row_phys(u.b, a.layer, g, s) * D + c : 0;
            cp16(k + r * RS + c, static_cast<const T *>(a.k) + e, real);
            cp16(v + r * RS + c, static_cast<const T *>(a.v) + e, real);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int st = step_from(0), buf = 0;
    if (st < steps) fetch(st, 0);
    for (int i = tid; i < kSimtWarps * RPT * (D / 4); i += kSimtThreads) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        const RowsRow w = rows_row<D>(a, u, g, r);
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < rows && w.seq >= 0) x = load4(static_cast<const T *>(a.q) + w.q + c);
        *reinterpret_cast<float4 *>(sQ + r * QS + c) = x;
    }
    float m[RPT], l[RPT];  // l: of the lane's own slots
    float2 acc[RPT][NC];
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[i][c] = make_float2(0.f, 0.f);
    }
    for (int ahead; st < steps; st = ahead, buf ^= 1) {
        ahead = step_from(st + 1);
        if (ahead < steps) {
            fetch(ahead, buf ^ 1);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        } else {
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        }
        __syncthreads();
        const T *k = sK + buf * kStep * RS, *v = sV + buf * kStep * RS;
        const int s0 = first_slot(st);
        const bool masked = a.pos || s0 < u.lo || s0 + kStep - 1 > all_hi || (s0 < all_wlo && s0 + kStep > sh);
        // (sums of even and of odd channels: two products an instruction)
        float2 s2[RPT][2];
#pragma unroll
        for (int i = 0; i < RPT; ++i) s2[i][0] = s2[i][1] = make_float2(0.f, 0.f);
#pragma unroll 2
        for (int c = 0; c < D; c += 4) {
            const float4 k0 = load4(k + lane * RS + c), k1 = load4(k + (lane + 32) * RS + c);
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                const float4 q = load4(sQ + (r0 + i) * QS + c);
                s2[i][0] = fma2(make_float2(q.x, q.y), make_float2(k0.x, k0.y), s2[i][0]);
                s2[i][1] = fma2(make_float2(q.x, q.y), make_float2(k1.x, k1.y), s2[i][1]);
                s2[i][0] = fma2(make_float2(q.z, q.w), make_float2(k0.z, k0.w), s2[i][0]);
                s2[i][1] = fma2(make_float2(q.z, q.w), make_float2(k1.z, k1.w), s2[i][1]);
            }
        }
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            float z0 = s2[i][0].x + s2[i][0].y, z1 = s2[i][1].x + s2[i][1].y;
            if (masked) {
                const int4 x = sRow[r0 + i];
                RowsRow w;
                w.lo = u.lo;
                w.hi = x.y;
                w.wlo = x.z;
                w.sh = sh;
                w.pos = a.pos && x.x >= 0
                            ? a.pos + ((int64_t)x.x * a.rows_per_seq + (a.rows_per_seq == 1 ? 0 : g)) * a.cap
                            : nullptr;
                if (x.x < 0 || !rows_sees(w, u.S0, s0 + lane)) z0 = -INFINITY;
                if (x.x < 0 || !rows_sees(w, u.S0, s0 + lane + 32)) z1 = -INFINITY;
            }
            // The maximum only moves where a weight would grow past 2^8: a vote in place of a reduction.  (The
            // products unrounded: what the maximum is off by is common to all of the row's weights.)
            const float z = __fmul_rn(fmaxf(z0, z1), a.scale_log2);
            if (__any_sync(0xffffffffu, z > m[i] + 8.f)) {
                const float top = fmaxf(m[i], warp_max(z)), f = ex2(m[i] - top);
                l[i] *= f;
#pragma unroll
                for (int c = 0; c < NC; ++c) acc[i][c] = fma2(acc[i][c], make_float2(f, f), make_float2(0.f, 0.f));
                m[i] = top;
            }
            const float ref = m[i] == -INFINITY ? 0.f : m[i];  // no slot so far: nothing to scale
            const float p0 = ex2(__fmaf_rn(z0, a.scale_log2, -ref)), p1 = ex2(__fmaf_rn(z1, a.scale_log2, -ref));
            sP[(r0 + i) * PS + lane] = p0;
            sP[(r0 + i) * PS + lane + 32] = p1;
            l[i] += p0 + p1;
        }
        __syncwarp();  // (a row's weights are written and read by one warp)
#pragma unroll 2
        for (int x = 0; x < kStep; x += 4) {
            float2 w[4][NC];
#pragma unroll
            for (int y = 0; y < 4; ++y)
#pragma unroll
                for (int c = 0; c < NC; ++c) w[y][c] = load2(v + (x + y) * RS + 2 * lane + 64 * c);
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                const float4 p = load4(sP + (r0 + i) * PS + x);
#pragma unroll
                for (int c = 0; c < NC; ++c) {
                    acc[i][c] = fma2(make_float2(p.x, p.x), w[0][c], acc[i][c]);
                    acc[i][c] = fma2(make_float2(p.y, p.y), w[1][c], acc[i][c]);
                    acc[i][c] = fma2(make_float2(p.z, p.z), w[2][c], acc[i][c]);
                    acc[i][c] = fma2(make_float2(p.w, p.w), w[3][c], acc[i][c]);
                }
            }
        }
        __syncthreads();
    }
    // results.  A row whose output is not finite though its sum is may have met NaN or infinite V rows
    // that it does not see (0 * inf): it is computed once more, over what it sees alone.
    const bool begins = j0 == 0, whole = begins && n == u.nt && !a.prefix;
    const int64_t slot = whole ? 0 : rows_slot(a, head, u, unit, g, blockIdx.x, begins);
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const int r = r0 + i;
        if (sRow[r].x < 0) continue;  // (the warp's)
        const float sum = warp_sum(l[i]);
        bool bad = false;
#pragma unroll
        for (int c = 0; c < NC; ++c) bad |= !(fabsf(acc[i][c].x) < INFINITY) || !(fabsf(acc[i][c].y) < INFINITY);
        if (__any_sync(0xffffffffu, bad) && !isnan(sum)) {
            rows_redo<D, T>(a, unit, g, j0, n, whole, slot, r);
            continue;
        }
        if (whole) {
            T *to = static_cast<T *>(a.out) + rows_row<D>(a, u, g, r).out + 2 * lane;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                store_as(to + 64 * c, over_sum(acc[i][c].x, sum));
                store_as(to + 64 * c + 1, over_sum(acc[i][c].y, sum));
            }
        } else {
            const int step = rows_part_step(a, u);
#pragma unroll
            for (int c = 0; c < NC; ++c)
                *reinterpret_cast<float2 *>(rows_part_o<D>(a, u, slot, r) + (int64_t)(lane / 2 + 16 * c) * step +
                                            lane % 2 * 2) = acc[i][c];
            if (lane == 0) rows_store_ml(a, u, slot, r, m[i], sum);
        }
    }
}

template <int D, typename T>
__global__ void __launch_bounds__(kSimtThreads, D == 64 ? 2 : 1) rows_simt_kernel(const RowsArgs a) {
    pdl_wait();
    extern __shared__ __align__(16) unsigned char smem[];
    float *sQ = reinterpret_cast<float *>(smem);
    T *sK = reinterpret_cast<T *>(sQ + kRowsSimt * (D + 4));
    T *sV = sK + 2 * kStep * row_stride<D, T>();
    float *sP = reinterpret_cast<float *>(sV + 2 * kStep * row_stride<D, T>());
    __shared__ int4 sRow[kRowsSimt];
    RowsHead head;
    head.n_pre = __ldcg(&a.head->n_pre);
    RowsWalk w;
    w.begin(__ldcg(reinterpret_cast<const int4 *>(a.start + blockIdx.x)));
    while (w.left > 0) {
        const RowsUnit u = rows_unit(a, w.unit);
        int j0;
        const int n = w.part(a, u, j0);
        if (n > 0) {
            if (u.n * a.group <= 16)
                simt_part<D, T, 2>(a, head, u, w.unit, w.g, j0, n, sQ, sK, sV, sP, sRow);
            else
                simt_part<D, T, 8>(a, head, u, w.unit, w.g, j0, n, sQ, sK, sV, sP, sRow);
        }
        w.next(a, u);
    }
}

template <int D, typename T>
cudaError_t launch_simt(const RowsArgs &a, cudaStream_t st) {
    constexpr size_t bytes = simt_smem<D, T>();
    static std::atomic<uint64_t> done{0};
    const cudaError_t e = allow_smem(rows_simt_kernel<D, T>, bytes, done);
    if (e != cudaSuccess) return e;
    return launch_k(rows_simt_kernel<D, T>, dim3(a.ctas), dim3(kSimtThreads), bytes, st, a);
}

}  // namespace

// shared memory: 184 KB (fp32) or 119 KB (bf16) at 128 channels, 102 KB or 70 KB at 64
int rows_simt_ctas_per_sm(int head_dim) { return head_dim == 64 ? 2 : 1; }

cudaError_t launch_rows_simt(const RowsArgs &a, int dtype, int head_dim, cudaStream_t st) {
    cudaError_t e;
    if (dtype == IKV_BF16)
        e = head_dim == 64 ? launch_simt<64, __nv_bfloat16>(a, st) : launch_simt<128, __nv_bfloat16>(a, st);
    else
        e = head_dim == 64 ? launch_simt<64, float>(a, st) : launch_simt<128, float>(a, st);
    note_launch();
    return e;
}

}  // namespace ikv
