// Packed-row attention without tensor cores: fp32 caches, and bf16 ones in pages whose size is no multiple
// of 8.  One pass over the slots with a running maximum and sum (online softmax):
//     S = Q K^T, m' = max(m, max_j S_j), p_j = 2^(S_j - m'), l' = l 2^(m - m') + sum p, O' = O 2^(m - m') + p V
// in fp32 on the FMA units, 64 slots of K and V a step, copied asynchronously a step ahead.
//
// A CTA of 256 threads holds 64 rows (16 where a part has no more): thread (ty, tx) has rows RPT ty ..,
// slots tx + 16 j of S and channels 4 tx + 64 k .. of O, so that a row's 16 threads share a half-warp: its
// maximum and its weights never leave the warp.
#include "merge.cuh"
#include "rows.cuh"
#include "rows_redo.cuh"

namespace ikv {
namespace {

constexpr int kStep = 64;           // slots of K and V a step
constexpr int kSimtThreads = 256;

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

__device__ __forceinline__ void fma4(float *acc, float p, float4 v) {
    const float2 pp = make_float2(p, p);
    float2 *a = reinterpret_cast<float2 *>(acc);
    a[0] = fma2(pp, make_float2(v.x, v.y), a[0]);
    a[1] = fma2(pp, make_float2(v.z, v.w), a[1]);
}

// One part: tiles [j0, j0 + n) of pair (unit, g).  (whole: its rows' outputs are final)
template <int D, typename T, int RPT>
__device__ void simt_part(const RowsArgs &a, const RowsHead &head, const RowsUnit &u, int unit, int g, int j0, int n,
                          float *sQ, T *sK, T *sV, float *sP) {
    constexpr int RS = row_stride<D, T>(), NC = D / 16, CH = D * (int)sizeof(T) / 16;
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15, lane = tid & 31;
    const int rows = u.n * a.group;
    int seq[RPT], hi[RPT], wlo[RPT];  // of its rows (the rest of a RowsRow again where it is needed)
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        const RowsRow w = rows_row<D>(a, u, g, ty * RPT + i);
        seq[i] = ty * RPT + i < rows ? w.seq : -1;
        hi[i] = w.hi;
        wlo[i] = w.wlo;
    }
    const int sh = a.prefix ? u.lo : u.S0 + a.sinks;
    __syncthreads();  // (the last part's shared memory has been read)
    for (int i = tid; i < 16 * RPT * (D / 4); i += kSimtThreads) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        const RowsRow w = rows_row<D>(a, u, g, r);
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (r < rows && w.seq >= 0) x = load4(static_cast<const T *>(a.q) + w.q + c);
        *reinterpret_cast<float4 *>(sQ + r * (D + 4) + c) = x;
    }
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
    float m[RPT], l[RPT];
    alignas(8) float acc[RPT][NC];
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) acc[i][c] = 0.f;
    }
    int st = step_from(0), buf = 0;
    if (st < steps) fetch(st, 0);
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
        // (sums of even and of odd channels: two products an instruction)
        float2 s2[RPT][4];
#pragma unroll
        for (int i = 0; i < RPT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s2[i][j] = make_float2(0.f, 0.f);
#pragma unroll 4
        for (int c = 0; c < D; c += 4) {
            float4 kk[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) kk[j] = load4(k + (tx + 16 * j) * RS + c);
#pragma unroll
            for (int i = 0; i < RPT; ++i) {
                const float4 q = load4(sQ + (ty * RPT + i) * (D + 4) + c);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    s2[i][j] = fma2(make_float2(q.x, q.y), make_float2(kk[j].x, kk[j].y), s2[i][j]);
                    s2[i][j] = fma2(make_float2(q.z, q.w), make_float2(kk[j].z, kk[j].w), s2[i][j]);
                }
            }
        }
        float s[RPT][4];
#pragma unroll
        for (int i = 0; i < RPT; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) s[i][j] = s2[i][j].x + s2[i][j].y;
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            float mx = m[i];
            if (seq[i] < 0 || a.pos || s0 < u.lo || s0 + kStep - 1 > hi[i] || (s0 < wlo[i] && s0 + kStep > sh)) {
                RowsRow w;
                w.lo = u.lo;
                w.hi = hi[i];
                w.wlo = wlo[i];
                w.sh = sh;
                w.pos = a.pos && seq[i] >= 0
                            ? a.pos + ((int64_t)seq[i] * a.rows_per_seq + (a.rows_per_seq == 1 ? 0 : g)) * a.cap
                            : nullptr;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (seq[i] < 0 || !rows_sees(w, u.S0, s0 + tx + 16 * j)) s[i][j] = -INFINITY;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) mx = fmaxf(mx, __fmul_rn(s[i][j], a.scale_log2));
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
            const float ref = mx == -INFINITY ? 0.f : mx;  // no slot so far: nothing to scale
            const float f = exp2f(m[i] - ref);
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                // (the product unrounded: what the maximum is off by is common to all of the row's weights)
                const float p = exp2f(__fmaf_rn(s[i][j], a.scale_log2, -ref));
                sum += p;
                sP[(ty * RPT + i) * (kStep + 4) + tx + 16 * j] = p;
            }
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            l[i] = l[i] * f + sum;
            m[i] = mx;
#pragma unroll
            for (int c = 0; c < NC; ++c) acc[i][c] *= f;
        }
        __syncwarp();  // (a row's weights are written and read by one half-warp)
#pragma unroll 2
        for (int x = 0; x < kStep; x += 4) {
            float4 p[RPT];
#pragma unroll
            for (int i = 0; i < RPT; ++i) p[i] = load4(sP + (ty * RPT + i) * (kStep + 4) + x);
#pragma unroll
            for (int kc = 0; kc < D / 64; ++kc) {
                float4 w[4];
#pragma unroll
                for (int y = 0; y < 4; ++y) w[y] = load4(v + (x + y) * RS + 4 * tx + 64 * kc);
#pragma unroll
                for (int i = 0; i < RPT; ++i) {
                    fma4(acc[i] + 4 * kc, p[i].x, w[0]);
                    fma4(acc[i] + 4 * kc, p[i].y, w[1]);
                    fma4(acc[i] + 4 * kc, p[i].z, w[2]);
                    fma4(acc[i] + 4 * kc, p[i].w, w[3]);
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
        const int r = ty * RPT + i;
        bool bad = false;
#pragma unroll
        for (int c = 0; c < NC; ++c) bad |= !(fabsf(acc[i][c]) < INFINITY);
        bad = bad && seq[i] >= 0 && !isnan(l[i]);
        const unsigned redo = __ballot_sync(0xffffffffu, bad);
        const bool again = (redo >> (lane & 16)) & 0xffffu;
        if (seq[i] >= 0 && !again) {
            const RowsRow w = rows_row<D>(a, u, g, r);
#pragma unroll
            for (int kc = 0; kc < D / 64; ++kc)
                rows_store4<D, T>(a, u, w, whole, slot, r, 4 * tx + 64 * kc, acc[i] + 4 * kc, l[i]);
            if (!whole && tx == 0) rows_store_ml(a, u, slot, r, m[i], l[i]);
        }
        for (int half = 0; half < 2; ++half)
            if ((redo >> (16 * half)) & 0xffffu)
                rows_redo<D, T>(a, unit, g, j0, n, whole, slot, ((tid >> 5) * 2 + half) * RPT + i);
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
                simt_part<D, T, 1>(a, head, u, w.unit, w.g, j0, n, sQ, sK, sV, sP);
            else
                simt_part<D, T, 4>(a, head, u, w.unit, w.g, j0, n, sQ, sK, sV, sP);
        }
        w.next(a, u);
    }
}

template <int D, typename T>
cudaError_t launch_simt(const RowsArgs &a, cudaStream_t st) {
    constexpr size_t bytes = simt_smem<D, T>();
    const cudaError_t e = cudaFuncSetAttribute(rows_simt_kernel<D, T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
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
