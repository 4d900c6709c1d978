// Where a row of a packed-row attention leaves its result, and the recomputation of single rows.
#pragma once
#include "merge.cuh"
#include "rows.cuh"

namespace ikv {
namespace {

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// two at a time: x y + z, x + y
__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(r)
        : "l"(*reinterpret_cast<unsigned long long *>(&x)), "l"(*reinterpret_cast<unsigned long long *>(&y)),
          "l"(*reinterpret_cast<unsigned long long *>(&z)));
    return *reinterpret_cast<float2 *>(&r);
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;"
        : "=l"(r)
        : "l"(*reinterpret_cast<unsigned long long *>(&x)), "l"(*reinterpret_cast<unsigned long long *>(&y)));
    return *reinterpret_cast<float2 *>(&r);
}

__device__ __forceinline__ float load_as_float(const float *p) { return __ldg(p); }
__device__ __forceinline__ float load_as_float(const __nv_bfloat16 *p) { return __bfloat162float(*p); }

__device__ __forceinline__ void store4(float *p, float a, float b, float c, float d) {
    *reinterpret_cast<float4 *>(p) = make_float4(a, b, c, d);
}
__device__ __forceinline__ void store4(__nv_bfloat16 *p, float a, float b, float c, float d) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b), y = __floats2bfloat162_rn(c, d);
    uint2 w;
    w.x = *reinterpret_cast<const uint32_t *>(&x);
    w.y = *reinterpret_cast<const uint32_t *>(&y);
    *reinterpret_cast<uint2 *>(p) = w;
}

// Channels 0 .. 3 of partial row r of a slot, and the distance to the next four
template <int D>
__device__ __forceinline__ float *rows_part_o(const RowsArgs &a, const RowsUnit &u, int64_t slot, int r) {
    return a.prefix && u.m0 < 0 ? a.own_o + slot * a.group * D + 4 * r : a.part_o + slot * a.rows_cap * D + 4 * r;
}
__device__ __forceinline__ int rows_part_step(const RowsArgs &a, const RowsUnit &u) {
    return 4 * (a.prefix && u.m0 < 0 ? a.group : a.rows_cap);
}
__device__ __forceinline__ float2 *rows_part_ml(const RowsArgs &a, const RowsUnit &u, int64_t slot, int r) {
    return a.prefix && u.m0 < 0 ? a.own_ml + slot * a.group + r : a.part_ml + slot * a.rows_cap + r;
}
__device__ __forceinline__ void rows_store_ml(const RowsArgs &a, const RowsUnit &u, int64_t slot, int r, float m,
                                              float l) {
    *rows_part_ml(a, u, slot, r) = make_float2(m, l);
}

// Four values of a row
__device__ __forceinline__ float4 load4_as_float(const float *p) { return __ldg(reinterpret_cast<const float4 *>(p)); }
__device__ __forceinline__ float4 load4_as_float(const __nv_bfloat16 *p) {
    const uint2 x = __ldg(reinterpret_cast<const uint2 *>(p));
    return make_float4(__uint_as_float(x.x << 16), __uint_as_float(x.x & 0xffff0000u), __uint_as_float(x.y << 16),
                       __uint_as_float(x.y & 0xffff0000u));
}

// Row r of a part by one warp, over the slots that it sees and no others: the products of a whole tile
// multiply rows of V that a row does not see by 0, which leaves NaN where those are not finite.  32 slots at a
// time, a lane a slot for the scores, a lane D / 32 channels for the output.
template <int D, typename T>
__device__ __noinline__ void rows_redo(const RowsArgs &a, int unit, int g, int j0, int n, bool whole, int64_t slot,
                                       int r) {
    constexpr int E = D / 32;
    constexpr unsigned kAll = 0xffffffffu;
    const RowsUnit u = rows_unit(a, unit);
    const int lane = threadIdx.x & 31;
    const RowsRow row = rows_row<D>(a, u, g, r);
    const T *q = static_cast<const T *>(a.q) + row.q;
    float acc[E], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    for (int i = 4 * j0; i < 4 * (j0 + n); ++i) {
        const int s = rows_tile(u, i / 4) * kRowsTile + i % 4 * 32 + lane;
        const bool sees = rows_sees(row, u.S0, s);
        const unsigned all = __ballot_sync(kAll, sees);
        if (!all) continue;
        const int64_t at = sees ? a.pv.row_phys(u.b, a.layer, g, s) * D : 0;
        float z = -INFINITY;
        if (sees) {
            const T *k = static_cast<const T *>(a.k) + at;
            float2 z2 = make_float2(0.f, 0.f);
#pragma unroll 8
            for (int c = 0; c < D; c += 4) {
                const float4 x = load4_as_float(k + c), y = load4_as_float(q + c);
                z2 = fma2(make_float2(x.x, x.y), make_float2(y.x, y.y), z2);
                z2 = fma2(make_float2(x.z, x.w), make_float2(y.z, y.w), z2);
            }
            z = z2.x + z2.y;
        }
        const float mx = fmaxf(m, warp_max(__fmul_rn(z, a.scale_log2))), ref = mx == -INFINITY ? 0.f : mx;
        const float f = exp2f(m - ref), p = sees ? exp2f(__fmaf_rn(z, a.scale_log2, -ref)) : 0.f;
        l = l * f + warp_sum(p);
        m = mx;
#pragma unroll
        for (int e = 0; e < E; ++e) acc[e] *= f;
#pragma unroll 8
        for (int x = 0; x < 32; ++x) {
            const float w = __shfl_sync(kAll, p, x);
            const T *v = static_cast<const T *>(a.v) + __shfl_sync(kAll, at, x) + lane;
            if ((all >> x) & 1u) {
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] += w * load_as_float(v + 32 * e);
            }
        }
    }
    if (whole) {
#pragma unroll
        for (int e = 0; e < E; ++e) store_as(static_cast<T *>(a.out) + row.out + lane + 32 * e, over_sum(acc[e], l));
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) {
            const int c = lane + 32 * e;
            rows_part_o<D>(a, u, slot, r)[(int64_t)(c / 4) * rows_part_step(a, u) + c % 4] = acc[e];
        }
        if (lane == 0) rows_store_ml(a, u, slot, r, m, l);
    }
}

}  // namespace
}  // namespace ikv
