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

// Row r of a part by one warp, over the slots that it sees and no others: the products of a whole tile
// multiply rows of V that a row does not see by 0, which leaves NaN where those are not finite.  Rare,
// so simple: a slot at a time.
template <int D, typename T>
__device__ __noinline__ void rows_redo(const RowsArgs &a, int unit, int g, int j0, int n, bool whole, int64_t slot,
                                       int r) {
    constexpr int E = D / 32;
    const RowsUnit u = rows_unit(a, unit);
    const int lane = threadIdx.x & 31;
    const RowsRow row = rows_row<D>(a, u, g, r);
    float q[E], acc[E], m = -INFINITY, l = 0.f;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        q[e] = load_as_float(static_cast<const T *>(a.q) + row.q + lane + 32 * e);
        acc[e] = 0.f;
    }
    for (int j = j0; j < j0 + n; ++j) {
        const int t0 = rows_tile(u, j) * kRowsTile;
        for (int s = t0; s < t0 + kRowsTile; ++s) {
            if (!rows_sees(row, u.S0, s)) continue;
            const int64_t at = a.pv.row_phys(u.b, a.layer, g, s) * D + lane;
            float z = 0.f;
#pragma unroll
            for (int e = 0; e < E; ++e) z += q[e] * load_as_float(static_cast<const T *>(a.k) + at + 32 * e);
            z = warp_sum(z);
            const float mx = fmaxf(m, __fmul_rn(z, a.scale_log2)), ref = mx == -INFINITY ? 0.f : mx;
            const float f = exp2f(m - ref), p = exp2f(__fmaf_rn(z, a.scale_log2, -ref));
            l = l * f + p;
            m = mx;
#pragma unroll
            for (int e = 0; e < E; ++e) acc[e] = acc[e] * f + p * load_as_float(static_cast<const T *>(a.v) + at + 32 * e);
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
