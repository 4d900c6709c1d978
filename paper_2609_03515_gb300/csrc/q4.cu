// Rows of K and V into and out of a cache held in 4 bits.
#include "q4.cuh"

namespace ikv {

__device__ unsigned int g_q4_error = 0;  // bit 5: rows outside a sequence's slot space; bit 8: outside those granted

namespace {

constexpr int kMoveThreads = 256;

// Where a row's channels lie.  A mma over 16 channels takes 4 of them from each lane of a quad,
// and a group's scale has to cover the whole mma; so a row is 8 units of D / 16 bytes, and unit
// u holds, for each group y, the two bytes of channels 32 y + 4 u .. + 3.  A lane of the
// attention reads two units of K or one of V in one load, and finds the same few channels of
// every group there.  Here 8 threads take a row, a unit each: on the dense side that is D / 32
// runs of 4 channels, 64 or 128 bytes for the eight of them, and nothing has to change lanes.
constexpr int kUnits = 8;

// The scale of a group whose largest magnitude is a, and what its values are multiplied by
// before they are rounded.  The product with 1 / 6 may be an ulp off, the comparison that
// follows is exact (6 s has 11 bits), so s is the smallest bf16 number with 6 s >= a.
__device__ __forceinline__ uint32_t group_scale(float a) {
    uint32_t bits = __float_as_uint(a * (1.f / 6.f)) & 0xffff0000u;
    if (__uint_as_float(bits) * 6.f < a) bits += 0x10000u;
    if (a < 0x1p-120f) bits = 0u;
    return a <= 0x1p127f ? bits : 0x7fc00000u;  // (false for NaN)
}

// Eight codes, the first in the lowest bits.
__device__ __forceinline__ uint32_t to_codes(const float2 (&y)[4]) {
    uint32_t r;
    asm("{\n\t.reg .b8 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
        "mov.b32 %0, {a, b, c, d};\n\t}"
        : "=r"(r) : "f"(y[0].x), "f"(y[0].y), "f"(y[1].x), "f"(y[1].y), "f"(y[2].x), "f"(y[2].y), "f"(y[3].x), "f"(y[3].y));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float f) {  // both at once
    uint64_t r;
    asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%1, %2};\n\tmov.b64 y, {%3, %3};\n\tmul.rn.f32x2 %0, x, y;\n\t}"
        : "=l"(r) : "f"(a.x), "f"(a.y), "f"(f));
    return make_float2(__uint_as_float((uint32_t)r), __uint_as_float((uint32_t)(r >> 32)));
}
// 1 / s to an ulp or two
__device__ __forceinline__ float inverse(float s) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(s));
    return s > 0.f ? r : 0.f;
}

// 4 channels of a row; two of them (groups y and y + 1) make a word of codes.
template <typename T> struct Quad;
template <> struct Quad<__nv_bfloat16> {
    uint2 w;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { w = __ldcs(reinterpret_cast<const uint2 *>(p)); }
    __device__ __forceinline__ void zero() { w = make_uint2(0u, 0u); }
    static __device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) {  // of two pairs of magnitudes, or NaN
        const __nv_bfloat162 r = __hmax2_nan(__habs2(*reinterpret_cast<const __nv_bfloat162 *>(&a)),
                                             __habs2(*reinterpret_cast<const __nv_bfloat162 *>(&b)));
        return *reinterpret_cast<const uint32_t *>(&r);
    }
    // the largest magnitudes of two groups over the row's threads (bits of a float; NaN above all)
    static __device__ __forceinline__ void amax2(const Quad &a, const Quad &b, uint32_t &m0, uint32_t &m1) {
        const uint32_t x = larger(a.w.x, a.w.y), y = larger(b.w.x, b.w.y);
        uint32_t two = larger(__byte_perm(x, y, 0x5410), __byte_perm(x, y, 0x7632));
#pragma unroll
        for (int d = 1; d < kUnits; d <<= 1) two = larger(two, __shfl_xor_sync(0xffffffffu, two, d));
        m0 = two << 16;
        m1 = two & 0xffff0000u;
    }
    // |x| / s against a midpoint m: both x and m s have at most 11 bits, so they are equal or
    // 2^-11 apart, and a factor 1 + 2^-14 puts ties on the upper side and moves nothing else
    static __device__ __forceinline__ uint32_t codes2(const Quad &a, const Quad &b, float, float, float r0, float r1) {
        r0 *= 1.f + 0x1p-14f;
        r1 *= 1.f + 0x1p-14f;
        auto both = [](uint32_t x) { return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)); };
        const float2 y[4] = {mul2(both(a.w.x), r0), mul2(both(a.w.y), r0), mul2(both(b.w.x), r1), mul2(both(b.w.y), r1)};
        return to_codes(y);
    }
    static __device__ __forceinline__ void store(__nv_bfloat16 *p, float2 a, float2 b) {
        const __nv_bfloat162 x = __floats2bfloat162_rn(a.x, a.y), y = __floats2bfloat162_rn(b.x, b.y);
        __stcs(reinterpret_cast<uint2 *>(p),
               make_uint2(*reinterpret_cast<const uint32_t *>(&x), *reinterpret_cast<const uint32_t *>(&y)));
    }
};
template <> struct Quad<float> {
    float4 w;
    __device__ __forceinline__ void load(const float *p) { w = __ldcs(reinterpret_cast<const float4 *>(p)); }
    __device__ __forceinline__ void zero() { w = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ uint32_t amax() const {
        const uint32_t m = 0x7fffffffu;
        return max(max(__float_as_uint(w.x) & m, __float_as_uint(w.y) & m), max(__float_as_uint(w.z) & m, __float_as_uint(w.w) & m));
    }
    static __device__ __forceinline__ void amax2(const Quad &a, const Quad &b, uint32_t &m0, uint32_t &m1) {
        m0 = a.amax();
        m1 = b.amax();
#pragma unroll
        for (int d = 1; d < kUnits; d <<= 1) {
            m0 = max(m0, __shfl_xor_sync(0xffffffffu, m0, d));
            m1 = max(m1, __shfl_xor_sync(0xffffffffu, m1, d));
        }
    }
    // x may lie an ulp from a midpoint: where a factor of 1 +- 2^-20, which covers the errors of
    // the reciprocal and the product, makes a difference, m s decides, which is exact
    static __device__ __forceinline__ uint32_t codes2(const Quad &a, const Quad &b, float s0, float s1, float r0, float r1) {
        const float4 p = a.w, q = b.w;
        auto all = [&](float f) {
            const float2 y[4] = {mul2(make_float2(p.x, p.y), r0 * f), mul2(make_float2(p.z, p.w), r0 * f),
                                 mul2(make_float2(q.x, q.y), r1 * f), mul2(make_float2(q.z, q.w), r1 * f)};
            return to_codes(y);
        };
        uint32_t c = all(1.f + 0x1p-20f);
        const uint32_t differ = c ^ all(1.f - 0x1p-20f);
        if (differ) {
            const float x[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = fabsf(x[i]), s = i < 4 ? s0 : s1;
                const uint32_t n = (v >= 0.25f * s) + (v >= 0.75f * s) + (v >= 1.25f * s) + (v >= 1.75f * s) +
                                   (v >= 2.5f * s) + (v >= 3.5f * s) + (v >= 5.f * s);
                if (differ >> (4 * i) & 15u) c = (c & ~(15u << (4 * i))) | (n | (x[i] < 0.f ? 8u : 0u)) << (4 * i);
            }
        }
        return c;
    }
    static __device__ __forceinline__ void store(float *p, float2 a, float2 b) {
        __stcs(reinterpret_cast<float4 *>(p), make_float4(a.x, a.y, b.x, b.y));
    }
};

// The rows of a CTA, K and V alike, ROWS rows a thread; row r of a sequence is KV head r % kv_heads of
// its token r / kv_heads, so a CTA's dense side is one run of memory.  All of a thread's loads, K's and
// V's, go out before the first is used.  Four layers of a 32k prompt of 8 heads of 128 (688 MB each
// way): stored in 120 us (5.7 TB/s; 80 % of the issue slots), loaded in 103 (6.7 TB/s, memory).
// A row of 16 threads with its words exchanged between them took 150 and 127.
template <typename T, int D, bool STORE, int ROWS>
__global__ void __launch_bounds__(kMoveThreads, 3) q4_move_kernel(const Q4MoveArgs a) {
    pdl_wait();
    constexpr int Y = D / kQ4Group;
    const int RPP = blockDim.x / kUnits;  // rows of a pass
    const int blk = blockIdx.x % a.blocks, lb = blockIdx.x / a.blocks;
    const int b = lb % a.batch, li = lb / a.batch;
    const int G = a.pv.kv_heads;
    int n = min(a.count ? a.count[b] : a.max_count, a.max_count);
    int first;
    if (a.first) {
        first = a.first[b];
        if (first < 0) return;  // no rows of this sequence
    } else {
        n = min(n, a.len[b]);
        first = a.len[b] - n;
    }
    if (n <= 0) return;
    const int S = a.pv.start_of(b);
    if (first > a.cap - S - n) {
        if (threadIdx.x == 0) atomicOr(&g_q4_error, 32u);
        return;
    }
    if (STORE && a.writable) {
        const int lo = a.writable[2 * b], hi = a.writable[2 * b + 1];
        if (first < lo || first + n > hi) {
            if (threadIdx.x == 0 && lo < hi) atomicOr(&g_q4_error, 256u);
            return;
        }
    }
    const int rows = n * G;
    if (blk * RPP * ROWS >= rows) return;
    const int u = threadIdx.x & (kUnits - 1), r0 = blk * RPP * ROWS + threadIdx.x / kUnits;
    const int64_t dense0 = (int64_t)li * a.rows.layer + (a.rows.row0 ? a.rows.row0[b] * a.rows.token : b * a.rows.seq) + u * 4;
    T *dk = static_cast<T *>(a.rows.k) + dense0, *dv = static_cast<T *>(a.rows.v) + dense0;
    int64_t dense[ROWS], paged[ROWS];
    bool in[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int r = r0 + j * RPP;
        in[j] = r < rows;
        const int i = in[j] ? (a.head_shift >= 0 ? r >> a.head_shift : r / G) : 0, g = in[j] ? r - i * G : 0;
        dense[j] = i * a.rows.token + g * a.rows.head;
        paged[j] = a.pv.row_phys(b, a.layer0 + li, g, S + first + i);
    }
    if (STORE) {
        Quad<T> x[2][ROWS][Y];
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int j = 0; j < ROWS; ++j)
#pragma unroll
                for (int y = 0; y < Y; ++y)
                    if (in[j]) x[kv][j][y].load((kv ? dv : dk) + dense[j] + y * kQ4Group);
                    else x[kv][j][y].zero();
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            unsigned char *codes = kv ? a.v : a.k;
            uint16_t *scales = kv ? a.vs : a.ks;
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                uint32_t m[Y];
#pragma unroll
                for (int y = 0; y < Y; y += 2) Quad<T>::amax2(x[kv][j][y], x[kv][j][y + 1], m[y], m[y + 1]);
                // thread u works out group u % Y's scale for all
                uint32_t mine = m[0];
#pragma unroll
                for (int y = 1; y < Y; ++y)
                    if (u % Y == y) mine = m[y];
                const uint32_t s_mine = group_scale(__uint_as_float(mine));
                const float r_mine = inverse(__uint_as_float(s_mine));
                uint32_t c[Y / 2];
#pragma unroll
                for (int y = 0; y < Y; y += 2) {
                    float s[2] = {0.f, 0.f}, r[2];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        if (sizeof(T) == 4) s[i] = __uint_as_float(__shfl_sync(0xffffffffu, s_mine, y + i, kUnits));
                        r[i] = __shfl_sync(0xffffffffu, r_mine, y + i, kUnits);
                    }
                    c[y / 2] = Quad<T>::codes2(x[kv][j][y], x[kv][j][y + 1], s[0], s[1], r[0], r[1]);
                }
                if (!in[j]) continue;
                unsigned char *to = codes + paged[j] * (D / 2) + u * (D / 16);
                if (Y == 4) *reinterpret_cast<uint2 *>(to) = make_uint2(c[0], c[Y / 2 - 1]);
                else *reinterpret_cast<uint32_t *>(to) = c[0];
                if (u < Y) scales[paged[j] * Y + u] = (uint16_t)(s_mine >> 16);
            }
        }
    } else {
        uint32_t w[2][ROWS][Y / 2], s[2][ROWS][Y / 2];
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                const unsigned char *c = (kv ? a.v : a.k) + paged[j] * (D / 2) + u * (D / 16);
                const uint16_t *f = (kv ? a.vs : a.ks) + paged[j] * Y;
                if (Y == 4) {
                    const uint2 x = in[j] ? __ldg(reinterpret_cast<const uint2 *>(c)) : make_uint2(0u, 0u);
                    const uint2 z = in[j] ? __ldg(reinterpret_cast<const uint2 *>(f)) : make_uint2(0u, 0u);
                    w[kv][j][0] = x.x;
                    w[kv][j][Y / 2 - 1] = x.y;
                    s[kv][j][0] = z.x;
                    s[kv][j][Y / 2 - 1] = z.y;
                } else {
                    w[kv][j][0] = in[j] ? __ldg(reinterpret_cast<const uint32_t *>(c)) : 0u;
                    s[kv][j][0] = in[j] ? __ldg(reinterpret_cast<const uint32_t *>(f)) : 0u;
                }
            }
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                if (!in[j]) continue;
                T *to = (kv ? dv : dk) + dense[j];
#pragma unroll
                for (int y = 0; y < Y; ++y) {
                    const uint32_t x = s[kv][j][y >> 1];
                    const float f = __uint_as_float((y & 1) ? x & 0xffff0000u : x << 16);
                    float2 p = __half22float2(e2m1_pair(w[kv][j][y >> 1], 2 * (y & 1)));
                    float2 q = __half22float2(e2m1_pair(w[kv][j][y >> 1], 2 * (y & 1) + 1));
                    Quad<T>::store(to + y * kQ4Group, make_float2(p.x * f, p.y * f), make_float2(q.x * f, q.y * f));
                }
            }
    }
}

template <typename T, int D, bool STORE>
cudaError_t launch_move_t(Q4MoveArgs a, cudaStream_t st) {
    // rows a thread: as many as their registers allow
    constexpr int kRows = !STORE ? 4 : (sizeof(T) * D <= 128 ? 4 : sizeof(T) * D <= 256 ? 2 : 1);
    // single tokens: a row a thread, in CTAs no larger than a sequence's rows need
    const int64_t rows = (int64_t)a.max_count * a.pv.kv_heads;
    const bool few = rows * kUnits <= kMoveThreads;
    const int threads = few ? (int)((rows * kUnits + 31) / 32 * 32) : kMoveThreads;
    const int per = threads / kUnits * (few ? 1 : kRows);
    a.blocks = (int)((rows + per - 1) / per);
    const int64_t ctas = (int64_t)a.blocks * a.batch * a.n_layers;
    if (ctas == 0) return cudaSuccess;
    if (ctas > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const cudaError_t e = launch_k(few ? q4_move_kernel<T, D, STORE, 1> : q4_move_kernel<T, D, STORE, kRows>,
                                   dim3((unsigned)ctas), dim3(threads), 0, st, a);
    note_launch();
    return e;
}
template <bool STORE>
cudaError_t launch_move(const Q4MoveArgs &a, int dtype, cudaStream_t st) {
    const bool wide = a.pv.head_dim == 128;
    if (dtype == IKV_BF16)
        return wide ? launch_move_t<__nv_bfloat16, 128, STORE>(a, st) : launch_move_t<__nv_bfloat16, 64, STORE>(a, st);
    return wide ? launch_move_t<float, 128, STORE>(a, st) : launch_move_t<float, 64, STORE>(a, st);
}

}  // namespace

cudaError_t launch_q4_store(const Q4MoveArgs &a, int dtype, cudaStream_t st) { return launch_move<true>(a, dtype, st); }
cudaError_t launch_q4_load(const Q4MoveArgs &a, int dtype, cudaStream_t st) { return launch_move<false>(a, dtype, st); }

cudaError_t read_clear_q4_error(unsigned int *v) {
    unsigned int z = 0;
    cudaError_t e = cudaMemcpyFromSymbol(v, g_q4_error, sizeof(*v));
    if (e == cudaSuccess && *v) e = cudaMemcpyToSymbol(g_q4_error, &z, sizeof(z));
    return e;
}

}  // namespace ikv
