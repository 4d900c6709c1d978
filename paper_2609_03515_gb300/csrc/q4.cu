// Rows of K and V into and out of a cache held in 4 bits.
#include "q4.cuh"

namespace ikv {

__device__ unsigned int g_q4_error = 0;  // bit 5: rows outside a sequence's slot space

namespace {

constexpr int kMoveThreads = 256;
constexpr int kMoveRows = 4;  // rows a thread has in flight

// Where a row's channels lie.  A mma over 16 channels takes 4 of them from each lane of a quad,
// and a group's scale has to cover the whole mma; so a row is 8 units of D / 16 bytes, and unit
// u holds, for each group y, the two bytes of channels 32 y + 4 u .. + 3.  A lane of the
// attention reads two units of K or one of V in one load, and finds the same few channels of
// every group there.
// Thread p of a row's D / 8 holds channels 8 p .. 8 p + 7 as a word (its lower half belongs to
// unit 2 (p % 4), its upper half to the next); memory wants word m of the row.  to_units turns
// the first into the second among the row's threads, from_units turns it back.
template <int D>
__device__ __forceinline__ uint32_t to_units(uint32_t w) {
    constexpr int TPR = D / 8, per = D / 64;
    const int m = threadIdx.x & (TPR - 1), u = m / per, half = m % per;
    const int p = 8 * half + (u >> 1);
    const uint32_t x = __shfl_sync(0xffffffffu, w, p, TPR), y = __shfl_sync(0xffffffffu, w, p + 4, TPR);
    return __byte_perm(x, y, (u & 1) ? 0x7632 : 0x5410);
}
template <int D>
__device__ __forceinline__ uint32_t from_units(uint32_t w) {
    constexpr int TPR = D / 8, per = D / 64;
    const int p = threadIdx.x & (TPR - 1), y = p >> 2;
    const int m = 2 * (p & 3) * per + (y >> 1);
    const uint32_t lo = __shfl_sync(0xffffffffu, w, m, TPR), hi = __shfl_sync(0xffffffffu, w, m + per, TPR);
    return __byte_perm(lo, hi, (y & 1) ? 0x7632 : 0x5410);
}

// The scale of a group whose largest magnitude is a, and what its values are multiplied by
// before they are rounded.  The product with 1 / 6 may be an ulp off, the comparison that
// follows is exact (6 s has 11 bits), so s is the smallest bf16 number with 6 s >= a.
__device__ __forceinline__ uint32_t group_scale(float a) {
    uint32_t bits = __float_as_uint(a * (1.f / 6.f)) & 0xffff0000u;
    if (__uint_as_float(bits) * 6.f < a) bits += 0x10000u;
    if (a < 0x1p-120f) bits = 0u;
    return a <= 0x1p127f ? bits : 0x7fc00000u;  // (false for NaN)
}

__device__ __forceinline__ uint32_t to_codes(float lo, float hi) {  // two codes in the low byte
    uint32_t r;
    asm("{\n\t.reg .b8 b;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %1, %2;\n\tcvt.u32.u8 %0, b;\n\t}" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ uint32_t pack_codes(const float *y) {
    return to_codes(y[0], y[1]) | to_codes(y[2], y[3]) << 8 | to_codes(y[4], y[5]) << 16 | to_codes(y[6], y[7]) << 24;
}

template <typename T> struct Chunk;  // 8 channels
template <> struct Chunk<__nv_bfloat16> {
    uint4 w;
    __device__ __forceinline__ void load(const __nv_bfloat16 *p) { w = __ldcs(reinterpret_cast<const uint4 *>(p)); }
    __device__ __forceinline__ void zero() { w = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ uint32_t amax() const {  // bits of the largest magnitude, NaN above all
        const uint32_t m = 0x7fff7fffu;
        const uint32_t x = __vmaxu2(__vmaxu2(w.x & m, w.y & m), __vmaxu2(w.z & m, w.w & m));
        return max(x << 16, x & 0xffff0000u);
    }
    // |x| / s against a midpoint m: both x and m s have at most 11 bits, so they are equal or
    // 2^-11 apart, and a factor 1 + 2^-14 puts ties on the upper side and moves nothing else
    __device__ __forceinline__ uint32_t codes(float s) const {
        const float r = s > 0.f ? __frcp_rn(s) * (1.f + 0x1p-14f) : 0.f;
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
        float y[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y[2 * i] = __uint_as_float(x[i] << 16) * r;
            y[2 * i + 1] = __uint_as_float(x[i] & 0xffff0000u) * r;
        }
        return pack_codes(y);
    }
    __device__ __forceinline__ void set(const float *y) {
        uint32_t x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(y[2 * i], y[2 * i + 1]);
            x[i] = *reinterpret_cast<const uint32_t *>(&b);
        }
        w = make_uint4(x[0], x[1], x[2], x[3]);
    }
    __device__ __forceinline__ void store(__nv_bfloat16 *p) const { __stcs(reinterpret_cast<uint4 *>(p), w); }
};
template <> struct Chunk<float> {
    float4 w[2];
    __device__ __forceinline__ void load(const float *p) {
        w[0] = __ldcs(reinterpret_cast<const float4 *>(p));
        w[1] = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
    }
    __device__ __forceinline__ void zero() { w[0] = w[1] = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ uint32_t amax() const {
        const uint32_t *x = reinterpret_cast<const uint32_t *>(w);
        uint32_t a = 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i) a = max(a, x[i] & 0x7fffffffu);
        return a;
    }
    // x may lie an ulp from a midpoint: where a factor of 1 +- 2^-20, which covers the errors of
    // the reciprocal and the product, makes a difference, m s decides, which is exact
    __device__ __forceinline__ uint32_t codes(float s) const {
        const float *x = reinterpret_cast<const float *>(w);
        const float r = s > 0.f ? __frcp_rn(s) : 0.f;
        const float ru = r * (1.f + 0x1p-20f), rd = r * (1.f - 0x1p-20f);
        float y[8], z[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            y[i] = x[i] * ru;
            z[i] = x[i] * rd;
        }
        uint32_t c = pack_codes(y);
        if (c != pack_codes(z) && s > 0.f) {
            c = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float a = fabsf(x[i]);
                const uint32_t n = (a >= 0.25f * s) + (a >= 0.75f * s) + (a >= 1.25f * s) + (a >= 1.75f * s) +
                                   (a >= 2.5f * s) + (a >= 3.5f * s) + (a >= 5.f * s);
                c |= (n | (x[i] < 0.f ? 8u : 0u)) << (4 * i);
            }
        }
        return c;
    }
    __device__ __forceinline__ void set(const float *y) {
        w[0] = make_float4(y[0], y[1], y[2], y[3]);
        w[1] = make_float4(y[4], y[5], y[6], y[7]);
    }
    __device__ __forceinline__ void store(float *p) const {
        __stcs(reinterpret_cast<float4 *>(p), w[0]);
        __stcs(reinterpret_cast<float4 *>(p) + 1, w[1]);
    }
};

// The rows of a CTA: D / 8 threads a row, K and V alike, ROWS rows a thread; row r of a sequence is KV
// head r % kv_heads of its token r / kv_heads, so a CTA's dense side is one run of memory.  Bound by
// memory: all of a thread's loads, K's and V's, go out before the first is used.
template <typename T, int D, bool STORE, int ROWS>
__global__ void __launch_bounds__(kMoveThreads, 3) q4_move_kernel(const Q4MoveArgs a) {
    pdl_wait();
    constexpr int TPR = D / 8, Y = D / kQ4Group;
    const int RPP = blockDim.x / TPR;  // rows of a pass
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
    const int rows = n * G;
    if (blk * RPP * ROWS >= rows) return;
    const int p = threadIdx.x & (TPR - 1), r0 = blk * RPP * ROWS + threadIdx.x / TPR;
    const int64_t dense0 = (int64_t)li * a.rows.layer + (a.rows.row0 ? a.rows.row0[b] * a.rows.token : b * a.rows.seq) + p * 8;
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
        Chunk<T> x[2][ROWS];
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int j = 0; j < ROWS; ++j)
                if (in[j]) x[kv][j].load((kv ? dv : dk) + dense[j]);
                else x[kv][j].zero();
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
            unsigned char *codes = kv ? a.v : a.k;
            uint16_t *scales = kv ? a.vs : a.ks;
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                uint32_t m = x[kv][j].amax();
                m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
                m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
                const uint32_t s = group_scale(__uint_as_float(m));
                const uint32_t w = to_units<D>(x[kv][j].codes(__uint_as_float(s)));
                if (!in[j]) continue;
                *reinterpret_cast<uint32_t *>(codes + paged[j] * (D / 2) + p * 4) = w;
                if ((p & 3) == 0) scales[paged[j] * Y + (p >> 2)] = (uint16_t)(s >> 16);
            }
        }
    } else {
        uint32_t w[2][ROWS], s[2][ROWS];
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                w[kv][j] = in[j] ? __ldg(reinterpret_cast<const uint32_t *>((kv ? a.v : a.k) + paged[j] * (D / 2) + p * 4)) : 0u;
                s[kv][j] = in[j] ? __ldg((kv ? a.vs : a.ks) + paged[j] * Y + (p >> 2)) : 0u;
            }
#pragma unroll
        for (int kv = 0; kv < 2; ++kv)
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                const uint32_t c = from_units<D>(w[kv][j]);
                const float f = __uint_as_float(s[kv][j] << 16);
                float y[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float2 v = __half22float2(e2m1_pair(c, i));
                    y[2 * i] = v.x * f;
                    y[2 * i + 1] = v.y * f;
                }
                Chunk<T> x;
                x.set(y);
                if (in[j]) x.store((kv ? dv : dk) + dense[j]);
            }
    }
}

template <typename T, int D, bool STORE>
cudaError_t launch_move_t(Q4MoveArgs a, cudaStream_t st) {
    // single tokens: a row a thread, in CTAs no larger than a sequence's rows need
    const int64_t rows = (int64_t)a.max_count * a.pv.kv_heads;
    const bool few = rows * (D / 8) <= kMoveThreads;
    const int threads = few ? (int)((rows * (D / 8) + 31) / 32 * 32) : kMoveThreads;
    const int per = threads / (D / 8) * (few ? 1 : kMoveRows);
    a.blocks = (int)((rows + per - 1) / per);
    const int64_t ctas = (int64_t)a.blocks * a.batch * a.n_layers;
    if (ctas == 0) return cudaSuccess;
    if (ctas > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const cudaError_t e = launch_k(few ? q4_move_kernel<T, D, STORE, 1> : q4_move_kernel<T, D, STORE, kMoveRows>,
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
    if (e == cudaSuccess) e = cudaMemcpyToSymbol(g_q4_error, &z, sizeof(z));
    return e;
}

}  // namespace ikv
