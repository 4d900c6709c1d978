// Decode attention over a cache held in 4 bits.
#include "merge.cuh"
#include "q4.cuh"

namespace ikv {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kStages = 4;            // tiles a warp has in flight or in use
constexpr int kCtasPerSm = 4;
constexpr float kMaxSlack = 6.f;      // log2: how far a logit may lie above the running reference
constexpr float kScaleRoom = 256.f;   // how far a V scale may grow, normalised, before it is renormalised

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const void *src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t dst, const void *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 unpack_half(uint32_t x) { return __half22float2(*reinterpret_cast<const __half2 *>(&x)); }
// The lower term of a weight is held 2^11 times too large, so that it has its bits where the upper
// term is subnormal, and meets codes 2^-11 times too small (0.5 becomes 2^-12, a normal number).
constexpr float kLowUp = 2048.f;
__device__ __forceinline__ uint32_t shrink(uint32_t x) {
    const __half2 h = __hmul2(*reinterpret_cast<const __half2 *>(&x), __float2half2_rn(1.f / kLowUp));
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float bf16_lo(uint32_t x) { return __uint_as_float(x << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t x) { return __uint_as_float(x & 0xffff0000u); }

// One tile of a warp's ring: 16 tokens of one KV head.
template <int D>
struct Tile {
    static constexpr int kRow = D / 2, kScaleRow = D / 16;  // bytes
    unsigned char k[kQ4Tile * kRow];   // row r: token perm(r)
    unsigned char v[kQ4Tile * kRow];   // row t: token t, its 16-byte pieces swizzled
    unsigned char ks[kQ4Tile * kScaleRow], vs[kQ4Tile * kScaleRow];  // by token
    int32_t pos[kQ4Tile];
};

// A tile's row r stands for token perm(r): lane (g, t) of the second product then finds its
// four tokens t, 4 + t, 8 + t, 12 + t, whose 8-byte units lie in different banks.
__device__ __forceinline__ int perm_of_row(int r) { return ((r >> 1) & 3) + 4 * (r & 1) + 8 * (r >> 3); }
__device__ __forceinline__ int row_of_token(int t) { return 2 * (t & 3) + ((t >> 2) & 1) + 8 * (t >> 3); }

// softmax(q K^T / sqrt d) V for one (sequence, KV head), a chunk of its slots a CTA, and the
// log2-domain logits of those slots.
//
// S^T = K q^T: the tile's 16 tokens are the rows of an mma, its 8 columns the heads of the
// group (a group of 8 or fewer), 16 channels its depth.  A group of 32 channels is two of them
// and has one scale, so codes are converted to fp16 as they are (exact) and the scale
// multiplies the group's fp32 sum.  q is scaled by a power of two to [2^7, 2^8) and held in fp16
// (bf16 queries: exact down to 2^-22 of the largest; fp32 queries: two terms).
// O^T = V^T P^T: the rows are channels, the depth the 16 tokens; V's scales, which differ from
// token to token, multiply the probabilities instead, once for each group of channels, in fp32
// before they are rounded to fp16 (fp32 outputs: two terms).  Normalised by a power of two
// that follows the largest scale seen, they stay within fp16's range.
// The softmax runs on a reference that is at most 2^6 below the largest logit, so the sums are
// rescaled a few times a sequence and no tile waits for a maximum across lanes.
template <int D, typename T>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) q4_attend_kernel(const Q4AttendArgs a) {
    constexpr int Y = D / kQ4Group;        // groups of a row
    constexpr int NP = sizeof(T) == 4 ? 2 : 1;  // fp16 terms of q and of the probabilities
    constexpr int kPieces = D / 32;        // 16-byte pieces of a row of codes
    extern __shared__ __align__(128) unsigned char smem[];
    Tile<D> *ring = reinterpret_cast<Tile<D> *>(smem) + (threadIdx.x >> 5) * kStages;
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int chunk = blockIdx.x % a.n_chunks, unit = blockIdx.x / a.n_chunks;
    const int kvh = a.pv.kv_heads, b = unit / kvh, kv = unit % kvh;
    const int G = a.q_heads / kvh;
    const int L = a.len[b], S = a.pv.start_of(b);
    const int64_t head0 = (int64_t)b * a.q_heads + (int64_t)kv * G;
    // tiles of the sequence: those that hold its slots S .. S + L - 1
    const int tile0 = S / kQ4Tile;
    const int tiles = L > 0 ? (S + L + kQ4Tile - 1) / kQ4Tile - tile0 : 0;
    const int chunks = min((tiles + a.chunk_tiles - 1) / a.chunk_tiles, a.n_chunks);
    if (chunk >= max(chunks, 1)) return;
    const int first = chunk * a.chunk_tiles, last = min(first + a.chunk_tiles, tiles);  // within the sequence

    // q: lane (g, t) holds head g's channels 32 y + 8 t .. + 7
    uint32_t q[NP][Y][4];
    float post[2];  // what turns the mma's sums into log2-domain logits, heads 2 t and 2 t + 1
    {
        float x[Y][8], m = 0.f;
        const T *src = static_cast<const T *>(a.q) + (head0 + g) * D + 8 * t;
#pragma unroll
        for (int y = 0; y < Y; ++y) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[y][e] = 0.f;
            if (g < G) {
                if (NP == 1) {
                    const uint4 w = *reinterpret_cast<const uint4 *>(src + 32 * y);
                    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        x[y][2 * e] = bf16_lo(u[e]);
                        x[y][2 * e + 1] = bf16_hi(u[e]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float4 w = reinterpret_cast<const float4 *>(src + 32 * y)[e];
                        x[y][4 * e] = w.x;
                        x[y][4 * e + 1] = w.y;
                        x[y][4 * e + 2] = w.z;
                        x[y][4 * e + 3] = w.w;
                    }
                }
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) m = fmaxf(m, fabsf(x[y][e]));
        }
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
        int e = m > 0.f && m < INFINITY ? ilogbf(m) : 7;  // (7: a factor of 1)
        e = max(e, -100);
        const float up = ldexpf(1.f, 7 - e);
#pragma unroll
        for (int y = 0; y < Y; ++y)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float lo = x[y][2 * i] * up, hi = x[y][2 * i + 1] * up;
                q[0][y][i] = pack_half(lo, hi);
                if (NP == 2) {
                    const float2 f = unpack_half(q[0][y][i]);
                    q[NP - 1][y][i] = pack_half(lo - f.x, hi - f.y);
                }
            }
        const float mine = a.scale_log2 * ldexpf(1.f, e - 7);
        post[0] = __shfl_sync(0xffffffffu, mine, 8 * t);
        post[1] = __shfl_sync(0xffffffffu, mine, 8 * t + 4);
    }

    float o[2 * Y][4];  // O^T of channels 32 y + 4 g + 2 h (+ 1), heads 2 t, 2 t + 1
#pragma unroll
    for (int i = 0; i < 2 * Y; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
    float ref[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
    float norm = 1.f, room = -1.f;  // V scales times norm stay within kScaleRoom while they are <= room
    int norm_e = 0;                 // norm = 2^norm_e

    const int32_t *pos = a.pos ? a.pos + (int64_t)(a.rows_per_seq == 1 ? b : b * a.rows_per_seq + kv) * a.cap : nullptr;
    // this warp's tiles: first + warp, + kWarps, ...; lane i knows the first row of the i-th of
    // the 32 that start at base_i
    const int mine = last - first - warp > 0 ? (last - first - warp + kWarps - 1) / kWarps : 0;
    auto row_of = [&](int i) -> int64_t {  // row of the paged arrays where my tile i starts
        const int slot = (tile0 + first + warp + i * kWarps) * kQ4Tile;
        return i < mine ? a.pv.row_phys(b, a.layer, kv, slot) : 0;
    };
    int64_t my_row = row_of(lane);
    auto issue = [&](int i) {
        if (i < mine) {
            if (i > 0 && (i & 31) == 0) my_row = row_of(i + lane);
            const int64_t row = __shfl_sync(0xffffffffu, my_row, i & 31);
            Tile<D> &s = ring[i % kStages];
            const unsigned char *ks = a.k + row * Tile<D>::kRow, *vs = a.v + row * Tile<D>::kRow;
#pragma unroll
            for (int j = 0; j < kQ4Tile * kPieces / 32; ++j) {
                const int c = lane + 32 * j, tok = c / kPieces, piece = c % kPieces;
                const int swz = D == 128 ? piece ^ (tok & 2) : piece;
                copy16(smem_u32(s.k + row_of_token(tok) * Tile<D>::kRow + piece * 16), ks + c * 16);
                copy16(smem_u32(s.v + tok * Tile<D>::kRow + swz * 16), vs + c * 16);
            }
            constexpr int kScalePieces = kQ4Tile * Tile<D>::kScaleRow / 16;  // 8 or 4
            if (lane < kScalePieces)
                copy16(smem_u32(s.ks + lane * 16), reinterpret_cast<const unsigned char *>(a.ks) + row * Tile<D>::kScaleRow + lane * 16);
            else if (lane >= 8 && lane < 8 + kScalePieces)
                copy16(smem_u32(s.vs + (lane - 8) * 16), reinterpret_cast<const unsigned char *>(a.vs) + row * Tile<D>::kScaleRow + (lane - 8) * 16);
            else if (lane >= 16 && pos) {
                const int j = (tile0 + first + warp + i * kWarps) * kQ4Tile + lane - 16 - S;
                if (j >= 0 && j < L) copy4(smem_u32(s.pos + lane - 16), pos + j);
            }
        }
        copy_commit();
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) issue(i);

    const int tok0 = perm_of_row(g);  // tokens of rows g and g + 8: tok0, tok0 + 8
    for (int i = 0; i < mine; ++i) {
        copy_wait<kStages - 2>();
        __syncwarp();
        issue(i + kStages - 1);  // into the stage that the previous iteration left
        const Tile<D> &s = ring[i % kStages];
        // ---- logits
        float z[4] = {0.f, 0.f, 0.f, 0.f};
        {
            uint32_t kw[2][D / 32];  // rows g, g + 8: two units
            if (D == 128) {
                *reinterpret_cast<uint4 *>(kw[0]) = *reinterpret_cast<const uint4 *>(s.k + g * Tile<D>::kRow + t * 16);
                *reinterpret_cast<uint4 *>(kw[1]) = *reinterpret_cast<const uint4 *>(s.k + (g + 8) * Tile<D>::kRow + t * 16);
            } else {
                *reinterpret_cast<uint2 *>(kw[0]) = *reinterpret_cast<const uint2 *>(s.k + g * Tile<D>::kRow + t * 8);
                *reinterpret_cast<uint2 *>(kw[1]) = *reinterpret_cast<const uint2 *>(s.k + (g + 8) * Tile<D>::kRow + t * 8);
            }
            uint32_t sc[2][Y / 2];
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int y = 0; y < Y / 2; ++y)
                    sc[r][y] = reinterpret_cast<const uint32_t *>(s.ks + (tok0 + 8 * r) * Tile<D>::kScaleRow)[y];
#pragma unroll
            for (int y = 0; y < Y; ++y) {
                float c[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // unit 2 t + h: words h * Y / 2 ..; group y's two bytes
                    const int w = h * (Y / 2) + (y >> 1), byte = 2 * (y & 1);
                    const uint32_t f[4] = {e2m1_bits(kw[0][w], byte), e2m1_bits(kw[1][w], byte),
                                           e2m1_bits(kw[0][w], byte + 1), e2m1_bits(kw[1][w], byte + 1)};
#pragma unroll
                    for (int n = 0; n < NP; ++n) mma16816(c, f, q[n][y][2 * h], q[n][y][2 * h + 1]);
                }
                const float s0 = (y & 1) ? bf16_hi(sc[0][y >> 1]) : bf16_lo(sc[0][y >> 1]);
                const float s1 = (y & 1) ? bf16_hi(sc[1][y >> 1]) : bf16_lo(sc[1][y >> 1]);
                z[0] += s0 * c[0];
                z[1] += s0 * c[1];
                z[2] += s1 * c[2];
                z[3] += s1 * c[3];
            }
        }
        const int slot = (tile0 + first + warp + i * kWarps) * kQ4Tile + tok0 - S;  // cache slot of row g
        bool in[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int j = slot + 8 * r;
            const bool have = j >= 0 && j < L;
            in[r] = have && (!pos || s.pos[tok0 + 8 * r] >= 0);
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                z[2 * r + c] = in[r] ? z[2 * r + c] * post[c] : -INFINITY;
                if (a.logits && have && 2 * t + c < G) a.logits[(head0 + 2 * t + c) * a.lstride + j] = z[2 * r + c];
            }
        }
        // ---- running reference and sums
        if (__any_sync(0xffffffffu, fmaxf(z[0], z[2]) > ref[0] + kMaxSlack || fmaxf(z[1], z[3]) > ref[1] + kMaxSlack)) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float m = fmaxf(z[c], z[2 + c]);
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
                m = fmaxf(m, ref[c]);
                const float f = ref[c] == m ? 1.f : exp2f(ref[c] - m);
                ref[c] = m;
                sum[c] *= f;
#pragma unroll
                for (int j = 0; j < 2 * Y; ++j) {
                    o[j][c] *= f;
                    o[j][2 + c] *= f;
                }
            }
        }
        float p[4];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const float m = ref[c] == -INFINITY ? 0.f : ref[c];
            p[c] = exp2f(z[c] - m);
            p[2 + c] = exp2f(z[2 + c] - m);
            sum[c] += p[c] + p[2 + c];
        }
        // ---- V scales of rows g and g + 8 (0 where the slot is none of the sequence's, whatever it holds)
        float vs[2][Y], big = 0.f;
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int y = 0; y < Y / 2; ++y) {
                const uint32_t w = in[r] ? reinterpret_cast<const uint32_t *>(s.vs + (tok0 + 8 * r) * Tile<D>::kScaleRow)[y] : 0u;
                vs[r][2 * y] = bf16_lo(w);
                vs[r][2 * y + 1] = bf16_hi(w);
                big = fmaxf(big, fmaxf(vs[r][2 * y], vs[r][2 * y + 1]));
            }
        if (__any_sync(0xffffffffu, big > room)) {
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
            int e = norm_e;
            if (big > 0.f) e = 4 - max(ilogbf(big), -120);
            const float f = room < 0.f ? 1.f : ldexpf(1.f, e - norm_e);  // (nothing summed before the first)
            norm_e = e;
            norm = ldexpf(1.f, e);
            room = big > 0.f ? kScaleRoom * ldexpf(1.f, -e) : 0.f;
#pragma unroll
            for (int j = 0; j < 2 * Y; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) o[j][c] *= f;
        }
        // ---- outputs
        uint32_t vw[4][Y / 2];  // unit g of tokens t, 4 + t, 8 + t, 12 + t
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const unsigned char *row = s.v + (4 * j + t) * Tile<D>::kRow;
            if (D == 128)
                *reinterpret_cast<uint2 *>(vw[j]) = *reinterpret_cast<const uint2 *>(row + (((g >> 1) ^ (t & 2)) << 4) + ((g & 1) << 3));
            else
                vw[j][0] = *reinterpret_cast<const uint32_t *>(row + g * 4);
        }
#pragma unroll
        for (int y2 = 0; y2 < Y / 2; ++y2) {
            // bytes with a channel's codes of two tokens: the even channels, the odd ones
            uint32_t x[2][2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t u = vw[2 * j][y2], w = vw[2 * j + 1][y2];
                x[j][0] = (u & 0x0f0f0f0fu) | ((w << 4) & 0xf0f0f0f0u);
                x[j][1] = ((u >> 4) & 0x0f0f0f0fu) | (w & 0xf0f0f0f0u);
            }
#pragma unroll
            for (int yy = 0; yy < 2; ++yy) {
                const int y = 2 * y2 + yy;
                uint32_t bf[NP][2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const float f = vs[r][y] * norm;
                    const float w0 = p[2 * r] * f, w1 = p[2 * r + 1] * f;
                    const uint32_t w = pack_half(w0, w1);
                    bf[0][r] = transpose8x8(w);
                    if (NP == 2) {
                        const float2 back = unpack_half(w);
                        bf[NP - 1][r] = transpose8x8(pack_half((w0 - back.x) * kLowUp, (w1 - back.y) * kLowUp));
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int byte = 2 * yy + h;
                    const uint32_t f[4] = {e2m1_bits(x[0][0], byte), e2m1_bits(x[0][1], byte), e2m1_bits(x[1][0], byte),
                                           e2m1_bits(x[1][1], byte)};
                    mma16816(o[2 * y + h], f, bf[0][0], bf[0][1]);
                    if (NP == 2) {
                        const uint32_t low[4] = {shrink(f[0]), shrink(f[1]), shrink(f[2]), shrink(f[3])};
                        mma16816(o[2 * y + h], low, bf[NP - 1][0], bf[NP - 1][1]);
                    }
                }
            }
        }
    }
    copy_wait<0>();

    // ---- the warps' results joined: (reference, sum) and outputs through shared memory
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum[c] += __shfl_xor_sync(0xffffffffu, sum[c], d);
    __syncthreads();  // every ring is done with
    float2 *ml = reinterpret_cast<float2 *>(smem);                          // [kWarps][8]
    float *po = reinterpret_cast<float *>(smem + kWarps * 8 * sizeof(float2));  // [kWarps][8][D]
    const float back = ldexpf(1.f, -norm_e);
    if (g == 0) {
        ml[warp * 8 + 2 * t] = make_float2(ref[0], sum[0]);
        ml[warp * 8 + 2 * t + 1] = make_float2(ref[1], sum[1]);
    }
#pragma unroll
    for (int y = 0; y < Y; ++y)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int c = 0; c < 2; ++c)
                *reinterpret_cast<float2 *>(po + (warp * 8 + 2 * t + c) * D + 32 * y + 4 * g + 2 * h) =
                    make_float2(o[2 * y + h][c] * back, o[2 * y + h][2 + c] * back);
    __syncthreads();
    for (int i = threadIdx.x; i < G * (D / 4); i += kThreads) {
        const int h = i / (D / 4), e = i % (D / 4) * 4;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) m = fmaxf(m, ml[w * 8 + h].x);
        const float base = m == -INFINITY ? 0.f : m;
        float l = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float2 y = ml[w * 8 + h];
            const float f = exp2f(y.x - base);
            const float4 v = *reinterpret_cast<const float4 *>(po + (w * 8 + h) * D + e);
            l += f * y.y;
            x.x += f * v.x;
            x.y += f * v.y;
            x.z += f * v.z;
            x.w += f * v.w;
        }
        const int64_t head = head0 + h;
        if (chunks <= 1) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            T *dst = static_cast<T *>(a.out) + head * D + e;
            store_as(dst, x.x * inv);
            store_as(dst + 1, x.y * inv);
            store_as(dst + 2, x.z * inv);
            store_as(dst + 3, x.w * inv);
            if (e == 0) a.lse2[head] = l == 0.f ? -INFINITY : m + log2f(l);
        } else {
            const int64_t at = head * a.n_chunks + chunk;
            *reinterpret_cast<float4 *>(a.part_o + at * D + e) = x;
            if (e == 0) reinterpret_cast<float2 *>(a.part_ml)[at] = make_float2(m, l);
        }
    }
}

template <int D, typename T>
cudaError_t launch_t(const Q4AttendArgs &a, cudaStream_t st) {
    constexpr size_t ring = sizeof(Tile<D>) * kStages * kWarps;
    constexpr size_t join = kWarps * 8 * (sizeof(float2) + D * sizeof(float));
    constexpr size_t smem = ring > join ? ring : join;
    static_assert(smem <= 48 << 10, "more shared memory needs an attribute");
    const int64_t ctas = (int64_t)a.batch * a.pv.kv_heads * a.n_chunks;
    if (ctas > 0x7fffffff) return cudaErrorInvalidConfiguration;
    const cudaError_t e = launch_k(q4_attend_kernel<D, T>, dim3((unsigned)ctas), dim3(kThreads), smem, st, a);
    note_launch();
    return e;
}

}  // namespace

// The chunk count that finishes first when the CTAs run in whole waves: waves x tiles of a
// chunk, plus what a CTA costs besides (its ramp and join, as tiles).
void q4_attend_plan(const ikv_shape *s, int32_t max_len, int sms, int32_t *chunk_tiles, int32_t *n_chunks) {
    // a start offset may put the first slot anywhere in its tile
    const int64_t tiles = max_len > 0 ? ((int64_t)max_len + 2 * kQ4Tile - 2) / kQ4Tile : 1;
    const int64_t units = (int64_t)s->batch * s->kv_heads, slots = (int64_t)sms * kCtasPerSm;
    int64_t best = INT64_MAX, best_tiles = tiles;
    for (int64_t n = 1; n <= kMaxSplits && n <= tiles; ++n) {
        const int64_t per = ((tiles + n - 1) / n + kWarps - 1) / kWarps * kWarps;
        const int64_t used = (tiles + per - 1) / per;
        const int64_t waves = (units * used + slots - 1) / slots;
        const int64_t cost = waves * (per + 8) + (used > 1 ? 8 : 0);
        if (cost < best) {
            best = cost;
            best_tiles = per;
        }
    }
    *chunk_tiles = (int32_t)best_tiles;
    *n_chunks = (int32_t)((tiles + best_tiles - 1) / best_tiles);
}

cudaError_t launch_q4_attend(const Q4AttendArgs &a, int dtype, int head_dim, cudaStream_t st) {
    if (dtype == IKV_BF16)
        return head_dim == 128 ? launch_t<128, __nv_bfloat16>(a, st) : launch_t<64, __nv_bfloat16>(a, st);
    return head_dim == 128 ? launch_t<128, float>(a, st) : launch_t<64, float>(a, st);
}

}  // namespace ikv
