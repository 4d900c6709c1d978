// Decode attention over a cache held in 4 bits.
#include <cfloat>
#include <cstddef>
#include <type_traits>

#include "merge.cuh"
#include "q4.cuh"

namespace ikv {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kPair = 2;              // tiles of an iteration
constexpr int kStages = 3;            // pairs of tiles a warp has in flight or in use
constexpr int kCtasPerSm = 3;
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
__device__ __forceinline__ void mma16816_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ float exp2_fast(float x) {  // results below 2^-126 are 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float r;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
    return r;
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

// How the work is cut.  A unit (sequence, KV head) is rounds of kRound slots, counted from the tile
// that holds its first slot; the units' rounds, one unit behind another, are dealt to the CTAs in
// equal runs of `per`, so a batch of uneven lengths loads them evenly, and a CTA's run is one or
// more segments, each of one unit.  A unit's n segments leave partials 0 .. n - 1.  Everything
// follows from the lengths on the device; each kernel works it out for itself.
constexpr int kRoundTiles = kWarps * kPair, kRound = kRoundTiles * kQ4Tile;
struct Span {  // of a sequence
    int tile0, tiles, rounds;
};
__device__ __forceinline__ Span span_of(int L, int S) {
    Span s;
    s.tile0 = S / kQ4Tile;
    s.tiles = L > 0 ? (S + L + kQ4Tile - 1) / kQ4Tile - s.tile0 : 0;
    s.rounds = (s.tiles + kRoundTiles - 1) / kRoundTiles;
    return s;
}
struct Deal {
    int64_t per;     // rounds of a CTA
    int64_t before;  // rounds (of one KV head) of the sequences in front of one
};
// The deal to `ctas` CTAs, and for the sequence that `pick` finds, given the rounds in front of a
// sequence, its own and per (true for one sequence at most): its number, through *found (-1: none).
// All threads of the CTA; each takes a run of sequences.
template <int NT, typename Pick>
__device__ __forceinline__ Deal deal_rounds(const int32_t *len, const int32_t *start, int batch, int kv_heads, int ctas,
                                            Pick pick, int *found) {
    __shared__ int64_t sums[NT / 32];
    __shared__ int tops[NT / 32];
    __shared__ int64_t s_before;
    __shared__ int s_found;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int run = (batch + NT - 1) / NT, b0 = threadIdx.x * run, b1 = min(b0 + run, batch);
    int64_t mine = 0;
    int top = 0;
    for (int b = b0; b < b1; ++b) {
        const int r = span_of(len[b], start ? start[b] : 0).rounds;
        mine += r;
        top = max(top, r);
    }
    int64_t scan = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, scan, d);
        if (lane >= d) scan += y;
        top = max(top, __shfl_xor_sync(0xffffffffu, top, d));
    }
    if (threadIdx.x == 0) s_found = -1;
    if (lane == 31) {
        sums[warp] = scan;
        tops[warp] = top;
    }
    __syncthreads();
    int64_t total = 0, base = scan - mine;
#pragma unroll
    for (int w = 0; w < NT / 32; ++w) {
        if (w < warp) base += sums[w];
        total += sums[w];
        top = max(top, tops[w]);
    }
    Deal deal;
    // (a unit is cut into kMaxSplits segments at most: two of them may be parts of a run)
    deal.per = max(max((total * kv_heads + ctas - 1) / ctas, ((int64_t)top + kMaxSplits - 3) / (kMaxSplits - 2)), (int64_t)1);
    for (int b = b0; b < b1; ++b) {
        const int r = span_of(len[b], start ? start[b] : 0).rounds;
        if (pick(b, base, r, deal.per)) {
            s_before = base;
            s_found = b;
        }
        base += r;
    }
    __syncthreads();
    *found = s_found;
    deal.before = s_before;
    return deal;
}

// softmax(q K^T / sqrt d) V for a CTA's segments, and the log2-domain logits of their slots.
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
template <int D, typename T, bool SCORE>
__global__ void __launch_bounds__(kThreads, kCtasPerSm) q4_attend_kernel(const Q4AttendArgs a) {
    constexpr int Y = D / kQ4Group;        // groups of a row
    constexpr int NP = sizeof(T) == 4 ? 2 : 1;  // fp16 terms of q and of the probabilities
    constexpr int kPieces = D / 32;        // 16-byte pieces of a row of codes
    extern __shared__ __align__(128) unsigned char smem[];
    Tile<D> *ring = reinterpret_cast<Tile<D> *>(smem) + (threadIdx.x >> 5) * (kStages * kPair);
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int kvh = a.pv.kv_heads;
    const int G = a.q_heads / kvh;
    int b;
    int64_t at = 0;  // the run starts at this round
    const Deal deal = deal_rounds<kThreads>(a.len, a.pv.start, a.batch, kvh, (int)gridDim.x,
        [&](int, int64_t before, int rounds, int64_t per) {
            const int64_t x = blockIdx.x * per;
            return x >= before * kvh && x < (before + rounds) * kvh;
        }, &b);
    if (b < 0) return;  // past the last round
    at = blockIdx.x * deal.per - deal.before * kvh;  // within the sequence's units
    int64_t before = deal.before, left = deal.per;
    Span sp = span_of(a.len[b], a.pv.start_of(b));
    int kv = (int)(at / sp.rounds), round = (int)(at % sp.rounds);
    while (left > 0) {
    const int L = a.len[b], S = a.pv.start_of(b);
    const int64_t head0 = (int64_t)b * a.q_heads + (int64_t)kv * G;
    const int tile0 = sp.tile0, take = (int)min((int64_t)(sp.rounds - round), left);
    const int first = round * kRoundTiles, last = min(first + take * kRoundTiles, sp.tiles);  // tiles of the sequence
    // the unit's segments: the runs that its rounds lie in
    const int64_t unit0 = before * kvh + (int64_t)kv * sp.rounds;
    const int seg0 = (int)(unit0 / deal.per), segs = (int)((unit0 + sp.rounds - 1) / deal.per) - seg0 + 1;

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
    float ref[2] = {-FLT_MAX, -FLT_MAX}, sum[2] = {0.f, 0.f};
    float norm = 1.f, room = -1.f;  // V scales times norm stay within kScaleRoom while they are <= room
    int norm_e = 0;                 // norm = 2^norm_e

    const int32_t *pos = a.pos ? a.pos + (int64_t)(a.rows_per_seq == 1 ? b : b * a.rows_per_seq + kv) * a.cap : nullptr;
    // this warp's pairs of tiles: first / 2 + warp, + kWarps, ...; lane i knows where the i-th of
    // the 32 tiles from base on start
    const int pairs = (last - first + kPair - 1) / kPair;
    const int mine = pairs > warp ? (pairs - warp + kWarps - 1) / kWarps : 0;
    auto tile_of = [&](int i) { return first + ((i >> 1) * kWarps + warp) * kPair + (i & 1); };  // my i-th tile
    auto row_of = [&](int i) -> int64_t {  // row of the paged arrays where it starts
        const int x = tile_of(i);
        return x < last ? a.pv.row_phys(b, a.layer, kv, (tile0 + x) * kQ4Tile) : 0;
    };
    int64_t my_row = row_of(lane);
    // where a lane's pieces of a tile go: K's rows permuted, V's pieces swizzled
    constexpr int kCopies = kQ4Tile * kPieces / 32;
    constexpr int kScalePieces = kQ4Tile * Tile<D>::kScaleRow / 16;  // 8 or 4
    const uint32_t ring_at = smem_u32(ring);
    uint32_t to_k[kCopies], to_v[kCopies];
#pragma unroll
    for (int j = 0; j < kCopies; ++j) {
        const int c = lane + 32 * j, tok = c / kPieces, piece = c % kPieces;
        to_k[j] = offsetof(Tile<D>, k) + row_of_token(tok) * Tile<D>::kRow + piece * 16;
        to_v[j] = offsetof(Tile<D>, v) + tok * Tile<D>::kRow + (D == 128 ? piece ^ (tok & 2) : piece) * 16;
    }
    const unsigned char *scales = reinterpret_cast<const unsigned char *>(lane < 8 ? a.ks : a.vs) + (lane & 7) * 16;
    const uint32_t to_s = (lane < 8 ? offsetof(Tile<D>, ks) : offsetof(Tile<D>, vs)) + (lane & 7) * 16;
    auto issue = [&](int i, uint32_t stage) {
        if (i < mine) {
            if (i > 0 && (i & 15) == 0) my_row = row_of(2 * i + lane);
#pragma unroll
            for (int u = 0; u < kPair; ++u) {
                const int64_t row = __shfl_sync(0xffffffffu, my_row, (2 * i + u) & 31);
                const uint32_t dst = stage + u * sizeof(Tile<D>);
                if (u > 0 && tile_of(2 * i + u) >= last) break;
                const unsigned char *ks = a.k + row * Tile<D>::kRow + lane * 16, *vs = a.v + row * Tile<D>::kRow + lane * 16;
#pragma unroll
                for (int j = 0; j < kCopies; ++j) {
                    copy16(dst + to_k[j], ks + j * 512);
                    copy16(dst + to_v[j], vs + j * 512);
                }
                if ((lane & 7) < kScalePieces && lane < 16) copy16(dst + to_s, scales + row * Tile<D>::kScaleRow);
                else if (lane >= 16 && pos) {
                    const int j = (tile0 + tile_of(2 * i + u)) * kQ4Tile + lane - 16 - S;
                    if (j >= 0 && j < L) copy4(dst + offsetof(Tile<D>, pos) + (lane - 16) * 4, pos + j);
                }
            }
        }
        copy_commit();
    };
    constexpr uint32_t kStageBytes = kPair * sizeof(Tile<D>);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) issue(i, ring_at + i * kStageBytes);

    const int tok0 = perm_of_row(g);  // tokens of rows g and g + 8: tok0, tok0 + 8
    // One pair of tiles; MASK: some of its slots are not the sequence's, or dead
    auto pair_step = [&](const Tile<D> *tiles, int slot0, auto mask_tag) {
        constexpr bool MASK = decltype(mask_tag)::value;
        // ---- logits
        float z[kPair][4];
        bool in[kPair][2];
#pragma unroll
        for (int u = 0; u < kPair; ++u) {
            const Tile<D> &s = tiles[u];
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
                float c[4];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // unit 2 t + h: words h * Y / 2 ..; group y's two bytes
                    const int w = h * (Y / 2) + (y >> 1), byte = 2 * (y & 1);
                    const uint32_t f[4] = {e2m1_bits(kw[0][w], byte), e2m1_bits(kw[1][w], byte),
                                           e2m1_bits(kw[0][w], byte + 1), e2m1_bits(kw[1][w], byte + 1)};
#pragma unroll
                    for (int n = 0; n < NP; ++n)
                        if (h == 0 && n == 0) mma16816_first(c, f, q[n][y][2 * h], q[n][y][2 * h + 1]);
                        else mma16816(c, f, q[n][y][2 * h], q[n][y][2 * h + 1]);
                }
                const float s0 = (y & 1) ? bf16_hi(sc[0][y >> 1]) : bf16_lo(sc[0][y >> 1]);
                const float s1 = (y & 1) ? bf16_hi(sc[1][y >> 1]) : bf16_lo(sc[1][y >> 1]);
#pragma unroll
                for (int e = 0; e < 4; ++e) z[u][e] = y == 0 ? (e < 2 ? s0 : s1) * c[e] : z[u][e] + (e < 2 ? s0 : s1) * c[e];
            }
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int j = slot0 + u * kQ4Tile + 8 * r + tok0;  // cache slot of row g + 8 r
                const bool have = !MASK || (j >= 0 && j < L);
                in[u][r] = have && (!MASK || !pos || s.pos[tok0 + 8 * r] >= 0);
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    z[u][2 * r + c] = in[u][r] ? z[u][2 * r + c] * post[c] : -INFINITY;
                    if (SCORE && have && 2 * t + c < G) a.logits[(head0 + 2 * t + c) * a.lstride + j] = z[u][2 * r + c];
                }
            }
        }
        // ---- V scales of rows g and g + 8 (0 where the slot is none of the sequence's, whatever it holds)
        uint32_t sv[kPair][2][Y / 2];
        float big = 0.f;
#pragma unroll
        for (int u = 0; u < kPair; ++u)
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int y = 0; y < Y / 2; ++y) {
                    const uint32_t w = reinterpret_cast<const uint32_t *>(tiles[u].vs + (tok0 + 8 * r) * Tile<D>::kScaleRow)[y];
                    sv[u][r][y] = in[u][r] ? w : 0u;
                    big = max3(big, bf16_lo(sv[u][r][y]), bf16_hi(sv[u][r][y]));
                }
        // ---- running reference of the logits, norm of the scales
        float over = -FLT_MAX;
#pragma unroll
        for (int u = 0; u < kPair; ++u)
#pragma unroll
            for (int c = 0; c < 2; ++c) over = max3(over, z[u][c] - ref[c], z[u][2 + c] - ref[c]);
        if (__any_sync(0xffffffffu, over > kMaxSlack || big > room)) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float m = ref[c];
#pragma unroll
                for (int u = 0; u < kPair; ++u) m = max3(m, z[u][c], z[u][2 + c]);
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, d));
                const float f = exp2_fast(ref[c] - m);
                ref[c] = m;
                sum[c] *= f;
#pragma unroll
                for (int j = 0; j < 2 * Y; ++j) {
                    o[j][c] *= f;
                    o[j][2 + c] *= f;
                }
            }
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, d));
            if (big > room) {
                const int e = big > 0.f ? 4 - max(ilogbf(big), -114) : norm_e;
                const float f = room < 0.f ? 1.f : ldexpf(1.f, e - norm_e);  // (nothing summed before the first)
                norm_e = e;
                norm = ldexpf(1.f, e);
                room = big > 0.f ? kScaleRoom * ldexpf(1.f, -e) : 0.f;
#pragma unroll
                for (int j = 0; j < 2 * Y; ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c) o[j][c] *= f;
            }
        }
#pragma unroll
        for (int u = 0; u < kPair; ++u) {
            float p[4];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                p[c] = exp2_fast(z[u][c] - ref[c]);
                p[2 + c] = exp2_fast(z[u][2 + c] - ref[c]);
                sum[c] += p[c] + p[2 + c];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) p[e] *= norm;
            // ---- outputs
            uint32_t vw[4][Y / 2];  // unit g of tokens t, 4 + t, 8 + t, 12 + t
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned char *row = tiles[u].v + (4 * j + t) * Tile<D>::kRow;
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
                    const uint32_t lo = vw[2 * j][y2], hi = vw[2 * j + 1][y2];
                    x[j][0] = (lo & 0x0f0f0f0fu) | ((hi << 4) & 0xf0f0f0f0u);
                    x[j][1] = ((lo >> 4) & 0x0f0f0f0fu) | (hi & 0xf0f0f0f0u);
                }
#pragma unroll
                for (int yy = 0; yy < 2; ++yy) {
                    uint32_t bf[NP][2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const float f = yy ? bf16_hi(sv[u][r][y2]) : bf16_lo(sv[u][r][y2]);
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
                        const int y = 2 * y2 + yy, byte = 2 * yy + h;
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
    };
    uint32_t use = 0, fill = (kStages - 1) * kStageBytes;  // stages, as offsets
    for (int i = 0; i < mine; ++i) {
        copy_wait<kStages - 2>();
        __syncwarp();
        issue(i + kStages - 1, ring_at + fill);  // into the stage that the previous iteration left
        const Tile<D> *tiles = reinterpret_cast<const Tile<D> *>(reinterpret_cast<const unsigned char *>(ring) + use);
        const int slot0 = (tile0 + tile_of(2 * i)) * kQ4Tile - S;  // cache slot of the pair's first token
        if (!pos && slot0 >= 0 && slot0 + kPair * kQ4Tile <= L) pair_step(tiles, slot0, std::false_type{});
        else pair_step(tiles, slot0, std::true_type{});
        fill = use;
        use = use + kStageBytes == kStages * kStageBytes ? 0u : use + kStageBytes;
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
        if (ref[c] == -FLT_MAX) ref[c] = -INFINITY;  // no live slot
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
        if (segs == 1) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            T *dst = static_cast<T *>(a.out) + head * D + e;
            store_as(dst, x.x * inv);
            store_as(dst + 1, x.y * inv);
            store_as(dst + 2, x.z * inv);
            store_as(dst + 3, x.w * inv);
            if (e == 0) a.lse2[head] = l == 0.f ? -INFINITY : m + log2f(l);
        } else {
            const int64_t to = head * kMaxSplits + ((int)blockIdx.x - seg0);
            *reinterpret_cast<float4 *>(a.part_o + to * D + e) = x;
            if (e == 0) reinterpret_cast<float2 *>(a.part_ml)[to] = make_float2(m, l);
        }
    }
    // ---- the run goes on in the next unit
    left -= take;
    round = 0;
    if (++kv == kvh) {
        kv = 0;
        before += sp.rounds;
        do {
            if (++b >= a.batch) return;
            sp = span_of(a.len[b], a.pv.start_of(b));
        } while (sp.rounds == 0);
    }
    __syncthreads();  // the shared memory is read
    }
}

// The rest of a call: outputs of units of several segments (or of none: 0), Eq. 1's scores and Eq. 4.
//
// The first CTAs take a utility row's tokens, kFinishThreads / HS of them each, HS threads a token
// that share the row's heads; the others merge eight heads' outputs.  A head's log-sum-exp comes from
// its segments' (reference, sum) pairs, so no pass of its own has to gather it.
constexpr int kFinishThreads = 256;
template <int HS>
__global__ void __launch_bounds__(kFinishThreads) q4_finish_kernel(const Q4FinishArgs a) {
    constexpr int kTok = kFinishThreads / HS, kAhead = 8;
    extern __shared__ float lse[];  // [heads of a row]
    __shared__ float wq[kFinishThreads / 32][kMaxSplits];
    __shared__ float part[HS > 1 ? kFinishThreads : 1];
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int G = a.q_heads / a.kv_heads;
    const bool merge = (int)blockIdx.x >= a.token_ctas;
    const int blocks = a.token_ctas > 0 ? a.token_ctas / (a.batch * a.rows_per_seq) : 1;
    int b, r = 0, token = 0;
    if (merge) {
        b = ((int)blockIdx.x - a.token_ctas) / a.merge_ctas;
    } else {
        r = blockIdx.x / blocks;
        b = r / a.rows_per_seq;
        token = blockIdx.x % blocks * kTok + (threadIdx.x & (kTok - 1));
        if (blockIdx.x % blocks * kTok >= a.len[b]) return;
    }
    const int L = a.len[b];
    const int rounds = span_of(L, a.start ? a.start[b] : 0).rounds;
    const int h0 = merge || a.rows_per_seq == 1 ? 0 : r % a.rows_per_seq * G;
    const int nh = merge || a.rows_per_seq == 1 ? a.q_heads : G;
    // the first of the thread's logits, before anything that they wait for
    const int hs = threadIdx.x / kTok;
    const float *zp = a.logits + ((int64_t)b * a.q_heads + h0) * a.lstride + token;
    float z[kAhead], was = 0.f;
    auto load = [&](int j0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int h = (j0 + j) * HS + hs;
            z[j] = h < nh && token < L ? __ldcg(zp + (int64_t)h * a.lstride) : -INFINITY;
        }
    };
    if (!merge) {
        load(0);
        if (a.ema && hs == 0 && token < L) was = a.ema[(int64_t)r * a.cap + token];
    }
    int found;
    const Deal deal = deal_rounds<kFinishThreads>(a.len, a.start, a.batch, a.kv_heads, a.attend_ctas,
                                                  [&](int x, int64_t, int, int64_t) { return x == b; }, &found);
    auto segments = [&](int h) {  // of the unit that head h of sequence b belongs to
        const int64_t unit0 = deal.before * a.kv_heads + (int64_t)(h / G) * rounds;
        return rounds > 0 ? (int)((unit0 + rounds - 1) / deal.per - unit0 / deal.per) + 1 : 0;
    };
    if (merge) {
        const int h = ((int)blockIdx.x - a.token_ctas) % a.merge_ctas * (kFinishThreads / 32) + warp;
        if (h >= a.q_heads) return;
        const int n = segments(h);
        if (n == 1) return;
        const int64_t hh = (int64_t)b * a.q_heads + h;
        const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + hh * kMaxSplits;
        const float *po = a.part_o + hh * kMaxSplits * a.head_dim;
        if (a.bf16) {
            __nv_bfloat16 *o = static_cast<__nv_bfloat16 *>(a.out) + hh * a.head_dim;
            if (a.head_dim == 128) merge_head<4>(ml, po, n, wq[warp], o, (float *)nullptr);
            else merge_head<2>(ml, po, n, wq[warp], o, (float *)nullptr);
        } else {
            float *o = static_cast<float *>(a.out) + hh * a.head_dim;
            if (a.head_dim == 128) merge_head<4>(ml, po, n, wq[warp], o, (float *)nullptr);
            else merge_head<2>(ml, po, n, wq[warp], o, (float *)nullptr);
        }
        return;
    }
    for (int h = warp; h < nh; h += kFinishThreads / 32) {
        const int n = segments(h0 + h);
        const int64_t hh = (int64_t)b * a.q_heads + h0 + h;
        float x;
        if (n == 1) {
            x = __ldcg(a.lse2 + hh);
        } else {
            const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + hh * kMaxSplits;
            float2 y[kMaxSplits / 32];
            float m = -INFINITY, w = 0.f;
#pragma unroll
            for (int k = 0; k < kMaxSplits / 32; ++k) {
                y[k] = lane + 32 * k < n ? __ldcg(ml + lane + 32 * k) : make_float2(-INFINITY, 0.f);
                m = fmaxf(m, y[k].x);
            }
            m = warp_max(m);
            const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int k = 0; k < kMaxSplits / 32; ++k) w += y[k].y * exp2f(y[k].x - base);
            w = warp_sum(w);
            x = w == 0.f ? -INFINITY : m + log2f(w);
        }
        if (lane == 0) lse[h] = x == -INFINITY ? INFINITY : x;  // no live slot: probabilities 0
    }
    __syncthreads();
    float acc = 0.f;
    for (int j0 = 0; j0 * HS < nh; j0 += kAhead) {
        if (j0) load(j0);
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int h = (j0 + j) * HS + hs;
            if (h < nh) acc += exp2f(z[j] - lse[h]);
        }
    }
    if (HS > 1) {
        part[threadIdx.x] = acc;
        __syncthreads();
        if (hs > 0) return;
#pragma unroll
        for (int k = 1; k < HS; ++k) acc += part[threadIdx.x + k * kTok];
    }
    if (token >= L) return;
    const float s = acc * (1.f / (float)nh);
    const int64_t to = (int64_t)r * a.cap + token;
    if (a.score) a.score[to] = s;
    if (a.ema) a.ema[to] = a.alpha * was + (1.f - a.alpha) * s;
}

template <int D, typename T>
cudaError_t launch_t(const Q4AttendArgs &a, int ctas, cudaStream_t st) {
    constexpr size_t ring = sizeof(Tile<D>) * kPair * kStages * kWarps;
    constexpr size_t join = kWarps * 8 * (sizeof(float2) + D * sizeof(float));
    constexpr size_t smem = ring > join ? ring : join;
    auto kernel = a.logits ? q4_attend_kernel<D, T, true> : q4_attend_kernel<D, T, false>;
    if (smem > 48 << 10) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    const cudaError_t e = launch_k(kernel, dim3((unsigned)ctas), dim3(kThreads), smem, st, a);
    note_launch();
    return e;
}

template <int HS>
cudaError_t launch_finish_t(Q4FinishArgs a, int64_t rows, int32_t max_len, cudaStream_t st) {
    constexpr int tok = kFinishThreads / HS;
    const int64_t tokens = rows * ((max_len + tok - 1) / tok), merges = (int64_t)a.batch * a.merge_ctas;
    if (tokens + merges > 0x7fffffff) return cudaErrorInvalidConfiguration;
    a.token_ctas = (int32_t)tokens;
    const int nh = a.rows_per_seq > 1 ? a.q_heads / a.kv_heads : a.q_heads;
    const cudaError_t e = launch_k(q4_finish_kernel<HS>, dim3((unsigned)(tokens + merges)), dim3(kFinishThreads),
                                   sizeof(float) * nh, st, a);
    note_launch();
    return e;
}

}  // namespace

// One wave of CTAs at most, one round each at least.
int32_t q4_attend_ctas(const ikv_shape *s, int32_t max_len, int sms) {
    // a start offset may put the first slot anywhere in its tile
    const int64_t rounds = max_len > 0 ? ((int64_t)max_len + kQ4Tile - 1 + kRound - 1) / kRound : 1;
    const int64_t units = (int64_t)s->batch * s->kv_heads, wave = (int64_t)sms * kCtasPerSm;
    return (int32_t)(rounds * units < wave ? rounds * units : wave);
}

cudaError_t launch_q4_attend(const Q4AttendArgs &a, int dtype, int head_dim, int32_t ctas, cudaStream_t st) {
    if (dtype == IKV_BF16)
        return head_dim == 128 ? launch_t<128, __nv_bfloat16>(a, ctas, st) : launch_t<64, __nv_bfloat16>(a, ctas, st);
    return head_dim == 128 ? launch_t<128, float>(a, ctas, st) : launch_t<64, float>(a, ctas, st);
}

cudaError_t launch_q4_finish(const Q4FinishArgs &args, int32_t max_len, int sms, cudaStream_t st) {
    Q4FinishArgs a = args;
    a.merge_ctas = (a.q_heads + kFinishThreads / 32 - 1) / (kFinishThreads / 32);
    const int64_t rows = a.score || a.ema ? (int64_t)a.batch * a.rows_per_seq : 0;
    // as many threads a token as it takes to give every SM a CTA
    if (rows * ((max_len + kFinishThreads - 1) / kFinishThreads) >= sms) return launch_finish_t<1>(a, rows, max_len, st);
    if (rows * ((max_len + kFinishThreads / 4 - 1) / (kFinishThreads / 4)) >= sms)
        return launch_finish_t<4>(a, rows, max_len, st);
    return launch_finish_t<8>(a, rows, max_len, st);
}

}  // namespace ikv
