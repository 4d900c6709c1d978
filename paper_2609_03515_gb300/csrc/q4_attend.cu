// Decode attention over a cache held in 4 bits.
#include <algorithm>
#include <cfloat>
#include <climits>
#include <cstddef>
#include <type_traits>

#include "merge.cuh"
#include "q4.cuh"

namespace ikv {
namespace {

constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kPair = 2;              // tiles of an iteration
constexpr int kStages = 2;            // pairs of tiles a warp has in flight or in use
// CTAs an SM holds: at 4, 128 channels lack the registers that 3 leave (32 x 16k, 28 / 4 heads: 56.3 us
// where 3 took 52.6); 64 channels of bf16 queries have them (16 / 4 heads: 33.7 against 35.5)
constexpr int ctas_per_sm(int head_dim, int elem_bytes) { return head_dim == 64 && elem_bytes == 2 ? 4 : 3; }
constexpr int kSwitch = 12;           // what going from one unit to the next costs a CTA, in pairs of tiles
constexpr float kMaxSlack = 7.f;      // log2: how far a logit may lie above the running reference
constexpr float kScaleRoom = 256.f;   // a V scale's most, normalised, before its group is normalised again (a weight's: 2^15)
// powers of two that V scales are multiplied by: the first of a group brings its smallest (2^-123) to 2^3 and
// its inverse is a normal number; the largest scale takes 2^-120
constexpr int kNormFirst = 126;

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
// The cache is read once: it goes out of L2 before the logits and partials, which are read again.
__device__ __forceinline__ uint64_t read_once_policy() {
    uint64_t p;
    asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(p));
    return p;
}
__device__ __forceinline__ void copy16(uint32_t dst, const void *src, uint64_t policy) {
    asm volatile("cp.async.cg.shared.global.L2::cache_hint [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "l"(policy) : "memory");
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
// 2^e for whole e <= 127: exact, 0 below 2^-126 (and for a NaN)
__device__ __forceinline__ float pow2(float e) { return __int_as_float(((int)fmaxf(e, -127.f) + 127) << 23); }
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {  // (of a number and NaN: the number)
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// A group's power of two, in the half of norm that starts at bit `at`: such that its largest scale, in the
// same half of most, comes to 2^4 .. 2^5.  Returns what its outputs so far are multiplied by (0 where
// they are nothing beside the new ones).
__device__ __forceinline__ float renorm(uint32_t &norm, uint32_t most, int at) {
    const int was = norm >> (at + 7) & 255, e = 127 + 4 + 127 - (int)min(most >> (at + 7) & 255u, 251u);
    norm = (norm & ~(0xffffu << at)) | (uint32_t)e << (at + 7);
    return pow2((float)(e - was));
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

template <int D>
constexpr size_t kJoinBytes = kWarps * 8 * (sizeof(float2) + D * sizeof(float));  // in place of the rings

// A tile's row r stands for token perm(r): lane (g, t) of the second product then finds its
// four tokens t, 4 + t, 8 + t, 12 + t, whose 8-byte units lie in different banks.
__device__ __forceinline__ int perm_of_row(int r) { return ((r >> 1) & 3) + 4 * (r & 1) + 8 * (r >> 3); }
__device__ __forceinline__ int row_of_token(int t) { return 2 * (t & 3) + ((t >> 2) & 1) + 8 * (t >> 3); }

// How the work is cut.  A unit (sequence, KV head) is pairs of tiles, counted from the tile that
// holds its first slot.  The units are laid one behind another, each a little longer than its pairs,
// and that length is dealt to one wave of CTAs in equal runs: a batch of uneven lengths loads them
// evenly, and a CTA's run is one or more segments, each of one unit.  A unit's n segments leave
// partials 0 .. n - 1 and n in segs.
struct Span {  // of a sequence
    int L, S, tile0, tiles, pairs;
};
__device__ __forceinline__ Span span_of(const Q4AttendArgs &a, int b) {
    Span s;
    s.L = a.len[b];
    s.S = a.pv.start_of(b);
    s.tile0 = s.S / kQ4Tile;
    s.tiles = s.L > 0 ? (s.S + s.L + kQ4Tile - 1) / kQ4Tile - s.tile0 : 0;
    s.pairs = (s.tiles + kPair - 1) / kPair;
    return s;
}
struct Segment {
    int b, kv;          // its unit
    int pairs;          // the unit's pairs that are the CTA's
    int seg0, segs;     // the CTA of the unit's first segment, the unit's segments
};
// Where a CTA's run starts and how long it is.
struct Run {
    int b, before;      // its first sequence, and the length (of one KV head) in front of that; b < 0: none
    int per;            // length of a run
    int whole;          // > 0: every unit is as long as its pairs rounded up to runs; 0: kSwitch longer than its pairs
    __device__ __forceinline__ int length(int pairs) const {
        return pairs == 0 ? 0 : whole ? whole : pairs + kSwitch;
    }
    // n sequences with slots, of `total` pairs, low to top each
    __device__ __forceinline__ void deal(int total, int n, int low, int top, int kvh, int ctas) {
        const int units = n * kvh;
        // (a unit of kMaxSplits - 2 whole runs at most: it may begin and end inside two more)
        const int least = (top + kMaxSplits - 3) / (kMaxSplits - 2);
        per = max(max((total * kvh + units * kSwitch + ctas - 1) / ctas, least), 1);
        whole = 0;
        if (top == low && units <= ctas) {
            // units of one length, cut evenly, each into runs of its own, if that makes them no longer
            const int each_unit = ctas / units, cut = max((top + each_unit - 1) / each_unit, least);
            // (a few pairs: as many for every warp)
            const int even = cut > 2 * kWarps ? cut : (cut + kWarps - 1) / kWarps * kWarps;
            if (even <= per + kSwitch) {
                per = even;
                whole = (top + even - 1) / even * even;
            }
        }
    }
    // whether the CTA's run starts in a sequence of that length, `base` in front of it
    __device__ __forceinline__ bool starts_in(int base, int len, int kvh) const {
        const int64_t x = (int64_t)blockIdx.x * per;
        return x >= base * kvh && x < (base + len) * kvh;
    }
};
// Up to 32 sequences: each warp for itself, a sequence a lane, with no barrier (1 x 3277 slots: 10.3 ->
// 9.7 us).  sp: the span of the first.
__device__ __forceinline__ Run run_of_few(const Q4AttendArgs &a, Span &sp) {
    const int lane = threadIdx.x & 31;
    Span mine{0, 0, 0, 0, 0};
    if (lane < a.batch) mine = span_of(a, lane);
    Run run;
    run.deal(__reduce_add_sync(0xffffffffu, mine.pairs), __popc(__ballot_sync(0xffffffffu, mine.pairs > 0)),
             __reduce_min_sync(0xffffffffu, mine.pairs > 0 ? mine.pairs : INT_MAX),
             __reduce_max_sync(0xffffffffu, mine.pairs), a.pv.kv_heads, (int)gridDim.x);
    const int len = run.length(mine.pairs);
    int end = len;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, end, d);
        if (lane >= d) end += y;
    }
    run.b = __ffs(__ballot_sync(0xffffffffu, run.starts_in(end - len, len, a.pv.kv_heads))) - 1;
    run.before = __shfl_sync(0xffffffffu, end - len, max(run.b, 0));
    sp.L = __shfl_sync(0xffffffffu, mine.L, max(run.b, 0));
    sp.S = __shfl_sync(0xffffffffu, mine.S, max(run.b, 0));
    sp.tile0 = __shfl_sync(0xffffffffu, mine.tile0, max(run.b, 0));
    sp.tiles = __shfl_sync(0xffffffffu, mine.tiles, max(run.b, 0));
    sp.pairs = __shfl_sync(0xffffffffu, mine.pairs, max(run.b, 0));
    return run;
}
// Any number: every thread of the CTA takes some sequences.
__device__ __forceinline__ Run run_of(const Q4AttendArgs &a, Span &sp) {
    __shared__ int sums[kWarps], counts[kWarps], tops[kWarps], lows[kWarps], found[2];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int each = (a.batch + kThreads - 1) / kThreads, b0 = threadIdx.x * each, b1 = min(b0 + each, a.batch);
    int mine = 0, n_mine = 0, top = 0, low = INT_MAX;
    for (int b = b0; b < b1; ++b) {
        const int pairs = span_of(a, b).pairs;
        mine += pairs;
        n_mine += pairs > 0;
        top = max(top, pairs);
        if (pairs > 0) low = min(low, pairs);
    }
    int scan = mine, n_scan = n_mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int y = __shfl_up_sync(0xffffffffu, scan, d), z = __shfl_up_sync(0xffffffffu, n_scan, d);
        if (lane >= d) {
            scan += y;
            n_scan += z;
        }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    low = __reduce_min_sync(0xffffffffu, low);
    if (threadIdx.x == 0) found[0] = -1;
    if (lane == 31) {
        sums[warp] = scan;
        counts[warp] = n_scan;
        tops[warp] = top;
        lows[warp] = low;
    }
    __syncthreads();
    int total = 0, n = 0, base = scan - mine, n_base = n_scan - n_mine;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) {
            base += sums[w];
            n_base += counts[w];
        }
        total += sums[w];
        n += counts[w];
        top = max(top, tops[w]);
        low = min(low, lows[w]);
    }
    Run run;
    run.deal(total, n, low, top, a.pv.kv_heads, (int)gridDim.x);
    base = run.whole ? n_base * run.whole : base + n_base * kSwitch;
    for (int b = b0; b < b1; ++b) {
        const int len = run.length(span_of(a, b).pairs);
        if (run.starts_in(base, len, a.pv.kv_heads)) {
            found[0] = b;
            found[1] = base;
        }
        base += len;
    }
    __syncthreads();
    run.b = found[0];
    run.before = found[1];
    if (run.b >= 0) sp = span_of(a, run.b);
    return run;
}

// softmax(q K^T / sqrt d) V for a CTA's segments, and the logits of their slots, over a.post.
//
// S^T = K q^T: the tile's 16 tokens are the rows of an mma, its 8 columns the heads of the
// group (a group of 8 or fewer), 16 channels its depth.  A group of 32 channels is two of them
// and has one scale, so codes are converted to fp16 as they are (exact) and the scale
// multiplies the group's fp32 sum.  q is scaled by a power of two to [2^7, 2^8) and held in fp16
// (bf16 queries: exact down to 2^-22 of the largest; fp32 queries: two terms, 2^-22 of each).
// O^T = V^T P^T: the rows are channels, the depth the 16 tokens; V's scales, which differ from
// token to token, multiply the probabilities instead, once for each group of channels, in fp32
// before they are rounded to fp16 (fp32 outputs: two terms, 2^-22 of a weight; bf16 outputs: one, 2^-11
// of each, at most an eighth of what the output's own rounding does).  Each group of channels has a power of
// two that follows its largest scale seen and that its scales are multiplied by (exactly, two
// groups an instruction), so the weights stay within fp16's range however large or small V is,
// and a group of small channels beside one of large loses nothing.
// The softmax runs on a whole number of log2 units as its reference, at most 2^7 below the largest
// logit: the sums are rescaled a few times a sequence, exactly, and no tile waits for a
// maximum across lanes.  Weights and their sums know nothing of V's scales.
// DUAL (groups of four heads or fewer): a pair of tiles shares the columns, the first's logits in
// columns 0 to 3 and the second's in 4 to 7, each with an operand that is zero in the other's
// columns; logits, weights and scales then take half the instructions, and a head's two columns
// are joined like two warps (16 ragged sequences of 4k to 8k, 32 / 8 heads: 39.0 -> 36.7 us).
//
// Memory allows a tile of 128 channels 99 cycles of an SM.  It takes about 265 instructions (229
// DUAL), 64 of them conversions of codes that fill the ALU pipe for 32 cycles; 12 warps issue some
// 2.2 a cycle, which hides most of them.  32 sequences of 12k to 16k, 28 / 4 heads: 264 MB in
// 53.0 us with the merge (5.0 TB/s), of which waiting for the tiles alone takes 47.8; one of 32k,
// 32 / 8 heads, 38 MB in 12 us, 17.8 with its scores: lengths, table and first tiles are 4 of them,
// the join 1.5.  A third stage was slower (54.5 us where two took 52.6).
template <int D, typename T, bool SCORE, bool DUAL>
__global__ void __launch_bounds__(kThreads, ctas_per_sm(D, sizeof(T))) q4_attend_kernel(const Q4AttendArgs a) {
    constexpr int Y = D / kQ4Group;        // groups of a row
    constexpr int NP = sizeof(T) == 4 ? 2 : 1;  // fp16 terms of q and of the probabilities
    constexpr int kPieces = D / 32;        // 16-byte pieces of a row of codes
    extern __shared__ __align__(128) unsigned char smem[];
    float2 *ml = reinterpret_cast<float2 *>(smem);                              // [kWarps][8]
    float *po = reinterpret_cast<float *>(smem + kWarps * 8 * sizeof(float2));  // [kWarps][8][D]
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int g = lane >> 2, t = lane & 3;
    const Tile<D> *ring = reinterpret_cast<const Tile<D> *>(smem) + warp * (kStages * kPair);
    pdl_wait();
    const int kvh = a.pv.kv_heads, G = a.q_heads / kvh;
    Span sp;
    const Run run = a.batch <= 32 ? run_of_few(a, sp) : run_of(a, sp);
    if (run.b < 0) return;  // past the last run

    // where a lane's pieces of a tile go: K's rows permuted, V's pieces swizzled
    constexpr int kCopies = kQ4Tile * kPieces / 32;
    constexpr int kScalePieces = kQ4Tile * Tile<D>::kScaleRow / 16;  // 8 or 4
    constexpr uint32_t kStageBytes = kPair * sizeof(Tile<D>);
    const uint32_t ring_at = smem_u32(ring);
    // (its second piece of each lies 8 tokens on: the same distance in memory and in the ring)
    const int c_tok = lane / kPieces, c_piece = lane % kPieces;
    const uint32_t to_k = offsetof(Tile<D>, k) + row_of_token(c_tok) * Tile<D>::kRow + c_piece * 16;
    const uint32_t to_v = offsetof(Tile<D>, v) + c_tok * Tile<D>::kRow + (D == 128 ? c_piece ^ (c_tok & 2) : c_piece) * 16;
    const bool has_scale = lane < 16 && (lane & 7) < kScalePieces;
    const unsigned char *scales = reinterpret_cast<const unsigned char *>(lane < 8 ? a.ks : a.vs) + (lane & 7) * 16;
    const uint32_t to_s = (lane < 8 ? offsetof(Tile<D>, ks) : offsetof(Tile<D>, vs)) + (lane & 7) * 16;

    // the segment at hand
    int before = run.before, left = run.per;
    Segment sg;
    const int32_t *pos = nullptr;
    int first = 0, last = 0, mine = 0;  // its tiles [first, last) of the sequence, this warp's pairs of them
    auto enter = [&](int b, int kv, int pair) {
        sg.b = b;
        sg.kv = kv;
        sg.pairs = min(sp.pairs - pair, left);
        left -= run.length(sp.pairs) - pair;
        pos = a.pos ? a.pos + (int64_t)(a.rows_per_seq == 1 ? b : b * a.rows_per_seq + kv) * a.cap : nullptr;
        first = pair * kPair;
        last = min(first + sg.pairs * kPair, sp.tiles);
        mine = sg.pairs > warp ? (sg.pairs - warp + kWarps - 1) / kWarps : 0;
    };
    // the unit behind (b, kv), if the run reaches it
    auto enter_next = [&](int b, int kv) -> bool {
        if (left <= 0) return false;
        if (++kv == kvh) {
            kv = 0;
            before += run.length(sp.pairs);
            do {
                if (++b >= a.batch) return false;
                sp = span_of(a, b);
            } while (sp.pairs == 0);
        }
        enter(b, kv, 0);
        return true;
    };
    // the warp's pairs of tiles: first / 2 + warp, + kWarps, ...; lane i knows where the i-th of
    // the 32 tiles from a multiple of 32 on starts
    auto tile_of = [&](int i) { return first + ((i >> 1) * kWarps + warp) * kPair + (i & 1); };  // my i-th tile
    auto place_of = [&](int i) -> uint32_t {  // the tile of the paged arrays (its row / kQ4Tile)
        const int x = tile_of(i);
        return x < last ? (uint32_t)(a.pv.row_phys(sg.b, a.layer, sg.kv, (sp.tile0 + x) * kQ4Tile) / kQ4Tile) : 0u;
    };
    uint32_t places = 0;
    const uint64_t policy = read_once_policy();
    const unsigned char *const from_k = a.k + lane * 16, *const from_v = a.v + lane * 16;
    auto issue = [&](int i, uint32_t stage) {
        if (i < mine) {
            if ((i & 15) == 0) places = place_of(2 * i + lane);
            const uint32_t at_k = stage + to_k, at_v = stage + to_v, at_s = stage + to_s;
            const bool both = tile_of(2 * i + 1) < last;
#pragma unroll
            for (int u = 0; u < kPair; ++u) {
                const uint32_t place = __shfl_sync(0xffffffffu, places, (2 * i + u) & 31);
                if (u > 0 && !both) break;
                const unsigned char *k = from_k + (uint64_t)place * (kQ4Tile * Tile<D>::kRow);
                const unsigned char *v = from_v + (uint64_t)place * (kQ4Tile * Tile<D>::kRow);
#pragma unroll
                for (int j = 0; j < kCopies; ++j) {
                    copy16(at_k + u * sizeof(Tile<D>) + j * 512, k + j * 512, policy);
                    copy16(at_v + u * sizeof(Tile<D>) + j * 512, v + j * 512, policy);
                }
                if (has_scale) copy16(at_s + u * sizeof(Tile<D>), scales + (uint64_t)place * (kQ4Tile * Tile<D>::kScaleRow), policy);
                if (pos && lane >= 16) {
                    const int j = (sp.tile0 + tile_of(2 * i + u)) * kQ4Tile + lane - 16 - sp.S;
                    if (j >= 0 && j < sp.L) copy4(stage + u * sizeof(Tile<D>) + offsetof(Tile<D>, pos) + (lane - 16) * 4, pos + j);
                }
            }
        }
        copy_commit();
    };
    uint32_t use = 0;  // the stage of the next pair, as an offset
    auto stage_after = [&](uint32_t x, int n) {  // n < kStages
        x += n * kStageBytes;
        return x >= kStages * kStageBytes ? x - kStages * kStageBytes : x;
    };
    auto prologue = [&]() {
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) issue(i, ring_at + stage_after(use, i));
    };
    {
        const int at = (int)((int64_t)blockIdx.x * run.per - (int64_t)run.before * kvh);  // within the sequence's units
        const int length = run.length(sp.pairs), kv = at / length, pair = at % length;
        if (pair < sp.pairs) {
            enter(run.b, kv, pair);
        } else {  // behind the unit's last pair
            left -= length - pair;
            if (!enter_next(run.b, kv)) return;
        }
    }
    prologue();
    while (true) {
    // the unit's segments: the runs that its pairs lie in
    {
        const int unit0 = before * kvh + sg.kv * run.length(sp.pairs);
        sg.seg0 = unit0 / run.per;
        sg.segs = (unit0 + sp.pairs - 1) / run.per - sg.seg0 + 1;
        if (threadIdx.x == 0 && first == 0) a.segs[sg.b * kvh + sg.kv] = sg.segs;
    }
    const int L = sp.L, S = sp.S, tile0 = sp.tile0;
    const int64_t head0 = (int64_t)sg.b * a.q_heads + (int64_t)sg.kv * G;

    // q: lane (g, t) holds channels 32 y + 8 t .. + 7 of its column's head; DUAL: the first tile's
    // operand, with columns 4 to 7 zero, and the second's
    uint32_t q[DUAL ? 2 : 1][NP][Y][4];
    float post[2];  // what turns the mma's sums into log2-domain logits, columns 2 t and 2 t + 1
    {
        float x[Y][8], m = 0.f;
        const int head = DUAL ? g & 3 : g;
        const T *src = static_cast<const T *>(a.q) + (head0 + head) * D + 8 * t;
#pragma unroll
        for (int y = 0; y < Y; ++y) {
#pragma unroll
            for (int e = 0; e < 8; ++e) x[y][e] = 0.f;
            if (head < G) {
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
                q[0][0][y][i] = pack_half(lo, hi);
                if (NP == 2) {
                    const float2 f = unpack_half(q[0][0][y][i]);
                    q[0][NP - 1][y][i] = pack_half(lo - f.x, hi - f.y);
                }
                if constexpr (DUAL) {
#pragma unroll
                    for (int n = 0; n < NP; ++n) {
                        q[1][n][y][i] = g < 4 ? 0u : q[0][n][y][i];
                        q[0][n][y][i] = g < 4 ? q[0][n][y][i] : 0u;
                    }
                }
            }
        const float mine = a.scale_log2 * ldexpf(1.f, e - 7);
        if (SCORE && first == 0 && threadIdx.x < 32 && t == 0 && g < G && (!DUAL || g < 4)) a.post[head0 + g] = mine;
        post[0] = __shfl_sync(0xffffffffu, mine, 8 * t);
        post[1] = __shfl_sync(0xffffffffu, mine, 8 * t + 4);
    }

    // where the logits of columns 2 t and 2 t + 1 go, by cache slot
    const int col = DUAL ? 2 * (t & 1) : 2 * t;  // their heads: col, col + 1
    float *const lg = SCORE ? a.logits + (head0 + col) * a.lstride : nullptr;
    const bool lg0 = col < G, lg1 = col + 1 < G;

    float o[2 * Y][4];  // O^T of channels 32 y + 4 g + 2 h (+ 1), columns 2 t, 2 t + 1
#pragma unroll
    for (int i = 0; i < 2 * Y; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] = 0.f;
    float ref[2] = {-FLT_MAX, -FLT_MAX}, sum[2] = {0.f, 0.f};
    uint32_t norm[Y / 2];  // bf16: what the scales of groups 2 y and 2 y + 1 are multiplied by
#pragma unroll
    for (int y = 0; y < Y / 2; ++y) norm[y] = (uint32_t)(kNormFirst + 127) * 0x00800080u;

    const int tok0 = perm_of_row(g);  // tokens of rows g and g + 8: tok0, tok0 + 8
    // One pair of tiles; MASK: some of its slots are not the sequence's, or dead.  A lane's columns
    // belong to both tiles one after the other (NZ = 2 sets of logits), or DUAL to one of them.
    constexpr int NZ = DUAL ? 1 : kPair;
    const int my_tile = DUAL ? t >> 1 : 0;
    auto pair_step = [&](const Tile<D> *tiles, int slot0, auto mask_tag) {
        constexpr bool MASK = decltype(mask_tag)::value;
        // ---- logits
        float z[NZ][4];
        bool in[NZ][2];
        uint32_t kw[kPair][2][D / 32];  // rows g, g + 8: two units
#pragma unroll
        for (int u = 0; u < kPair; ++u)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const unsigned char *row = tiles[u].k + (g + 8 * r) * Tile<D>::kRow + t * (D / 8);
                if (D == 128) *reinterpret_cast<uint4 *>(kw[u][r]) = *reinterpret_cast<const uint4 *>(row);
                else *reinterpret_cast<uint2 *>(kw[u][r]) = *reinterpret_cast<const uint2 *>(row);
            }
        uint32_t sc[NZ][2][Y / 2];
#pragma unroll
        for (int v = 0; v < NZ; ++v)
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int y = 0; y < Y / 2; ++y)
                    sc[v][r][y] = reinterpret_cast<const uint32_t *>(tiles[v + my_tile].ks + (tok0 + 8 * r) * Tile<D>::kScaleRow)[y];
#pragma unroll
        for (int y = 0; y < Y; ++y) {
            float c[NZ][4];
#pragma unroll
            for (int u = 0; u < kPair; ++u)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    // unit 2 t + h: words h * Y / 2 ..; group y's two bytes
                    const int w = h * (Y / 2) + (y >> 1), byte = 2 * (y & 1);
                    const uint32_t f[4] = {e2m1_bits(kw[u][0][w], byte), e2m1_bits(kw[u][1][w], byte),
                                           e2m1_bits(kw[u][0][w], byte + 1), e2m1_bits(kw[u][1][w], byte + 1)};
                    const auto &qu = q[DUAL ? u : 0];
                    float(&cu)[4] = c[DUAL ? 0 : u];
#pragma unroll
                    for (int n = 0; n < NP; ++n)
                        if (h == 0 && n == 0 && !(DUAL && u > 0)) mma16816_first(cu, f, qu[n][y][2 * h], qu[n][y][2 * h + 1]);
                        else mma16816(cu, f, qu[n][y][2 * h], qu[n][y][2 * h + 1]);
                }
#pragma unroll
            for (int v = 0; v < NZ; ++v) {
                const float s0 = (y & 1) ? bf16_hi(sc[v][0][y >> 1]) : bf16_lo(sc[v][0][y >> 1]);
                const float s1 = (y & 1) ? bf16_hi(sc[v][1][y >> 1]) : bf16_lo(sc[v][1][y >> 1]);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    z[v][e] = y == 0 ? (e < 2 ? s0 : s1) * c[v][e] : z[v][e] + (e < 2 ? s0 : s1) * c[v][e];
            }
        }
#pragma unroll
        for (int v = 0; v < NZ; ++v)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int j = slot0 + (v + my_tile) * kQ4Tile + 8 * r + tok0;  // cache slot of row g + 8 r
                const bool have = !MASK || (j >= 0 && j < L);
                in[v][r] = have && (!MASK || !pos || tiles[v + my_tile].pos[tok0 + 8 * r] >= 0);
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (!in[v][r]) z[v][2 * r + c] = -INFINITY;
                if (SCORE && have) {
                    if (lg0) lg[j] = z[v][2 * r];
                    if (lg1) lg[j + a.lstride] = z[v][2 * r + 1];
                }
            }
        // ---- V scales of rows g and g + 8 (0 where the slot is none of the sequence's, whatever it holds),
        // normalised
        auto scale_of = [&](int v, int r, int y) -> uint32_t {
            const uint32_t w = reinterpret_cast<const uint32_t *>(tiles[v + my_tile].vs + (tok0 + 8 * r) * Tile<D>::kScaleRow)[y];
            return in[v][r] ? w : 0u;
        };
        uint32_t sv[NZ][2][Y / 2];
        float big = 0.f;
#pragma unroll
        for (int v = 0; v < NZ; ++v)
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int y = 0; y < Y / 2; ++y) {
                    sv[v][r][y] = mul_bf16x2(scale_of(v, r, y), norm[y]);
                    big = max3(big, bf16_lo(sv[v][r][y]), bf16_hi(sv[v][r][y]));
                }
        // ---- running reference of the logits, norms of the scales; a weight is 2^(logit - ref)
        float d[NZ][4], over = -FLT_MAX;
        auto weigh = [&]() {
#pragma unroll
            for (int v = 0; v < NZ; ++v)
#pragma unroll
                for (int e = 0; e < 4; ++e) d[v][e] = fmaf(z[v][e], post[e & 1], -ref[e & 1]);
        };
        weigh();
#pragma unroll
        for (int v = 0; v < NZ; ++v)
#pragma unroll
            for (int c = 0; c < 2; ++c) over = max3(over, d[v][c], d[v][2 + c]);
        if (__any_sync(0xffffffffu, over > kMaxSlack || big > kScaleRoom)) {
            float f[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                float m = -INFINITY;
#pragma unroll
                for (int v = 0; v < NZ; ++v) m = max3(m, z[v][c], z[v][2 + c]);
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
                m = fmaxf(ref[c], floorf(m * post[c]));
                f[c] = pow2(ref[c] - m);
                ref[c] = m;
                sum[c] *= f[c];
            }
            weigh();
#pragma unroll
            for (int y = 0; y < Y / 2; ++y) {
                uint32_t m = 0u;  // the largest scales of two groups
#pragma unroll
                for (int v = 0; v < NZ; ++v)
#pragma unroll
                    for (int r = 0; r < 2; ++r) m = max_bf16x2(m, scale_of(v, r, y));
#pragma unroll
                for (int x = 1; x < 32; x <<= 1) m = max_bf16x2(m, __shfl_xor_sync(0xffffffffu, m, x));
                const uint32_t most = mul_bf16x2(m, norm[y]);
                float up[2] = {1.f, 1.f};
                if (bf16_lo(most) > kScaleRoom) up[0] = renorm(norm[y], m, 0);
                if (bf16_hi(most) > kScaleRoom) up[1] = renorm(norm[y], m, 16);
#pragma unroll
                for (int yy = 0; yy < 2; ++yy)
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[2 * (2 * y + yy) + h][e] *= f[e & 1] * up[yy];
#pragma unroll
                for (int v = 0; v < NZ; ++v)
#pragma unroll
                    for (int r = 0; r < 2; ++r) sv[v][r][y] = mul_bf16x2(scale_of(v, r, y), norm[y]);
            }
        }
        float p[NZ][4];
#pragma unroll
        for (int v = 0; v < NZ; ++v) {
#pragma unroll
            for (int e = 0; e < 4; ++e) p[v][e] = exp2_fast(d[v][e]);
#pragma unroll
            for (int c = 0; c < 2; ++c) sum[c] += p[v][c] + p[v][2 + c];
        }
        // ---- outputs
        // unit g of tokens t, 4 + t, 8 + t, 12 + t: bytes with a channel's codes of two tokens, the
        // even channels in x[0], the odd ones in x[1]
        auto load_v = [&](int u, uint32_t(&vw)[4][Y / 2]) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const unsigned char *row = tiles[u].v + (4 * j + t) * Tile<D>::kRow;
                if (D == 128)
                    *reinterpret_cast<uint2 *>(vw[j]) = *reinterpret_cast<const uint2 *>(row + (((g >> 1) ^ (t & 2)) << 4) + ((g & 1) << 3));
                else
                    vw[j][0] = *reinterpret_cast<const uint32_t *>(row + g * 4);
            }
        };
        auto mix_v = [&](const uint32_t(&vw)[4][Y / 2], int y2, uint32_t(&x)[2][2]) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t lo = vw[2 * j][y2], hi = vw[2 * j + 1][y2];
                x[j][0] = (lo & 0x0f0f0f0fu) | ((hi << 4) & 0xf0f0f0f0u);
                x[j][1] = ((lo >> 4) & 0x0f0f0f0fu) | (hi & 0xf0f0f0f0u);
            }
        };
        // P^T times the scales of group 2 y2 + yy, as an mma's second operand
        auto weights = [&](int v, int y2, int yy, uint32_t(&bf)[NP][2]) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float f = yy ? bf16_hi(sv[v][r][y2]) : bf16_lo(sv[v][r][y2]);
                const float w0 = p[v][2 * r] * f, w1 = p[v][2 * r + 1] * f;
                const uint32_t w = pack_half(w0, w1);
                bf[0][r] = transpose8x8(w);
                if (NP == 2) {
                    const float2 back = unpack_half(w);
                    bf[NP - 1][r] = transpose8x8(pack_half((w0 - back.x) * kLowUp, (w1 - back.y) * kLowUp));
                }
            }
        };
        auto add_v = [&](const uint32_t(&x)[2][2], int y2, int yy, int h, const uint32_t(&bf)[NP][2]) {
            float(&to)[4] = o[2 * (2 * y2 + yy) + h];
            const int byte = 2 * yy + h;
            const uint32_t f[4] = {e2m1_bits(x[0][0], byte), e2m1_bits(x[0][1], byte), e2m1_bits(x[1][0], byte),
                                   e2m1_bits(x[1][1], byte)};
            mma16816(to, f, bf[0][0], bf[0][1]);
            if (NP == 2) {
                const uint32_t low[4] = {shrink(f[0]), shrink(f[1]), shrink(f[2]), shrink(f[3])};
                mma16816(to, low, bf[NP - 1][0], bf[NP - 1][1]);
            }
        };
        if constexpr (DUAL) {
            uint32_t vw[kPair][4][Y / 2];
#pragma unroll
            for (int u = 0; u < kPair; ++u) load_v(u, vw[u]);
            const uint32_t keep = g < 4 ? 0xffffffffu : 0u;  // columns of the first tile
#pragma unroll
            for (int y2 = 0; y2 < Y / 2; ++y2) {
                uint32_t x[kPair][2][2];
#pragma unroll
                for (int u = 0; u < kPair; ++u) mix_v(vw[u], y2, x[u]);
#pragma unroll
                for (int yy = 0; yy < 2; ++yy) {
                    uint32_t bf[kPair][NP][2];
                    weights(0, y2, yy, bf[0]);
#pragma unroll
                    for (int n = 0; n < NP; ++n)
#pragma unroll
                        for (int r = 0; r < 2; ++r) {
                            bf[1][n][r] = bf[0][n][r] & ~keep;
                            bf[0][n][r] &= keep;
                        }
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int u = 0; u < kPair; ++u) add_v(x[u], y2, yy, h, bf[u]);
                }
            }
        } else {
#pragma unroll
            for (int u = 0; u < kPair; ++u) {
                uint32_t vw[4][Y / 2];
                load_v(u, vw);
#pragma unroll
                for (int y2 = 0; y2 < Y / 2; ++y2) {
                    uint32_t x[2][2];
                    mix_v(vw, y2, x);
#pragma unroll
                    for (int yy = 0; yy < 2; ++yy) {
                        uint32_t bf[NP][2];
                        weights(u, y2, yy, bf);
#pragma unroll
                        for (int h = 0; h < 2; ++h) add_v(x, y2, yy, h, bf);
                    }
                }
            }
        }
    };
    for (int i = 0; i < mine; ++i) {
        copy_wait<kStages - 2>();
        __syncwarp();
        issue(i + kStages - 1, ring_at + stage_after(use, kStages - 1));  // into the stage that the previous iteration left
        const Tile<D> *tiles = reinterpret_cast<const Tile<D> *>(reinterpret_cast<const unsigned char *>(ring) + use);
        const int slot0 = (tile0 + tile_of(2 * i)) * kQ4Tile - S;  // cache slot of the pair's first token
        if (!pos && slot0 >= 0 && slot0 + kPair * kQ4Tile <= L) pair_step(tiles, slot0, std::false_type{});
        else pair_step(tiles, slot0, std::true_type{});
        use = stage_after(use, 1);
    }
#pragma unroll
    for (int c = 0; c < 2; ++c)
        if (ref[c] == -FLT_MAX) ref[c] = -INFINITY;  // no live slot
    // ---- the warps' results joined: (reference, sum) and outputs through shared memory
#pragma unroll
    for (int c = 0; c < 2; ++c)
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum[c] += __shfl_xor_sync(0xffffffffu, sum[c], d);
    __syncthreads();  // every ring is done with
    // Sums are brought into [1/2, 1) by the reference, which stays a whole number: outputs are then no
    // larger than the largest value, whatever the number of tokens.
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const int bits = __float_as_int(sum[c]) >> 23, up = bits > 0 && bits < 255 ? bits - 126 : 0;
        const float down = pow2((float)-up);
        if (g == 0) ml[warp * 8 + 2 * t + c] = make_float2(ref[c] + (float)up, sum[c] * down);
#pragma unroll
        for (int y = 0; y < Y; ++y) {
            const float back = __uint_as_float((254u - (norm[y >> 1] >> (16 * (y & 1) + 7) & 255u)) << 23);
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<float2 *>(po + (warp * 8 + 2 * t + c) * D + 32 * y + 4 * g + 2 * h) =
                    make_float2(o[2 * y + h][c] * down * back, o[2 * y + h][2 + c] * down * back);
        }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < G * (D / 4); i += kThreads) {
        const int h = i / (D / 4), e = i % (D / 4) * 4;
        // its columns: one a warp, or two that took turns
        constexpr int kParts = DUAL ? 2 * kWarps : kWarps;
        auto part = [&](int w) { return DUAL ? (w >> 1) * 8 + 4 * (w & 1) + h : w * 8 + h; };
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < kParts; ++w) m = fmaxf(m, ml[part(w)].x);
        // (so far above the largest that neither the sum over the warps here nor the one over the
        // segments later passes the largest value)
        const float base = m == -INFINITY ? 0.f : m + (sg.segs == 1 ? 3.f : 10.f);
        static_assert(kParts <= 8 && kMaxSplits <= 128, "2^3 and 2^7 of them");
        float l = 0.f;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kParts; ++w) {
            const float2 y = ml[part(w)];
            const float f = pow2(y.x - base);
            const float4 v = *reinterpret_cast<const float4 *>(po + part(w) * D + e);
            l += f * y.y;
            x.x += f * v.x;
            x.y += f * v.y;
            x.z += f * v.z;
            x.w += f * v.w;
        }
        const int64_t head = head0 + h, to = head * kMaxSplits + ((int)blockIdx.x - sg.seg0);
        if (sg.segs == 1) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            T *dst = static_cast<T *>(a.out) + head * D + e;
            store_as(dst, x.x * inv);
            store_as(dst + 1, x.y * inv);
            store_as(dst + 2, x.z * inv);
            store_as(dst + 3, x.w * inv);
        } else {
            *reinterpret_cast<float4 *>(a.part_o + to * D + e) = x;
        }
        if (e == 0) reinterpret_cast<float2 *>(a.part_ml)[to] = make_float2(m == -INFINITY ? m : base, l);
    }
    // ---- the run goes on in the next unit
    if (!enter_next(sg.b, sg.kv)) return;
    __syncthreads();  // the join is read
    prologue();
    }
}

// The rest of a call: outputs of units of several segments (or of none: 0), Eq. 1's scores and Eq. 4.
//
// The first token_ctas CTAs take the utility rows' tokens, row_ctas of them a row: a block of
// kFinishThreads / HS tokens each, with HS threads a token that share the row's heads, or (V = 4) every
// row_ctas-th block of V kFinishThreads, with V tokens a thread.  The CTAs behind them merge the heads'
// outputs: MANY, a CTA a head, each of whose warps sums a part of the segments; else a warp a head.  A head's reference and sum come from
// its segments' pairs of them, so no pass of its own has to gather them; a probability is
// 2^(logit - reference) / sum, with the logit's factor applied here, as in the sum, without another rounding.
constexpr int kFinishThreads = 512;

// One CTA merges one head's segments: every warp sums some of them, 32 E channels wide.
template <int E, typename T>
__device__ __forceinline__ void merge_segments(const Q4FinishArgs &a, int hh, float *sum) {
    constexpr int kW = kFinishThreads / 32, D = 32 * E, kLoads = 2;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + (int64_t)hh * kMaxSplits;
    const float *po = a.part_o + (int64_t)hh * kMaxSplits * D + lane * E;
    // the loads go out with the count of segments: those that are none are read and dropped
    float2 y[kMaxSplits / 32];
    y[0] = __ldcg(ml + lane);
    float v[kLoads][E];
    auto load = [&](int k0) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const float *p = po + (int64_t)(k0 + j * kW) * D;
#pragma unroll
            for (int e = 0; e < E; e += 2) {
                const float2 x = k0 + j * kW < kMaxSplits ? __ldcg(reinterpret_cast<const float2 *>(p + e)) : make_float2(0.f, 0.f);
                v[j][e] = x.x;
                v[j][e + 1] = x.y;
            }
        }
    };
    load(warp);
    const int n = a.len[hh / a.q_heads] > 0 ? __ldcg(a.segs + hh / (a.q_heads / a.kv_heads)) : 0;
    if (n == 1) return;
    float m = -INFINITY, w = 0.f;
#pragma unroll
    for (int k = 0; k < kMaxSplits / 32; ++k) {
        if (k > 0 && 32 * k < n) y[k] = __ldcg(ml + lane + 32 * k);
        if (lane + 32 * k >= n) y[k] = make_float2(-INFINITY, 0.f);
        m = fmaxf(m, y[k].x);
    }
    m = warp_max(m);
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int k = 0; k < kMaxSplits / 32; ++k) {
        y[k].x = exp2f(y[k].x - base);
        w += y[k].y * y[k].x;
    }
    w = warp_sum(w);
    float acc[E];
#pragma unroll
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    for (int k0 = warp; k0 < n; k0 += kLoads * kW) {
        if (k0 != warp) load(k0);
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int k = k0 + j * kW;
            float mine = y[0].x;
#pragma unroll
            for (int i = 1; i < kMaxSplits / 32; ++i)
                if (k >> 5 == i) mine = y[i].x;
            const float f = __shfl_sync(0xffffffffu, mine, k & 31);
            if (k < n) {
#pragma unroll
                for (int e = 0; e < E; ++e) acc[e] += f * v[j][e];
            }
        }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) sum[warp * D + lane * E + e] = acc[e];
    __syncthreads();
    if (threadIdx.x < D) {
        float x = 0.f;
#pragma unroll
        for (int k = 0; k < kW; ++k) x += sum[k * D + threadIdx.x];
        store_as(static_cast<T *>(a.out) + (int64_t)hh * D + threadIdx.x, w == 0.f ? 0.f : x / w);
    }
}

// CTA x of those that merge: of one head (MANY), or of a head a warp.
template <bool MANY, int E, typename T>
__device__ __forceinline__ void merge_any(const Q4FinishArgs &a, int x, float *room) {
    if (MANY) {
        merge_segments<E, T>(a, x, room);
        return;
    }
    const int warp = threadIdx.x >> 5, hh = x * (kFinishThreads / 32) + warp;
    if (hh >= a.batch * a.q_heads) return;
    const int n = a.len[hh / a.q_heads] > 0 ? __ldcg(a.segs + hh / (a.q_heads / a.kv_heads)) : 0;
    if (n != 1)
        merge_head<E>(reinterpret_cast<const float2 *>(a.part_ml) + (int64_t)hh * kMaxSplits,
                      a.part_o + (int64_t)hh * kMaxSplits * 32 * E, n, room + warp * kMaxSplits,
                      static_cast<T *>(a.out) + (int64_t)hh * 32 * E, (float *)nullptr);
}

// A thread's V tokens.
template <int V>
struct Floats {
    alignas(V * sizeof(float)) float x[V];
    __device__ __forceinline__ void fill(float f) {
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = f;
    }
    __device__ __forceinline__ void load(const float *p) {
        if (V == 4) *reinterpret_cast<float4 *>(x) = __ldcg(reinterpret_cast<const float4 *>(p));
        else x[0] = __ldcg(p);
    }
    __device__ __forceinline__ void store(float *p, int n) const {  // n of them
        if (V == 4 && n >= V) {
            *reinterpret_cast<float4 *>(p) = *reinterpret_cast<const float4 *>(x);
        } else {
#pragma unroll
            for (int v = 0; v < V; ++v)
                if (v < n) p[v] = x[v];
        }
    }
};

template <int HS, bool MANY, int V>
__global__ void __launch_bounds__(kFinishThreads, V == 1 ? 0 : 2) q4_finish_kernel(const Q4FinishArgs a) {
    static_assert(HS == 1 || V == 1, "a thread's tokens are its own");
    constexpr int kTok = kFinishThreads / HS * V, kAhead = V == 4 ? 4 : 8, kWarpsF = kFinishThreads / 32, kHeads = 2;
    extern __shared__ float4 whole[];  // [heads of a row] the logits' factor, reference, 1 / sum, -
    __shared__ float part[HS > 1 ? kFinishThreads : 1];
    __shared__ float room[kWarpsF * 128];  // of those that merge
    static_assert(kMaxSplits <= 128, "a warp's weights");
    pdl_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int G = a.q_heads / a.kv_heads;
    if ((int)blockIdx.x >= a.token_ctas) {
        const int x = (int)blockIdx.x - a.token_ctas;
        if (a.bf16) {
            if (a.head_dim == 128) merge_any<MANY, 4, __nv_bfloat16>(a, x, room);
            else merge_any<MANY, 2, __nv_bfloat16>(a, x, room);
        } else {
            if (a.head_dim == 128) merge_any<MANY, 4, float>(a, x, room);
            else merge_any<MANY, 2, float>(a, x, room);
        }
        return;
    }
    const int r = blockIdx.x / a.row_ctas, b = r / a.rows_per_seq, block = blockIdx.x % a.row_ctas;
    int token = block * kTok + (threadIdx.x & (kFinishThreads / HS - 1)) * V;
    const int hs = threadIdx.x / (kFinishThreads / HS);
    const int h0 = a.rows_per_seq == 1 ? 0 : r % a.rows_per_seq * G;
    const int nh = a.rows_per_seq == 1 ? a.q_heads : G;
    const int64_t head0 = (int64_t)b * a.q_heads + h0;
    // whatever has an address goes out before anything is waited for
    const int L = a.len[b];
    Floats<V> z[kAhead], was;
    const int64_t next = (int64_t)HS * a.lstride;  // from one of the thread's heads to its next
    const int mine = (nh - hs + HS - 1) / HS;      // the thread's heads: hs, hs + HS, ...
    const float *zp = a.logits + (head0 + hs) * a.lstride + min(token, a.lstride - V);
    auto load = [&](int j0) {
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (j0 + j < mine) z[j].load(zp + (j0 + j) * next);
            else z[j].fill(-INFINITY);
        }
    };
    load(0);
    was.fill(0.f);
    if (a.ema && hs == 0 && token < a.cap) was.load(a.ema + (int64_t)r * a.cap + token);
    if (block * kTok >= L) return;  // (a sequence without slots has no segment count either)
    // the sum brought into [1, 2) by the reference, which is a whole number; no live slot: probabilities 0
    auto norm_of = [&](float post, float m, float w) {
        const int bits = __float_as_int(w) >> 23, up = bits > 0 && bits < 255 ? bits - 127 : 0;
        return make_float4(post, m == -INFINITY ? 0.f : m + (float)up, w == 0.f ? 0.f : 1.f / (w * pow2((float)-up)), 0.f);
    };
    if (!MANY) {  // few segments: a head a thread
        for (int h = threadIdx.x; h < nh; h += kFinishThreads) {
            constexpr int kFew = 4;
            const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + (head0 + h) * kMaxSplits;
            const int n = __ldcg(a.segs + (head0 + h) / G);
            const float post = __ldcg(a.post + head0 + h);
            float2 y[kFew];
#pragma unroll
            for (int k = 0; k < kFew; ++k) y[k] = __ldcg(ml + k);
            float m = -INFINITY, w = 0.f;
#pragma unroll
            for (int k = 0; k < kFew; ++k) m = k < n ? fmaxf(m, y[k].x) : m;
            for (int k = kFew; k < n; ++k) m = fmaxf(m, __ldcg(&ml[k].x));
            const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int k = 0; k < kFew; ++k) w += k < n ? y[k].y * pow2(y[k].x - base) : 0.f;
            for (int k = kFew; k < n; ++k) {
                const float2 v = __ldcg(ml + k);
                w += v.y * pow2(v.x - base);
            }
            whole[h] = norm_of(post, m, w);
        }
    }
    for (int hb = warp; MANY && hb < nh; hb += kHeads * kWarpsF) {
        int n[kHeads];
        float post[kHeads];
        constexpr int PL = 2;  // pairs a lane loads before it knows how many there are
        float2 y[kHeads][PL];
#pragma unroll
        for (int j = 0; j < kHeads; ++j) {
            const int h = hb + j * kWarpsF;
            const bool have = h < nh;
            n[j] = have ? __ldcg(a.segs + (head0 + h) / G) : 0;
            post[j] = have ? __ldcg(a.post + head0 + h) : 0.f;
#pragma unroll
            for (int k = 0; k < PL; ++k)
                y[j][k] = have ? __ldcg(reinterpret_cast<const float2 *>(a.part_ml) + (head0 + h) * kMaxSplits + lane + 32 * k)
                               : make_float2(0.f, 0.f);
        }
#pragma unroll
        for (int j = 0; j < kHeads; ++j) {
            const int h = hb + j * kWarpsF;
            if (h >= nh) break;
            const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + (head0 + h) * kMaxSplits;
            float m = -INFINITY, w = 0.f;
#pragma unroll
            for (int k = 0; k < PL; ++k)
                if (lane + 32 * k < n[j]) m = fmaxf(m, y[j][k].x);
            for (int k = 32 * PL + lane; k < n[j]; k += 32) m = fmaxf(m, __ldcg(&ml[k].x));
            m = warp_max(m);
            const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
            for (int k = 0; k < PL; ++k)
                if (lane + 32 * k < n[j]) w += y[j][k].y * pow2(y[j][k].x - base);
            for (int k = 32 * PL + lane; k < n[j]; k += 32) {
                const float2 v = __ldcg(ml + k);
                w += v.y * pow2(v.x - base);
            }
            w = warp_sum(w);
            if (lane == 0) whole[h] = norm_of(post[j], m, w);
        }
    }
    __syncthreads();
    while (true) {
        Floats<V> s;
        s.fill(0.f);
        for (int j0 = 0; j0 < mine; j0 += kAhead) {
            if (j0) load(j0);
#pragma unroll
            for (int j = 0; j < kAhead; ++j) {
                const float4 n = whole[min((j0 + j) * HS + hs, nh - 1)];  // (past the last: 0)
#pragma unroll
                for (int v = 0; v < V; ++v) s.x[v] = fmaf(exp2_fast(fmaf(z[j].x[v], n.x, -n.y)), n.z, s.x[v]);
            }
        }
        if (HS > 1) {
            part[threadIdx.x] = s.x[0];
            __syncthreads();
            if (hs > 0) return;
#pragma unroll
            for (int k = 1; k < HS; ++k) s.x[0] += part[threadIdx.x + k * kTok];
        }
        const int64_t to = (int64_t)r * a.cap + token;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            // (each rounding named: every variant of the kernel gives the same bits)
            s.x[v] = __fmul_rn(s.x[v], 1.f / (float)nh);
            was.x[v] = __fmaf_rn(a.alpha, was.x[v], __fmul_rn(1.f - a.alpha, s.x[v]));
        }
        if (a.score) s.store(a.score + to, L - token);
        if (a.ema) was.store(a.ema + to, L - token);
        if (V == 1) return;  // (a block a CTA)
        token += a.row_ctas * kTok;
        if (token >= L) return;
        zp += a.row_ctas * kTok;
        load(0);
        if (a.ema) was.load(a.ema + (int64_t)r * a.cap + token);
    }
}

template <int D, typename T>
cudaError_t launch_t(const Q4AttendArgs &a, int ctas, cudaStream_t st) {
    constexpr size_t ring = sizeof(Tile<D>) * kPair * kStages * kWarps, smem = ring > kJoinBytes<D> ? ring : kJoinBytes<D>;
    static_assert(smem <= 48 << 10, "more shared memory needs an attribute of the kernel");
    // two tiles share the columns of a group of 4 or fewer, where the registers hold q for both
    constexpr bool kDual = sizeof(T) * D <= 256;
    const bool dual = kDual && a.q_heads <= 4 * a.pv.kv_heads;
    auto kernel = dual ? (a.logits ? q4_attend_kernel<D, T, true, kDual> : q4_attend_kernel<D, T, false, kDual>)
                       : (a.logits ? q4_attend_kernel<D, T, true, false> : q4_attend_kernel<D, T, false, false>);
    const cudaError_t e = launch_k(kernel, dim3((unsigned)ctas), dim3(kThreads), smem, st, a);
    note_launch();
    return e;
}

template <int HS, bool MANY, int V>
cudaError_t launch_finish_t(Q4FinishArgs a, int64_t rows, int32_t max_len, int sms, cudaStream_t st) {
    constexpr int tok = kFinishThreads / HS * V, heads = MANY ? 1 : kFinishThreads / 32;
    const int blocks = (max_len + tok - 1) / tok;
    a.row_ctas = V == 1 ? blocks : (int)std::min((int64_t)blocks, std::max(2 * (int64_t)sms / rows, (int64_t)1));
    const int64_t tokens = rows * a.row_ctas, merges = ((int64_t)a.batch * a.q_heads + heads - 1) / heads;
    if (tokens + merges > 0x7fffffff) return cudaErrorInvalidConfiguration;
    a.token_ctas = (int32_t)tokens;
    const int nh = a.rows_per_seq > 1 ? a.q_heads / a.kv_heads : a.q_heads;
    const int smem = (int)sizeof(float4) * nh;
    constexpr int kDefault = 32 << 10;  // with the kernel's own arrays within 48 KB
    cudaError_t e = cudaSuccess;
    if (smem > kDefault)
        e = cudaFuncSetAttribute(q4_finish_kernel<HS, MANY, V>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 (int)sizeof(float4) * kMaxQ4Heads);
    if (e != cudaSuccess) return e;
    e = launch_k(q4_finish_kernel<HS, MANY, V>, dim3((unsigned)(tokens + merges)), dim3(kFinishThreads), smem, st, a);
    note_launch();
    return e;
}
template <bool MANY>
cudaError_t launch_finish(const Q4FinishArgs &a, int32_t max_len, int sms, cudaStream_t st) {
    const int64_t rows = a.score || a.ema ? (int64_t)a.batch * a.rows_per_seq : 0;
    // Four tokens a thread from as many tokens on as take half of the SMs then: a CTA gathers its row's references
    // and sums once for several blocks of them.  us with the attention, one token a thread / four, batches of
    // 4k to 8k: 32 heads, a row a sequence, 64 blocks of 2048 tokens 31.7 / 33.4, 80 37.6 / 39.0, 96 45.8 / 45.6, 128
    // 56.8 / 55.7, 192 81.4 / 77.0; 16 heads, 64 17.5 / 17.6, 80 19.9 / 19.5, 192 34.7 / 30.8; 28 heads, a row for
    // each of 4 KV heads, 64 12.9 / 12.5, 96 16.3 / 15.1, 256 27.8 / 21.7.
    const bool aligned = (reinterpret_cast<uintptr_t>(a.score) | reinterpret_cast<uintptr_t>(a.ema)) % 16 == 0;
    if (aligned && rows > 0 && 2 * rows * ((max_len + 4 * kFinishThreads - 1) / (4 * kFinishThreads)) >= sms)
        return launch_finish_t<1, MANY, 4>(a, rows, max_len, sms, st);
    // else as many threads a token as it takes to give every SM a CTA
    if (rows * ((max_len + kFinishThreads - 1) / kFinishThreads) >= sms) return launch_finish_t<1, MANY, 1>(a, rows, max_len, sms, st);
    if (rows * ((max_len + kFinishThreads / 4 - 1) / (kFinishThreads / 4)) >= sms)
        return launch_finish_t<4, MANY, 1>(a, rows, max_len, sms, st);
    return launch_finish_t<8, MANY, 1>(a, rows, max_len, sms, st);
}

}  // namespace

// One wave of CTAs at most, a pair for each warp at least.
int32_t q4_attend_ctas(const ikv_shape *s, int32_t max_len, int sms) {
    // a start offset may put the first slot anywhere in its tile
    constexpr int kSlots = kPair * kQ4Tile;
    const int64_t pairs = max_len > 0 ? ((int64_t)max_len + kQ4Tile - 1 + kSlots - 1) / kSlots : 1;
    const int64_t ctas = (int64_t)s->batch * s->kv_heads * ((pairs + kWarps - 1) / kWarps), wave = (int64_t)sms * ctas_per_sm(s->head_dim, s->dtype == IKV_BF16 ? 2 : 4);
    return (int32_t)(ctas < wave ? ctas : wave);
}

cudaError_t launch_q4_attend(const Q4AttendArgs &a, int dtype, int head_dim, int32_t ctas, cudaStream_t st) {
    if (dtype == IKV_BF16)
        return head_dim == 128 ? launch_t<128, __nv_bfloat16>(a, ctas, st) : launch_t<64, __nv_bfloat16>(a, ctas, st);
    return head_dim == 128 ? launch_t<128, float>(a, ctas, st) : launch_t<64, float>(a, ctas, st);
}

cudaError_t launch_q4_finish(const Q4FinishArgs &a, int32_t ctas, int32_t max_len, int sms, cudaStream_t st) {
    // A CTA a head from a mean of 8 segments a unit on.  us with the attention, a warp a head / a CTA, without and with
    // scores (8 KV heads, 32 heads): one sequence, 8 segments 7.7 / 7.4 and 8.1 / 7.8, 16 8.1 / 7.9 and 10.0 / 8.6,
    // 57 18.4 / 15.9 and 26.5 / 18.0; two, 8 7.7 / 8.1 and 8.6 / 8.7, 28 22.9 / 21.3 and 34.0 / 27.6; four, 14 33.8 /
    // 33.2 and 39.4 / 41.0; six, 9.5 45.7 / 45.7 and 55.0 / 56.6; eight, 7 21.1 / 21.3 and 25.2 / 28.3; sixteen, 3.6
    // 34.9 / 37.6 and 39.1 / 44.0.  The host knows the mean alone: one long sequence among short ones
    // (60000 and 15 of 300: 25.4 / 23.0 and 38.2 / 32.6) goes by a warp a head.
    return ctas > 8 * (int64_t)a.batch * a.kv_heads ? launch_finish<true>(a, max_len, sms, st)
                                                     : launch_finish<false>(a, max_len, sms, st);
}

}  // namespace ikv
