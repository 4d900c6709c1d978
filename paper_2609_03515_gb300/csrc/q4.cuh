// Caches held in 4 bits (ikv_q4_*), and page pools (ikv_pages_*): internal declarations.
#pragma once
#include <cuda_fp16.h>

#include "ikv_internal.cuh"

namespace ikv {

// A group of 32 channels shares a scale s, the smallest bf16 number with 6 s >= the group's
// largest magnitude; a code is a sign and one of the magnitudes 0, .5, 1, 1.5, 2, 3, 4, 6 of s
// (the E2M1 numbers, which the GPU converts two at a time).
constexpr int kQ4Group = 32;
constexpr int kMaxQ4Heads = 8192;  // query heads
constexpr int kQ4Tile = 16;  // page sizes are multiples of it: the rows of one mma tile lie in one page

// the two codes in byte i of w, as fp16 (exact)
__device__ __forceinline__ uint32_t e2m1_bits(uint32_t w, int i) {
    uint32_t r;
    if (i == 0)
        asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}" : "=r"(r) : "r"(w));
    else if (i == 1)
        asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, b;\n\t}" : "=r"(r) : "r"(w));
    else if (i == 2)
        asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, c;\n\t}" : "=r"(r) : "r"(w));
    else
        asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, d;\n\t}" : "=r"(r) : "r"(w));
    return r;
}
__device__ __forceinline__ __half2 e2m1_pair(uint32_t w, int i) {
    const uint32_t r = e2m1_bits(w, i);
    return *reinterpret_cast<const __half2 *>(&r);
}

struct Q4Rows {  // dense rows on the caller's side: element (li, b, i, g, e)
    void *k, *v;
    int64_t layer, seq, token, head;  // strides, in elements
    const int32_t *row0;              // [batch] sequence b starts at token row0[b], or null (seq strides)
};

struct Q4MoveArgs {
    unsigned char *k, *v;             // codes: row of D / 2 bytes
    uint16_t *ks, *vs;                // scales: row of D / 32 bf16
    PagedView pv;
    Q4Rows rows;
    const int32_t *len, *first, *count;  // [batch]; first null: the newest slots, up to count; count null: max_count
    const int32_t *writable;          // [batch][2] slots that a store may write, or null: all
    int32_t batch, layer0, n_layers, max_count, cap;
    int32_t head_shift;               // log2(kv_heads), or -1
    int32_t blocks;                   // CTAs of one sequence's rows; set by the launcher
};
cudaError_t launch_q4_store(const Q4MoveArgs &a, int dtype, cudaStream_t st);
cudaError_t launch_q4_load(const Q4MoveArgs &a, int dtype, cudaStream_t st);

struct Q4AttendArgs {
    const unsigned char *k, *v;
    const uint16_t *ks, *vs;
    PagedView pv;
    const int32_t *len, *pos;         // pos: [rows][cap] with -1 at dead slots, or null
    const void *q;                    // [batch][q_heads][D] (dtype)
    void *out;                        // the same
    int32_t batch, q_heads, layer, rows_per_seq, cap;
    float scale_log2;
    float *logits;                    // [batch][q_heads][lstride] logits; post of their head times them is
                                      // log2 of the weights.  Or null
    float *post;                      // [batch][q_heads] (of sequences that have a slot)
    int32_t lstride;
    float *part_ml, *part_o;          // [batch][q_heads][kMaxSplits][2], [..][D]: reference and sum of each
                                      // segment, and outputs of units of several
    int32_t *segs;                    // [batch][kv_heads] segments of a unit (of sequences that have a slot)
};
// CTAs of an attention launch at lengths up to max_len
int32_t q4_attend_ctas(const ikv_shape *s, int32_t max_len, int sms);
cudaError_t launch_q4_attend(const Q4AttendArgs &a, int dtype, int head_dim, int32_t ctas, cudaStream_t st);

struct Q4FinishArgs {
    const int32_t *len;
    int32_t batch, q_heads, kv_heads, rows_per_seq, cap, head_dim, bf16;
    const float *logits;
    int32_t lstride;
    const float *post, *part_ml, *part_o;
    const int32_t *segs;
    void *out;
    float alpha;
    float *score, *ema;               // [rows][cap] or null
    int32_t token_ctas, row_ctas;     // CTAs of all rows' tokens, of a row's; set by the launcher
};
// ctas: of the attention launch before
cudaError_t launch_q4_finish(const Q4FinishArgs &a, int32_t ctas, int32_t max_len, int sms, cudaStream_t st);

// ---- page pools (pages.cu)
constexpr int kMaxPlanes = IKV_MAX_PLANES;
struct PagesArgs {
    unsigned char *plane[kMaxPlanes];
    int32_t row_bytes[kMaxPlanes];
    int32_t n_planes;
    int32_t *refs;                    // [num_pages] holders of a page
    int32_t *table;                   // [batch][max_pages], 0 = none
    int32_t num_pages, page_size, max_pages, kv_heads, layers, batch, rows_per_seq, cap;
    int32_t *len, *next_pos, *start, *pos;
    int2 *writable;                   // [batch] slots granted, or null
    float *ema, *vnorm;
};
// scratch of one call: what its kernels hand to one another
struct PagesWs {
    int32_t *total;                   // [4]: jobs; whether there were pages enough (compaction);
                                      // rows of the longest copy (writable); -
    int32_t *free_ids;                // [batch * max_pages] the free pages that the call takes, ascending
    int32_t *count, *last;            // [num_pages] writers of a shared page, the last of them
    int32_t *jobs;                    // [batch * max_pages][4]; a compaction's old table entries
    int32_t *begin, *base;            // [batch + 1] first page made anew, jobs of the sequences before
};
size_t pages_ws(int32_t batch, int32_t max_pages, int32_t num_pages, void *ws, PagesWs *w);
cudaError_t launch_pages_release(const PagesArgs &a, int32_t extra, cudaStream_t st);
cudaError_t launch_pages_fork(const PagesArgs &a, int32_t n, const int32_t *src, const int32_t *dst, cudaStream_t st);
cudaError_t launch_pages_writable(const PagesArgs &a, const PagesWs &w, const int32_t *first, const int32_t *count,
                                  int32_t max_count, int32_t *lacking, int sms, cudaStream_t st);
cudaError_t launch_pages_compact(const PagesArgs &a, const PagesWs &w, const int32_t *keep, const int32_t *keep_len,
                                 int32_t *lacking, int sms, cudaStream_t st);

}  // namespace ikv
