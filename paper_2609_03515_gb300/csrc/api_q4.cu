// C ABI of the 4-bit caches and the page pools: argument checks and launches.
#include <cmath>

#include "q4.cuh"

using namespace ikv;

namespace {

ikv_status check_q4(const ikv_shape *s, const ikv_cache *c, const ikv_q4 *q) {
    clear_error();
    ikv_status e = check_shape(s);
    if (e) return e;
    if ((e = check_cache(s, c, false))) return e;
    if (!q || !q->k_scale || !q->v_scale) return report(IKV_ERR_ARG, "q4 or its scale pools are NULL");
    if (!aligned16(q->k_scale) || !aligned16(q->v_scale)) return report(IKV_ERR_ALIGN, "scale pools must be 16-byte aligned");
    if (c->page_size % kQ4Tile) return report(IKV_ERR_UNSUPPORTED, "page_size must be a multiple of %d", kQ4Tile);
    return IKV_OK;
}

ikv_status move_rows(const ikv_shape *s, const ikv_cache *c, const ikv_q4 *q, int32_t layer0, int32_t n_layers,
                     const void *k, const void *v, const ikv_rows *rows, const int32_t *first, const int32_t *count,
                     int32_t max_count, bool store, cudaStream_t st) {
    if (layer0 < 0 || n_layers < 0 || layer0 > s->layers - n_layers)
        return report(IKV_ERR_ARG, "layers [%d, %d + %d) out of range", layer0, layer0, n_layers);
    if (max_count < 0 || max_count > cap_of(c)) return report(IKV_ERR_SHAPE, "max_count %d outside [0, cap]", max_count);
    if ((int64_t)max_count * s->kv_heads > 0x7fff0000)  // (the kernel counts a CTA's rows past them)
        return report(IKV_ERR_SHAPE, "max_count * kv_heads too large");
    if (max_count == 0 || n_layers == 0) return IKV_OK;  // (whatever the rows of nothing are)
    if (!k || !v || !rows) return report(IKV_ERR_ARG, "k/v/rows is NULL");
    const int64_t unit = s->dtype == IKV_BF16 ? 8 : 4;  // elements of 16 bytes
    if (!aligned16(k) || !aligned16(v) || rows->layer % unit || rows->seq % unit || rows->token % unit || rows->head % unit)
        return report(IKV_ERR_ALIGN, "k/v rows must lie on 16-byte boundaries");
    Q4MoveArgs a{};
    a.k = static_cast<unsigned char *>(c->k);
    a.v = static_cast<unsigned char *>(c->v);
    a.ks = static_cast<uint16_t *>(q->k_scale);
    a.vs = static_cast<uint16_t *>(q->v_scale);
    a.pv = view_of(s, c);
    a.rows = Q4Rows{const_cast<void *>(k), const_cast<void *>(v), rows->layer, rows->seq, rows->token, rows->head, rows->row0};
    a.len = c->len;
    a.first = first;
    a.count = count;
    a.writable = c->writable;
    a.batch = s->batch;
    a.layer0 = layer0;
    a.n_layers = n_layers;
    a.max_count = max_count;
    a.cap = cap_of(c);
    a.head_shift = (s->kv_heads & (s->kv_heads - 1)) == 0 ? __builtin_ctz((unsigned)s->kv_heads) : -1;
    PdlScope pdl;
    IKV_TRY_CUDA(store ? launch_q4_store(a, s->dtype, st) : launch_q4_load(a, s->dtype, st),
                 store ? "4-bit store launch" : "4-bit load launch");
    return IKV_OK;
}

ikv_status check_pages(const ikv_shape *s, const ikv_cache *c, const ikv_pages *p, bool need_pos, PagesArgs *a) {
    clear_error();
    ikv_status e = check_shape(s);
    if (e) return e;
    if (!c) return report(IKV_ERR_ARG, "cache is NULL");
    ikv_cache same = *c;  // (no page call goes by max_len, so a bound past the slot space is one too)
    if (c->max_len > 0) same.max_len = 0;
    if ((e = check_cache(s, &same, need_pos))) return e;
    if (!p || !p->refs) return report(IKV_ERR_ARG, "pages or its refs is NULL");
    if (reinterpret_cast<uintptr_t>(c->writable) % sizeof(int2)) return report(IKV_ERR_ALIGN, "cache->writable must be 8-byte aligned");
    if (c->num_pages > 0x7fff0000) return report(IKV_ERR_SHAPE, "too many pages");  // (the search counts past them)
    if (p->n_planes < 1 || p->n_planes > kMaxPlanes) return report(IKV_ERR_SHAPE, "n_planes outside [1, %d]", kMaxPlanes);
    for (int i = 0; i < p->n_planes; ++i) {
        if (!p->plane[i]) return report(IKV_ERR_ARG, "plane %d is NULL", i);
        if (!aligned16(p->plane[i])) return report(IKV_ERR_ALIGN, "planes must be 16-byte aligned");
        if (p->row_bytes[i] <= 0 || p->row_bytes[i] % 4)
            return report(IKV_ERR_SHAPE, "row_bytes must be positive multiples of 4");
        if ((int64_t)p->row_bytes[i] * c->page_size > (int64_t)1 << 24) return report(IKV_ERR_SHAPE, "page too large");
        a->plane[i] = static_cast<unsigned char *>(p->plane[i]);
        a->row_bytes[i] = p->row_bytes[i];
    }
    a->n_planes = p->n_planes;
    a->refs = p->refs;
    a->table = const_cast<int32_t *>(c->block_table);
    a->num_pages = c->num_pages;
    a->page_size = c->page_size;
    a->max_pages = c->max_pages;
    a->kv_heads = s->kv_heads;
    a->layers = s->layers;
    a->batch = s->batch;
    a->rows_per_seq = rows_per_seq(s);
    a->cap = cap_of(c);
    a->len = c->len;
    a->next_pos = c->next_pos;
    a->start = c->start;
    a->pos = c->pos;
    a->writable = reinterpret_cast<int2 *>(c->writable);
    a->vnorm = c->vnorm;
    return IKV_OK;
}

ikv_status check_pages_ws(const PagesArgs &a, void *ws, size_t bytes, PagesWs *w) {
    const size_t need = pages_ws(a.batch, a.max_pages, a.num_pages, ws, w);
    if (!ws || bytes < need) return report(IKV_ERR_WORKSPACE, "workspace needs %zu bytes", need);
    if (!aligned16(ws)) return report(IKV_ERR_ALIGN, "workspace must be 16-byte aligned");
    return IKV_OK;
}

}  // namespace

extern "C" {

ikv_status ikv_q4_store(const ikv_shape *shape, const ikv_cache *cache, const ikv_q4 *q4, int32_t layer0,
                        int32_t n_layers, const void *k, const void *v, const ikv_rows *rows, const int32_t *first,
                        const int32_t *count, int32_t max_count, cudaStream_t stream) {
    const ikv_status e = check_q4(shape, cache, q4);
    return e ? e : move_rows(shape, cache, q4, layer0, n_layers, k, v, rows, first, count, max_count, true, stream);
}

ikv_status ikv_q4_load(const ikv_shape *shape, const ikv_cache *cache, const ikv_q4 *q4, int32_t layer0,
                       int32_t n_layers, void *k, void *v, const ikv_rows *rows, const int32_t *first,
                       const int32_t *count, int32_t max_count, cudaStream_t stream) {
    const ikv_status e = check_q4(shape, cache, q4);
    return e ? e : move_rows(shape, cache, q4, layer0, n_layers, k, v, rows, first, count, max_count, false, stream);
}

ikv_status ikv_q4_append_token(const ikv_shape *shape, ikv_cache *cache, const ikv_q4 *q4, const void *k_new,
                               const void *v_new, float *ema, int32_t init_mean, int32_t *slot, cudaStream_t stream) {
    ikv_status e = check_q4(shape, cache, q4);
    if (e) return e;
    if ((e = check_cache(shape, cache, true))) return e;
    if (!slot) return report(IKV_ERR_ARG, "slot is NULL");
    if (!k_new != !v_new) return report(IKV_ERR_ARG, "one of k_new/v_new is NULL");
    if (k_new && (!aligned16(k_new) || !aligned16(v_new)))
        return report(IKV_ERR_ALIGN, "k_new/v_new must be 16-byte aligned");
    if (cache->max_len + 1 > cap_of(cache)) return report(IKV_ERR_SHAPE, "no free slot: max_len + 1 > cap");
    AppendArgs a{};
    a.pv = view_of(shape, cache);
    a.batch = shape->batch;
    a.layers = shape->layers;
    a.rows_per_seq = rows_per_seq(shape);
    a.cap = cap_of(cache);
    a.len = cache->len;
    a.pos = cache->pos;
    a.next_pos = cache->next_pos;
    a.ema = ema;
    a.init_mean = ema ? init_mean : 0;
    a.dead_slots = cache->dead_slots ? 1 : 0;
    a.slot = slot;
    a.writable = cache->writable;
    PdlScope pdl;
    IKV_TRY_CUDA(launch_append(a, stream), "append launch");
    if (!k_new) return IKV_OK;
    const int64_t head = shape->head_dim, seq = head * shape->kv_heads;
    const ikv_rows rows{seq * shape->batch, seq, seq, head, nullptr};
    return move_rows(shape, cache, q4, 0, shape->layers, k_new, v_new, &rows, slot, nullptr, 1, true, stream);
}

ikv_status ikv_q4_attend_score(const ikv_shape *shape, const ikv_cache *cache, const ikv_q4 *q4, int32_t layer,
                               const void *q, void *out, float *score, float *ema, float alpha, void *ws,
                               size_t ws_bytes, cudaStream_t stream) {
    const ikv_status e = check_q4(shape, cache, q4);
    if (e) return e;
    if (layer < 0 || layer >= shape->layers) return report(IKV_ERR_ARG, "layer %d out of range", layer);
    if (!q || !out) return report(IKV_ERR_ARG, "q/out is NULL");
    if (!aligned16(q) || !aligned16(out)) return report(IKV_ERR_ALIGN, "q/out must be 16-byte aligned");
    if (ema && !(alpha >= 0.f && alpha <= 1.f)) return report(IKV_ERR_ARG, "alpha must be in [0, 1]");
    if (shape->q_heads > kMaxQ4Heads) return report(IKV_ERR_SHAPE, "more than %d query heads", kMaxQ4Heads);
    const bool want_score = score || ema;
    const AttendWs w = attend_ws(shape, cap_of(cache), 1, want_score);
    if (!ws || ws_bytes < w.end) return report(IKV_ERR_WORKSPACE, "workspace needs %zu bytes", w.end);
    if (!aligned16(ws)) return report(IKV_ERR_ALIGN, "workspace must be 16-byte aligned");
    Q4AttendArgs a{};
    a.k = static_cast<const unsigned char *>(cache->k);
    a.v = static_cast<const unsigned char *>(cache->v);
    a.ks = static_cast<const uint16_t *>(q4->k_scale);
    a.vs = static_cast<const uint16_t *>(q4->v_scale);
    a.pv = view_of(shape, cache);
    a.len = cache->len;
    a.pos = cache->dead_slots ? cache->pos : nullptr;
    a.q = q;
    a.out = out;
    a.batch = shape->batch;
    a.q_heads = shape->q_heads;
    a.layer = layer;
    a.rows_per_seq = rows_per_seq(shape);
    a.cap = cap_of(cache);
    a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)shape->head_dim));
    a.logits = want_score ? at<float>(ws, w.logits) : nullptr;
    a.post = at<float>(ws, w.lse2);  // (the same size)
    a.lstride = logit_stride(a.cap);
    a.part_ml = at<float>(ws, w.part_ml);
    a.part_o = at<float>(ws, w.part_o);
    a.segs = at<int32_t>(ws, w.arrivals);
    // (the kernels count the sequences' pairs of tiles in 32 bits, with some to spare for each unit)
    if ((int64_t)shape->batch * shape->kv_heads * (a.cap / 32 + 64) > 0x30000000)
        return report(IKV_ERR_SHAPE, "batch * kv_heads * cap too large");
    // (and name a pool's tiles in 32 bits)
    if ((uint64_t)shape->layers * shape->kv_heads * cache->num_pages * (cache->page_size / kQ4Tile) > 0xffffffffu)
        return report(IKV_ERR_SHAPE, "pool too large");
    PdlScope pdl;
    const int32_t ctas = q4_attend_ctas(shape, cache->max_len, sm_count());
    IKV_TRY_CUDA(launch_q4_attend(a, shape->dtype, shape->head_dim, ctas, stream), "4-bit attend launch");
    Q4FinishArgs f{};
    f.len = cache->len;
    f.batch = shape->batch;
    f.q_heads = shape->q_heads;
    f.kv_heads = shape->kv_heads;
    f.rows_per_seq = a.rows_per_seq;
    f.cap = a.cap;
    f.head_dim = shape->head_dim;
    f.bf16 = shape->dtype == IKV_BF16;
    f.segs = a.segs;
    f.logits = a.logits;
    f.post = a.post;
    f.lstride = a.lstride;
    f.part_ml = a.part_ml;
    f.part_o = a.part_o;
    f.out = out;
    f.alpha = alpha;
    f.score = score;
    f.ema = ema;
    IKV_TRY_CUDA(launch_q4_finish(f, ctas, cache->max_len, sm_count(), stream), "4-bit score launch");
    return IKV_OK;
}

ikv_status ikv_pages_workspace_size(const ikv_shape *shape, const ikv_cache *cache, const ikv_pages *pages,
                                    size_t *bytes) {
    PagesArgs a{};
    const ikv_status e = check_pages(shape, cache, pages, false, &a);
    if (e) return e;
    if (!bytes) return report(IKV_ERR_ARG, "bytes is NULL");
    *bytes = pages_ws(a.batch, a.max_pages, a.num_pages, nullptr, nullptr);
    return IKV_OK;
}

ikv_status ikv_pages_release(const ikv_shape *shape, ikv_cache *cache, const ikv_pages *pages, int32_t extra,
                             cudaStream_t stream) {
    PagesArgs a{};
    const ikv_status e = check_pages(shape, cache, pages, false, &a);
    if (e) return e;
    if (extra < 0) return report(IKV_ERR_ARG, "extra must be >= 0");
    PdlScope pdl;
    IKV_TRY_CUDA(launch_pages_release(a, extra, stream), "page release launch");
    return IKV_OK;
}

ikv_status ikv_pages_fork(const ikv_shape *shape, ikv_cache *cache, const ikv_pages *pages, int32_t n,
                          const int32_t *src, const int32_t *dst, float *ema, cudaStream_t stream) {
    PagesArgs a{};
    const ikv_status e = check_pages(shape, cache, pages, false, &a);
    if (e) return e;
    if (cache->pos_cap > 0) return report(IKV_ERR_UNSUPPORTED, "pos and ema laid out for per-layer eviction");
    if (n < 0 || n > shape->batch || n > 65535) return report(IKV_ERR_SHAPE, "n %d outside [0, batch]", n);
    if (n == 0) return IKV_OK;
    if (!src || !dst) return report(IKV_ERR_ARG, "src/dst is NULL");
    a.ema = ema;
    PdlScope pdl;
    IKV_TRY_CUDA(launch_pages_fork(a, n, src, dst, stream), "page fork launch");
    return IKV_OK;
}

ikv_status ikv_pages_writable(const ikv_shape *shape, ikv_cache *cache, const ikv_pages *pages, const int32_t *first,
                              const int32_t *count, int32_t max_count, int32_t *lacking, void *ws, size_t ws_bytes,
                              cudaStream_t stream) {
    PagesArgs a{};
    PagesWs w;
    ikv_status e = check_pages(shape, cache, pages, false, &a);
    if (e) return e;
    if (max_count < 0 || max_count > a.cap) return report(IKV_ERR_SHAPE, "max_count %d outside [0, cap]", max_count);
    if ((e = check_pages_ws(a, ws, ws_bytes, &w))) return e;
    if (max_count == 0 && !lacking) return IKV_OK;
    PdlScope pdl;
    IKV_TRY_CUDA(launch_pages_writable(a, w, first, count, max_count, lacking, sm_count(), stream), "page writable launch");
    return IKV_OK;
}

ikv_status ikv_pages_compact(const ikv_shape *shape, ikv_cache *cache, const ikv_pages *pages, const int32_t *keep,
                             const int32_t *keep_len, float *ema, int32_t *lacking, void *ws, size_t ws_bytes,
                             cudaStream_t stream) {
    PagesArgs a{};
    PagesWs w;
    ikv_status e = check_pages(shape, cache, pages, false, &a);
    if (e) return e;
    if (cache->pos_cap > 0) return report(IKV_ERR_UNSUPPORTED, "pos and ema laid out for per-layer eviction");
    if (!keep || !keep_len) return report(IKV_ERR_ARG, "keep/keep_len is NULL");
    if ((e = check_pages_ws(a, ws, ws_bytes, &w))) return e;
    a.ema = ema;
    PdlScope pdl;
    IKV_TRY_CUDA(launch_pages_compact(a, w, keep, keep_len, lacking, sm_count(), stream), "page compaction launch");
    return IKV_OK;
}

}  // extern "C"
