// C ABI of the shared-prefix decode and of the sliding window: argument checks, workspace, launches.
#include <cmath>

#include "rows.cuh"

using namespace ikv;

namespace {

ikv_status check_rows(const ikv_shape *s, const ikv_cache *c) {
    clear_error();
    ikv_status e = check_shape(s);
    if (e) return e;
    if ((e = check_dense(s, c, false))) return e;
    if (s->q_heads > 8192) return report(IKV_ERR_SHAPE, "more than 8192 query heads");
    return IKV_OK;
}

// (a CTA's share of a call's cost is counted in 32 bits: `units` sets of query rows over up to cap slots)
ikv_status check_cost(const ikv_shape *s, const ikv_cache *c, int64_t units) {
    const int64_t pairs = units * s->kv_heads, tiles = cap_of(c) / kRowsTile + 4;
    if (pairs / sm_count() > ((int64_t)1 << 31) / (kTileTwo * tiles + kExtraTwo) - 1)
        return report(IKV_ERR_SHAPE, "too many query rows over too long a slot space");
    return IKV_OK;
}

ikv_status check_prefix(const ikv_shape *s, const ikv_cache *c, const ikv_prefix *p) {
    const ikv_status e = check_rows(s, c);
    if (e) return e;
    if (!p) return report(IKV_ERR_ARG, "prefix is NULL");
    if (p->n_groups < 0) return report(IKV_ERR_ARG, "n_groups must be >= 0");
    if (p->n_groups > 0 && (!p->first || !p->member || !p->len))
        return report(IKV_ERR_ARG, "prefix first/member/len is NULL");
    if (p->n_groups > (1 << 20) || (int64_t)s->batch * s->q_heads > 1 << 28)
        return report(IKV_ERR_SHAPE, "too many groups or query rows");
    return check_cost(s, c, 2 * (int64_t)s->batch + p->n_groups);
}

ikv_status check_window(const ikv_shape *s, const ikv_cache *c, const ikv_window *w) {
    const ikv_status e = check_rows(s, c);
    if (e) return e;
    if (!w) return report(IKV_ERR_ARG, "window is NULL");
    if (w->window < 0 || w->sinks < 0) return report(IKV_ERR_ARG, "window and sinks must be >= 0");
    if (w->max_count < 0) return report(IKV_ERR_ARG, "max_count must be >= 0");
    if ((int64_t)s->batch * w->max_count > ((int64_t)1 << 30) / s->q_heads)
        return report(IKV_ERR_SHAPE, "batch * max_count * q_heads too large");
    const int64_t row = (int64_t)s->q_heads * s->head_dim, unit = s->dtype == IKV_BF16 ? 8 : 4;
    for (const int64_t x : {w->q_stride, w->out_stride}) {
        if (x == 0) continue;
        if (x < row) return report(IKV_ERR_SHAPE, "a token's row holds %lld elements", (long long)row);
        if (x % unit) return report(IKV_ERR_ALIGN, "rows of q and out must lie on 16-byte boundaries");
    }
    // (16 query rows a unit at least but for its last)
    return check_cost(s, c, (int64_t)s->batch * (w->max_count / (16 / (s->q_heads / s->kv_heads)) + 1));
}

// The arguments of a call but for its pointers to q and results, and its workspace: *bytes of it, at ws
// if there is one.
// (score: the call's score pass needs its own; sizes are with it)
RowsArgs rows_args(const ikv_shape *s, const ikv_cache *c, const ikv_prefix *p, const ikv_window *w, void *ws,
                   size_t *bytes, bool score = true) {
    RowsArgs a{};
    a.k = c->k;
    a.v = c->v;
    a.pv = view_of(s, c);
    a.len = c->len;
    a.pos = c->dead_slots ? c->pos : nullptr;
    a.rows_per_seq = rows_per_seq(s);
    a.cap = cap_of(c);
    a.batch = s->batch;
    a.q_heads = s->q_heads;
    a.group = s->q_heads / s->kv_heads;
    a.scale_log2 = (float)(1.4426950408889634 / std::sqrt((double)s->head_dim));
    a.q_stride = a.out_stride = (int64_t)s->q_heads * s->head_dim;
    const bool tc = rows_tc_supported(s, c);
    a.ctas = sm_count() * (tc ? 1 : rows_simt_ctas_per_sm(s->head_dim));
    if (a.ctas > kRowsMaxCtas) a.ctas = kRowsMaxCtas;
    const int n = p ? s->batch : w->max_count;
    const int most = tc ? 2 * (128 / a.group) : kRowsSimt / a.group;  // (tensor cores: two row tiles)
    a.tile_n = tc ? 128 / a.group : most;
    a.unit_n = n <= a.tile_n ? a.tile_n : most;
    a.rows_cap = (n < most ? n : most) * a.group;
    int64_t units;
    if (w) {
        if (w->q_stride) a.q_stride = w->q_stride;
        if (w->out_stride) a.out_stride = w->out_stride;
        a.window = w->window > 0 && w->window < 1 << 30 ? w->window : 1 << 30;
        a.sinks = w->sinks < 1 << 30 ? w->sinks : (1 << 30) - 1;
        a.row0 = w->row0;
        a.count = w->count;
        a.max_count = w->max_count;
        a.seq_units = (w->max_count + a.unit_n - 1) / a.unit_n;
        units = (int64_t)s->batch * a.seq_units;
        a.small = units <= 32;
    } else {
        a.prefix = 1;
        a.n_groups = p->n_groups;
        a.first = p->first;
        a.member = p->member;
        a.group_len = p->len;
        a.small = s->batch <= 32 && p->n_groups <= 32 && s->batch <= a.unit_n;
        units = (int64_t)p->n_groups + s->batch / a.unit_n + s->batch;
    }
    // (64 units, each with at most cap / 128 + 2 tiles of cost 4 and 12 more, and twice that many items)
    a.small = a.small && (int64_t)(a.cap / kRowsTile + 8) * s->kv_heads * 64 * 4 < (int64_t)1 << 31;
    size_t off = 0;
    auto take = [&](auto *&x, size_t count) {
        x = ws ? at<std::remove_reference_t<decltype(*x)>>(ws, off) : nullptr;
        off = align256(off + count * sizeof(*x));
    };
    take(a.head, 1);
    take(a.start, a.ctas);
    take(a.units, units);
    if (a.pos && tc) {  // (the kernels without tensor cores read the positions themselves)
        a.live_words = (a.cap + 31) / 32;
        take(a.live, (size_t)a.batch * a.rows_per_seq * a.live_words);
    }
    if (tc && p) {
        // (64 columns a thread: an item's members, half of them each, are 2 (64 / G))
        a.item_n = 2 * (64 / a.group);
        // a utility row a KV head: an item each while there are few, else one for all of them, which looks up its
        // unit and members once.  (One prefix, 8 KV heads, one item / one each, us a call: 4 members of 2k 31.5 / 27.9, 8
        // of 2k 32.5 / 30.0, 8 of 8k 39.4 / 41.2, 16 of 8k, the first that take one, 47.3 / 50.4, 64 of 8k 95 / 115)
        a.item_subs = a.rows_per_seq > 1 && (int64_t)s->batch * (c->max_len / kRowsTile + 1) < 4 * a.ctas ? s->kv_heads : 1;
        take(a.items, a.ctas);
        take(a.icum, units);
        if (!score) {
            a.items = nullptr;
            a.icum = nullptr;
        }
    }
    const size_t pre = p ? (size_t)(p->n_groups + s->batch / a.unit_n) * s->kv_heads + a.ctas : 2 * (size_t)a.ctas;
    take(a.part_ml, pre * a.rows_cap);
    take(a.part_o, pre * a.rows_cap * s->head_dim);
    if (p) {
        const size_t nb = s->batch, own = (nb * s->kv_heads + a.ctas) * a.group;
        take(a.owner, nb);
        take(a.vm, nb);
        take(a.entry_group, nb);
        take(a.group_p, p->n_groups);
        take(a.group_lead, p->n_groups);
        take(a.group_unit, p->n_groups);
        take(a.seq, nb);
        take(a.norm, nb * s->q_heads);
        take(a.own_ml, own);
        take(a.own_o, own * s->head_dim);
    }
    *bytes = off;
    return a;
}

ikv_status check_call(const ikv_shape *s, int32_t layer, const void *q, const void *out, const void *ws, size_t ws_bytes,
                      size_t need) {
    if (layer < 0 || layer >= s->layers) return report(IKV_ERR_ARG, "layer %d out of range", layer);
    if (!q || !out) return report(IKV_ERR_ARG, "q/out is NULL");
    if (!aligned16(q) || !aligned16(out)) return report(IKV_ERR_ALIGN, "q/out must be 16-byte aligned");
    if (!ws || ws_bytes < need) return report(IKV_ERR_WORKSPACE, "workspace needs %zu bytes", need);
    if (!aligned16(ws)) return report(IKV_ERR_ALIGN, "workspace must be 16-byte aligned");
    return IKV_OK;
}

ikv_status attend(const RowsArgs &a, const ikv_shape *s, const ikv_cache *c, cudaStream_t st) {
    IKV_TRY_CUDA(launch_rows_plan(a, st), "row plan launch");
    IKV_TRY_CUDA(rows_tc_supported(s, c) ? launch_rows_tc(a, s->head_dim, st) : launch_rows_simt(a, s->dtype, s->head_dim, st),
                 "row attention launch");
    IKV_TRY_CUDA(launch_rows_merge(a, s->dtype, s->head_dim, st), "row merge launch");
    return IKV_OK;
}

}  // namespace

extern "C" {

ikv_status ikv_prefix_workspace_size(const ikv_shape *shape, const ikv_cache *cache, const ikv_prefix *prefix,
                                     size_t *bytes) {
    const ikv_status e = check_prefix(shape, cache, prefix);
    if (e) return e;
    if (!bytes) return report(IKV_ERR_ARG, "bytes is NULL");
    rows_args(shape, cache, prefix, nullptr, nullptr, bytes);
    return IKV_OK;
}

ikv_status ikv_prefix_attend_score(const ikv_shape *shape, const ikv_cache *cache, const ikv_prefix *prefix,
                                   int32_t layer, const void *q, void *out, float *score, float *ema, float alpha,
                                   void *ws, size_t ws_bytes, cudaStream_t stream) {
    ikv_status e = check_prefix(shape, cache, prefix);
    if (e) return e;
    size_t need = 0;
    RowsArgs a = rows_args(shape, cache, prefix, nullptr, ws, &need, score || ema);
    if ((e = check_call(shape, layer, q, out, ws, ws_bytes, need))) return e;
    if (ema && !(alpha >= 0.f && alpha <= 1.f)) return report(IKV_ERR_ARG, "alpha must be in [0, 1]");
    a.layer = layer;
    a.q = q;
    a.out = out;
    PdlScope pdl;
    if ((e = attend(a, shape, cache, stream))) return e;
    if (!score && !ema) return IKV_OK;
    const RowsScoreArgs sc{alpha, score, ema, cache->max_len};
    IKV_TRY_CUDA(a.items ? launch_rows_score_tc(a, sc, shape->head_dim, stream)
                         : launch_rows_score(a, sc, shape->dtype, shape->head_dim, stream),
                 "row score launch");
    return IKV_OK;
}

ikv_status ikv_window_workspace_size(const ikv_shape *shape, const ikv_cache *cache, const ikv_window *window,
                                     size_t *bytes) {
    const ikv_status e = check_window(shape, cache, window);
    if (e) return e;
    if (!bytes) return report(IKV_ERR_ARG, "bytes is NULL");
    rows_args(shape, cache, nullptr, window, nullptr, bytes);
    return IKV_OK;
}

ikv_status ikv_window_attend(const ikv_shape *shape, const ikv_cache *cache, const ikv_window *window, int32_t layer,
                             const void *q, void *out, void *ws, size_t ws_bytes, cudaStream_t stream) {
    ikv_status e = check_window(shape, cache, window);
    if (e) return e;
    size_t need = 0;
    RowsArgs a = rows_args(shape, cache, nullptr, window, ws, &need);
    if ((e = check_call(shape, layer, q, out, ws, ws_bytes, need))) return e;
    if (window->max_count == 0) return IKV_OK;
    a.layer = layer;
    a.q = q;
    a.out = out;
    PdlScope pdl;
    return attend(a, shape, cache, stream);
}

}  // extern "C"
