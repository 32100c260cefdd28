// group_ops.cpp -- the operators of include/corun.h for sequences that share a
// beginning: host-side checks, then the launches.  Nothing here allocates, waits
// or keeps anything from one call for the next.
#include <hip/hip_runtime.h>

#include "cache_ops.h"
#include "groups.h"

using namespace corun;

#define TRY(expr)                       \
    do {                                \
        corun_status s_ = (expr);       \
        if (s_ != CORUN_OK) return s_;  \
    } while (0)

extern "C" int64_t corun_beam_select_workspace(int32_t vocab, int32_t groups, int32_t beams, int32_t n_keep)
{
    if (vocab < 1 || vocab > (1 << 19)) return set_errorf(CORUN_E_SHAPE, "vocab %d outside [1, 2^19]", vocab);
    if (beams < 1 || beams > CORUN_MAX_BEAMS)
        return set_errorf(CORUN_E_SHAPE, "beams %d outside [1, %d]", beams, CORUN_MAX_BEAMS);
    if (n_keep < 1 || n_keep > CORUN_MAX_BEAMS)
        return set_errorf(CORUN_E_SHAPE, "n_keep %d outside [1, %d]", n_keep, CORUN_MAX_BEAMS);
    if (groups < 1 || (int64_t)groups * beams > 65535)
        return set_errorf(CORUN_E_SHAPE, "%d groups of %d beams: 1 to 65535 rows are supported", groups, beams);
    return (int64_t)beam_ws(vocab, groups, beams, n_keep);
}

extern "C" corun_status corun_beam_select(const float *logits, int64_t ld, int32_t vocab, int32_t groups, int32_t beams,
                                          const float *scores, const uint8_t *valid, const uint8_t *finished,
                                          const float *weights, int32_t end_token, int32_t n_keep, int32_t *tokens,
                                          int32_t *parents, float *out_scores, uint8_t *out_finished, void *ws,
                                          int64_t ws_bytes, void *stream)
{
    const int64_t need = corun_beam_select_workspace(vocab, groups, beams, n_keep);
    if (need < 0) return (corun_status)need;
    if (!logits || !scores || !tokens || !parents || !out_scores) return set_error(CORUN_E_INVAL, "null argument");
    if (((uintptr_t)logits & 3) != 0) return set_error(CORUN_E_INVAL, "logits must start on 4 bytes");
    if (ld < vocab) return set_errorf(CORUN_E_SHAPE, "logits row stride %lld below vocab %d", (long long)ld, vocab);
    if (end_token < -1 || end_token >= vocab)
        return set_errorf(CORUN_E_INVAL, "end_token %d outside [-1, %d)", end_token, vocab);
    if (finished && end_token < 0) return set_error(CORUN_E_INVAL, "finished rows need an end_token");
    TRY(check_ws(ws, ws_bytes, need));
    BeamArgs a;
    a.logits = logits;
    a.ld = ld;
    a.vocab = vocab;
    a.groups = groups;
    a.beams = beams;
    a.keep = n_keep;
    a.end_token = end_token;
    a.scores = scores;
    a.weights = weights;
    a.valid = valid;
    a.finished = finished;
    a.tokens = tokens;
    a.parents = parents;
    a.out_scores = out_scores;
    a.out_finished = out_finished;
    return launched(launch_beam_select(a, ws, (hipStream_t)stream));
}

namespace {

corun_status check_pages(const corun_kv *kv)
{
    if (!kv) return set_error(CORUN_E_INVAL, "null kv");
    TRY(check_cache(kv));
    if (kv->layout != CORUN_KV_PAGED) return set_error(CORUN_E_INVAL, "pages of a paged cache are assigned");
    if (kv->page_size > (1 << 20)) return set_error(CORUN_E_SHAPE, "page_size above 2^20");
    if (kv->n_slots < 1) return set_error(CORUN_E_CAPACITY, "the cache has no slots");
    if (kv->n_slots > (1 << 20) || kv->num_pages > (1 << 20) ||
        (int64_t)kv->n_slots * kv->max_pages_per_seq > (1 << 28))
        return set_error(CORUN_E_SHAPE, "more than 2^20 slots or pages, or 2^28 entries of the page table");
    return CORUN_OK;
}

// The layers of a call, COPY_LAYERS at a time.
struct Layers {
    const corun_kv *kv;
    int n;
};
void layers_from(const void *of, int first, PageLayers *out)
{
    const Layers &l = *(const Layers *)of;
    out->n = l.n - first < COPY_LAYERS ? l.n - first : COPY_LAYERS;
    for (int i = 0; i < out->n; ++i) {
        CacheLayer cl;
        (void)layer_of(l.kv, first + i, &cl);          // checked before
        out->k[i] = cl.k;
        out->v[i] = cl.v;
        out->ks[i] = cl.ks;
        out->vs[i] = cl.vs;
    }
}

corun_status pages_call(const corun_kv *kv, int32_t n_layers, int32_t n_kv_heads, int32_t head_dim, int32_t *page_table,
                        int32_t *held, const int32_t *src, const int32_t *keep, const int32_t *hold, int32_t *status,
                        void *ws, int64_t ws_bytes, void *stream)
{
    TRY(check_pages(kv));
    TRY(check_heads(kv, n_kv_heads, n_kv_heads, head_dim));
    const int64_t page_bytes = (int64_t)n_kv_heads * kv->page_size * head_dim * (kv->dtype == CORUN_KV_E4M3 ? 1 : 2);
    if (page_bytes > 1ll << 35) return set_error(CORUN_E_SHAPE, "a page above 2^35 bytes of a layer's keys");
    if (n_layers < 1) return set_errorf(CORUN_E_INVAL, "n_layers %d", n_layers);
    for (int l = 0; l < n_layers; ++l) {
        CacheLayer cl;
        TRY(layer_of(kv, l, &cl));
    }
    if (!page_table || !held || !status) return set_error(CORUN_E_INVAL, "null argument");
    if (page_table != kv->page_table) return set_error(CORUN_E_INVAL, "page_table is not the cache's");
    TRY(check_ws(ws, ws_bytes, corun_pages_workspace(kv)));
    const CacheView cv = cache_view(kv);
    PageShape s;
    s.slots = kv->n_slots;
    s.width = kv->max_pages_per_seq;
    s.pages = kv->num_pages;
    s.page_size = kv->page_size;
    s.nkv = n_kv_heads;
    s.block = 1 << cv.blk_shift;
    s.blocks = kv->page_size >> cv.blk_shift;
    s.row = (long long)s.block * head_dim * (cv.e4m3 ? 1 : 2);
    s.scales = cv.e4m3;
    const Layers of{kv, n_layers};
    return launched(launch_pages(s, page_table, held, src, keep, hold, status, n_layers, layers_from, &of, ws,
                                 (hipStream_t)stream));
}

}  // namespace

extern "C" int64_t corun_pages_workspace(const corun_kv *kv)
{
    TRY(check_pages(kv));
    return (int64_t)pages_ws(kv->n_slots, kv->max_pages_per_seq, kv->num_pages);
}

extern "C" corun_status corun_pages_assign(const corun_kv *kv, int32_t n_layers, int32_t n_kv_heads, int32_t head_dim,
                                           int32_t *page_table, int32_t *held, const int32_t *src, const int32_t *keep,
                                           const int32_t *hold, int32_t *status, void *ws, int64_t ws_bytes,
                                           void *stream)
{
    if (!src || !keep) return set_error(CORUN_E_INVAL, "null argument");
    return pages_call(kv, n_layers, n_kv_heads, head_dim, page_table, held, src, keep, hold, status, ws, ws_bytes,
                      stream);
}

extern "C" corun_status corun_pages_compact(const corun_kv *kv, int32_t n_layers, int32_t n_kv_heads, int32_t head_dim,
                                            int32_t *page_table, const int32_t *held, int32_t *status, void *ws,
                                            int64_t ws_bytes, void *stream)
{
    return pages_call(kv, n_layers, n_kv_heads, head_dim, page_table, const_cast<int32_t *>(held), nullptr, nullptr,
                      nullptr, status, ws, ws_bytes, stream);
}

namespace {

// The call's groups, the longest prefix and suffix that it covers, and its launch.
corun_status shared_call(const corun_kv *kv, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim, int32_t n_groups,
                         const int32_t *group_rows, int32_t max_prefix, int32_t max_suffix, GroupTable *g, int *most,
                         SharedShape *shape)
{
    TRY(check_heads(kv, n_heads, n_kv_heads, head_dim));
    if (!group_rows) return set_error(CORUN_E_INVAL, "null group_rows");
    static_assert(CORUN_MAX_GROUPS == MOST_GROUPS, "a call's groups fit the table");
    if (n_groups < 1 || n_groups > CORUN_MAX_GROUPS)
        return set_errorf(CORUN_E_INVAL, "n_groups %d outside [1, %d]", n_groups, CORUN_MAX_GROUPS);
    g->n = n_groups;
    long long rows = 0;
    for (int i = 0; i < n_groups; ++i) {
        if (group_rows[i] < 1) return set_errorf(CORUN_E_INVAL, "group_rows[%d] = %d", i, group_rows[i]);
        g->row0[i] = (uint16_t)rows;
        rows += group_rows[i];
        if (rows > 65535) return set_error(CORUN_E_SHAPE, "more than 65535 rows");
    }
    g->row0[n_groups] = (uint16_t)rows;
    if (rows > kv->n_slots)
        return set_errorf(CORUN_E_CAPACITY, "KV cache has %d slots < %lld rows", kv->n_slots, rows);
    const int cap = cache_view(kv).cap;
    if (max_prefix < 0 || max_prefix > cap || max_suffix < 0 || max_suffix > cap)
        return set_errorf(CORUN_E_CAPACITY, "max_prefix %d or max_suffix %d outside [0, %d]", max_prefix, max_suffix, cap);
    most[0] = max_prefix == 0 ? cap : max_prefix;
    most[1] = max_suffix == 0 ? cap : max_suffix;
    *shape = shared_shape(*g, n_heads, n_kv_heads, most[0], most[1]);
    if (shared_workgroups(*g, *shape, n_kv_heads) >= 1 << 24)
        return set_errorf(CORUN_E_SHAPE, "%lld rows of %d kv heads and their splits: at most 2^24 - 1 workgroups", rows,
                          n_kv_heads);
    return CORUN_OK;
}

}  // namespace

extern "C" int64_t corun_shared_attention_workspace(const corun_kv *kv, int32_t n_heads, int32_t n_kv_heads,
                                                    int32_t head_dim, int32_t n_groups, const int32_t *group_rows,
                                                    int32_t max_prefix, int32_t max_suffix)
{
    GroupTable g;
    SharedShape shape;
    int most[2];
    TRY(shared_call(kv, n_heads, n_kv_heads, head_dim, n_groups, group_rows, max_prefix, max_suffix, &g, most, &shape));
    return (int64_t)shared_ws(shape, n_kv_heads, head_dim);
}

extern "C" corun_status corun_shared_attention(const corun_kv *kv, int32_t layer, int32_t n_heads, int32_t n_kv_heads,
                                               int32_t head_dim, int32_t n_groups, const int32_t *group_rows,
                                               const void *q, int64_t ld_q, const uint8_t *valid, const int32_t *lens,
                                               const int32_t *prefix_slots, const int32_t *prefix_lens,
                                               int32_t max_prefix, int32_t max_suffix, void *out, int64_t ld_out,
                                               void *ws, int64_t ws_bytes, void *stream)
{
    GroupTable g;
    SharedShape shape;
    int most[2];
    TRY(shared_call(kv, n_heads, n_kv_heads, head_dim, n_groups, group_rows, max_prefix, max_suffix, &g, most, &shape));
    CacheLayer cl;
    TRY(layer_of(kv, layer, &cl));
    TRY(check_rows("q", q, ld_q, (int64_t)n_heads * head_dim));
    TRY(check_rows("out", out, ld_out, (int64_t)n_heads * head_dim));
    if (!lens || !prefix_lens) return set_error(CORUN_E_INVAL, "null argument");
    SharedArgs a;
    a.q = (const uint16_t *)q;
    a.ldq = ld_q;
    a.out = (uint16_t *)out;
    a.ldo = ld_out;
    a.valid = valid;
    a.lens = lens;
    a.prefix_slots = prefix_slots;
    a.prefix_lens = prefix_lens;
    a.nq = n_heads;
    a.nkv = n_kv_heads;
    a.d = head_dim;
    a.max_prefix = most[0];
    a.max_suffix = most[1];
    TRY(check_ws(ws, ws_bytes, (int64_t)shared_ws(shape, n_kv_heads, head_dim)));
    return launched(launch_shared(a, g, shape, cache_view(kv), cl, (float *)ws, (hipStream_t)stream));
}
