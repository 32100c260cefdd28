// cache_ops.cpp -- the cache operators of include/corun.h: host-side checks,
// then one launch (two for attention that is split).  Nothing here
// allocates, waits or keeps anything from one call for the next.
#include "cache_ops.h"

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdarg>
#include <cstdio>

namespace corun {

corun_status set_errorf(corun_status s, const char *fmt, ...)
{
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof buf, fmt, ap);
    va_end(ap);
    return set_error(s, buf);
}

corun_status check_cache(const corun_kv *kv)
{
    if (kv->layout == CORUN_KV_CONTIGUOUS) {
        if (kv->max_seq_len <= 0 || kv->max_seq_len % 16 != 0)
            return set_error(CORUN_E_CAPACITY, "max_seq_len must be a positive multiple of 16");
    } else if (kv->layout == CORUN_KV_PAGED) {
        if (kv->page_size <= 0 || kv->page_size % 16 != 0 || kv->num_pages <= 0 || kv->max_pages_per_seq <= 0)
            return set_error(CORUN_E_CAPACITY, "bad paged-cache geometry (page_size must be a multiple of 16)");
    } else {
        return set_errorf(CORUN_E_INVAL, "unknown KV layout %d", kv->layout);
    }
    if (kv->dtype == CORUN_KV_BF16) return CORUN_OK;   // scale_block and the scales are not looked at
    if (kv->dtype != CORUN_KV_E4M3) return set_errorf(CORUN_E_INVAL, "unknown KV dtype %d", kv->dtype);
    const int b = kv->scale_block, unit = kv->layout == CORUN_KV_PAGED ? kv->page_size : kv->max_seq_len;
    if (b != 16 && b != 32 && b != 64) return set_errorf(CORUN_E_SHAPE, "scale_block %d is not 16, 32 or 64", b);
    if (unit % b != 0)
        return set_errorf(CORUN_E_SHAPE, "scale_block %d does not divide %d tokens of a slot or page", b, unit);
    return CORUN_OK;
}

bool plain_rope(const corun_rope &r)
{
    return r.layout == CORUN_ROPE_HALF && r.rot_dim == r.head_dim && r.magnitude == 1.f;
}

static bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

corun_status layer_of(const corun_kv *kv, int32_t layer, CacheLayer *out)
{
    if (layer < 0) return set_errorf(CORUN_E_INVAL, "layer %d", layer);
    if (!kv->k || !kv->v || !kv->k[layer] || !kv->v[layer]) return set_error(CORUN_E_INVAL, "missing KV pointers");
    if (kv->layout == CORUN_KV_PAGED && !kv->page_table) return set_error(CORUN_E_INVAL, "paged cache needs page_table");
    out->k = kv->k[layer];
    out->v = kv->v[layer];
    if (!aligned16(out->k) || !aligned16(out->v)) return set_error(CORUN_E_INVAL, "cache buffers must start on 16 bytes");
    if (kv->dtype == CORUN_KV_E4M3) {
        if (!kv->k_scale || !kv->v_scale || !kv->k_scale[layer] || !kv->v_scale[layer])
            return set_error(CORUN_E_INVAL, "an e4m3 cache needs k_scale and v_scale");
        out->ks = kv->k_scale[layer];
        out->vs = kv->v_scale[layer];
    }
    return CORUN_OK;
}

corun_status check_rope(const corun_rope *r)
{
    if (!r) return set_error(CORUN_E_INVAL, "null rope");
    if (r->head_dim != 64 && r->head_dim != 128) return set_error(CORUN_E_SHAPE, "head_dim must be 64 or 128");
    if (r->rot_dim < 2 || r->rot_dim > r->head_dim || r->rot_dim % 2 != 0)
        return set_errorf(CORUN_E_SHAPE, "rot_dim %d is not an even number from 2 to head_dim", r->rot_dim);
    if (r->layout != CORUN_ROPE_HALF && r->layout != CORUN_ROPE_INTERLEAVED)
        return set_errorf(CORUN_E_INVAL, "unknown rope layout %d", r->layout);
    if (!(r->magnitude > 0.f) || std::isinf(r->magnitude)) return set_error(CORUN_E_INVAL, "bad rope magnitude");
    for (int i = 0; i < r->rot_dim / 2; ++i)
        if (!std::isfinite(r->freq[i])) return set_errorf(CORUN_E_INVAL, "rope frequency %d is not finite", i);
    return CORUN_OK;
}

CacheView cache_view(const corun_kv *kv)
{
    CacheView v;
    v.kv.layout = kv->layout;
    v.kv.max_seq_len = kv->max_seq_len;
    v.kv.page_size = kv->page_size;
    v.kv.max_pages_per_seq = kv->max_pages_per_seq;
    v.kv.page_table = kv->page_table;
    v.n_slots = kv->n_slots;
    v.num_pages = kv->num_pages;
    const bool paged = kv->layout == CORUN_KV_PAGED;
    const long long cap = paged ? (long long)kv->max_pages_per_seq * kv->page_size : kv->max_seq_len;
    v.cap = (int)(cap < (1 << 30) ? cap : (1 << 30));   // positions stay far from 2^31 in the kernels
    v.e4m3 = kv->dtype == CORUN_KV_E4M3;
    v.blk_shift = !v.e4m3 || kv->scale_block == 16 ? 4 : kv->scale_block == 32 ? 5 : 6;
    v.page_inv = paged ? 1.0f / (float)kv->page_size : 0.f;
    return v;
}

RopeArgs rope_args(const corun_rope &r)
{
    RopeArgs a{};
    a.mag = r.magnitude;
    a.rot = r.rot_dim;
    a.interleaved = r.layout == CORUN_ROPE_INTERLEAVED;
    for (int i = 0; i < r.rot_dim / 2; ++i) a.turns[i] = r.freq[i] / 6.283185307179586476925;
    return a;
}

corun_status check_heads(const corun_kv *kv, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim)
{
    if (!kv) return set_error(CORUN_E_INVAL, "null kv");
    corun_status s = check_cache(kv);
    if (s != CORUN_OK) return s;
    if (kv->n_slots < 1) return set_error(CORUN_E_CAPACITY, "the cache has no slots");
    if (kv->layout == CORUN_KV_PAGED && kv->page_size > (1 << 20))
        return set_error(CORUN_E_SHAPE, "page_size above 2^20");
    if (head_dim != 64 && head_dim != 128) return set_error(CORUN_E_SHAPE, "head_dim must be 64 or 128");
    if (n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads != 0 || n_heads / n_kv_heads > 16 || n_heads > 4096)
        return set_errorf(CORUN_E_SHAPE, "%d query heads over %d kv heads: groups of 1 to 16 are supported", n_heads,
                          n_kv_heads);
    return CORUN_OK;
}

corun_status check_rows(const char *name, const void *p, int64_t ld, int64_t width)
{
    if (!p) return set_errorf(CORUN_E_INVAL, "null %s", name);
    if (!aligned16(p) || ld % 8 != 0) return set_errorf(CORUN_E_INVAL, "%s rows must start on 16-byte boundaries", name);
    if (ld < width)
        return set_errorf(CORUN_E_SHAPE, "%s row stride %lld below its width %lld", name, (long long)ld, (long long)width);
    return CORUN_OK;
}

corun_status check_ws(const void *ws, int64_t bytes, int64_t need)
{
    if (need > 0 && (!ws || !aligned16(ws))) return set_error(CORUN_E_INVAL, "the workspace must start on 16 bytes");
    if (bytes < need)
        return set_errorf(CORUN_E_CAPACITY, "workspace of %lld bytes, %lld needed", (long long)bytes, (long long)need);
    return CORUN_OK;
}

corun_status launched(hipError_t e)
{
    return e == hipSuccess ? CORUN_OK : set_errorf(CORUN_E_HIP, "launch: %s", hipGetErrorString(e));
}

}  // namespace corun

using namespace corun;

extern "C" corun_status corun_rope_init(const corun_rope_cfg *c, corun_rope *out)
{
    if (!c || !out) return set_error(CORUN_E_INVAL, "null argument");
    corun_rope r{};
    r.head_dim = c->head_dim;
    r.rot_dim = c->rot_dim == 0 ? c->head_dim : c->rot_dim;
    r.layout = c->layout;
    r.magnitude = c->magnitude == 0.f ? 1.f : c->magnitude;
    if (!(c->theta > 1.0) || std::isinf(c->theta)) return set_error(CORUN_E_INVAL, "theta must be above 1");
    if (c->scaling < CORUN_ROPE_UNSCALED || c->scaling > CORUN_ROPE_BANDS)
        return set_errorf(CORUN_E_INVAL, "unknown rope scaling %d", c->scaling);
    if (c->scaling != CORUN_ROPE_UNSCALED && (!(c->factor >= 1.0) || std::isinf(c->factor)))
        return set_error(CORUN_E_INVAL, "the scaling factor must be at least 1");
    if (c->scaling == CORUN_ROPE_BANDS &&
        (c->trained_len < 1 || !(c->low >= 0.0) || !(c->high > c->low) || std::isinf(c->high)))
        return set_error(CORUN_E_INVAL, "bands need trained_len >= 1 and 0 <= low < high");
    corun_status s = check_rope(&r);                   // shapes, before the frequencies
    if (s != CORUN_OK) return s;
    for (int i = 0; i < r.rot_dim / 2; ++i) {
        double f = std::pow(c->theta, -2.0 * i / r.rot_dim);
        if (c->scaling == CORUN_ROPE_LINEAR) f /= c->factor;
        if (c->scaling == CORUN_ROPE_BANDS) {
            const double n = c->trained_len * f / 6.283185307179586476925;
            const double g = std::fmin(1.0, std::fmax(0.0, (n - c->low) / (c->high - c->low)));
            f *= g + (1.0 - g) / c->factor;
        }
        r.freq[i] = f;
    }
    *out = r;
    return CORUN_OK;
}

namespace {

corun_status check_step_rows(const corun_kv *kv, int32_t rows)
{
    if (rows < 1 || rows > 65535) return set_errorf(CORUN_E_SHAPE, "rows %d outside [1, 65535]", rows);
    if (rows > kv->n_slots) return set_errorf(CORUN_E_CAPACITY, "KV cache has %d slots < %d rows", kv->n_slots, rows);
    return CORUN_OK;
}

// slots == nullptr: only the sizes are looked at
corun_status sequences(const corun_kv *kv, int32_t n, const int32_t *lens, const int32_t *starts, const int32_t *slots,
                       SeqTable *out)
{
    if (!lens) return set_error(CORUN_E_INVAL, "null argument");
    if (n < 1 || n > CORUN_MAX_PREFILL_BATCH)
        return set_errorf(CORUN_E_INVAL, "n = %d outside [1, %d]", n, CORUN_MAX_PREFILL_BATCH);
    static_assert(CORUN_MAX_PREFILL_BATCH == sizeof(SeqTable::len) / sizeof(int), "a call's sequences fit the table");
    const long long cap = cache_view(kv).cap;
    long long rows = 0;
    out->n = n;
    for (int i = 0; i < n; ++i) {
        const int32_t start = starts ? starts[i] : 0;
        if (lens[i] < 1) return set_errorf(CORUN_E_INVAL, "lens[%d] = %d", i, lens[i]);
        if (start < 0) return set_errorf(CORUN_E_INVAL, "starts[%d] = %d", i, start);
        if ((long long)start + lens[i] > cap)
            return set_errorf(CORUN_E_CAPACITY, "sequence %d: positions %d .. %lld exceed the cache capacity %lld", i, start,
                              (long long)start + lens[i] - 1, cap);
        const int slot = slots ? slots[i] : 0;
        if (slot < 0 || slot >= kv->n_slots)
            return set_errorf(CORUN_E_INVAL, "slots[%d] = %d outside [0, %d)", i, slot, kv->n_slots);
        for (int j = 0; slots && j < i; ++j)
            if (slots[j] == slot) return set_errorf(CORUN_E_INVAL, "slot %d given twice", slot);
        out->row0[i] = (int)rows;
        out->len[i] = lens[i];
        out->start[i] = start;
        out->slot[i] = slot;
        rows += lens[i];
    }
    if (rows > (1 << 24)) return set_errorf(CORUN_E_SHAPE, "%lld rows in one call: at most 2^24", rows);
    return CORUN_OK;
}

// A launch has fewer than 2^32 threads: head_dim / 16 to a head of a row of a
// decode append, 512 to at most eight units of 32 rows of a head of prefill
// attention (a sequence's last unit and workgroup may be partly empty).
corun_status check_total(long long rows, long long heads, int log2_most)
{
    if (rows * heads <= 1ll << log2_most) return CORUN_OK;
    return set_errorf(CORUN_E_SHAPE, "%lld rows of %lld heads in one call: at most 2^%d", rows, heads, log2_most);
}

long long rows_of(const SeqTable &seq) { return (long long)seq.row0[seq.n - 1] + seq.len[seq.n - 1]; }

int longest(const corun_kv *kv, int32_t max_len)
{
    const int cap = cache_view(kv).cap;
    return max_len == 0 ? cap : max_len;
}

corun_status check_attention(const corun_kv *kv, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim)
{
    corun_status s = check_heads(kv, n_heads, n_kv_heads, head_dim);
    if (s != CORUN_OK) return s;
    if (kv->dtype != CORUN_KV_E4M3) return set_error(CORUN_E_INVAL, "attention of this entry point reads e4m3 caches");
    return CORUN_OK;
}

}  // namespace

#define TRY(expr)                       \
    do {                                \
        corun_status s_ = (expr);       \
        if (s_ != CORUN_OK) return s_;  \
    } while (0)

extern "C" corun_status corun_decode_append(const corun_kv *kv, int32_t layer, int32_t n_heads, int32_t n_kv_heads,
                                            const corun_rope *rope, int32_t rows, const void *qkv, int64_t ld_qkv,
                                            const uint8_t *valid, const int32_t *positions, void *q, int64_t ld_q,
                                            void *stream)
{
    TRY(check_rope(rope));
    const int d = rope->head_dim;
    TRY(check_heads(kv, n_heads, n_kv_heads, d));
    CacheLayer cl;
    TRY(layer_of(kv, layer, &cl));
    TRY(check_step_rows(kv, rows));
    TRY(check_rows("qkv", qkv, ld_qkv, (int64_t)(n_heads + 2 * n_kv_heads) * d));
    TRY(check_rows("q", q, ld_q, (int64_t)n_heads * d));
    if (!positions) return set_error(CORUN_E_INVAL, "null positions");
    TRY(check_total(rows, n_heads + 2 * n_kv_heads, 28));
    QkvRows in;
    in.bf16 = (const uint16_t *)qkv;
    in.ld = ld_qkv;
    return launched(launch_append_rows(in, rows, valid, positions, n_heads, n_kv_heads, d, rope_args(*rope), (uint16_t *)q,
                                       ld_q, cache_view(kv), cl, (hipStream_t)stream));
}

extern "C" corun_status corun_prefill_append(const corun_kv *kv, int32_t layer, int32_t n_heads, int32_t n_kv_heads,
                                             const corun_rope *rope, int32_t n, const int32_t *lens,
                                             const int32_t *starts, const int32_t *slots, const void *qkv,
                                             int64_t ld_qkv, void *q, int64_t ld_q, void *stream)
{
    TRY(check_rope(rope));
    const int d = rope->head_dim;
    TRY(check_heads(kv, n_heads, n_kv_heads, d));
    CacheLayer cl;
    TRY(layer_of(kv, layer, &cl));
    if (!slots) return set_error(CORUN_E_INVAL, "null argument");
    SeqTable seq;
    TRY(sequences(kv, n, lens, starts, slots, &seq));
    TRY(check_rows("qkv", qkv, ld_qkv, (int64_t)(n_heads + 2 * n_kv_heads) * d));
    TRY(check_rows("q", q, ld_q, (int64_t)n_heads * d));
    QkvRows in;
    in.bf16 = (const uint16_t *)qkv;
    in.ld = ld_qkv;
    return launched(launch_append_seqs(in, seq, n_heads, n_kv_heads, d, rope_args(*rope), (uint16_t *)q, ld_q,
                                       cache_view(kv), cl, (hipStream_t)stream));
}

extern "C" int64_t corun_decode_attention_workspace(const corun_kv *kv, int32_t n_heads, int32_t n_kv_heads,
                                                    int32_t head_dim, int32_t rows, int32_t max_len)
{
    TRY(check_attention(kv, n_heads, n_kv_heads, head_dim));
    TRY(check_step_rows(kv, rows));
    if (max_len < 0 || max_len > cache_view(kv).cap)
        return set_errorf(CORUN_E_CAPACITY, "max_len %d outside [0, %d]", max_len, cache_view(kv).cap);
    const int64_t most = longest(kv, max_len), chunk = attn8_chunk(rows, n_kv_heads, (int)most);
    if (chunk >= most) return 0;
    return (int64_t)sizeof(float) * rows * n_heads * ((most + chunk - 1) / chunk) * (head_dim + 2);
}

extern "C" corun_status corun_decode_attention(const corun_kv *kv, int32_t layer, int32_t n_heads, int32_t n_kv_heads,
                                               int32_t head_dim, int32_t rows, const void *q, int64_t ld_q,
                                               const uint8_t *valid, const int32_t *lens, int32_t max_len, void *out,
                                               int64_t ld_out, void *ws, int64_t ws_bytes, void *stream)
{
    const int64_t need = corun_decode_attention_workspace(kv, n_heads, n_kv_heads, head_dim, rows, max_len);
    if (need < 0) return (corun_status)need;
    CacheLayer cl;
    TRY(layer_of(kv, layer, &cl));
    TRY(check_rows("q", q, ld_q, (int64_t)n_heads * head_dim));
    TRY(check_rows("out", out, ld_out, (int64_t)n_heads * head_dim));
    if (!lens) return set_error(CORUN_E_INVAL, "null lens");
    TRY(check_ws(ws, ws_bytes, need));
    const CacheView cv = cache_view(kv);
    const int most = longest(kv, max_len), chunk = attn8_chunk(rows, n_kv_heads, most);
    const bool one = chunk >= most;                    // one split to a row: written straight to out
    TRY(launched(launch_attn8_split((const uint16_t *)q, ld_q, rows, valid, lens, 0, n_heads, n_kv_heads, head_dim, cv, cl,
                                    most, chunk, (float *)ws, (hipStream_t)stream, nullptr,
                                    one ? (uint16_t *)out : nullptr, ld_out)));
    if (one) return CORUN_OK;
    return launched(launch_attn8_merge((const float *)ws, rows, valid, lens, 0, n_heads, n_kv_heads, head_dim, most, chunk,
                                       (uint16_t *)out, ld_out, (hipStream_t)stream));
}

extern "C" int64_t corun_prefill_attention_workspace(const corun_kv *kv, int32_t n_heads, int32_t n_kv_heads,
                                                     int32_t head_dim, int32_t n, const int32_t *lens,
                                                     const int32_t *starts)
{
    TRY(check_attention(kv, n_heads, n_kv_heads, head_dim));
    SeqTable seq;
    TRY(sequences(kv, n, lens, starts, nullptr, &seq));
    return (int64_t)attn8_seqs_ws(seq, n_heads, n_kv_heads, head_dim);
}

extern "C" corun_status corun_prefill_attention(const corun_kv *kv, int32_t layer, int32_t n_heads, int32_t n_kv_heads,
                                                int32_t head_dim, int32_t n, const int32_t *lens, const int32_t *starts,
                                                const int32_t *slots, const void *q, int64_t ld_q, void *out,
                                                int64_t ld_out, void *ws, int64_t ws_bytes, void *stream)
{
    TRY(check_attention(kv, n_heads, n_kv_heads, head_dim));
    CacheLayer cl;
    TRY(layer_of(kv, layer, &cl));
    if (!slots) return set_error(CORUN_E_INVAL, "null argument");
    SeqTable seq;
    TRY(sequences(kv, n, lens, starts, slots, &seq));
    TRY(check_total(rows_of(seq), n_heads, 30));
    TRY(check_rows("q", q, ld_q, (int64_t)n_heads * head_dim));
    TRY(check_rows("out", out, ld_out, (int64_t)n_heads * head_dim));
    TRY(check_ws(ws, ws_bytes, (int64_t)attn8_seqs_ws(seq, n_heads, n_kv_heads, head_dim)));
    return launched(launch_attn8_seqs((const uint16_t *)q, ld_q, seq, n_heads, n_kv_heads, head_dim, cache_view(kv), cl,
                                      (uint16_t *)out, ld_out, (float *)ws, (hipStream_t)stream));
}
