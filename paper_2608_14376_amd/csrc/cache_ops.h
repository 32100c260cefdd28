// cache_ops.h -- a corun_kv's checks and its kernels' view of it, shared by
// the engine and the cache operators.
#pragma once
#include "cache.h"
#include "corun.h"

namespace corun {

corun_status set_error(corun_status s, const char *msg);
corun_status set_errorf(corun_status s, const char *fmt, ...);

// Layout, type and sizes of a cache (the pointers are not looked at).
corun_status check_cache(const corun_kv *kv);
// One layer of it: its pointers, which the kernels of this file's operators
// want on 16-byte boundaries.
corun_status layer_of(const corun_kv *kv, int32_t layer, CacheLayer *out);
// Whether the rotation is the one that the kernels with a QKV epilogue of
// their own apply: half pairs over the whole of a head, no magnitude.
bool plain_rope(const corun_rope &rope);
corun_status check_rope(const corun_rope *rope);
CacheView cache_view(const corun_kv *kv);
RopeArgs rope_args(const corun_rope &rope);
// A cache and the heads on it; rows of bf16 heads; a workspace.
corun_status check_heads(const corun_kv *kv, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim);
corun_status check_rows(const char *name, const void *p, int64_t ld, int64_t width);
corun_status check_ws(const void *ws, int64_t bytes, int64_t need);
// A launch's status.
corun_status launched(hipError_t e);

}  // namespace corun
