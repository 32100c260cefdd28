// cache.h -- what cache.hip's kernels take and their launchers: rotary forms, the
// append to bf16 and e4m3 caches, attention over e4m3 caches.
#pragma once
#include "kernels.h"

namespace corun {

// A cache of corun_kv as its kernels see it.  Codes are e4m3, one byte each,
// in the element order of a bf16 cache; the scale of a block of 1 << blk_shift
// tokens of one kv head is 2^(byte - 127), the bytes in block order where the
// tokens stand: [n_slots][nkv][max_seq_len >> blk_shift] or
// [num_pages][nkv][page_size >> blk_shift].
struct CacheView {
    KvView kv{};
    int n_slots = 0, num_pages = 0, cap = 0;   // cap: tokens per slot
    int e4m3 = 0, blk_shift = 4;               // bf16 caches: blk_shift groups tokens into work units only
    float page_inv = 0.f;                      // 1 / page_size
};
// One layer of it.
struct CacheLayer {
    void *k = nullptr, *v = nullptr;
    uint8_t *ks = nullptr, *vs = nullptr;
};

// Rotary positions: pair i < rot / 2 of a head turns by turns[i] per position;
// pairs are (i, i + rot / 2) or, interleaved, (2 i, 2 i + 1); the rotated
// elements are scaled by mag.
struct RopeArgs {
    double turns[64];
    float mag;
    int rot, interleaved;
};

// Packed QKV rows (q heads, k heads, v heads): bf16 rows of ld elements, or
// (bf16 == nullptr) fp32 split partials [S][rows][ld], summed in split order
// and rounded to bf16.
struct QkvRows {
    const uint16_t *bf16 = nullptr;
    const float *part = nullptr;
    int S = 1;
    long long stride = 0, ld = 0;
};

// Sequences of a prefill call, by value: sequence i owns rows row0[i] .. +
// len[i] - 1, positions start[i] .. of cache slot slot[i], and the launch's
// units from unit0[i] on.
struct SeqTable {
    int n = 0;
    int row0[64], len[64], start[64], slot[64], unit0[64];
};
// How they are split over their keys, and where their partial results start (in
// units of 32 rows of a head).
struct SplitTable {
    int splits[64], part0[64];
};

// cos / sin table of frequencies freq[i] (radians per position) of the d / 2 half
// pairs of a head, as launch_rope_table's.
hipError_t launch_rope_table_of(float2 *tab, int max_pos, int d, const double *freq, hipStream_t st);

// Row r of a decode step (padding rows, valid[r] == 0, skipped): q heads
// rotated at position pos[r] to q [rows][ldq], the rotated k and the v heads
// appended at that position of slot r.  A row whose position or page is
// outside the cache appends nothing and its q row is NaN.
hipError_t launch_append_rows(const QkvRows &in, int rows, const uint8_t *valid, const int32_t *pos, int nq, int nkv,
                              int d, const RopeArgs &rope, uint16_t *q, long long ldq, const CacheView &cv,
                              const CacheLayer &cl, hipStream_t st);
// The same for the sequences of a prefill call (unit0 is filled in here);
// positions and slots are the caller's to check, pages are checked as above.
hipError_t launch_append_seqs(const QkvRows &in, SeqTable &seq, int nq, int nkv, int d, const RopeArgs &rope,
                              uint16_t *q, long long ldq, const CacheView &cv, const CacheLayer &cl, hipStream_t st);

// Attention of row r's query heads over tokens 0 .. lens[r] - 1 of slot r of
// an e4m3 cache (lens[r] = pos[r] + 1 where plus_one): out rows of padding
// rows and of empty ones are zero, of rows whose length or pages are outside
// the cache or max_len NaN.  Split over the tokens in chunks (attn8_chunk, or
// any multiple of 64), then merged; ws: [rows][nkv][ceil(max_len / chunk)][G (d +
// 2)] floats; workgroups take the rows in row_order if given.
int attn8_chunk(int rows, int nkv, int max_len);
hipError_t launch_attn8_split(const uint16_t *q, long long ldq, int rows, const uint8_t *valid, const int32_t *lens,
                              int plus_one, int nq, int nkv, int d, const CacheView &cv, const CacheLayer &cl, int max_len,
                              int chunk, float *ws, hipStream_t st, const int32_t *row_order = nullptr,
                              uint16_t *out = nullptr, long long ldo = 0);   // out: chunk >= max_len, nothing to merge
hipError_t launch_attn8_merge(const float *ws, int rows, const uint8_t *valid, const int32_t *lens, int plus_one, int nq,
                              int nkv, int d, int max_len, int chunk, uint16_t *out, long long ldo, hipStream_t st);
// Causal attention of a prefill call's queries: row row0 + t of sequence i
// sees tokens 0 .. start + t of its slot (unit0 is not looked at).  ws:
// attn8_seqs_ws bytes on a 16-byte boundary.
size_t attn8_seqs_ws(const SeqTable &seq, int nq, int nkv, int d);
size_t attn8_seq_ws_max(int d);                // the most that one sequence adds to it
hipError_t launch_attn8_seqs(const uint16_t *q, long long ldq, const SeqTable &given, int nq, int nkv, int d,
                             const CacheView &cv, const CacheLayer &cl, uint16_t *out, long long ldo, float *ws,
                             hipStream_t st);

}  // namespace corun
