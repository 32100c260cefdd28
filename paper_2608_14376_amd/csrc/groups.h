// groups.h -- what the kernels for sequences that share a beginning take, and
// their launchers: beam.hip (selection), pages.hip (pages of a cache given to
// slots), shared.hip (attention over shared prefixes).
#pragma once
#include "cache.h"

namespace corun {

// Beam selection: row r = group beams + beam; the pointers as corun_beam_select's.
struct BeamArgs {
    const float *logits;
    long long ld;
    int vocab, groups, beams, keep, end_token;
    const float *scores, *weights;
    const uint8_t *valid, *finished;
    int32_t *tokens, *parents;
    float *out_scores;
    uint8_t *out_finished;
};
constexpr int MOST_BEAMS = 64;
size_t beam_ws(int vocab, int groups, int beams, int keep);
hipError_t launch_beam_select(const BeamArgs &a, void *ws, hipStream_t st);

// A paged cache's pages as they are copied: per kv head `row` bytes of elements
// to a block of tokens and `blocks` blocks to a page, and one scale byte to a
// block where the cache has scales.
struct PageShape {
    int slots, width, pages, page_size;                // width: entries of a table row
    int nkv, blocks, block;                            // block: tokens copied together
    long long row;                                     // bytes of a block of one kv head
    int scales;
};
// Layers of one copying launch, by value.
constexpr int COPY_LAYERS = 64;
struct PageLayers {
    int n;
    void *k[COPY_LAYERS], *v[COPY_LAYERS];
    uint8_t *ks[COPY_LAYERS], *vs[COPY_LAYERS];
};
size_t pages_ws(int slots, int width, int pages);
// Plans and carries out an assignment (src, keep, hold) or, src == nullptr, a
// compaction; `layer` gives the layers from `first` on.
typedef void (*LayersOf)(const void *of, int first, PageLayers *out);
hipError_t launch_pages(const PageShape &s, int32_t *table, int32_t *held, const int32_t *src, const int32_t *keep,
                        const int32_t *hold, int32_t *status, int n_layers, LayersOf layers, const void *of, void *ws,
                        hipStream_t st);

// Groups of rows, by value: group g owns rows row0[g] .. row0[g + 1] - 1, of at
// most 65535.
constexpr int MOST_GROUPS = 256;
struct GroupTable {
    int n;
    uint16_t row0[MOST_GROUPS + 1];
};
struct SharedArgs {
    const uint16_t *q;
    long long ldq;
    uint16_t *out;
    long long ldo;
    const uint8_t *valid;
    const int32_t *lens, *prefix_slots, *prefix_lens;
    int nq, nkv, d, max_prefix, max_suffix;
};
// What a call's lengths and slots, which only the device sees, leave to read; plain
// functions of numbers, so that a host program can go over all of them.
// A group's prefix.  len < 0: out of the launch's range.
struct Prefix {
    int len, slot;
};
__host__ __device__ inline Prefix prefix_within(int len, int slot, int max_prefix, int n_slots)
{
    return {len < 0 || len > max_prefix || (unsigned)slot >= (unsigned)n_slots ? -1 : len, slot};
}
// Tokens that a row sees, its prefix included: 0 for padding, -1 out of range.
__host__ __device__ inline int tokens_within(const Prefix &p, int len, int live, int max_suffix, int cap)
{
    if (live == 0) return 0;
    return p.len < 0 || len < p.len || len - p.len > max_suffix || len > cap ? -1 : len;
}
// Tokens t_lo .. t_end - 1 of a slot: a split of a prefix, or of what row r has of its
// own behind it (n of tokens_within).  Nothing: t_lo >= t_end.
struct Span {
    int slot, t_lo, t_end;
};
__host__ __device__ inline Span prefix_span(const Prefix &p, int chunk, int split)
{
    const int t0 = split * chunk;
    return {p.slot, t0, p.len - t0 < chunk ? p.len : t0 + chunk};
}
__host__ __device__ inline Span own_span(const Prefix &p, int r, int n, int chunk, int split)
{
    if (p.len < 0 || n <= p.len) return {r, 0, 0};     // a padding row's n is 0, its prefix may be any
    const int t0 = (p.len & ~15) + split * chunk;
    return {r, t0 > p.len ? t0 : p.len, n - t0 < chunk ? n : t0 + chunk};
}
// A call's launch: where each group's 32-query blocks (of one kv head) and query
// tiles start, and the splits; by value.
struct SharedShape {
    bool alone;                                        // one launch, no splits: the rest is not looked at
    int G, mt;                                         // query heads to a kv head; queries of a prefix tile
    int blocks;                                        // 32-query blocks of a kv head, all groups
    int chunk_p, splits_p, chunk_s, splits_s;          // tokens of a split, splits
    int tiles;                                         // query tiles of all groups
    uint16_t qb0[MOST_GROUPS + 1], tile0[MOST_GROUPS + 1];
};
SharedShape shared_shape(const GroupTable &g, int nq, int nkv, int max_prefix, int max_suffix);
long long shared_workgroups(const GroupTable &g, const SharedShape &s, int nkv);   // of its largest launch
size_t shared_ws(const SharedShape &s, int nkv, int d);
hipError_t launch_shared(const SharedArgs &a, const GroupTable &g, const SharedShape &s, const CacheView &cv,
                         const CacheLayer &cl, float *ws, hipStream_t st);

}  // namespace corun
