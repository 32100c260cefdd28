// shared.hip -- attention of a decode step whose rows share prefixes
// (corun_shared_attention), over bf16 and e4m3 caches.
//
// The queries of a group's rows that read one kv head are one matrix: query u =
// (row in the group) G + head, G query heads to a kv head.  A group's prefix is
// split over its tokens, and each split is done once for a tile of queries; the
// tokens that a row has of its own are split likewise, for its G queries alone.
// Both are workgroups of one launch.  Every split leaves its queries' maximum,
// sum and weighted values, and a second launch joins them:
//     M = max_i m_i,  out = sum_i 2^(m_i - M) o_i / sum_i 2^(m_i - M) l_i
// with the prefix's splits before the row's own, in order.  Splits follow from the
// call's sizes and a row's lengths alone, and a query's arithmetic does not depend
// on its place in a tile, so rows stay position-invariant.
//
// Weights enter the matrix units as two bf16 halves, hi + lo: about 16 bits, however
// small a weight is, for a value may be met by small ones alone.  bf16 values and the
// codes of an e4m3 cache times their scale are exact there.
//
// The rows' own tokens are bound by reading (228 rows of 1024 bf16 tokens of 8 kv
// heads of 128: 5.1 TB/s, a large copy's rate), the prefixes by the products and
// the softmax of a wavefront in turn (below).  Prefixes' workgroups come first in
// the launch: mixed among the others they were spread unevenly over the CUs (128
// rows of 64 heads behind 32768 tokens: 313 us, 233 so).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "device.h"
#include "groups.h"

namespace corun {
namespace {

typedef __attribute__((address_space(3))) void lds_void;

__device__ __forceinline__ float qnan() { return __uint_as_float(0x7fc00000u); }

// The last of n entries of a rising table that is at most u: a load and a count
// for 64 entries, where a search would wait for one after another.
__device__ __forceinline__ int last_at_most(const uint16_t *t, int n, int u)
{
    const int lane = threadIdx.x & 63;
    int count = 0;
#pragma unroll
    for (int i = 0; i < MOST_GROUPS; i += 64)
        if (i < n) count += __popcll(__ballot(i + lane < n && t[i + lane] <= u));
    return __builtin_amdgcn_readfirstlane(count - 1);
}

using Shape = SharedShape;

__device__ __forceinline__ Prefix prefix_of(const SharedArgs &a, const GroupTable &gt, const CacheView &cv, int gi)
{
    // gi is the same for a wavefront, and so are these: told so, addresses from them stay scalar
    const int p = __builtin_amdgcn_readfirstlane(a.prefix_lens[gi]);
    const int slot = __builtin_amdgcn_readfirstlane(a.prefix_slots == nullptr ? gt.row0[gi] : a.prefix_slots[gi]);
    return prefix_within(p, slot, a.max_prefix, cv.n_slots);
}
__device__ __forceinline__ int row_len(const SharedArgs &a, const CacheView &cv, const Prefix &p, int r)
{
    const int n = a.lens[r], live = a.valid == nullptr ? 1 : a.valid[r];   // in flight together
    return tokens_within(p, n, live, a.max_suffix, cv.cap);
}

// What a split leaves of a 32-query block: values [D / 4][32][4], then (maximum in
// base 2, sum) [32][2].
template <int D>
__host__ __device__ constexpr int part_floats() { return 32 * D + 64; }
template <int D>
__device__ __forceinline__ float *part_at(float *ws, const Shape &s, int nkv, int split, int kvh, int block)
{
    return ws + (((size_t)split * nkv + kvh) * s.blocks + block) * part_floats<D>();
}

// Transposed LDS read of bytes (ds_read_b64_tr_b8): in each group of 16 lanes,
// lane a + 2 q points at eight bytes (row q, columns 8 a .. 8 a + 7) and lane i
// receives column i of rows 0 .. 7.
__device__ __forceinline__ uint2 read_tr8(const void *lds_ptr)
{
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
    const i32x2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
        (lds_i32x2 *)(const __attribute__((address_space(3))) void *)lds_ptr);
    return __builtin_bit_cast(uint2, v);
}

// The value of the other half of 32 (HALF 16) or 64 lanes (HALF 32).
template <int HALF>
__device__ __forceinline__ float other(float x)
{
    const uint32_t u = __float_as_uint(x);
    const bool upper = threadIdx.x & HALF;
    if constexpr (HALF == 16) {
        const auto two = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        return __uint_as_float(upper ? two[0] : two[1]);
    } else {
        const auto two = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        return __uint_as_float(upper ? two[0] : two[1]);
    }
}

// Four codes times a power of two, in bf16: exact.
__device__ __forceinline__ uint2 codes4(uint32_t w, float scale)
{
    uint2 o;
    o.x = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false));
    o.y = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true));
    return o;
}
__device__ __forceinline__ uint4 codes8(uint32_t w0, uint32_t w1, float scale)
{
    const uint2 a = codes4(w0, scale), b = codes4(w1, scale);
    return (uint4){a.x, a.y, b.x, b.y};
}

// A position (a multiple of 16) of a slot as it moves on: the entry of its page in
// the table, and its place in the page.  Uniform over a wavefront, and followed by
// additions where a division at every step would cost more than the step's loads.
struct Walk {
    int page, in, pages, rest;                         // pages, rest: what a step moves by
    __device__ __forceinline__ Walk(int t, int step, int ps)
    {
        page = t / ps;
        in = t - page * ps;
        pages = step / ps;
        rest = step - pages * ps;
    }
    __device__ __forceinline__ void next(int ps)
    {
        page += pages;
        in += rest;
        if (in >= ps) {
            in -= ps;
            ++page;
        }
    }
};

// Where 16 tokens from position t of a slot stand: their first row of one kv head,
// and their scale block.  Paged: at place `in` of a page.
struct Rows16 {
    size_t row, blk;
};
template <bool PAGED>
__device__ __forceinline__ Rows16 rows16(const CacheView &cv, int nkv, int kvh, int slot, int page, int in, int t)
{
    if constexpr (PAGED) {
        const int ps = cv.kv.page_size;
        const size_t head = (size_t)page * nkv + kvh;
        return {head * ps + in, head * (ps >> cv.blk_shift) + (in >> cv.blk_shift)};
    }
    const size_t head = (size_t)slot * nkv + kvh;
    return {head * cv.kv.max_seq_len + t, head * (cv.kv.max_seq_len >> cv.blk_shift) + (t >> cv.blk_shift)};
}

// ---------------------------------------------------------------------------
// Up to 16 MT queries over tokens t_lo .. t_end - 1 of one slot: what a row has of
// its own, or a tile of queries on a split of a prefix.  Four wavefronts, each
// with all the queries and 32 tokens of a step of 128, on its own: no barrier in
// the loop, keys and values are read once for all the queries, and converted once.
//  * S^T = K q^T on 16x16x32 MFMA.  Keys go from the cache to registers: the
//    contraction may take the dimensions in any order, so lane (row, l / 16) loads
//    the (l / 16)th quarter of its token's row in one piece, and the queries are
//    held in the same order.  Tile T's row m is token
//    8 (m / 4) + 4 T + m % 4, so that lane l ends with the scores of tokens
//    8 (l / 16) .. + 7 of query l % 16, which is the A operand of
//  * O += P V.  Values go global -> LDS by direct 16-byte loads and come back
//    through transposed reads.
// The next step's values are loaded once this step's are in registers, its keys
// once this step's scores are there.  Weights are 2^(s - ref), where ref follows
// the running maximum when that is more than LAG above it: most steps rescale
// nothing.
//
// For few queries this is bound by loads: a step is 16 KB (e4m3) or 32 KB for 16 or
// 32 queries.  48 and 64 queries in the same way were slower than the shared tiles
// below, from 33 queries on (128 rows of 4 heads to a kv head behind 8000 e4m3 tokens:
// 58 us, 49; 10 rows 31, 25): every wavefront then waits for loads of its own.
// ---------------------------------------------------------------------------
constexpr float LAG = 6.f;

template <int D, bool E4>
constexpr int few_lds() { return 4 * (32 * D * (E4 ? 1 : 2) > 16 * D * 4 ? 32 * D * (E4 ? 1 : 2) : 16 * D * 4); }

template <int D, bool E4, bool PAGED, int MT, int SPANS, class QueryOf, class Emit>
__device__ __forceinline__ void attend_few(char *lds, float (*cm)[64], float (*cl)[64], int *lost, const CacheView &cv,
                                           const CacheLayer &layer, int nkv, int kvh, const Span (&spans)[SPANS],
                                           int queries, QueryOf &&query, Emit &&emit)
{
    constexpr int EB = E4 ? 1 : 2, RB = D * EB, KCH = RB / 16;       // bytes of a row; its 16-byte units
    constexpr int NK = RB / 64, NV = 32 * RB / 1024, ET = D / 16, KK = D / 32;
    const int tid = threadIdx.x, lane = tid & 63, hl = lane & 15, kg = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    if (tid == 0) *lost = 0;
    char *mine = lds + wave * 32 * RB;
    bf16x8 qf[MT][KK];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const uint16_t *q = 16 * m + hl < queries ? query(16 * m + hl) : nullptr;
#pragma unroll
        for (int kk = 0; kk < KK; ++kk) {
            uint4 v = {0u, 0u, 0u, 0u};
            if (q != nullptr) v = *(const uint4 *)(q + kg * (D / 4) + 8 * kk);
            qf[m][kk] = __builtin_bit_cast(bf16x8, v);
        }
    }
    const float scale2 = 1.4426950408889634f / sqrtf((float)D);      // scores in base 2
    f32x4 acc[MT][ET];
    float mrun[MT], lrun[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        mrun[m] = -INFINITY;
        lrun[m] = 0.f;
#pragma unroll
        for (int et = 0; et < ET; ++et) acc[m][et] = (f32x4){0.f, 0.f, 0.f, 0.f};
    }
    const uint8_t *kc = (const uint8_t *)layer.k, *vc = (const uint8_t *)layer.v;
    bool bad = false;
#pragma unroll
    for (int sp = 0; sp < SPANS; ++sp) {
        const int slot = spans[sp].slot, t_lo = spans[sp].t_lo, t_end = spans[sp].t_end;
        if (t_lo >= t_end) continue;
        const int32_t *pt = PAGED ? cv.kv.page_table + (size_t)slot * cv.kv.max_pages_per_seq : nullptr;
        int tb = (t_lo & ~15) + 32 * wave, pg[2] = {0, 0}, in[2] = {0, 0};
        const int ps = PAGED ? cv.kv.page_size : 16;
        Walk walk(PAGED ? tb : 0, 128, ps);
        auto pages = [&](int t) {                          // of the wavefront's two groups of 16 tokens from t, one step on at every call
            if constexpr (PAGED) {
                const bool same = walk.in + 16 < ps;
                if (t < t_end) pg[0] = pt[walk.page];
                if (t + 16 < t_end) pg[1] = pt[walk.page + !same];
                in[0] = walk.in;
                in[1] = same ? walk.in + 16 : 0;
                walk.next(ps);
            }
        };
        uint4 kr[2][NK];
        uint32_t ks = 0, vs = 0;                           // scale bytes of this lane's keys, and of its eight value tokens
        const uint8_t *kp = nullptr;
        auto issue_values = [&](int t) {                   // and where the step's keys are
            Rows16 at[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                int page = __builtin_amdgcn_readfirstlane(pg[j]);
                if (PAGED && (unsigned)page >= (unsigned)cv.num_pages) {
                    if (t + 16 * j < t_end) bad = true;
                    page = 0;
                }
                at[j] = rows16<PAGED>(cv, nkv, kvh, slot, page, in[j], t + 16 * j < t_end ? t + 16 * j : t);
                if (t + 16 * j >= t_end) at[j] = at[0];    // past the end: the first group again, masked below
            }
            const Rows16 ka = hl & 8 ? at[1] : at[0];
            kp = kc + (ka.row + 8 * ((hl >> 2) & 1) + (hl & 3)) * RB + kg * (RB / 4);
            if constexpr (E4) {
                ks = layer.ks[ka.blk];
                vs = layer.vs[(kg & 2 ? at[1] : at[0]).blk];
            }
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int tk = (j * 64 + lane) / KCH, p = (j * 64 + lane) % KCH;
                int c;
                if constexpr (E4) c = p ^ (KCH == 8 ? (tk >> 1) & 7 : (tk >> 2) & 3);
                else c = p ^ vtile_swz<KCH>(tk);
                const size_t row = (j * 64 / KCH >= 16 ? at[1] : at[0]).row;
                __builtin_amdgcn_global_load_lds((const void *)(vc + row * RB + (tk & 15) * RB + 16 * c),
                                                 (lds_void *)(mine + 1024 * j), 16, 0, 0);
            }
        };
        auto issue_keys = [&]() {
#pragma unroll
            for (int T = 0; T < 2; ++T)
#pragma unroll
                for (int j = 0; j < NK; ++j) kr[T][j] = *(const uint4 *)(kp + 4 * T * RB + 16 * j);
        };
        if (tb < t_end) {
            pages(tb);
            issue_values(tb);
            issue_keys();
            pages(tb + 128);
        }
        for (; tb < t_end; tb += 128) {
            const bool more = tb + 128 < t_end;
            __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
            asm volatile("" ::: "memory");
            const float ksc = __uint_as_float(ks << 23), vsc = __uint_as_float(vs << 23);
            uint4 vr[ET];                                  // e4m3: the codes in the first two words
#pragma unroll
            for (int et = 0; et < ET; ++et) {
                if constexpr (E4) {
                    const int t = 8 * kg + (hl >> 1), swz = KCH == 8 ? (t >> 1) & 7 : (t >> 2) & 3;
                    const uint2 w = read_tr8(mine + 16 * (t * KCH + (et ^ swz)) + 8 * (hl & 1));
                    vr[et] = (uint4){w.x, w.y, 0u, 0u};
                } else {
                    uint2 w[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        const int t = 8 * kg + 4 * r + (hl >> 2), c = 2 * et + ((hl & 3) >> 1);
                        w[r] = lds_read_tr16(mine + 16 * (t * KCH + (c ^ vtile_swz<KCH>(t))) + 8 * (hl & 1));
                    }
                    vr[et] = (uint4){w[0].x, w[0].y, w[1].x, w[1].y};
                }
            }
            __builtin_amdgcn_s_waitcnt(0xC07F);            // lgkmcnt(0): the values are in registers
            asm volatile("" ::: "memory");
            if (more) issue_values(tb + 128);
            const bool edge = tb < t_lo || tb + 32 > t_end;   // wave-uniform: some of the 32 tokens are masked
            const int first = t_lo - (tb + 8 * kg), behind = t_end - (tb + 8 * kg);   // this lane's real tokens: first .. behind - 1 of 8
            if (edge) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool off = e < first || e >= behind;
#pragma unroll
                    for (int et = 0; et < ET; ++et) {
                        uint32_t *w = (uint32_t *)&vr[et];
                        if constexpr (E4) w[e / 4] &= off ? ~(0xffu << (8 * (e % 4))) : ~0u;
                        else w[e / 2] &= off ? ~(0xffffu << (16 * (e % 2))) : ~0u;
                    }
                }
            }
            f32x4 st[MT][2];
#pragma unroll
            for (int m = 0; m < MT; ++m) st[m][0] = st[m][1] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                bf16x8 kf[2];
#pragma unroll
                for (int T = 0; T < 2; ++T) {
                    if constexpr (E4) {
                        const uint4 w = kr[T][kk / 2];
                        kf[T] = __builtin_bit_cast(bf16x8, kk & 1 ? codes8(w.z, w.w, ksc) : codes8(w.x, w.y, ksc));
                    } else {
                        kf[T] = __builtin_bit_cast(bf16x8, kr[T][kk]);
                    }
                }
#pragma unroll
                for (int m = 0; m < MT; ++m)
#pragma unroll
                    for (int T = 0; T < 2; ++T) st[m][T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[T], qf[m][kk], st[m][T], 0, 0, 0);
            }
            if (more) {
                issue_keys();
                pages(tb + 256);
            }
            bf16x8 ph[MT], pl[MT];
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                float mt = -INFINITY;
#pragma unroll
                for (int T = 0; T < 2; ++T)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (edge) st[m][T][e] = 4 * T + e >= first && 4 * T + e < behind ? st[m][T][e] : -INFINITY;
                        mt = fmaxf(mt, st[m][T][e]);
                    }
                mt = fmaxf(mt, other<16>(mt));
                mt = fmaxf(mt, other<32>(mt)) * scale2;
                const float mnew = mt > mrun[m] + LAG ? mt : mrun[m], moff = mnew == -INFINITY ? 0.f : mnew;
                if (__ballot(mnew != mrun[m])) {           // lane l's sums belong to queries 4 (l / 16) + e
                    const float alpha = mnew == mrun[m] ? 1.f : __builtin_amdgcn_exp2f(mrun[m] - mnew);
                    lrun[m] *= alpha;
                    mrun[m] = mnew;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float ae = __shfl(alpha, 4 * kg + e, 64);
#pragma unroll
                        for (int et = 0; et < ET; ++et) acc[m][et][e] *= ae;
                    }
                }
                uint32_t hi[4], lo[4];
                float ls = 0.f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(st[m][i / 2][2 * (i % 2)], scale2, -moff));
                    const float b = __builtin_amdgcn_exp2f(__builtin_fmaf(st[m][i / 2][2 * (i % 2) + 1], scale2, -moff));
                    ls += a + b;
                    const uint32_t w = f2bf2(a, b);
                    hi[i] = w;
                    lo[i] = f2bf2(a - __uint_as_float(w << 16), b - __uint_as_float(w & 0xffff0000u));
                }
                lrun[m] += ls;
                ph[m] = __builtin_bit_cast(bf16x8, hi);
                pl[m] = __builtin_bit_cast(bf16x8, lo);
            }
#pragma unroll
            for (int et = 0; et < ET; ++et) {
                const bf16x8 vf = __builtin_bit_cast(bf16x8, E4 ? codes8(vr[et].x, vr[et].y, vsc) : vr[et]);
#pragma unroll
                for (int m = 0; m < MT; ++m) {
                    acc[m][et] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ph[m], vf, acc[m][et], 0, 0, 0);
                    acc[m][et] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pl[m], vf, acc[m][et], 0, 0, 0);
                }
            }
        }
    }
    // the four wavefronts in order, 16 queries at a time, through the idle buffers
    __syncthreads();
    if (bad) *lost = 1;
    float *ca = (float *)lds;                          // [4][16][D]
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        lrun[m] += other<16>(lrun[m]);
        lrun[m] += other<32>(lrun[m]);
        if (lane < 16) {
            cm[wave][16 * m + lane] = mrun[m];
            cl[wave][16 * m + lane] = lrun[m];
        }
#pragma unroll
        for (int et = 0; et < ET; ++et)
#pragma unroll
            for (int e = 0; e < 4; ++e) ca[(wave * 16 + 4 * kg + e) * D + 16 * et + hl] = acc[m][et][e];
        __syncthreads();
        const int here = min(16, queries - 16 * m);
        for (int i = tid; i < here * (D / 4); i += 256) {
            const int g = i / (D / 4), d4 = i % (D / 4);
            float M = -INFINITY, L = 0.f;
#pragma unroll
            for (int w = 0; w < 4; ++w) M = fmaxf(M, cm[w][16 * m + g]);
            const float off = M == -INFINITY ? 0.f : M;
            float4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const float f = __builtin_amdgcn_exp2f(cm[w][16 * m + g] - off);
                const float4 x = *(const float4 *)(ca + (w * 16 + g) * D + 4 * d4);
                L += cl[w][16 * m + g] * f;
                o.x += x.x * f;
                o.y += x.y * f;
                o.z += x.z * f;
                o.w += x.w * f;
            }
            emit(16 * m + g, d4, o, *lost ? qnan() : M, L);
        }
        __syncthreads();
    }
}

// Query u's result of a split, to the workspace.
template <int D>
__device__ __forceinline__ void emit_part(float *part, int u, int d4, const float4 &o, float m, float l)
{
    float *dst = part + (u / 32) * part_floats<D>();
    *(float4 *)(dst + (d4 * 32 + u % 32) * 4) = o;
    if (d4 == 0) *(float2 *)(dst + 32 * D + 2 * (u % 32)) = {m, l};
}

// ---------------------------------------------------------------------------
// A tile of 128 queries over tokens t0 .. t_end - 1 of a prefix: four wavefronts
// of 32 queries each on shared tiles of 64 tokens.  Wavefront w loads the w-th 16
// tokens of the next tile into registers while this one is computed, and writes
// them as bf16 (codes times their scale) to the other of two LDS buffers.
//  * S^T = K Q^T on 32x32x16 MFMA, key rows permuted (pf_key_of_row) so that lane l
//    ends with eight consecutive keys 16 s + 8 (l / 32) .. + 7 of query l % 32 in
//    each step s of 16 keys: the operand P^T of
//  * O^T += V^T P^T, V^T by transposed reads.
//
// Bound by a wavefront's products and softmax in turn: a call of 128 rows of 64
// heads behind 32768 tokens takes 273 us (e4m3, 0.50 PFLOP/s; its conversions come on
// top) or 259 (bf16, 0.53); the second product is done twice, for the weights' halves.
// A SIMD's two wavefronts hardly overlap products and softmax: of the time that a CU
// was busy the matrix units took 43% and the vector units 55%.  One fp16 product over
// e4m3 values was 70 us faster there and is not used: a weight far below the largest
// lost its bits, and with them values that the largest ones do not meet.  Raising a
// wavefront's priority around its products changed nothing; tiles of 32 tokens, whose
// registers and LDS let three workgroups on a CU, took 279 us for bf16 where this took
// 250.
// ---------------------------------------------------------------------------
template <int KCH>
__device__ __forceinline__ int val16_swz(int t) { return vtile_swz<KCH>(t) ^ (t & 1); }

template <int D>
constexpr int many_lds() { return 4 * 64 * D * 2; }

template <int D, bool E4, bool PAGED, class QueryOf>
__device__ __forceinline__ void attend_many(char *lds, int *lost, const CacheView &cv, const CacheLayer &layer, int nkv,
                                            int kvh, int slot, int t0, int t_end, int queries, QueryOf &&query,
                                            float *part)
{
    constexpr int EB = E4 ? 1 : 2, RB = D * EB, RU = RB / 16;        // a row's bytes and 16-byte units in the cache
    constexpr int NR = 16 * RB / 1024, KCH = D / 8, UNITS = 64 * KCH, DT = D / 32, KS = D / 16;
    const int tid = threadIdx.x, lane = tid & 63, r32 = lane & 31, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const bool active = 32 * wave < queries;           // wave-uniform
    uint4 *ring = (uint4 *)lds;                        // keys of both buffers, then values
    if (tid == 0) *lost = 0;
    bf16x8 qf[KS];
    {
        const uint16_t *q = 32 * wave + r32 < queries ? query(32 * wave + r32) : nullptr;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            uint4 v = {0u, 0u, 0u, 0u};
            if (q != nullptr) v = *(const uint4 *)(q + 16 * ks + 8 * h);
            qf[ks] = __builtin_bit_cast(bf16x8, v);
        }
    }
    const uint8_t *kc = (const uint8_t *)layer.k, *vc = (const uint8_t *)layer.v;
    const int32_t *pt = PAGED ? cv.kv.page_table + (size_t)slot * cv.kv.max_pages_per_seq : nullptr;
    int next = t0 + 16 * wave, page = 0, in = 0;       // the wavefront's group of the next tile to load
    const int ps = PAGED ? cv.kv.page_size : 16;
    Walk walk(PAGED ? next : 0, 64, ps);
    bool bad = false;
    auto fetch_page = [&]() {
        if constexpr (PAGED) {
            if (next < t_end) page = pt[walk.page];
            in = walk.in;
            walk.next(ps);
        }
    };
    // the wavefront's next group: whether there is one, and where it stands
    auto locate = [&](Rows16 &at) -> bool {
        const bool real = next < t_end;
        if (real) {
            int pg = __builtin_amdgcn_readfirstlane(page);
            if (PAGED && (unsigned)pg >= (unsigned)cv.num_pages) {
                bad = true;
                pg = 0;
            }
            at = rows16<PAGED>(cv, nkv, kvh, slot, pg, in, next);
        }
        next += 64;
        return real;
    };
    // e4m3: to registers, and from there converted to buffer b of the tile from token k0
    uint4 kraw[NR] = {}, vraw[NR] = {};
    uint32_t ks8 = 0, vs8 = 0;
    auto load = [&]() {                                // past the end: what was loaded before, masked below
        Rows16 at;
        if (!locate(at)) return;
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            kraw[j] = *(const uint4 *)(kc + at.row * RB + 1024 * j + 16 * lane);
            vraw[j] = *(const uint4 *)(vc + at.row * RB + 1024 * j + 16 * lane);
        }
        ks8 = layer.ks[at.blk];
        vs8 = layer.vs[at.blk];
    };
    auto store = [&](int k0, int b) {
        uint4 *K = ring + b * UNITS, *V = ring + (2 + b) * UNITS;
        const float ksc = __uint_as_float(__builtin_amdgcn_readfirstlane(ks8) << 23);
        const float vsc = __uint_as_float(__builtin_amdgcn_readfirstlane(vs8) << 23);
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            const int u = 64 * j + lane, row = 16 * wave + u / RU, c = u % RU;
            uint4 w = vraw[j];
            if (k0 + 64 > t_end) {
                const uint32_t use = k0 + row < t_end ? ~0u : 0u;
                w = (uint4){w.x & use, w.y & use, w.z & use, w.w & use};
            }
            K[pf_swz<KCH>(row, 2 * c)] = codes8(kraw[j].x, kraw[j].y, ksc);
            K[pf_swz<KCH>(row, 2 * c + 1)] = codes8(kraw[j].z, kraw[j].w, ksc);
            V[row * KCH + ((2 * c) ^ val16_swz<KCH>(row))] = codes8(w.x, w.y, vsc);
            V[row * KCH + ((2 * c + 1) ^ val16_swz<KCH>(row))] = codes8(w.z, w.w, vsc);
        }
    };
    // bf16: straight to buffer b; values past the end are cleared once they have landed
    auto direct = [&](int b) {
        Rows16 at;
        if (!locate(at)) return;
        uint4 *K = ring + b * UNITS + 16 * wave * KCH, *V = ring + (2 + b) * UNITS + 16 * wave * KCH;
#pragma unroll
        for (int j = 0; j < NR; ++j) {
            const int u = 64 * j + lane, row = u / KCH, p = u % KCH;
            const size_t off = (at.row + row) * RB;
            const int ck = pf_swz<KCH>(row, p) % KCH, cv16 = p ^ val16_swz<KCH>(row);   // rows of a group: the same swizzles at any group
            __builtin_amdgcn_global_load_lds((const void *)(kc + off + 16 * ck), (lds_void *)(K + 64 * j), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const void *)(vc + off + 16 * cv16), (lds_void *)(V + 64 * j), 16, 0, 0);
        }
    };
    auto clear = [&](int k0, int b) {
        uint4 *V = ring + (2 + b) * UNITS + 16 * wave * KCH;
        for (int u = lane; u < 16 * KCH; u += 64)
            if (k0 + 16 * wave + u / KCH >= t_end) V[u] = (uint4){0u, 0u, 0u, 0u};
    };
    f32x16 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[dt][j] = 0.f;
    float mrow = -INFINITY, lpart = 0.f;
    const float scale2 = 1.4426950408889634f / sqrtf((float)D);
    const int krow = pf_key_of_row(r32), a4 = lane & 3, qv = (lane >> 2) & 3, half16 = (lane >> 4) & 1;

    fetch_page();
    if constexpr (E4) {
        load();
        fetch_page();
        store(t0, 0);
        load();
    } else {
        direct(0);
    }
    fetch_page();
#pragma unroll 1
    for (int k0 = t0, b = 0; k0 < t_end; k0 += 64, b ^= 1) {
        if constexpr (!E4) {
            __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
            asm volatile("" ::: "memory");
            if (k0 + 64 > t_end) clear(k0, b);
        }
        __syncthreads();                               // the tile is in LDS, and the one before is done with
        if (k0 + 64 < t_end) {
            if constexpr (E4) {
                store(k0 + 64, b ^ 1);
                load();
            } else {
                direct(b ^ 1);
            }
            fetch_page();
        }
        if (!active) continue;
        const uint4 *Kt = ring + b * UNITS, *Vt = ring + (2 + b) * UNITS;
        f32x16 st[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int j = 0; j < 16; ++j) st[kt][j] = 0.f;
        constexpr int KD = 2;                          // key operands are read that many steps ahead
        bf16x8 kf[KD + 1][2];
        int kr = krow;
        asm volatile("" : "+v"(kr));                   // the steps' addresses are made anew: kept, they cost registers
        auto kread = [&](int ks) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
                kf[ks % (KD + 1)][kt] = __builtin_bit_cast(bf16x8, Kt[pf_swz<KCH>(32 * kt + kr, 2 * ks + h)]);
        };
#pragma unroll
        for (int ks = 0; ks < KD; ++ks) kread(ks);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            if (ks + KD < KS) kread(ks + KD);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
                st[kt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks % (KD + 1)][kt], qf[ks], st[kt], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        // lane: keys k0 + 32 kt + 16 (j / 8) + 8 h + j % 8 of its query
        if (k0 + 64 > t_end) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int j = 0; j < 16; ++j)
                    st[kt][j] = k0 + 32 * kt + 16 * (j >> 3) + 8 * h + (j & 7) < t_end ? st[kt][j] : -INFINITY;
        }
        float mt = -INFINITY;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int j = 0; j < 16; ++j) mt = fmaxf(mt, st[kt][j]);
        const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
        mt = fmaxf(__uint_as_float(two[0]), __uint_as_float(two[1])) * scale2;   // both halves of the query's keys
        const float mnew = mt > mrow + LAG ? mt : mrow, moff = mnew == -INFINITY ? 0.f : mnew;
        if (__ballot(mnew != mrow)) {
            const float alpha = mnew == mrow ? 1.f : __builtin_amdgcn_exp2f(mrow - mnew);
            lpart *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[dt][j] *= alpha;
            mrow = mnew;
        }
        bf16x8 ph[4], pl[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            uint32_t hi[4], lo[4];
            float ls = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(st[s / 2][8 * (s % 2) + 2 * e], scale2, -moff));
                const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(st[s / 2][8 * (s % 2) + 2 * e + 1], scale2, -moff));
                ls += x + y;
                const uint32_t w = f2bf2(x, y);
                hi[e] = w;
                lo[e] = f2bf2(x - __uint_as_float(w << 16), y - __uint_as_float(w & 0xffff0000u));
            }
            ph[s] = __builtin_bit_cast(bf16x8, hi);
            pl[s] = __builtin_bit_cast(bf16x8, lo);
            lpart += ls;
        }
        // operand f: step f / DT of 16 keys, dimensions 32 (f % DT) + l % 32
        constexpr int VD = 3;
        bf16x8 vf[VD + 1];
        auto vread = [&](int f) {
            uint2 w[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int key = 16 * (f / DT) + 8 * h + 4 * r + qv, c = 4 * (f % DT) + 2 * half16 + (a4 >> 1);
                w[r] = lds_read_tr16((const char *)(Vt + key * KCH + (c ^ val16_swz<KCH>(key))) + 8 * (a4 & 1));
            }
            vf[f % (VD + 1)] = __builtin_bit_cast(bf16x8, (uint4){w[0].x, w[0].y, w[1].x, w[1].y});
        };
#pragma unroll
        for (int f = 0; f < VD; ++f) vread(f);
#pragma unroll
        for (int f = 0; f < 4 * DT; ++f) {
            if (f + VD < 4 * DT) vread(f + VD);
            __builtin_amdgcn_sched_barrier(0);
            acc[f % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[f % (VD + 1)], ph[f / DT], acc[f % DT], 0, 0, 0);
            acc[f % DT] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[f % (VD + 1)], pl[f / DT], acc[f % DT], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (bad) *lost = 1;
    __syncthreads();
    if (!active) return;
    // lane: O^T[32 dt + 8 (j / 4) + 4 h + j % 4][query l % 32]
    const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(lpart), __float_as_uint(lpart), false, false);
    const float sum = __uint_as_float(two[0]) + __uint_as_float(two[1]);
    float *dst = part + wave * part_floats<D>();
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int j = 0; j < 16; j += 4)
            *(float4 *)(dst + 4 * ((8 * dt + j / 2 + h) * 32 + r32)) = {acc[dt][j], acc[dt][j + 1], acc[dt][j + 2], acc[dt][j + 3]};
    if (h == 0) *(float2 *)(dst + 32 * D + 2 * r32) = {*lost ? qnan() : mrow, sum};
}

// Workgroup: a kv head (running fastest) of a unit, which is a query tile and split
// of a prefix, or a split of a row's own tokens.
template <int D, bool E4, bool PAGED, int MT>
__global__ __launch_bounds__(256, 2) void k_shared_parts(SharedArgs a, GroupTable gt, Shape s, CacheView cv,
                                                         CacheLayer layer, float *__restrict__ ws)
{
    constexpr int FEW = few_lds<D, E4>(), LDS = MT == 128 && many_lds<D>() > FEW ? many_lds<D>() : FEW;
    __shared__ __attribute__((aligned(16))) char lds[LDS];
    __shared__ float cm[4][64], cl[4][64];
    __shared__ int lost;
    const int nkv = a.nkv, G = s.G, kvh = blockIdx.x % nkv, unit = blockIdx.x / nkv;
    const int np = s.tiles * s.splits_p;               // the prefixes' units come first
    if (unit < np) {
        const int tile = unit % s.tiles, split = unit / s.tiles;
        const int gi = last_at_most(s.tile0, gt.n, tile);
        const Prefix p = prefix_of(a, gt, cv, gi);
        const Span span = prefix_span(p, s.chunk_p, split);
        if (span.t_lo >= span.t_end) return;
        const int u0 = (tile - s.tile0[gi]) * MT, row0 = gt.row0[gi];
        const int queries = min(MT, (gt.row0[gi + 1] - row0) * G - u0);
        const auto query = [&](int m) {
            return a.q + (size_t)(row0 + (u0 + m) / G) * a.ldq + (size_t)(kvh * G + (u0 + m) % G) * D;
        };
        float *part = part_at<D>(ws, s, nkv, split, kvh, s.qb0[gi]);
        if constexpr (MT == 128)
            attend_many<D, E4, PAGED>(lds, &lost, cv, layer, nkv, kvh, span.slot, span.t_lo, span.t_end, queries, query,
                                      part + (u0 / 32) * part_floats<D>());
        else
            attend_few<D, E4, PAGED, MT / 16, 1>(
                lds, cm, cl, &lost, cv, layer, nkv, kvh, {span}, queries, query,
                [&](int u, int d4, const float4 &o, float m, float l) { emit_part<D>(part, u0 + u, d4, o, m, l); });
        return;
    }
    const int v = unit - np, split = v % s.splits_s, r = v / s.splits_s;
    const int gi = last_at_most(gt.row0, gt.n, r);
    const Prefix p = prefix_of(a, gt, cv, gi);
    const Span span = own_span(p, r, row_len(a, cv, p, r), s.chunk_s, split);
    if (span.t_lo >= span.t_end) return;
    const auto query = [&](int m) { return a.q + (size_t)r * a.ldq + (size_t)(kvh * G + m) * D; };
    float *part = part_at<D>(ws, s, nkv, s.splits_p + split, kvh, s.qb0[gi]);
    const int u0 = (r - gt.row0[gi]) * G;
    attend_few<D, E4, PAGED, 1, 1>(lds, cm, cl, &lost, cv, layer, nkv, kvh, {span}, G, query,
                                   [&](int u, int d4, const float4 &o, float m, float l) {
                                       emit_part<D>(part, u0 + u, d4, o, m, l);
                                   });
}

// The smallest calls in one launch: a workgroup to a row and kv head, which goes
// over the prefix and the row's own tokens by itself.
template <int D, bool E4, bool PAGED>
__global__ __launch_bounds__(256, 2) void k_shared_alone(SharedArgs a, GroupTable gt, CacheView cv, CacheLayer layer)
{
    __shared__ __attribute__((aligned(16))) char lds[few_lds<D, E4>()];
    __shared__ float cm[4][64], cl[4][64];
    __shared__ int lost;
    const int nkv = a.nkv, G = a.nq / nkv, kvh = blockIdx.x % nkv, r = blockIdx.x / nkv;
    const int gi = last_at_most(gt.row0, gt.n, r);
    const Prefix p = prefix_of(a, gt, cv, gi);
    const int n = row_len(a, cv, p, r);
    uint16_t *out = a.out + (size_t)r * a.ldo + (size_t)kvh * G * D;
    if (n <= 0) {
        for (int i = threadIdx.x; i < G * D; i += 256) out[i] = n < 0 ? (uint16_t)0x7fc0 : (uint16_t)0;
        return;
    }
    const auto query = [&](int m) { return a.q + (size_t)r * a.ldq + (size_t)(kvh * G + m) * D; };
    attend_few<D, E4, PAGED, 1, 2>(lds, cm, cl, &lost, cv, layer, nkv, kvh, {{p.slot, 0, p.len}, {r, p.len, n}}, G, query,
                                   [&](int u, int d4, const float4 &o, float m, float l) {
                                       const float inv = (m != m ? m : 1.0f) / l;
                                       *(uint2 *)(out + (size_t)u * D + 4 * d4) = {f2bf2(o.x * inv, o.y * inv),
                                                                                  f2bf2(o.z * inv, o.w * inv)};
                                   });
}

// Joins the splits: a workgroup takes four dimension fours (y) of a 32-query block
// of a kv head (x); thread (four, query).  Sixteen splits' loads are in flight at
// once: latency, 4.5 us for 32 queries of 13 splits, 8 to 10 for 1024 (with eight, after a
// pass over the maxima, 11.4 for the 32).
template <int D>
__global__ __launch_bounds__(128) void k_shared_join(SharedArgs a, GroupTable gt, Shape s, CacheView cv,
                                                     float *__restrict__ ws)
{
    constexpr int PF = 16;                             // splits whose values are in flight at once
    const int nkv = a.nkv, G = s.G, kvh = blockIdx.x % nkv, block = blockIdx.x / nkv;
    const int tid = threadIdx.x, u32 = tid & 31, d4 = 4 * blockIdx.y + (tid >> 5);
    const int gi = last_at_most(s.qb0, gt.n, block);
    const int u = 32 * (block - s.qb0[gi]) + u32, r = gt.row0[gi] + u / G;
    if (r >= gt.row0[gi + 1]) return;
    const Prefix p = prefix_of(a, gt, cv, gi);
    const int n = row_len(a, cv, p, r);
    uint16_t *out = a.out + (size_t)r * a.ldo + (size_t)(kvh * G + u % G) * D + 4 * d4;
    if (n <= 0) {
        const uint32_t w = n < 0 ? 0x7fc07fc0u : 0u;
        *(uint2 *)out = {w, w};
        return;
    }
    const int np = (p.len + s.chunk_p - 1) / s.chunk_p;
    const int parts = np + (n > p.len ? (n - (p.len & ~15) + s.chunk_s - 1) / s.chunk_s : 0);
    const float *base = part_at<D>(ws, s, nkv, 0, kvh, block);
    const size_t split = (size_t)nkv * s.blocks * part_floats<D>();
    float M = -INFINITY, L = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    for (int i0 = 0; i0 < parts; i0 += PF) {           // in order, relative to the largest maximum so far
        f32x4 x[PF];
        f32x2 ml[PF];
#pragma unroll
        for (int j = 0; j < PF; ++j) {
            const int i = i0 + j;
            x[j] = (f32x4){0.f, 0.f, 0.f, 0.f};
            ml[j] = (f32x2){-INFINITY, 0.f};
            if (i < parts) {
                const float *b = base + (size_t)(i < np ? i : s.splits_p + i - np) * split;
                x[j] = *(const f32x4 *)(b + (d4 * 32 + u32) * 4);
                ml[j] = *(const f32x2 *)(b + 32 * D + 2 * u32);
            }
        }
        float m = M;
#pragma unroll
        for (int j = 0; j < PF; ++j) m = fmaxf(m, ml[j].x);   // a NaN shows in the sums
        const float off = m == -INFINITY ? 0.f : m, down = __builtin_amdgcn_exp2f(M - off);
        M = m;
        L *= down;
        o *= down;
#pragma unroll
        for (int j = 0; j < PF; ++j) {
            const float f = __builtin_amdgcn_exp2f(ml[j].x - off);   // 0 past the last split
            L += ml[j].y * f;
            o += x[j] * f;
        }
    }
    const float inv = 1.0f / L;
    *(uint2 *)out = {f2bf2(o.x * inv, o.y * inv), f2bf2(o.z * inv, o.w * inv)};
}

}  // namespace

// Whether a call is one launch of a workgroup to a row and kv head: few enough that
// all run at once, and not over four steps of 128 tokens.
static bool alone(const GroupTable &g, int nkv, int max_prefix, int max_suffix)
{
    return (long long)max_prefix + max_suffix <= 512 && (long long)g.row0[g.n] * nkv <= 512;
}

SharedShape shared_shape(const GroupTable &g, int nq, int nkv, int max_prefix, int max_suffix)
{
    SharedShape s;
    s.alone = alone(g, nkv, max_prefix, max_suffix);
    s.G = nq / nkv;
    int most = 0;
    for (int i = 0; i < g.n; ++i) most = std::max(most, (g.row0[i + 1] - g.row0[i]) * s.G);
    s.mt = most <= 16 ? 16 : most <= 32 ? 32 : 128;
    s.blocks = s.tiles = 0;
    for (int i = 0; i < g.n; ++i) {
        const int queries = (g.row0[i + 1] - g.row0[i]) * s.G;
        s.qb0[i] = (uint16_t)s.blocks;
        s.tile0[i] = (uint16_t)s.tiles;
        s.blocks += (queries + 31) / 32;
        s.tiles += (queries + s.mt - 1) / s.mt;
    }
    s.qb0[g.n] = (uint16_t)s.blocks;
    s.tile0[g.n] = (uint16_t)s.tiles;   // rows bound all of them
    // Tokens of a split: about `wgs` workgroups in all, splits of at least 256 tokens
    // (8 rows behind 4000 in bf16: 17 us, 18.6 with 128) and of at most `longest`, 256
    // splits at most.
    const auto chunk = [](long long tokens, long long units, long long wgs, long long longest) {
        long long n = std::max<long long>(1, wgs / std::max<long long>(1, units));
        n = std::min<long long>(std::max(std::min(n, (tokens + 255) / 256), (tokens + longest - 1) / longest), 256);
        const long long per = (tokens + n - 1) / n;
        return (int)std::min<long long>((per + 127) / 128 * 128, 1 << 30);
    };
    // One group: a workgroup to each CU (8000 tokens in bf16 for 128 rows of 8 kv heads
    // and 32: 53 us, 59 with 512 workgroups, 81 with 128; 64 rows 35, 40, 47).  Of
    // several, some may be shorter than the longest, and workgroups of many tokens then
    // end late (four of 11 to 30 thousand tokens: 159 us with splits of 1664, 238 of
    // 7424; eight of 500 to 8000: 60 of 1024, 71 of 2048).  Prefixes of up to 15 K tokens
    // take splits of 1024, longer ones fifteen or sixteen splits: a fifteenth rounded
    // down, since rounded up the documents' 1920 became 2048 (145 us, 175 so).
    s.chunk_p = chunk(max_prefix, (long long)s.tiles * nkv, 256, g.n == 1 ? 1 << 30 : std::max(1024, max_prefix / 15));
    s.splits_p = (int)(((long long)max_prefix + s.chunk_p - 1) / s.chunk_p);
    const long long suffix = (long long)max_suffix + 15;
    s.chunk_s = chunk(suffix, (long long)g.row0[g.n] * nkv, 2048, 1 << 30);
    s.splits_s = (int)((suffix + s.chunk_s - 1) / s.chunk_s);
    return s;
}

long long shared_workgroups(const GroupTable &g, const SharedShape &s, int nkv)
{
    if (s.alone) return (long long)g.row0[g.n] * nkv;
    return std::max(((long long)s.tiles * s.splits_p + (long long)g.row0[g.n] * s.splits_s) * nkv, (long long)s.blocks * nkv);
}

size_t shared_ws(const SharedShape &s, int nkv, int d)
{
    if (s.alone) return 0;
    return (size_t)(s.splits_p + s.splits_s) * nkv * s.blocks * (d == 128 ? part_floats<128>() : part_floats<64>()) *
           sizeof(float);
}

hipError_t launch_shared(const SharedArgs &a, const GroupTable &g, const SharedShape &s, const CacheView &cv,
                         const CacheLayer &cl, float *ws, hipStream_t st)
{
    const long long wgs = shared_workgroups(g, s, a.nkv);
    const bool paged = cv.kv.layout == 1;
    if (s.alone) {
        const dim3 grid((unsigned)g.row0[g.n] * a.nkv);
#define CORUN_ALONE(D_, E_) \
    if (a.d == D_ && cv.e4m3 == E_ && paged) KLAUNCH((k_shared_alone<D_, E_, true>), grid, dim3(256), 0, st, a, g, cv, cl); \
    if (a.d == D_ && cv.e4m3 == E_ && !paged) KLAUNCH((k_shared_alone<D_, E_, false>), grid, dim3(256), 0, st, a, g, cv, cl)
        CORUN_ALONE(128, 1);
        CORUN_ALONE(128, 0);
        CORUN_ALONE(64, 1);
        CORUN_ALONE(64, 0);
#undef CORUN_ALONE
        return hipGetLastError();
    }
#define CORUN_SHARED(D_, E_, P_, M_) \
    KLAUNCH((k_shared_parts<D_, E_, P_, M_>), dim3((unsigned)wgs), dim3(256), 0, st, a, g, s, cv, cl, ws)
#define CORUN_SHARED_M(D_, E_, P_)                     \
    do {                                               \
        if (s.mt == 16) CORUN_SHARED(D_, E_, P_, 16);  \
        else if (s.mt == 32) CORUN_SHARED(D_, E_, P_, 32); \
        else CORUN_SHARED(D_, E_, P_, 128);            \
    } while (0)
#define CORUN_SHARED_P(D_, E_)                  \
    do {                                        \
        if (paged) CORUN_SHARED_M(D_, E_, true); \
        else CORUN_SHARED_M(D_, E_, false);     \
    } while (0)
    if (a.d == 128 && cv.e4m3) CORUN_SHARED_P(128, true);
    else if (a.d == 128) CORUN_SHARED_P(128, false);
    else if (a.d == 64 && cv.e4m3) CORUN_SHARED_P(64, true);
    else if (a.d == 64) CORUN_SHARED_P(64, false);
    else return hipErrorInvalidValue;
#undef CORUN_SHARED_P
#undef CORUN_SHARED_M
#undef CORUN_SHARED
    const dim3 grid((unsigned)s.blocks * a.nkv, a.d / 16);
    if (a.d == 128) KLAUNCH(k_shared_join<128>, grid, dim3(128), 0, st, a, g, s, cv, ws);
    else KLAUNCH(k_shared_join<64>, grid, dim3(128), 0, st, a, g, s, cv, ws);
    return hipGetLastError();
}

}  // namespace corun
