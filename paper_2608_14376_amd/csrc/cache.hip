// cache.hip -- rotary positions, the append to bf16 and e4m3 caches, and
// attention over e4m3 caches.
//
// An e4m3 cache holds one byte per element and, for every block of 16, 32 or
// 64 tokens of one kv head, a power-of-two scale 2^e as the byte e + 127: an
// element is code 2^e.  A code has four significant bits, so the element is
// exact in bf16, and scaling by a power of two moves no mantissa: when a later
// token of a block needs a larger scale, its earlier codes are divided by a
// power of two, which rounds only values that fall among the subnormals.
// A scale is the smallest power of two with amax <= 448 2^e over the tokens
// appended by one call (448 is the largest code), never smaller than what the
// block's earlier tokens have.
//
// Like every kernel of the step, these are position-invariant: a row's work
// follows from its own data and length, in a fixed order, with no atomics.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "cache.h"
#include "device.h"

namespace corun {
namespace {

constexpr int E_MIN = -100;    // smallest scale exponent: every nonzero value stays a normal bf16 number

// The page of token t of a slot, or -1 where the table's entry is no page.
__device__ __forceinline__ int page_of(const CacheView &cv, int slot, int t)
{
    const int p = cv.kv.page_table[(size_t)slot * cv.kv.max_pages_per_seq + t / cv.kv.page_size];
    return (unsigned)p < (unsigned)cv.num_pages ? p : -1;
}

// A token's row of d elements, and the block it is in, of one kv head: indices
// into the codes (or bf16 rows) and the scale bytes.  page: page_of, paged
// caches only.
struct Place {
    size_t row, blk;
};
__device__ __forceinline__ Place place(const CacheView &cv, int nkv, int kvh, int slot, int page, int t)
{
    if (cv.kv.layout == 1) {
        const int at = t % cv.kv.page_size;
        const size_t head = (size_t)page * nkv + kvh;
        return {head * cv.kv.page_size + at, head * (cv.kv.page_size >> cv.blk_shift) + (at >> cv.blk_shift)};
    }
    const size_t head = (size_t)slot * nkv + kvh;
    return {head * cv.kv.max_seq_len + t, head * (cv.kv.max_seq_len >> cv.blk_shift) + (t >> cv.blk_shift)};
}

// The sequence that unit u of a call belongs to: one load and a count, where a
// walk through the table would wait for every entry.
__device__ __forceinline__ int seq_of(const SeqTable &seq, int u)
{
    static_assert(sizeof(SeqTable::unit0) == 64 * sizeof(int), "a lane to a sequence");
    const int lane = threadIdx.x & 63;
    const bool before = lane < seq.n && seq.unit0[lane] <= u;
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(before)) - 1);
}

__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }   // -126 .. 127

// The scale exponent that the largest finite magnitude (as bits) needs: the
// smallest e with amax <= 448 2^e = 1.75 2^(e + 8).
__device__ __forceinline__ int scale_exp(uint32_t amax)
{
    const int e = (int)(amax >> 23) - 127 - 8 + ((amax & 0x7fffffu) > 0x600000u);
    return max(e, E_MIN);
}

// Magnitude bits of a finite value; 0 for infinities and NaN, which get the
// NaN code whatever the scale.
__device__ __forceinline__ uint32_t finite_bits(float x)
{
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < 0x7f800000u ? u : 0u;
}

// Four codes: values times m (a power of two), rounded to nearest, ties to even.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float e, float m)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a * m, b * m, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * m, e * m, w, true);
}

// Four codes times m <= 1, rounded again.
__device__ __forceinline__ uint32_t rescale4(uint32_t w, float m)
{
    return encode4(__builtin_amdgcn_cvt_f32_fp8(w, 0), __builtin_amdgcn_cvt_f32_fp8(w, 1),
                   __builtin_amdgcn_cvt_f32_fp8(w, 2), __builtin_amdgcn_cvt_f32_fp8(w, 3), m);
}

// cos and sin of t turns, 64 bits.  The nearest quarter turn is taken off, and
// the rest, |x| <= pi / 4, goes through the Taylor series to x^15 and x^14
// (next terms below 1e-15).
__device__ __forceinline__ void turn_cos_sin(double turns, double pos, double &c, double &s)
{
    const double whole = turns * pos;
    const double u = __builtin_fma(turns, pos, -__builtin_rint(whole));   // within half a turn of 0
    const double quarter = __builtin_rint(4.0 * u);
    const double x = 6.283185307179586476925 * __builtin_fma(-0.25, quarter, u), z = x * x;
    double sn = -1.0 / 1307674368000.0, cn = -1.0 / 87178291200.0;
    sn = __builtin_fma(sn, z, 1.0 / 6227020800.0);
    sn = __builtin_fma(sn, z, -1.0 / 39916800.0);
    sn = __builtin_fma(sn, z, 1.0 / 362880.0);
    sn = __builtin_fma(sn, z, -1.0 / 5040.0);
    sn = __builtin_fma(sn, z, 1.0 / 120.0);
    sn = __builtin_fma(sn, z, -1.0 / 6.0);
    sn = __builtin_fma(sn * z, x, x);
    cn = __builtin_fma(cn, z, 1.0 / 479001600.0);
    cn = __builtin_fma(cn, z, -1.0 / 3628800.0);
    cn = __builtin_fma(cn, z, 1.0 / 40320.0);
    cn = __builtin_fma(cn, z, -1.0 / 720.0);
    cn = __builtin_fma(cn, z, 1.0 / 24.0);
    cn = __builtin_fma(cn, z, -0.5);
    cn = __builtin_fma(cn, z, 1.0);
    const int q = (int)quarter & 3;
    const double a = q & 1 ? sn : cn, b = q & 1 ? cn : sn;
    c = q == 1 || q == 2 ? -a : a;
    s = q >= 2 ? -b : b;
}

// 64 -> 32 bits, inexact results to the neighbour with an odd last bit: a
// further rounding to fewer bits then gives what rounding the 64-bit value
// once would.
__device__ __forceinline__ float to_odd(double y)
{
    float r = (float)y;
    const double back = (double)r;
    uint32_t u = __float_as_uint(r);
    if (back != y && !(u & 1u)) u += __builtin_fabs(back) > __builtin_fabs(y) ? 0xffffffffu : 1u;
    return __uint_as_float(u);
}

// ---------------------------------------------------------------------------
// Append.  A thread owns eight pairs of one token and keeps their cosines and
// sines while it goes from head to head: two runs of eight elements from a0 and
// b0 on, (8 j, 8 j + rot / 2) for rotated half pairs, otherwise the 16
// elements from 16 j on, whose pairs stand side by side.  Half pairs of a rot
// that is no multiple of 16 are read one element at a time (VEC false), pair j +
// t D / 16 in turn, so that a token's threads read side by side (4000 tokens of 32 +
// 8 + 8 heads, rot 52: 43 us, 78 with eight pairs in a row; rot 64, in runs: 25).
//
// q is rotated in fp32 and rounded once to bf16, as are bf16 keys.  Keys that
// become codes are rotated in 64 bits and rounded to odd, so that a code is the
// nearest one to the exact product however close it is to a tie; kv heads alone
// take that.
//
// Bound by reading the rows and writing q and the cache: 32768 tokens of 64 + 8 +
// 8 heads of 128 in 282 us, 4.5 TB/s (a large copy reaches 5.2); cosines are made
// once per token and pair instead of per head or read from a table.
// ---------------------------------------------------------------------------
template <int D, bool VEC>
struct Pairs {
    int j, a0, b0, rot2;           // thread of the token; runs; rotated pairs of the head
    bool half;

    __device__ __forceinline__ Pairs(const RopeArgs &r, int j_)
    {
        j = j_;
        rot2 = r.rot / 2;
        half = !r.interleaved && 8 * j < rot2;
        a0 = half ? 8 * j : 16 * j;
        b0 = half ? 8 * j + rot2 : 16 * j + 8;
    }
    __device__ __forceinline__ int pair(int t) const { return VEC ? 8 * j + t : j + t * (D / 16); }
    __device__ __forceinline__ bool rotated(int t) const { return pair(t) < rot2; }
    // element offsets of pair t where the runs do not hold it
    __device__ __forceinline__ int at(int t, int which) const
    {
        const int i = pair(t);
        return i < rot2 ? i + which * rot2 : 2 * i + which;
    }
};

// Cosines and sines of a thread's pairs at a position.
struct Turn64 {
    double c[8], s[8];
    template <class P>
    __device__ __forceinline__ void init(const RopeArgs &r, const P &p, int pos)
    {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            turn_cos_sin(r.turns[p.pair(t)], (double)pos, c[t], s[t]);
            c[t] *= r.mag;
            s[t] *= r.mag;
        }
    }
};

// What a thread loads of a head, as loaded: 16 bf16 values (fp32 partials are
// summed and rounded).  Pair t of a VEC thread: elements t and 8 + t (half), or
// 2 t and 2 t + 1.
struct Raw {
    uint32_t w[8];
};

template <int D, bool VEC>
__device__ __forceinline__ Raw load_raw(const QkvRows &in, const Pairs<D, VEC> &p, long long row, int head)
{
    const size_t off = (size_t)row * in.ld + (size_t)head * D;
    Raw r;
    if (in.bf16 != nullptr) {
        const uint16_t *src = in.bf16 + off;
        if constexpr (VEC) {
            const uint4 a = *(const uint4 *)(src + p.a0), b = *(const uint4 *)(src + p.b0);
            r.w[0] = a.x; r.w[1] = a.y; r.w[2] = a.z; r.w[3] = a.w;
            r.w[4] = b.x; r.w[5] = b.y; r.w[6] = b.z; r.w[7] = b.w;
        } else {
#pragma unroll
            for (int t = 0; t < 8; ++t) r.w[t] = (uint32_t)src[p.at(t, 0)] | ((uint32_t)src[p.at(t, 1)] << 16);
        }
        return r;
    }
    float e[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) e[i] = 0.f;
    for (int sp = 0; sp < in.S; ++sp) {
        const float *src = in.part + sp * in.stride + off;
        if constexpr (VEC) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 f = *(const float4 *)(src + (i < 2 ? p.a0 : p.b0) + 4 * (i & 1));
                e[4 * i] += f.x;
                e[4 * i + 1] += f.y;
                e[4 * i + 2] += f.z;
                e[4 * i + 3] += f.w;
            }
        } else {
#pragma unroll
            for (int t = 0; t < 8; ++t) {
                e[2 * t] += src[p.at(t, 0)];
                e[2 * t + 1] += src[p.at(t, 1)];
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) r.w[i] = f2bf2(e[2 * i], e[2 * i + 1]);
    return r;
}

__device__ __forceinline__ float lo_f(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The pairs' first and second elements.
template <int D, bool VEC>
__device__ __forceinline__ void to_pairs(const Raw &r, const Pairs<D, VEC> &p, float (&x0)[8], float (&x1)[8])
{
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        if (VEC && p.half) {
            x0[t] = t & 1 ? hi_f(r.w[t / 2]) : lo_f(r.w[t / 2]);
            x1[t] = t & 1 ? hi_f(r.w[4 + t / 2]) : lo_f(r.w[4 + t / 2]);
        } else {
            x0[t] = lo_f(r.w[t]);
            x1[t] = hi_f(r.w[t]);
        }
    }
}

template <int D, bool VEC>
__device__ __forceinline__ void rotate(const Pairs<D, VEC> &p, const float (&c)[8], const float (&s)[8], float (&x0)[8],
                                       float (&x1)[8])
{
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        const float y0 = __builtin_fmaf(x0[t], c[t], -(x1[t] * s[t])), y1 = __builtin_fmaf(x1[t], c[t], x0[t] * s[t]);
        x0[t] = p.rotated(t) ? y0 : x0[t];
        x1[t] = p.rotated(t) ? y1 : x1[t];
    }
}

template <int D, bool VEC>
__device__ __forceinline__ void rotate_exact(const Pairs<D, VEC> &p, const Turn64 &tu, float (&x0)[8], float (&x1)[8])
{
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        const double u = x0[t], w = x1[t];
        const float y0 = to_odd(__builtin_fma(u, tu.c[t], -(w * tu.s[t]))), y1 = to_odd(__builtin_fma(w, tu.c[t], u * tu.s[t]));
        x0[t] = p.rotated(t) ? y0 : x0[t];
        x1[t] = p.rotated(t) ? y1 : x1[t];
    }
}

template <int D, bool VEC>
__device__ __forceinline__ void store_bf16(uint16_t *dst, const Pairs<D, VEC> &p, const float (&y0)[8], const float (&y1)[8])
{
    if constexpr (!VEC) {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            dst[p.at(t, 0)] = f2bf(y0[t]);
            dst[p.at(t, 1)] = f2bf(y1[t]);
        }
    } else {
        uint32_t w[8];
        if (p.half) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                w[t] = f2bf2(y0[2 * t], y0[2 * t + 1]);
                w[4 + t] = f2bf2(y1[2 * t], y1[2 * t + 1]);
            }
        } else {
#pragma unroll
            for (int t = 0; t < 8; ++t) w[t] = f2bf2(y0[t], y1[t]);
        }
        *(uint4 *)(dst + p.a0) = (uint4){w[0], w[1], w[2], w[3]};
        *(uint4 *)(dst + p.b0) = (uint4){w[4], w[5], w[6], w[7]};
    }
}

template <int D, bool VEC>
__device__ __forceinline__ void store_codes(uint8_t *dst, const Pairs<D, VEC> &p, const float (&y0)[8], const float (&y1)[8],
                                            int e)
{
    const float m = exp2_int(-e);
    if constexpr (!VEC) {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const uint32_t w = encode4(y0[t], y1[t], 0.f, 0.f, m);
            dst[p.at(t, 0)] = (uint8_t)w;
            dst[p.at(t, 1)] = (uint8_t)(w >> 8);
        }
    } else if (p.half) {
        *(uint2 *)(dst + p.a0) = (uint2){encode4(y0[0], y0[1], y0[2], y0[3], m), encode4(y0[4], y0[5], y0[6], y0[7], m)};
        *(uint2 *)(dst + p.b0) = (uint2){encode4(y1[0], y1[1], y1[2], y1[3], m), encode4(y1[4], y1[5], y1[6], y1[7], m)};
    } else {
        *(uint4 *)(dst + p.a0) =
            (uint4){encode4(y0[0], y1[0], y0[1], y1[1], m), encode4(y0[2], y1[2], y0[3], y1[3], m),
                    encode4(y0[4], y1[4], y0[5], y1[5], m), encode4(y0[6], y1[6], y0[7], y1[7], m)};
    }
}

__device__ __forceinline__ uint32_t top_of(const float (&y0)[8], const float (&y1)[8])
{
    uint32_t u = 0u;
#pragma unroll
    for (int t = 0; t < 8; ++t) u = max(u, max(finite_bits(y0[t]), finite_bits(y1[t])));
    return u;
}

__device__ __forceinline__ uint4 rescale16(uint4 v, float m)
{
    return (uint4){rescale4(v.x, m), rescale4(v.y, m), rescale4(v.z, m), rescale4(v.w, m)};
}

constexpr float QNAN = __builtin_nanf("");

// One decode step's rows: D / 16 threads to a (row, head).  What does not wait
// for the position (the values, the row's flags) is loaded first: one short
// chain of latencies is the whole time, 5 us for 162 rows of 32 + 8 + 8 heads
// (3.7 MB) as for one.
template <int D, bool VEC, bool E4>
__global__ __launch_bounds__(256) void k_append_rows(QkvRows in, int rows, const uint8_t *__restrict__ valid,
                                                     const int32_t *__restrict__ pos, int nq, int nkv, RopeArgs rope,
                                                     uint16_t *__restrict__ q, long long ldq, CacheView cv, CacheLayer cl)
{
    constexpr int LPT = D / 16;
    const int unit = (blockIdx.x * 256 + threadIdx.x) / LPT, j = threadIdx.x % LPT;
    const int nh = nq + 2 * nkv, r = unit / nh, h = unit % nh;
    if (r >= rows) return;
    const uint8_t live = valid != nullptr ? valid[r] : 1;
    const int t = pos[r];
    if (!live) return;                                // nothing of a padding row is read
    const Pairs<D, VEC> p(rope, j);
    const Raw raw = load_raw<D, VEC>(in, p, r, h);
    bool bad = t < 0 || t >= cv.cap;
    int page = 0;
    if (!bad && cv.kv.layout == 1) {
        page = page_of(cv, r, t);
        bad = page < 0;
    }
    Turn64 tu;
    const bool key = h >= nq && h < nq + nkv;
    if (h < nq + nkv) tu.init(rope, p, t);
    float x0[8], x1[8];
    to_pairs(raw, p, x0, x1);
    if (h < nq || (key && !E4)) {
        float c[8], s[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            c[i] = (float)tu.c[i];
            s[i] = (float)tu.s[i];
        }
        rotate(p, c, s, x0, x1);
    }
    if (h < nq) {
        if (bad)
#pragma unroll
            for (int i = 0; i < 8; ++i) x0[i] = x1[i] = QNAN;
        store_bf16(q + (size_t)r * ldq + (size_t)h * D, p, x0, x1);
        return;
    }
    if (bad) return;
    const int kvh = h - nq - (key ? 0 : nkv);
    const Place pl = place(cv, nkv, kvh, r, page, t);
    if constexpr (!E4) {
        store_bf16((uint16_t *)(key ? cl.k : cl.v) + pl.row * D, p, x0, x1);
        return;
    }
    if (key) rotate_exact(p, tu, x0, x1);
    uint8_t *codes = (uint8_t *)(key ? cl.k : cl.v) + pl.row * D;
    uint8_t *scale = (key ? cl.ks : cl.vs) + pl.blk;
    uint32_t top = top_of(x0, x1);
#pragma unroll
    for (int o = 1; o < LPT; o *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, o, LPT));
    const int kept = t & ((1 << cv.blk_shift) - 1);
    const int need = scale_exp(top), old = kept ? (int)*scale - 127 : need, e = max(old, need);
    store_codes(codes, p, x0, x1, e);
    if (old < e) {   // the block's earlier tokens move to the larger scale, four of them in flight
        const float m = e - old > 120 ? 0.f : exp2_int(old - e);
        for (int i = 1; i <= kept; i += 4) {
            uint4 v[4];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u <= kept) v[u] = *(const uint4 *)(codes - (size_t)(i + u) * D + 16 * j);
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u <= kept) *(uint4 *)(codes - (size_t)(i + u) * D + 16 * j) = rescale16(v[u], m);
        }
    }
    if (j == 0 && (kept == 0 || e != old)) *scale = (uint8_t)(e + 127);
}

// A prefill call's sequences.  Workgroup: one scale block of tokens of one
// sequence (x), a slice of the heads (y); thread (head group, token, j), so
// that a head group's wavefronts hold every new token of the block and agree
// on its scale through LDS, once per pair of key and value heads.  Threads of
// the block's earlier tokens move those to a scale that grew.  The query heads
// follow, four loads in flight to a thread.
template <int D, bool VEC, bool E4>
__global__ __launch_bounds__(512) void k_append_seqs(QkvRows in, SeqTable seq, int nq, int nkv, RopeArgs rope,
                                                     uint16_t *__restrict__ q, long long ldq, CacheView cv, CacheLayer cl)
{
    constexpr int LPT = D / 16;
    const int blk = 1 << cv.blk_shift, tid = threadIdx.x;
    const int gt = blk * LPT, groups = blockDim.x / gt;      // threads of a head group
    const int hg = tid / gt, tok = tid % gt / LPT, j = tid % LPT;
    const int i = seq_of(seq, blockIdx.x);
    const int start = seq.start[i], len = seq.len[i], slot = seq.slot[i];
    const int t0 = (start / blk + (int)blockIdx.x - seq.unit0[i]) * blk, t = t0 + tok;
    const bool fresh = t >= start && t - start < len;
    const long long row = seq.row0[i] + (long long)(t - start);
    int page = 0;
    bool bad = false;
    if (cv.kv.layout == 1) {
        page = page_of(cv, slot, t0);
        bad = page < 0;
    }
    const Pairs<D, VEC> p(rope, j);
    Turn64 tu;
    tu.init(rope, p, t);
    float c[8], s[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
        c[u] = (float)tu.c[u];
        s[u] = (float)tu.s[u];
    }
    const int ns = gridDim.y, sl = blockIdx.y;
    const int k_lo = (int)((long long)nkv * sl / ns), k_hi = (int)((long long)nkv * (sl + 1) / ns);
    if constexpr (!E4) {
        if (fresh && !bad)
            for (int h = k_lo + hg; h < k_hi; h += groups) {
                const Place pl = place(cv, nkv, h, slot, page, t);
                const Raw rk = load_raw<D, VEC>(in, p, row, nq + h), rv = load_raw<D, VEC>(in, p, row, nq + nkv + h);
                float x0[8], x1[8];
                to_pairs(rk, p, x0, x1);
                rotate(p, c, s, x0, x1);
                store_bf16((uint16_t *)cl.k + pl.row * D, p, x0, x1);
                to_pairs(rv, p, x0, x1);
                store_bf16((uint16_t *)cl.v + pl.row * D, p, x0, x1);
            }
    } else if (!bad) {                                // bad is uniform, as are the barriers
        __shared__ uint32_t tops[2][8][2];
        const int kept = max(0, start - t0);          // earlier tokens of the block
        const int wave = tid >> 6, gw = gt / 64;      // wavefronts of a head group
        const int per = (k_hi - k_lo + groups - 1) / groups;
        for (int it = 0; it < per; ++it) {
            const int h = k_lo + hg + it * groups;
            const bool on = h < k_hi;
            uint32_t tk = 0u, tv = 0u;
            float x0[8], x1[8], y0[8], y1[8];
            if (on && fresh) {
                const Raw rk = load_raw<D, VEC>(in, p, row, nq + h), rv = load_raw<D, VEC>(in, p, row, nq + nkv + h);
                to_pairs(rk, p, y0, y1);
                rotate_exact(p, tu, y0, y1);
                to_pairs(rv, p, x0, x1);
                tk = top_of(y0, y1);
                tv = top_of(x0, x1);
            }
#pragma unroll
            for (int o = 1; o < 64; o *= 2) {
                tk = max(tk, (uint32_t)__shfl_xor((int)tk, o, 64));
                tv = max(tv, (uint32_t)__shfl_xor((int)tv, o, 64));
            }
            if ((tid & 63) == 0) {
                tops[it & 1][wave][0] = tk;
                tops[it & 1][wave][1] = tv;
            }
            __syncthreads();                          // the other buffer's readers passed the last one
            for (int w = 0; w < gw; ++w) {
                tk = max(tk, tops[it & 1][hg * gw + w][0]);
                tv = max(tv, tops[it & 1][hg * gw + w][1]);
            }
            int ok = 0, ov = 0, ek = 0, ev = 0;
            const Place pl = place(cv, nkv, on ? h : k_lo, slot, page, t);
            if (on) {
                ek = scale_exp(tk);
                ev = scale_exp(tv);
                ok = kept ? (int)cl.ks[pl.blk] - 127 : ek;
                ov = kept ? (int)cl.vs[pl.blk] - 127 : ev;
                ek = max(ok, ek);
                ev = max(ov, ev);
                uint8_t *ck = (uint8_t *)cl.k + pl.row * D, *vk = (uint8_t *)cl.v + pl.row * D;
                if (fresh) {
                    store_codes(ck, p, y0, y1, ek);
                    store_codes(vk, p, x0, x1, ev);
                } else if (tok < kept) {
                    auto move = [&](uint8_t *at, int old, int e) {
                        if (old >= e) return;
                        const float m = e - old > 120 ? 0.f : exp2_int(old - e);
                        *(uint4 *)(at + 16 * j) = rescale16(*(const uint4 *)(at + 16 * j), m);
                    };
                    move(ck, ok, ek);
                    move(vk, ov, ev);
                }
            }
            if (kept) __syncthreads();                // every thread of a group has read the old scales (kept is uniform)
            if (on && tid % gt == 0) {
                cl.ks[pl.blk] = (uint8_t)(ek + 127);
                cl.vs[pl.blk] = (uint8_t)(ev + 127);
            }
        }
    }
    // query heads of this slice
    if (!fresh) return;
    const int q_lo = (int)((long long)nq * sl / ns), q_hi = (int)((long long)nq * (sl + 1) / ns);
    constexpr int PF = 4;
    for (int h = q_lo + hg; h < q_hi; h += PF * groups) {
        Raw raw[PF];
#pragma unroll
        for (int u = 0; u < PF; ++u)
            if (h + u * groups < q_hi) raw[u] = load_raw<D, VEC>(in, p, row, h + u * groups);
#pragma unroll
        for (int u = 0; u < PF; ++u) {
            if (h + u * groups >= q_hi) break;
            float x0[8], x1[8];
            to_pairs(raw[u], p, x0, x1);
            rotate(p, c, s, x0, x1);
            if (bad)
#pragma unroll
                for (int v = 0; v < 8; ++v) x0[v] = x1[v] = QNAN;
            store_bf16(q + (size_t)row * ldq + (size_t)(h + u * groups) * D, p, x0, x1);
        }
    }
}

// ---------------------------------------------------------------------------
// Decode attention, split over the tokens.  A row of n tokens has ceil(n /
// chunk) splits, a function of its own length, and merges them in order.
//
// Workgroup (kv head, split, row), four wavefronts.  The chunk is walked in
// steps of 128 tokens whose key and value rows go global -> LDS by direct
// 16-byte loads that cover whole rows; a wavefront takes 32 tokens of a step,
// reads its operands into registers, and the next step's loads go out before
// it computes.  Codes become bf16 in registers, with their scale, exactly
// (v_cvt_scalef32_pk_bf16_fp8).
//  * S^T = K q^T on 16x16x32 MFMA, two tiles of 16 tokens, the group's query
//    heads in the columns; tile T's row m is token 8 (m / 4) + 4 T + m % 4,
//    so lane l ends with head l % 16's scores of tokens 8 (l / 16) .. + 7;
//  * the running maximum and sum of a softmax, per lane over its own tokens;
//  * O += P V: those eight weights are the lane's A operand, in two bf16 halves
//    hi + lo (about 16 bits), and one transposed 8-bit read gives the B operand,
//    eight tokens of a dimension.
// Tokens past the length: loads repeat the last token, scores are masked by
// selection, value codes are cleared.
//
// Bound by reading the cache: 162 rows of 512 to 4096 tokens (8 kv heads of 128)
// take 147 us, 5.2 TB/s, which is what a large copy reaches, though reads alone can
// be faster (the bf16 kernel takes these rows at 5.8); 32 paged rows of 1024 to
// 32768 tokens 127 us, 4.7 TB/s, where the longest row's last splits run alone.
// Three workgroups of 33 KB to a CU keep enough loads in flight; the weights' bf16
// halves hi + lo cost matrix instructions that the loads leave idle, where one bf16
// weight would lose 8 bits.
// ---------------------------------------------------------------------------

// Transposed LDS read of bytes (ds_read_b64_tr_b8): in each group of 16 lanes,
// lane a + 2 q points at eight bytes (row q, columns 8 a .. 8 a + 7) and lane i
// receives column i of rows 0 .. 7.
__device__ __forceinline__ uint2 lds_read_tr8(const void *lds_ptr)
{
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
    const i32x2 v = __builtin_amdgcn_ds_read_tr8_b64_v2i32(
        (lds_i32x2 *)(const __attribute__((address_space(3))) void *)lds_ptr);
    return __builtin_bit_cast(uint2, v);
}

// Eight codes times a power of two, in bf16: exact.
__device__ __forceinline__ bf16x8 codes_bf16(uint2 w, float scale)
{
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    bf16x2_t h[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, scale, false),
                     __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.x, scale, true),
                     __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, scale, false),
                     __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w.y, scale, true)};
    return __builtin_bit_cast(bf16x8, h);
}

// LDS: 16-byte unit c of token t's row (KB units) at t KB + (c ^ swizzle(t)).
// A key read's half wavefront takes one unit of the 16 tokens 8 a + 4 T + b (a,
// b < 4), a value read's one unit of 16 consecutive tokens: each lands on the
// 16 groups of four banks once.
template <int KB>
__device__ __forceinline__ int key_swz(int t)
{
    if constexpr (KB == 8) return (((t >> 3) & 3) << 1) | ((t >> 1) & 1);
    else return (t >> 3) & 3;
}
template <int KB>
__device__ __forceinline__ int val_swz(int t)
{
    if constexpr (KB == 8) return (t >> 1) & 7;
    else return (t >> 2) & 3;
}

// Tokens that row r attends to; -1 for a length outside the launch.
__device__ __forceinline__ int row_len(const uint8_t *valid, const int32_t *lens, int plus_one, int max_len, int r)
{
    const int n = lens[r];                            // in flight together with the flag
    const bool live = valid == nullptr || valid[r] != 0;
    return !live ? 0 : n < 0 || n > max_len - plus_one ? -1 : n + plus_one;
}

template <int D, bool PAGED>
__global__ __launch_bounds__(256, 3) void k_attn8_split(const uint16_t *__restrict__ q, long long ldq,
                                                     const uint8_t *__restrict__ valid, const int32_t *__restrict__ lens,
                                                     int plus_one, int G, int nkv, CacheView cv, CacheLayer cl, int chunk,
                                                     int max_splits, int max_len, float *__restrict__ ws,
                                                     const int32_t *__restrict__ row_order, uint16_t *__restrict__ out,
                                                     long long ldo)
{
    constexpr int ET = D / 16, KB = D / 16, STEP = 128, KU = STEP * KB, OPS = KU / 256;
    static_assert(4 * 16 * D * 4 <= 2 * KU * 16, "wavefront partials fit the tile");
    __shared__ __attribute__((aligned(16))) uint4 tile[2 * KU];       // keys, then values
    __shared__ float cm[4][16], cl_[4][16];
    __shared__ int32_t pgs[2][64];                    // paged: a step's pages, fetched one step ahead
    __shared__ int lost;
    typedef __attribute__((address_space(3))) void lds_void;

    const int kvh = blockIdx.x, split = blockIdx.y, r = row_order != nullptr ? row_order[blockIdx.z] : blockIdx.z;
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, hl = lane & 15, kg = lane >> 4;
    const int n = row_len(valid, lens, plus_one, max_len, r);
    const int t0 = split * chunk;
    // out: rows have one split, whose result is the row's
    uint16_t *orow = out == nullptr ? nullptr : out + (size_t)r * ldo + (size_t)kvh * G * D;
    if (t0 >= n) {
        if (orow != nullptr)
            for (int i = tid; i < G * D; i += 256) orow[i] = n < 0 ? (uint16_t)0x7fc0 : (uint16_t)0;
        return;
    }
    const int t1 = min(n, t0 + chunk), kmax = t1 - 1;
    if (tid == 0) lost = 0;

    // q^T (B operand of the scores): lane l supplies head l % 16, dims 32 kk + 8 (l / 16) .. + 7
    bf16x8 qf[D / 32];
    {
        const uint16_t *qr = q + (size_t)r * ldq + ((size_t)kvh * G + hl) * D + kg * 8;
#pragma unroll
        for (int kk = 0; kk < D / 32; ++kk) {
            uint4 v = {0u, 0u, 0u, 0u};
            if (hl < G) v = *(const uint4 *)(qr + 32 * kk);
            qf[kk] = __builtin_bit_cast(bf16x8, v);
        }
    }
    const float scale = 1.0f / sqrtf((float)D);
    f32x4 oacc[ET];
#pragma unroll
    for (int et = 0; et < ET; ++et) oacc[et] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float mrun = -INFINITY, lrun = 0.f;

    const int ps = PAGED ? cv.kv.page_size : 1, last_page = kmax / ps, bs = cv.blk_shift;
    const uint8_t *kc = (const uint8_t *)cl.k, *vc = (const uint8_t *)cl.v;
    const size_t head0 = ((size_t)r * nkv + kvh) * cv.kv.max_seq_len;                 // contiguous: the head's first row
    const size_t blk0 = ((size_t)r * nkv + kvh) * (cv.kv.max_seq_len >> bs);
    bool bad = false;
    auto fetch_pages = [&](int tb0, int buf) {        // wavefront 0, lane l: page tb0 / ps + l (clamped)
        if (PAGED && wave == 0) {
            const int pi = min(tb0 / ps + lane, last_page);
            __builtin_amdgcn_global_load_lds((const void *)(cv.kv.page_table + (size_t)r * cv.kv.max_pages_per_seq + pi),
                                             (lds_void *)&pgs[buf][0], 4, 0, 0);
        }
    };
    // paged: row of the real token that stands `in` tokens behind the first of
    // the step's first page, and its scale block
    auto at = [&](int in, int buf) -> Place {
        const int i = (int)(((float)in + 0.5f) * cv.page_inv);            // in / ps: exact below 2^21
        int page = pgs[buf][i];
        if ((unsigned)page >= (unsigned)cv.num_pages) {
            bad = true;
            page = 0;
        }
        in -= i * ps;
        const size_t head = (size_t)page * nkv + kvh;
        return {head * ps + in, head * (ps >> bs) + (in >> bs)};
    };
    uint32_t kb_next = 0, vb_next = 0;                // scale bytes of the lane's key rows and of its value tokens
    auto issue = [&](int tb0, int buf) {
        uint4 *base = tile + wave * 64;
        const int top = kmax - tb0, in0 = PAGED ? tb0 % ps : 0;           // last real token of the step; its place in a page
        const uint8_t *kb = kc + (head0 + tb0) * D, *vb = vc + (head0 + tb0) * D;   // contiguous
#pragma unroll
        for (int j = 0; j < OPS; ++j) {
            const int u = j * 256 + tid, tk = u / KB, c = u % KB, t = min(tk, top);
            const uint32_t kc16 = 16 * (c ^ key_swz<KB>(tk)), vc16 = 16 * (c ^ val_swz<KB>(tk));
            const uint8_t *ksrc, *vsrc;
            if constexpr (PAGED) {
                const size_t off = at(in0 + t, buf).row * D;
                ksrc = kc + off + kc16;
                vsrc = vc + off + vc16;
            } else {
                ksrc = kb + (uint32_t)(t * D + kc16);
                vsrc = vb + (uint32_t)(t * D + vc16);
            }
            __builtin_amdgcn_global_load_lds((const void *)ksrc, (lds_void *)(base + j * 256), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((const void *)vsrc, (lds_void *)(base + KU + j * 256), 16, 0, 0);
        }
        const int tk = min(32 * wave + 8 * (hl >> 2), top), tv = min(32 * wave + 8 * kg, top);
        if constexpr (PAGED) {
            kb_next = cl.ks[at(in0 + tk, buf).blk];
            vb_next = cl.vs[at(in0 + tv, buf).blk];
        } else {
            kb_next = cl.ks[blk0 + (uint32_t)((tb0 + tk) >> bs)];
            vb_next = cl.vs[blk0 + (uint32_t)((tb0 + tv) >> bs)];
        }
    };

    const int nsteps = (t1 - t0 + STEP - 1) / STEP;
    fetch_pages(t0, 0);
    __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
    lds_barrier();
    issue(t0, 0);
    if (nsteps > 1) fetch_pages(t0 + STEP, 1);
    for (int i = 0; i < nsteps; ++i) {
        const int tb0 = t0 + STEP * i, tb = tb0 + 32 * wave;
        __builtin_amdgcn_s_waitcnt(vmcnt_imm(0));
        lds_barrier();                                // the step (and the next step's pages) are in LDS
        const bool active = tb < t1;                  // wave-uniform: some token of the wavefront's 32 is real
        const float ksc = __uint_as_float(kb_next << 23), vsc = __uint_as_float(vb_next << 23);
        uint2 kr[2][D / 32], vr[ET];
        if (active) {
#pragma unroll
            for (int T = 0; T < 2; ++T) {
                const int tl = 32 * wave + 8 * (hl >> 2) + 4 * T + (hl & 3);
#pragma unroll
                for (int kk = 0; kk < D / 32; ++kk)
                    kr[T][kk] = *(const uint2 *)((const char *)(tile + tl * KB + ((2 * kk + (kg >> 1)) ^ key_swz<KB>(tl))) +
                                                 8 * (kg & 1));
            }
            const int tv = 32 * wave + 8 * kg + (hl >> 1);
#pragma unroll
            for (int et = 0; et < ET; ++et)
                vr[et] = lds_read_tr8((const char *)(tile + KU + tv * KB + (et ^ val_swz<KB>(tv))) + 8 * (hl & 1));
            const int nv = t1 - (tb + 8 * kg);        // the lane's real tokens, of eight
            if (nv < 8) {
                const unsigned long long keep = nv <= 0 ? 0ull : (1ull << (8 * nv)) - 1;
#pragma unroll
                for (int et = 0; et < ET; ++et) {
                    vr[et].x &= (uint32_t)keep;
                    vr[et].y &= (uint32_t)(keep >> 32);
                }
            }
        }
        __builtin_amdgcn_s_waitcnt(0xC07F);           // lgkmcnt(0): this wavefront's LDS reads are done
        lds_barrier();                                // the tile is free: the next step's loads go out
        if (i + 1 < nsteps) {
            issue(tb0 + STEP, (i + 1) & 1);
            if (i + 2 < nsteps) fetch_pages(tb0 + 2 * STEP, i & 1);
        }
        if (!active) continue;
        f32x4 st[2];
#pragma unroll
        for (int T = 0; T < 2; ++T) {
            st[T] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < D / 32; ++kk)
                st[T] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(codes_bf16(kr[T][kk], ksc), qf[kk], st[T], 0, 0, 0);
        }
        float mt = -INFINITY;
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float sv = (tb + 8 * kg + 4 * T + e < t1) ? st[T][e] * scale : -INFINITY;
                st[T][e] = sv;
                mt = fmaxf(mt, sv);
            }
        mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
        mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
        const float mnew = fmaxf(mrun, mt);           // every 32-token block has a real token (NaN scores aside)
        const float alpha = mnew == mrun ? 1.f : __expf(mrun - mnew);   // also where both are -inf (NaN scores only)
        const float moff = mnew == -INFINITY ? 0.f : mnew;
        uint32_t hi[4], lo[4];
        float ls = 0.f;
#pragma unroll
        for (int T = 0; T < 2; ++T)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const float a = __expf(st[T][e] - moff), b = __expf(st[T][e + 1] - moff);
                ls += a;
                ls += b;
                const uint32_t w = f2bf2(a, b);
                hi[2 * T + e / 2] = w;
                lo[2 * T + e / 2] = f2bf2(a - __uint_as_float(w << 16), b - __uint_as_float(w & 0xffff0000u));
            }
        lrun = lrun * alpha + ls;
        mrun = mnew;
        if (__ballot(alpha != 1.f)) {                 // lane l's accumulators belong to heads 4 (l / 16) + e
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float ae = __shfl(alpha, 4 * kg + e, 64);
#pragma unroll
                for (int et = 0; et < ET; ++et) oacc[et][e] *= ae;
            }
        }
        const bf16x8 ph = __builtin_bit_cast(bf16x8, hi), pl = __builtin_bit_cast(bf16x8, lo);
#pragma unroll
        for (int et = 0; et < ET; ++et) {
            const bf16x8 vf = codes_bf16(vr[et], vsc);
            oacc[et] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ph, vf, oacc[et], 0, 0, 0);
            oacc[et] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pl, vf, oacc[et], 0, 0, 0);
        }
    }
    lrun += __shfl_xor(lrun, 16, 64);
    lrun += __shfl_xor(lrun, 32, 64);

    // the four wavefronts in order, through the idle tile
    lds_barrier();
    if (bad) lost = 1;
    float *ca = reinterpret_cast<float *>(tile);      // [4][G D]
    if (lane < 16) {
        cm[wave][lane] = mrun;
        cl_[wave][lane] = lrun;
    }
#pragma unroll
    for (int et = 0; et < ET; ++et)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int g = 4 * kg + e;
            if (g < G) ca[(wave * G + g) * D + 16 * et + hl] = oacc[et][e];
        }
    __syncthreads();
    float *o = ws + (((size_t)r * nkv + kvh) * max_splits + split) * (G * (D + 2));
    for (int idx = tid; idx < G * D; idx += 256) {
        const int g = idx / D;
        float M = cm[0][g];
#pragma unroll
        for (int w = 1; w < 4; ++w) M = fmaxf(M, cm[w][g]);
        const float off = M == -INFINITY ? 0.f : M;   // NaN scores only
        float L = 0.f, A = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __expf(cm[w][g] - off);   // a wavefront without tokens: exp(-inf) = 0
            L += cl_[w][g] * f;
            A += ca[w * G * D + idx] * f;
        }
        if (orow != nullptr) {
            orow[idx] = f2bf(lost ? QNAN : A / L);
            continue;
        }
        o[2 * G + idx] = A;
        if (idx % D == 0) {
            o[g] = lost ? QNAN : M;
            o[G + g] = L;
        }
    }
}

// Merge: 256 / D query heads of one row to a workgroup, one thread to a
// dimension; a head's first wavefront turns its splits' maxima into weights and
// sums, every thread folds its dimension over the splits in order.  Latencies in
// a row: 5.4 us for one row, 7.7 for 256 of 32 heads.
template <int D>
__global__ __launch_bounds__(256) void k_attn8_merge(const float *__restrict__ ws, const uint8_t *__restrict__ valid,
                                                     const int32_t *__restrict__ lens, int plus_one, int nq, int nkv,
                                                     int chunk, int max_splits, int max_len, uint16_t *__restrict__ out,
                                                     long long ldo)
{
    constexpr int HB = 256 / D, PF = 16;              // splits whose values are in flight at once
    extern __shared__ float fs[];                     // [HB][2][max_splits] maxima, then weights; sums
    __shared__ float total[HB];
    const int hb = threadIdx.x / D, dd = threadIdx.x % D, lane = threadIdx.x & 63;
    const int h = blockIdx.x * HB + hb, r = blockIdx.y, G = nq / nkv;
    const int n = row_len(valid, lens, plus_one, max_len, r);
    uint16_t *o = out + (size_t)r * ldo + (size_t)h * D + dd;
    if (n <= 0) {
        if (h < nq) *o = n < 0 ? (uint16_t)0x7fc0 : (uint16_t)0;
        return;
    }
    const int ns = (n + chunk - 1) / chunk, kvh = min(h, nq - 1) / G, g = min(h, nq - 1) % G;
    const size_t stride = (size_t)G * (D + 2);
    const float *base = ws + ((size_t)r * nkv + kvh) * max_splits * stride;
    const float *a = base + 2 * G + g * D + dd;
    float v[PF];
#pragma unroll
    for (int u = 0; u < PF; ++u) v[u] = u < ns ? a[u * stride] : 0.f;
    float *f = fs + hb * 2 * max_splits, *fl = f + max_splits;
    if (dd < 64) {
        float M = -INFINITY, L = 0.f;
        for (int sp = lane; sp < ns; sp += 64) {      // both loads at once: the sums wait for no maximum
            const float m = base[sp * stride + g], l = base[sp * stride + G + g];
            f[sp] = m;
            fl[sp] = l;
            M = fmaxf(M, m);
        }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) M = fmaxf(M, __shfl_xor(M, off, 64));
        const float off_ = M == -INFINITY ? 0.f : M;
        for (int sp = lane; sp < ns; sp += 64) {
            const float w = __expf(f[sp] - off_);
            f[sp] = w;
            L += fl[sp] * w;
        }
#pragma unroll
        for (int off = 32; off >= 1; off >>= 1) L += __shfl_xor(L, off, 64);
        if (lane == 0) total[hb] = L;
    }
    __syncthreads();
    float acc = 0.f;
    for (int sp = 0; sp < ns; sp += PF) {
        if (sp > 0)
#pragma unroll
            for (int u = 0; u < PF; ++u) v[u] = sp + u < ns ? a[(size_t)(sp + u) * stride] : 0.f;
#pragma unroll
        for (int u = 0; u < PF; ++u)
            if (sp + u < ns) acc += v[u] * f[sp + u];
    }
    if (h < nq) *o = f2bf(acc / total[hb]);
}

// ---------------------------------------------------------------------------
// Prefill attention, causal: keys in tiles of 64 in order, online softmax in
// base 2.  A sequence of few rows behind many tokens is split over its tiles
// (attn8_seq_splits, a function of the sequence alone): each split's result and
// its maximum and sum go to the workspace, and k_attn8_join weighs them in order.
//
// A unit is 32 queries of one query head; a workgroup of NW = 4 or 8 wavefronts
// takes NW units of one kv head in [query block][head] order, latest first, one
// to a wavefront, on shared key and value tiles.  A tile's codes are read into
// registers one tile ahead, and become 16-bit LDS rows once for all its
// wavefronts: keys in bf16 with their scale (exact), values in fp16 under the
// largest scale of the tile (exact), which goes to the weights: these are fp16 of
// weight times scale, so that what they lose is small beside the largest such
// product, wherever the large scores and the large values stand; and they keep
// 11 bits where bf16 would keep 8.
//  * S^T = K Q^T on v_mfma_f32_32x32x16_bf16, two 32 x 32 tiles, key rows
//    permuted (pf_key_of_row) so that lane l ends with eight consecutive keys
//    16 s + 8 (l / 32) .. + 7 of each step s of query l % 32: the P^T operand of
//  * O^T += V^T P^T on v_mfma_f32_32x32x16_f16, V^T by transposed LDS reads.
// Weights are 2^(s + b - ref + P_UP), b the tile's scale byte, where ref follows the
// running maximum of s + b once that is more than P_LAG above it: at most 2^15;
// what is 2^-22 of the largest is still a normal number, what is 2^-33 of it
// becomes zero.  The row sum (fp32, of the weights before they are rounded) takes
// the scale out again, and the output is their quotient.  Where the groups of 16
// tokens of a tile have scales more than 2^B_NEAR apart, each group's scale goes
// to its own weights (`far`).  Bytes are within B_LOW .. B_HIGH (2^-60 .. 2^30; lower
// ones count as B_LOW, with their codes scaled down instead), so that no weight that
// the sum needs falls out of fp32.
//
// A wavefront's load takes rows of one 16-token group of a tile, so its page and
// row base are scalars and the loop has no vector address arithmetic.  Future keys
// and those past the sequence are masked by selection, value codes past it are
// cleared.  A NaN among the values would reach queries that do not see it
// (0 NaN), scales outside that range would lose weights or codes, and a page that
// is none is taken for zeros: a wavefront whose sums hold a NaN, or whose keys reach
// such a group, does its rows again one by one (attend_row); a split notes a NaN
// maximum for such a row and the join does it.
//
// Bound by the matrix units and the softmax's arithmetic of one wavefront in turn:
// a tile's 32 products are 1024 cycles of each SIMD's matrix unit, and with two
// wavefronts to a SIMD a tile takes 1.9 us, about 4500 cycles for 2048 of products.
// 2048 rows of 32 heads behind 14336 tokens: 539 to 554 us, 0.93 to 0.96 PFLOP/s
// (a large bf16 matrix product reaches 1.25); 615 where every tile is `far`.
// Products of the next tile between the steps of this tile's softmax (588 us) and
// halves of the wavefronts half a tile apart (5% longer) came out slower: two
// wavefronts already fill each other's gaps, and no reads of keys or values (2%
// each) or exponentials (5%) bound it alone.  Heads of 64 are held to the registers
// of three wavefronts to a SIMD (6000 paged tokens: 218 us, 259 with two).
// ---------------------------------------------------------------------------
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
constexpr int P_UP = 8, P_LAG = 7;
constexpr int B_LOW = 67, B_HIGH = 157, B_NEAR = 4;
constexpr int MOST_SPLITS = 64;

// Tiles of each of ns splits of Lk keys.
__host__ __device__ __forceinline__ int tiles_of_split(int Lk, int ns)
{
    return ((Lk + 63) / 64 + ns - 1) / ns;
}

// Sixteen codes times a power of two, as 32 bytes of bf16 or fp16.
template <bool F16>
__device__ __forceinline__ void codes_16(uint4 w, float scale, uint4 &lo, uint4 &hi)
{
    uint32_t o[8];
    const uint32_t in[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (F16) {
            o[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(in[i], scale, false));
            o[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(in[i], scale, true));
        } else {
            o[2 * i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(in[i], scale, false));
            o[2 * i + 1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(in[i], scale, true));
        }
    }
    lo = (uint4){o[0], o[1], o[2], o[3]};
    hi = (uint4){o[4], o[5], o[6], o[7]};
}

// One query row over its first n keys, by one wavefront in fp32: 64 keys at a
// time, a key to a lane for the scores, then D / 64 dimensions to a lane.  For
// rows that see a NaN, a scale out of the other pass's range or a page that is none
// (the whole row becomes NaN).  Slow: 6000 tokens of 32 heads whose first value
// holds a NaN take 97 ms (0.33 without it), 600 take 4.3.
template <int D>
__device__ __forceinline__ void attend_row(const uint16_t *q, int n, int kvh, int nkv, int slot, const CacheView &cv,
                                        const CacheLayer &cl, uint16_t *out)
{
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63;
    const float scale = 1.0f / sqrtf((float)D);
    float m = -INFINITY, l = 0.f, acc[E] = {};
    bool lost = false;
    for (int b = 0; b < n; b += 64) {
        const int t = min(b + lane, n - 1);
        int page = 0;
        if (cv.kv.layout == 1) page = page_of(cv, slot, t);
        lost |= page < 0;
        const Place pl = place(cv, nkv, kvh, slot, max(page, 0), t);
        const uint8_t *k = (const uint8_t *)cl.k + pl.row * D;
        float sc = 0.f;
#pragma unroll 1
        for (int i = 0; i < D; i += 4) {
            const uint32_t w = *(const uint32_t *)(k + i);
            sc += bf2f(q[i]) * __builtin_amdgcn_cvt_f32_fp8(w, 0);
            sc += bf2f(q[i + 1]) * __builtin_amdgcn_cvt_f32_fp8(w, 1);
            sc += bf2f(q[i + 2]) * __builtin_amdgcn_cvt_f32_fp8(w, 2);
            sc += bf2f(q[i + 3]) * __builtin_amdgcn_cvt_f32_fp8(w, 3);
        }
        sc *= __uint_as_float((uint32_t)cl.ks[pl.blk] << 23) * scale;
        const bool on = b + lane < n;
        float mt = on ? sc : -INFINITY;
        for (int o = 32; o; o >>= 1) mt = fmaxf(mt, __shfl_xor(mt, o, 64));
        const float mn = fmaxf(m, mt), off = mn == -INFINITY ? 0.f : mn;
        const float al = __expf(m - off), pe = on ? __expf(sc - off) : 0.f;
        float sum = pe;
        for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o, 64);
        l = l * al + sum;
        m = mn;
        for (int e = 0; e < E; ++e) acc[e] *= al;
        const float vsc = __uint_as_float((uint32_t)cl.vs[pl.blk] << 23);
        for (int i = 0; i < min(64, n - b); ++i) {
            const float w = __shfl(pe, i, 64), vs = __shfl(vsc, i, 64);
            const size_t row = __shfl((unsigned long long)pl.row, i, 64);
            for (int e = 0; e < E; ++e)
                acc[e] += w * (__builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)cl.v)[row * D + E * lane + e], 0) * vs);
        }
    }
    lost = __ballot(lost) != 0ull;
    for (int e = 0; e < E; ++e) out[E * lane + e] = f2bf(lost ? QNAN : acc[e] / l);
}

// LDS units of a value tile: vtile_swz, and odd rows' units in the other of two
// neighbours, so that the 16 lanes of a store phase (every second unit of two
// rows) land on different banks; a transposed read takes both neighbours.
template <int KCH>
__device__ __forceinline__ int val16_swz(int t) { return vtile_swz<KCH>(t) ^ (t & 1); }

// 256 + b of a byte b, by its bits: a scalar stays one
__device__ __forceinline__ float byte_256(int b) { return __uint_as_float(0x43800000u | (uint32_t)b << 15); }

// Floats that a split leaves of a unit: its rows' results, [D / 4][32 rows][4],
// then their maxima (log2) and sums, [32][2].
template <int D>
constexpr int PART = 32 * D + 64;

template <int D, bool PAGED, int NW>
__global__ __launch_bounds__(64 * NW, D == 64 ? 3 : 2) void k_attn8_prefill(const uint16_t *__restrict__ q, long long ldq, SeqTable seq,
                                                              SplitTable sp, int G, int nkv, CacheView cv, CacheLayer cl,
                                                              uint16_t *__restrict__ out, long long ldo,
                                                              float *__restrict__ ws)
{
    constexpr int QB = 32, BKT = 64;                  // queries of a unit; keys of a tile
    constexpr int DT = D / 32, KS = D / 16, KCH = D / 8;
    constexpr int UNITS = BKT * KCH;                  // 16-byte units of a tile's 16-bit keys, or values
    constexpr int OPITCH = D + 8;
    constexpr int LDS_UNITS = 4 * UNITS > NW * QB * OPITCH / 8 ? 4 * UNITS : NW * QB * OPITCH / 8;
    __shared__ __attribute__((aligned(16))) uint4 ring[LDS_UNITS];    // two key tiles, two value tiles; the output
    __shared__ int redo;

    const int kvh = blockIdx.x % nkv;
    const int si = seq_of(seq, blockIdx.x / nkv), in_seq = (int)(blockIdx.x / nkv) - seq.unit0[si];
    const int ns = sp.splits[si];
    const int grp = ns == 1 ? in_seq : in_seq / ns, split = in_seq - grp * ns;
    const int n = seq.len[si], p0 = seq.start[si], slot = seq.slot[si], Lk = p0 + n;
    q += (size_t)seq.row0[si] * ldq;
    out += (size_t)seq.row0[si] * ldo;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int r32 = lane & 31, h = lane >> 5;
    const int units = (n + QB - 1) / QB * G;
    const int u = units - 1 - (grp * NW + wave);
    const bool active = u >= 0;
    const int qb = active ? u / G : 0, g = active ? u % G : 0, hq = kvh * G + g, q0 = qb * QB;
    const int wg_last_q = p0 + min(n, ((units - 1 - grp * NW) / G + 1) * QB) - 1;
    const int my_last_q = active ? p0 + min(n, q0 + QB) - 1 : -1;
    const int per = ns == 1 ? INT32_MAX : tiles_of_split(Lk, ns);
    const int tile0 = ns == 1 ? 0 : split * per;      // a split's tiles: tile0 .. ntiles - 1
    const int ntiles = __builtin_amdgcn_readfirstlane(min(wg_last_q / BKT + 1, ns == 1 ? INT32_MAX : tile0 + per));
    if (tile0 >= ntiles) return;                      // all of the split is in the workgroup's future

    // Loads: R passes over a tile's rows, in each of which a thread takes 16-byte
    // unit c of row `row` + r ROWS of keys and values, in 16-token group sub + r
    // ROWS / 16.
    constexpr int KB = D / 16, R = BKT * KB / (64 * NW), ROWS = BKT / R;
    static_assert(R * 64 * NW == BKT * KB, "the threads cover a tile's units");
    const int row = tid / KB, c = tid % KB, sub = wave * (64 / KB) / 16;
    const int ps = PAGED ? cv.kv.page_size : 0, bs = cv.blk_shift;
    const int32_t *pt = PAGED ? cv.kv.page_table + (size_t)slot * cv.kv.max_pages_per_seq : nullptr;
    const size_t head0 = ((size_t)slot * nkv + kvh) * cv.kv.max_seq_len;
    const size_t blk0 = ((size_t)slot * nkv + kvh) * (cv.kv.max_seq_len >> bs);
    const uint32_t off = (uint32_t)((row & 15) * D + 16 * c);      // in the group's rows
    // The next tile to load: its groups start at tokens t + 16 j; paged, page
    // idx and row `in` of the wavefront's groups, and of the group whose value
    // scale this lane loads (lane & 3).
    int t = BKT * tile0, idx[R], in[R], l_idx = 0, l_in = 16 * (lane & 3);
    int page[R], l_page = 0;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        idx[r] = PAGED ? t / ps : 0;
        in[r] = (PAGED ? t % ps : 0) + 16 * sub + ROWS * r;
        page[r] = 0;
    }
    if constexpr (PAGED) {
        l_idx = t / ps;
        l_in += t % ps;
    }
    // Rows from here on are done again: the first group that this wavefront found
    // on a page that is none, or whose scale no row can hold beside the others.
    int redo_from = INT32_MAX;
    auto fetch_pages = [&]() {
        if constexpr (PAGED) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                while (in[r] >= ps) {
                    in[r] -= ps;
                    ++idx[r];
                }
                page[r] = 0;
                if (t + 16 * sub + ROWS * r < Lk) page[r] = pt[idx[r]];
            }
            const int step = (int)(((float)l_in + 0.5f) * cv.page_inv);   // l_in < page_size + 64: exact
            l_idx += step;
            l_in -= step * ps;
            l_page = 0;
            if (t + 16 * (lane & 3) < Lk) l_page = pt[l_idx];
        }
    };
    uint4 kraw[R], vraw[R];
    // scale bytes: of the wavefront's groups' keys, of group lane & 3's values (past
    // the sequence or on a page that is none: of a group before)
    uint32_t kb[R] = {}, vb = 0;
    auto load = [&]() {
        size_t vblk;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int t16 = t + 16 * sub + ROWS * r;
            kraw[r] = vraw[r] = (uint4){0u, 0u, 0u, 0u};
            size_t base, kblk;
            bool real = t16 < Lk;                     // the whole group stands in the slot
            if constexpr (PAGED) {
                const int pg = __builtin_amdgcn_readfirstlane(page[r]);
                if ((unsigned)pg >= (unsigned)cv.num_pages) {
                    redo_from = min(redo_from, t16);
                    real = false;
                }
                const size_t head = (size_t)pg * nkv + kvh;
                base = head * ps + in[r];
                kblk = head * (ps >> bs) + (in[r] >> bs);
                in[r] += BKT;
            } else {
                base = head0 + t16;
                kblk = blk0 + (t16 >> bs);
            }
            if (real) {
                kraw[r] = *(const uint4 *)((const uint8_t *)cl.k + base * D + off);
                kb[r] = cl.ks[kblk];
                vraw[r] = *(const uint4 *)((const uint8_t *)cl.v + base * D + off);
            }
        }
        bool in_seq16 = t + 16 * (lane & 3) < Lk;
        if constexpr (PAGED) {
            in_seq16 &= (unsigned)l_page < (unsigned)cv.num_pages;
            vblk = ((size_t)l_page * nkv + kvh) * (ps >> bs) + (l_in >> bs);
            l_in += BKT;
        } else {
            vblk = blk0 + ((t + 16 * (lane & 3)) >> bs);
        }
        if (in_seq16) vb = cl.vs[vblk];
        t += BKT;
    };
    // The loaded tile, from key k0, to LDS buffer b; sc: the scales of its values.
    struct Scales {
        int top, g[4];                                // bytes; top is at least B_LOW
        bool far;
    };
    auto store = [&](int k0, int b, Scales &sc) {
        const int v0 = __builtin_amdgcn_readlane(vb, 0), v1 = __builtin_amdgcn_readlane(vb, 1);
        const int v2 = __builtin_amdgcn_readlane(vb, 2), v3 = __builtin_amdgcn_readlane(vb, 3);
        sc.top = max(max(max(v0, v1), max(v2, v3)), B_LOW);
        sc.g[0] = v0;
        sc.g[1] = v1;
        sc.g[2] = v2;
        sc.g[3] = v3;
        sc.far = __ballot(max((int)vb, B_LOW) + B_NEAR < sc.top) != 0ull;
        if (sc.top > B_HIGH) redo_from = min(redo_from, k0);
        uint4 *K = ring + b * UNITS, *V = ring + (2 + b) * UNITS;
        uint4 lo, hi;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int rw = row + ROWS * r;
            codes_16<false>(kraw[r], __uint_as_float(__builtin_amdgcn_readfirstlane(kb[r]) << 23), lo, hi);
            K[pf_swz<KCH>(rw, 2 * c)] = lo;
            K[pf_swz<KCH>(rw, 2 * c + 1)] = hi;
            uint4 w = vraw[r];
            if (k0 + BKT > Lk) {
                const uint32_t use = k0 + rw < Lk ? 0xffffffffu : 0u;
                w = (uint4){w.x & use, w.y & use, w.z & use, w.w & use};
            }
            const int grp16 = sub + ROWS / 16 * r;
            const int byte = grp16 == 0 ? v0 : grp16 == 1 ? v1 : grp16 == 2 ? v2 : v3;
            const int up = max(byte - (sc.far ? max(byte, B_LOW) : sc.top), -60);
            // 2^-9 times this is below 2^-24: codes lose bits (codes of zero excepted)
            if (up < -15 && __ballot(((w.x | w.y | w.z | w.w) & 0x7f7f7f7fu) != 0u)) redo_from = min(redo_from, k0 + 16 * grp16);
            codes_16<true>(w, exp2_int(up), lo, hi);
            V[rw * KCH + ((2 * c) ^ val16_swz<KCH>(rw))] = lo;
            V[rw * KCH + ((2 * c + 1) ^ val16_swz<KCH>(rw))] = hi;
        }
    };

    // Q^T operand: lane l supplies query q0 + l % 32, dims 16 s + 8 (l / 32) .. + 7
    bf16x8 qf[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
        uint4 v = {0u, 0u, 0u, 0u};
        if (active && q0 + r32 < n) v = *(const uint4 *)(q + (size_t)(q0 + r32) * ldq + (size_t)hq * D + 16 * ks + 8 * h);
        qf[ks] = __builtin_bit_cast(bf16x8, v);
    }
    f32x16 acc[DT];
#pragma unroll
    for (int dt = 0; dt < DT; ++dt)
#pragma unroll
        for (int j = 0; j < 16; ++j) acc[dt][j] = 0.f;
    float mrow = -INFINITY, lpart = 0.f;              // reference and sum of the lane's own keys
    const float scale2 = 1.4426950408889634f / sqrtf((float)D);   // log2(e) / sqrt(d)
    const int qq = p0 + q0 + r32;
    // operand addresses in a tile: key unit 2 s + h of the row that this lane's
    // MFMA row stands for; transposed value reads (see vread)
    const int krow = pf_key_of_row(r32), a4 = lane & 3, qv = (lane >> 2) & 3, half16 = (lane >> 4) & 1;

    if (tid == 0) redo = INT32_MAX;
    Scales next;
    fetch_pages();
    load();
    fetch_pages();
    if (BKT * tile0 + 16 * (lane & 3) >= Lk) vb = __builtin_amdgcn_readlane(vb, 0);
    store(BKT * tile0, tile0 & 1, next);
    load();
    fetch_pages();
    for (int i = tile0; i < ntiles; ++i) {
        const int k0 = i * BKT, b = i & 1;
        __syncthreads();                              // tile i is in LDS, and tile i - 1's buffers are free
        const Scales sc = next;
        if (i + 1 < ntiles) {
            store(k0 + BKT, b ^ 1, next);
            load();                                   // past the last tile: groups past the sequence, or a tile not stored
            fetch_pages();
        }
        if (k0 > my_last_q) continue;                 // wave-uniform: the whole tile is in this unit's future

        const uint4 *Kt = ring + b * UNITS, *Vt = ring + (2 + b) * UNITS;
        f32x16 st[2];
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int j = 0; j < 16; ++j) st[kt][j] = 0.f;
        // key operands two steps ahead of their products, in a fixed order
        constexpr int KD = 2;
        bf16x8 kf[KD + 1][2];
        int kr = krow;
        asm volatile("" : "+v"(kr));                  // the steps' addresses are made anew: kept, they cost registers
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
        // lane: keys k0 + 32 kt + 16 (j / 8) + 8 h + j % 8 of query qq
        // the reference stays where the maximum is at most 2^P_LAG above it, so
        // most tiles rescale nothing
        auto reference = [&]() {
            float mt = -INFINITY;
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int j = 0; j < 16; ++j) mt = fmaxf(mt, st[kt][j]);
            const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
            mt = fmaxf(__uint_as_float(two[0]), __uint_as_float(two[1]));   // both halves of the query's keys
            mt = __builtin_fmaf(mt, scale2, byte_256(sc.top));
            return mt > mrow + P_LAG ? mt : mrow;
        };
        // what is added to scores in base 2 for a weight's exponent
        auto offset = [&](float ref) { return byte_256(sc.top) - ((ref == -INFINITY ? 0.f : ref) - P_UP); };
        float far = 0.f;
        if (k0 + BKT - 1 > p0 + q0 || k0 + BKT > Lk || sc.far) {
#pragma unroll
            for (int kt = 0; kt < 2; ++kt)
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const int key = k0 + 32 * kt + 16 * (j >> 3) + 8 * h + (j & 7);
                    st[kt][j] = (key <= qq && key < Lk) ? st[kt][j] : -INFINITY;
                }
            if (sc.far) {                             // each group's scale: on its scores, and out of its sum
#pragma unroll
                for (int f = 0; f < 4; ++f)
#pragma unroll
                    for (int j = 0; j < 8; ++j) st[f >> 1][8 * (f & 1) + j] += (float)(max(sc.g[f], B_LOW) - sc.top) * (1.0f / scale2);
                const float at = offset(reference());
#pragma unroll
                for (int f = 0; f < 4; ++f) {
                    float part = 0.f;
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        part += __builtin_amdgcn_exp2f(__builtin_fmaf(st[f >> 1][8 * (f & 1) + j], scale2, at));
                    far += part * exp2_int(min(sc.top - max(sc.g[f], B_LOW), B_HIGH - B_LOW));
                }
            }
        }
        const float mnew = reference(), at = offset(mnew);
        f16x8 pf[4];
        float ls = 0.f;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f16x2 w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    typedef float f32x2_t __attribute__((ext_vector_type(2)));
                    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kt][8 * half + 2 * e], scale2, at));
                    const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(st[kt][8 * half + 2 * e + 1], scale2, at));
                    ls += x + y;
                    w[e] = __builtin_convertvector((f32x2_t){x, y}, f16x2);
                }
                pf[2 * kt + half] = __builtin_bit_cast(f16x8, w);
            }
        if (__ballot(mnew != mrow)) {
            const float alpha = mnew == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mrow - mnew);
            lpart *= alpha;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt)
#pragma unroll
                for (int j = 0; j < 16; ++j) acc[dt][j] *= alpha;
        }
        lpart = __builtin_fmaf(sc.far ? far : ls, exp2_int(127 - sc.top), lpart);
        mrow = mnew;
        // operand f: 16-key step f / DT, output tile f % DT; lane l takes
        // dimension 32 dt + l % 32 of keys 16 s + 8 h .. + 7 by two transposed reads
        constexpr int VD = 3;                         // read three ahead of their products
        f16x8 vf[VD + 1];
        auto vread = [&](int f) {
            uint2 part[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int key = 16 * (f / DT) + 8 * h + 4 * r + qv;
                const int cc = 4 * (f % DT) + 2 * half16 + (a4 >> 1);
                part[r] = lds_read_tr16(reinterpret_cast<const char *>(Vt + key * KCH + (cc ^ val16_swz<KCH>(key))) + 8 * (a4 & 1));
            }
            vf[f % (VD + 1)] = __builtin_bit_cast(f16x8, (uint4){part[0].x, part[0].y, part[1].x, part[1].y});
        };
#pragma unroll
        for (int f = 0; f < VD; ++f) vread(f);
#pragma unroll
        for (int f = 0; f < 4 * DT; ++f) {
            if (f + VD < 4 * DT) vread(f + VD);
            __builtin_amdgcn_sched_barrier(0);
            acc[f % DT] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vf[f % (VD + 1)], pf[f / DT], acc[f % DT], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    if (lane == 0 && redo_from != INT32_MAX) atomicMin(&redo, redo_from);
    __syncthreads();                                  // every wavefront is done with the tiles

    // lane: O^T[32 dt + 8 (j / 4) + 4 h + j % 4][query l % 32]
    const auto two = __builtin_amdgcn_permlane32_swap(__float_as_uint(lpart), __float_as_uint(lpart), false, false);
    const float sum = __uint_as_float(two[0]) + __uint_as_float(two[1]), inv = 1.0f / sum;
    bool nan = false;
    if (ns > 1) {
        if (!active || my_last_q < BKT * tile0) return;   // no row of the unit sees the split's tiles
        const size_t all = (size_t)(units / G) * G * nkv, unit = (size_t)kvh * units + u;
        float *part = ws + ((size_t)sp.part0[si] + split * all + unit) * PART<D>;
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int j = 0; j < 16; j += 4) {
                float4 v;
                v.x = acc[dt][j] * inv;
                v.y = acc[dt][j + 1] * inv;
                v.z = acc[dt][j + 2] * inv;
                v.w = acc[dt][j + 3] * inv;
                nan |= v.x != v.x || v.y != v.y || v.z != v.z || v.w != v.w;
                *(float4 *)(part + 4 * ((8 * dt + j / 2 + h) * 32 + r32)) = v;
            }
        const unsigned long long bad = __ballot(nan || redo <= qq);
        if (h == 0) *(float2 *)(part + 32 * D + 2 * r32) = {((bad | bad >> 32) >> r32) & 1 ? QNAN : mrow, sum};
        return;
    }
    // through LDS for whole rows
    uint16_t *ost = (uint16_t *)ring + (size_t)wave * QB * OPITCH;
    {
#pragma unroll
        for (int dt = 0; dt < DT; ++dt)
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float v = acc[dt][j] * inv;
                nan |= v != v;
                ost[r32 * OPITCH + 32 * dt + 8 * (j >> 2) + 4 * h + (j & 3)] = f2bf(v);
            }
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);               // lgkmcnt(0): this wavefront's staging writes are done
    if (!active) return;
    if (redo <= my_last_q || __ballot(nan && q0 + r32 < n)) {
#pragma unroll 1
        for (int r = 0; r < QB && q0 + r < n; ++r)
            attend_row<D>(q + (size_t)(q0 + r) * ldq + (size_t)hq * D, p0 + q0 + r + 1, kvh, nkv, slot, cv, cl,
                          out + (size_t)(q0 + r) * ldo + (size_t)hq * D);
        return;
    }
#pragma unroll 4
    for (int it = lane; it < QB * (D / 8); it += 64) {
        const int qr = it / (D / 8), c8 = it % (D / 8), qo = q0 + qr;
        if (qo < n) *(uint4 *)(out + (size_t)qo * ldo + (size_t)hq * D + 8 * c8) = *(const uint4 *)(ost + qr * OPITCH + 8 * c8);
    }
}

// The splits of a unit's rows, weighed by their maxima and sums in order: by sum
// 2^maximum, where the sums' own exponents count (they carry their values' scales).
// Workgroup: one unit (x), D / 4 slices of 8 dimension fours (y); thread (four,
// row).  A row counts the splits that it sees; rows with a NaN maximum are done
// again by the first slice.
template <int D>
__global__ __launch_bounds__(256) void k_attn8_join(const float *__restrict__ ws, const uint16_t *__restrict__ q,
                                                    long long ldq, SeqTable seq, SplitTable sp, int G, int nkv, CacheView cv,
                                                    CacheLayer cl, uint16_t *__restrict__ out, long long ldo)
{
    __shared__ float w[MOST_SPLITS][32], l[MOST_SPLITS][32];
    __shared__ uint32_t again;
    const int si = seq_of(seq, blockIdx.x), ns = sp.splits[si], n = seq.len[si], p0 = seq.start[si], slot = seq.slot[si];
    const int unit = (int)blockIdx.x - seq.unit0[si], units = (n + 31) / 32 * G;
    const int kvh = unit / units, u = unit % units, q0 = u / G * 32, hq = kvh * G + u % G;
    const int tid = threadIdx.x, r = tid & 31, sl = tid >> 5, t = q0 + r;
    const int span = 64 * tiles_of_split(p0 + n, ns), seen = t < n ? (p0 + t) / span + 1 : 0;   // <= ns
    const size_t stride = (size_t)units * nkv * PART<D>;
    const float *part = ws + ((size_t)sp.part0[si] + unit) * PART<D>;
    for (int s = sl; s < seen; s += 8) {
        const float2 ml = *(const float2 *)(part + s * stride + 32 * D + 2 * r);
        w[s][r] = ml.x;
        l[s][r] = ml.y;
    }
    __syncthreads();
    if (tid < 32) {
        float M = -INFINITY, L = 0.f;
        bool bad = false;
        for (int s = 0; s < seen; ++s) {
            bad |= w[s][r] != w[s][r];
            M = fmaxf(M, w[s][r] + (float)__builtin_amdgcn_frexp_expf(l[s][r]));
        }
        for (int s = 0; s < seen; ++s) {
            const float sum = l[s][r], up = w[s][r] - M + (float)__builtin_amdgcn_frexp_expf(sum);
            const float x = __builtin_amdgcn_frexp_mantf(sum) * __builtin_amdgcn_exp2f(up);
            w[s][r] = x;
            L += x;
        }
        for (int s = 0; s < seen; ++s) w[s][r] /= L;
        const uint32_t rows = (uint32_t)__ballot(bad);
        if (tid == 0) again = rows;
    }
    __syncthreads();
    const uint32_t rows = again;
    const int c = 8 * blockIdx.y + sl;
    float4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int s = 0; s < seen; ++s) {
        const float4 v = *(const float4 *)(part + s * stride + 4 * (c * 32 + r));
        const float x = w[s][r];
        o.x += x * v.x;
        o.y += x * v.y;
        o.z += x * v.z;
        o.w += x * v.w;
    }
    if (t < n && !((rows >> r) & 1))
        *(uint2 *)(out + (size_t)(seq.row0[si] + t) * ldo + (size_t)hq * D + 4 * c) = (uint2){f2bf2(o.x, o.y), f2bf2(o.z, o.w)};
    if (blockIdx.y != 0) return;
#pragma unroll 1
    for (int i = tid >> 6; i < 32; i += 4)
        if ((rows >> i) & 1)                          // set for rows of the sequence only
            attend_row<D>(q + (size_t)(seq.row0[si] + q0 + i) * ldq + (size_t)hq * D, p0 + q0 + i + 1, kvh, nkv, slot, cv, cl,
                          out + (size_t)(seq.row0[si] + q0 + i) * ldo + (size_t)hq * D);
}

struct Freqs {
    double f[64];
};
__global__ void k_rope_table_of(float2 *tab, int half, Freqs fr)
{
    const int i = threadIdx.x;
    if (i >= half) return;
    double s, c;
    sincos((double)blockIdx.x * fr.f[i], &s, &c);
    tab[(size_t)blockIdx.x * half + i] = {(float)c, (float)s};
}

}  // namespace

hipError_t launch_rope_table_of(float2 *tab, int max_pos, int d, const double *freq, hipStream_t st)
{
    Freqs fr{};
    for (int i = 0; i < d / 2; ++i) fr.f[i] = freq[i];
    KLAUNCH(k_rope_table_of, dim3(max_pos), dim3(64), 0, st, tab, d / 2, fr);
    return hipGetLastError();
}

// f(head size, whether pairs come in 16-byte runs, whether the cache is e4m3)
template <class F>
static hipError_t append_variant(int d, const RopeArgs &rope, const CacheView &cv, F &&f)
{
    const bool vec = rope.interleaved || rope.rot % 16 == 0;
    const auto go = [&](auto dd) {
        if (vec) return cv.e4m3 ? f(dd, std::true_type{}, std::true_type{}) : f(dd, std::true_type{}, std::false_type{});
        return cv.e4m3 ? f(dd, std::false_type{}, std::true_type{}) : f(dd, std::false_type{}, std::false_type{});
    };
    if (d == 128) go(std::integral_constant<int, 128>{});
    else if (d == 64) go(std::integral_constant<int, 64>{});
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

hipError_t launch_append_rows(const QkvRows &in, int rows, const uint8_t *valid, const int32_t *pos, int nq, int nkv,
                              int d, const RopeArgs &rope, uint16_t *q, long long ldq, const CacheView &cv,
                              const CacheLayer &cl, hipStream_t st)
{
    const long long threads = (long long)rows * (nq + 2 * nkv) * (d / 16);
    const dim3 grid((unsigned)((threads + 255) / 256));
    return append_variant(d, rope, cv, [&](auto dd, auto vec, auto e4) {
        KLAUNCH((k_append_rows<decltype(dd)::value, decltype(vec)::value, decltype(e4)::value>), grid, dim3(256), 0, st, in,
                rows, valid, pos, nq, nkv, rope, q, ldq, cv, cl);
    });
}

hipError_t launch_append_seqs(const QkvRows &in, SeqTable &seq, int nq, int nkv, int d, const RopeArgs &rope,
                              uint16_t *q, long long ldq, const CacheView &cv, const CacheLayer &cl, hipStream_t st)
{
    const int blk = 1 << cv.blk_shift;
    int units = 0;
    for (int i = 0; i < seq.n; ++i) {
        seq.unit0[i] = units;
        units += (seq.start[i] + seq.len[i] - 1) / blk - seq.start[i] / blk + 1;
    }
    if (units == 0) return hipErrorInvalidValue;
    int slices = 1;
    while (slices < nkv && (long long)units * slices < 512) slices *= 2;
    slices = std::min(slices, nkv);
    const dim3 grid(units, slices), block(std::max(256, blk * (d / 16)));
    return append_variant(d, rope, cv, [&](auto dd, auto vec, auto e4) {
        KLAUNCH((k_append_seqs<decltype(dd)::value, decltype(vec)::value, decltype(e4)::value>), grid, block, 0, st, in, seq,
                nq, nkv, rope, q, ldq, cv, cl);
    });
}

// One split for lengths up to 512, whose four steps cost less than a second
// launch that merges (four slots of 128 tokens: 6.8 us a call, 10.2 with
// two).  Else the smallest chunk from 128 tokens up to 1024 for which rows of
// max_len have at most 2048 workgroups (162 rows of 512 to 4096 tokens: 154 us
// at 1024, 156 at 512, 157 at 2048; 32 rows of 1K to 32K: 132, 139, 142), or 4096
// for max_len up to 2048, where few splits divide the work badly (108 rows up to
// 1282 tokens: 22 us, 32 with 2048; 150 rows up to 700: 19, 26; 200 rows up to 2000:
// 58 either way); more where a row would have over 512 splits to merge.
int attn8_chunk(int rows, int nkv, int max_len)
{
    if (max_len <= 512) return 512;
    long long chunk = 128;
    const int most = max_len <= 2048 ? 4096 : 2048;
    while (chunk < 1024 && (long long)rows * nkv * ((max_len + chunk - 1) / chunk) > most) chunk *= 2;
    while ((max_len + chunk - 1) / chunk > 512) chunk *= 2;
    return (int)std::min<long long>(chunk, 1 << 30);
}

hipError_t launch_attn8_split(const uint16_t *q, long long ldq, int rows, const uint8_t *valid, const int32_t *lens,
                              int plus_one, int nq, int nkv, int d, const CacheView &cv, const CacheLayer &cl, int max_len,
                              int chunk, float *ws, hipStream_t st, const int32_t *row_order, uint16_t *out,
                              long long ldo)
{
    const int splits = (int)((max_len + (long long)chunk - 1) / chunk), G = nq / nkv;
    if (out != nullptr && splits != 1) return hipErrorInvalidValue;
    const dim3 grid(nkv, splits, rows);
    const bool paged = cv.kv.layout == 1;
#define CORUN_SPLIT8(D_, P_)                                                                                              \
    KLAUNCH((k_attn8_split<D_, P_>), grid, dim3(256), 0, st, q, ldq, valid, lens, plus_one, G, nkv, cv, cl, chunk, splits, \
            max_len, ws, row_order, out, ldo)
    if (d == 128 && paged) CORUN_SPLIT8(128, true);
    else if (d == 128) CORUN_SPLIT8(128, false);
    else if (d == 64 && paged) CORUN_SPLIT8(64, true);
    else if (d == 64) CORUN_SPLIT8(64, false);
    else return hipErrorInvalidValue;
#undef CORUN_SPLIT8
    return hipGetLastError();
}

hipError_t launch_attn8_merge(const float *ws, int rows, const uint8_t *valid, const int32_t *lens, int plus_one, int nq,
                              int nkv, int d, int max_len, int chunk, uint16_t *out, long long ldo, hipStream_t st)
{
    const int splits = (int)((max_len + (long long)chunk - 1) / chunk);
    const int hb = 256 / d;
    const dim3 grid((nq + hb - 1) / hb, rows);
    const size_t shm = sizeof(float) * hb * 2 * splits;
    if (d == 128)
        KLAUNCH((k_attn8_merge<128>), grid, dim3(256), shm, st, ws, valid, lens, plus_one, nq, nkv, chunk, splits, max_len,
                out, ldo);
    else if (d == 64)
        KLAUNCH((k_attn8_merge<64>), grid, dim3(256), shm, st, ws, valid, lens, plus_one, nq, nkv, chunk, splits, max_len,
                out, ldo);
    else
        return hipErrorInvalidValue;
    return hipGetLastError();
}

// Splits of a sequence over its tiles, from nothing but itself, so that its
// results stay the same beside others: where its workgroups of four would fill at
// most half of the chip's room for 512, as many as fill it, of at least eight
// tiles each (starting a split and joining it cost about four), or 32 where more
// than a quarter is filled already.  Heads of 8 over 32, behind 8192 tokens: 1 row
// 30 us, 204 unsplit; 256 rows 56, 210; 512 rows 88, 218; 1024 rows 160, 231.
static int attn8_seq_splits(int rows, int start, int nq, int nkv)
{
    const int G = nq / nkv, tiles = (int)(((long long)start + rows + 63) / 64);
    const long long wgs = (((long long)rows + 31) / 32 * G + 3) / 4 * nkv;
    if (wgs > 256) return 1;
    const int most = std::min({(int)(512 / wgs), tiles / (wgs > 128 ? 32 : 8), MOST_SPLITS});
    if (most < 2) return 1;
    const int per = (tiles + most - 1) / most;
    return (tiles + per - 1) / per;                   // no split without tiles
}

static size_t part_bytes(int d) { return (d == 128 ? PART<128> : PART<64>) * sizeof(float); }

// Splits times workgroups are at most 512, of at most four units each.
size_t attn8_seq_ws_max(int d) { return 2048 * part_bytes(d); }

size_t attn8_seqs_ws(const SeqTable &seq, int nq, int nkv, int d)
{
    size_t units = 0;
    for (int i = 0; i < seq.n; ++i) {
        const int ns = attn8_seq_splits(seq.len[i], seq.start[i], nq, nkv);
        if (ns > 1) units += (size_t)ns * ((seq.len[i] + 31) / 32) * nq;
    }
    return units * part_bytes(d);
}

hipError_t launch_attn8_seqs(const uint16_t *q, long long ldq, const SeqTable &given, int nq, int nkv, int d,
                             const CacheView &cv, const CacheLayer &cl, uint16_t *out, long long ldo, float *ws,
                             hipStream_t st)
{
    const int G = nq / nkv, n = given.n;
    if (n < 1 || n > 64) return hipErrorInvalidValue;
    // longest sequences first: the last workgroups of a call are short ones (12
    // prompts of 100 to 600 tokens: 47 us in the order given, 40 so)
    int by[64];
    for (int i = 0; i < n; ++i) by[i] = i;
    const auto keys = [&](int i) { return given.start[i] + given.len[i]; };
    std::stable_sort(by, by + n, [&](int a, int b) { return keys(a) > keys(b); });
    SeqTable seq, joined;
    SplitTable sp, jp;
    seq.n = n;
    joined.n = 0;
    long long groups8 = 0;
    int parts = 0, join_units = 0;
    for (int i = 0; i < n; ++i) {
        seq.row0[i] = given.row0[by[i]];
        seq.len[i] = given.len[by[i]];
        seq.start[i] = given.start[by[i]];
        seq.slot[i] = given.slot[by[i]];
        sp.splits[i] = attn8_seq_splits(seq.len[i], seq.start[i], nq, nkv);
        sp.part0[i] = parts;
        groups8 += ((seq.len[i] + 31) / 32 * G + 7) / 8 * sp.splits[i];
        if (sp.splits[i] == 1) continue;
        const int units = (seq.len[i] + 31) / 32 * nq, j = joined.n++;
        parts += units * sp.splits[i];
        joined.row0[j] = seq.row0[i];
        joined.len[j] = seq.len[i];
        joined.start[j] = seq.start[i];
        joined.slot[j] = seq.slot[i];
        joined.unit0[j] = join_units;
        jp.splits[j] = sp.splits[i];
        jp.part0[j] = sp.part0[i];
        join_units += units;
    }
    if (joined.n > 0 && ws == nullptr) return hipErrorInvalidValue;
    // Eight wavefronts share a tile's conversion; four are twice the workgroups,
    // and a tile takes them 1.7 us on a CU of their own where eight need 1.9.
    // Heads of 128 take four where eight would leave half of the 256 CUs idle
    // (behind 8192 tokens 64 rows: 35 us, 38 with eight; 256 rows: 60, 56; 1536: 318,
    // 275) and where no sequence has many tiles (600 tokens: 22 us, 26 with eight;
    // 1000: 32, 36; 2000: 62, 67; 4000: 174, 147).  Heads of 64 have units for four
    // wavefronts to load only.  A row's arithmetic is the same either way.
    const int NW = d == 64 || groups8 * nkv <= 128 || keys(by[0]) <= 2048 ? 4 : 8;
    int groups = 0;
    for (int i = 0; i < n; ++i) {
        seq.unit0[i] = groups;
        groups += ((seq.len[i] + 31) / 32 * G + NW - 1) / NW * sp.splits[i];
    }
    const dim3 grid((unsigned)groups * nkv);
    const bool paged = cv.kv.layout == 1;
#define CORUN_PREFILL8(D_, P_, NW_) \
    KLAUNCH((k_attn8_prefill<D_, P_, NW_>), grid, dim3(64 * NW_), 0, st, q, ldq, seq, sp, G, nkv, cv, cl, out, ldo, \
            ws)
    if (d == 128 && paged && NW == 8) CORUN_PREFILL8(128, true, 8);
    else if (d == 128 && paged) CORUN_PREFILL8(128, true, 4);
    else if (d == 128 && NW == 8) CORUN_PREFILL8(128, false, 8);
    else if (d == 128) CORUN_PREFILL8(128, false, 4);
    else if (d == 64 && paged) CORUN_PREFILL8(64, true, 4);
    else if (d == 64) CORUN_PREFILL8(64, false, 4);
    else return hipErrorInvalidValue;
#undef CORUN_PREFILL8
    if (joined.n > 0) {
        const dim3 jgrid(join_units, d / 32);
        if (d == 128)
            KLAUNCH((k_attn8_join<128>), jgrid, dim3(256), 0, st, ws, q, ldq, joined, jp, G, nkv, cv, cl, out, ldo);
        else
            KLAUNCH((k_attn8_join<64>), jgrid, dim3(256), 0, st, ws, q, ldq, joined, jp, G, nkv, cv, cl, out, ldo);
    }
    return hipGetLastError();
}

}  // namespace corun
