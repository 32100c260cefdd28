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

#include "device.h"
#include "kernels.h"

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
// that is no multiple of 16 are read one element at a time.
// ---------------------------------------------------------------------------
template <int D>
struct Pairs {
    int a0, b0, first, rot2;       // first pair; rotated pairs of the head
    bool half, vec;
    float c[8], s[8];
    double cd[8], sd[8];

    __device__ __forceinline__ bool rotated(int t) const { return first + t < rot2; }
    // element offsets of pair t where vec does not hold
    __device__ __forceinline__ int at(int t, int which) const
    {
        const int i = first + t;
        return i < rot2 ? i + which * rot2 : 2 * i + which;
    }
    __device__ __forceinline__ void init(const RopeArgs &r, int j, int pos)
    {
        first = 8 * j;
        rot2 = r.rot / 2;
        half = !r.interleaved && first < rot2;
        vec = r.interleaved || r.rot % 16 == 0;
        a0 = half ? 8 * j : 16 * j;
        b0 = half ? 8 * j + rot2 : 16 * j + 8;
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            turn_cos_sin(r.turns[first + t], (double)pos, cd[t], sd[t]);
            cd[t] *= r.mag;
            sd[t] *= r.mag;
            c[t] = (float)cd[t];
            s[t] = (float)sd[t];
        }
    }
    __device__ __forceinline__ void rotate(const float *x0, const float *x1, float *y0, float *y1) const
    {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            y0[t] = rotated(t) ? __builtin_fmaf(x0[t], c[t], -(x1[t] * s[t])) : x0[t];
            y1[t] = rotated(t) ? __builtin_fmaf(x1[t], c[t], x0[t] * s[t]) : x1[t];
        }
    }
    __device__ __forceinline__ void rotate_exact(const float *x0, const float *x1, float *y0, float *y1) const
    {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const double u = x0[t], w = x1[t];
            y0[t] = rotated(t) ? to_odd(__builtin_fma(u, cd[t], -(w * sd[t]))) : x0[t];
            y1[t] = rotated(t) ? to_odd(__builtin_fma(w, cd[t], u * sd[t])) : x1[t];
        }
    }
    // runs of eight elements <-> pairs: run A holds the pairs' first elements
    // and run B the second (half), or the two runs hold the pairs in turn
    __device__ __forceinline__ void to_pairs(const float *e, float *x0, float *x1) const
    {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            x0[t] = half ? e[t] : e[2 * t];
            x1[t] = half ? e[8 + t] : e[2 * t + 1];
        }
    }
    __device__ __forceinline__ void from_pairs(const float *x0, const float *x1, float *e) const
    {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            e[t] = half ? x0[t] : (t & 1 ? x1[t / 2] : x0[t / 2]);
            e[8 + t] = half ? x1[t] : (t & 1 ? x1[4 + t / 2] : x0[4 + t / 2]);
        }
    }
};

template <int D>
__device__ __forceinline__ void load_pairs(const QkvRows &in, const Pairs<D> &p, long long row, int head, float *x0, float *x1)
{
    const size_t off = (size_t)row * in.ld + (size_t)head * D;
    if (!p.vec) {
#pragma unroll
        for (int t = 0; t < 8; ++t)
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                float x = 0.f;
                if (in.bf16 != nullptr) x = bf2f(in.bf16[off + p.at(t, w)]);
                else {
                    for (int sp = 0; sp < in.S; ++sp) x += in.part[sp * in.stride + off + p.at(t, w)];
                    x = bf2f(f2bf(x));
                }
                (w ? x1 : x0)[t] = x;
            }
        return;
    }
    float e[16];
    if (in.bf16 != nullptr) {
        const uint4 a = *(const uint4 *)(in.bf16 + off + p.a0), b = *(const uint4 *)(in.bf16 + off + p.b0);
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            e[2 * i] = __uint_as_float(w[i] << 16);
            e[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = 0.f;
        for (int sp = 0; sp < in.S; ++sp) {
            const float *src = in.part + sp * in.stride + off;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 f = *(const float4 *)(src + (i < 2 ? p.a0 : p.b0) + 4 * (i & 1));
                e[4 * i] += f.x;
                e[4 * i + 1] += f.y;
                e[4 * i + 2] += f.z;
                e[4 * i + 3] += f.w;
            }
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) e[i] = bf2f(f2bf(e[i]));
    }
    p.to_pairs(e, x0, x1);
}

template <int D>
__device__ __forceinline__ void store_bf16(uint16_t *dst, const Pairs<D> &p, const float *y0, const float *y1)
{
    if (!p.vec) {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            dst[p.at(t, 0)] = f2bf(y0[t]);
            dst[p.at(t, 1)] = f2bf(y1[t]);
        }
        return;
    }
    float e[16];
    p.from_pairs(y0, y1, e);
    *(uint4 *)(dst + p.a0) = (uint4){f2bf2(e[0], e[1]), f2bf2(e[2], e[3]), f2bf2(e[4], e[5]), f2bf2(e[6], e[7])};
    *(uint4 *)(dst + p.b0) = (uint4){f2bf2(e[8], e[9]), f2bf2(e[10], e[11]), f2bf2(e[12], e[13]), f2bf2(e[14], e[15])};
}

template <int D>
__device__ __forceinline__ void store_codes(uint8_t *dst, const Pairs<D> &p, const float *y0, const float *y1, int e_)
{
    const float m = exp2_int(-e_);
    if (!p.vec) {
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            const uint32_t w = encode4(y0[t], y1[t], 0.f, 0.f, m);
            dst[p.at(t, 0)] = (uint8_t)w;
            dst[p.at(t, 1)] = (uint8_t)(w >> 8);
        }
        return;
    }
    float e[16];
    p.from_pairs(y0, y1, e);
    *(uint2 *)(dst + p.a0) = (uint2){encode4(e[0], e[1], e[2], e[3], m), encode4(e[4], e[5], e[6], e[7], m)};
    *(uint2 *)(dst + p.b0) = (uint2){encode4(e[8], e[9], e[10], e[11], m), encode4(e[12], e[13], e[14], e[15], m)};
}

__device__ __forceinline__ uint32_t top_of(const float *y0, const float *y1)
{
    uint32_t u = 0u;
#pragma unroll
    for (int t = 0; t < 8; ++t) u = max(u, max(finite_bits(y0[t]), finite_bits(y1[t])));
    return u;
}

constexpr float QNAN = __builtin_nanf("");

// One decode step's rows: D / 16 threads to a (row, head).
template <int D>
__global__ __launch_bounds__(256) void k_append_rows(QkvRows in, int rows, const uint8_t *__restrict__ valid,
                                                     const int32_t *__restrict__ pos, int nq, int nkv, RopeArgs rope,
                                                     uint16_t *__restrict__ q, long long ldq, CacheView cv, CacheLayer cl)
{
    constexpr int LPT = D / 16;
    const int unit = (blockIdx.x * 256 + threadIdx.x) / LPT, j = threadIdx.x % LPT;
    const int nh = nq + 2 * nkv, r = unit / nh, h = unit % nh;
    if (r >= rows || (valid != nullptr && !valid[r])) return;
    const int t = pos[r];
    bool bad = t < 0 || t >= cv.cap;
    int page = 0;
    if (!bad && cv.kv.layout == 1) {
        page = page_of(cv, r, t);
        bad = page < 0;
    }
    Pairs<D> p;
    float x0[8], x1[8], y0[8], y1[8];
    p.init(rope, j, t);
    load_pairs<D>(in, p, r, h, x0, x1);
    if (h < nq) {
        p.rotate(x0, x1, y0, y1);
        if (bad)
#pragma unroll
            for (int i = 0; i < 8; ++i) y0[i] = y1[i] = QNAN;
        store_bf16<D>(q + (size_t)r * ldq + (size_t)h * D, p, y0, y1);
        return;
    }
    if (bad) return;
    const bool key = h < nq + nkv;
    const int kvh = h - nq - (key ? 0 : nkv);
    const Place pl = place(cv, nkv, kvh, r, page, t);
    if (!cv.e4m3) {
        if (key) p.rotate(x0, x1, y0, y1);
        store_bf16<D>((uint16_t *)(key ? cl.k : cl.v) + pl.row * D, p, key ? y0 : x0, key ? y1 : x1);
        return;
    }
    if (key) {
        p.rotate_exact(x0, x1, y0, y1);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x0[i] = y0[i];
            x1[i] = y1[i];
        }
    }
    uint8_t *codes = (uint8_t *)(key ? cl.k : cl.v) + pl.row * D;
    uint8_t *scale = (key ? cl.ks : cl.vs) + pl.blk;
    uint32_t top = top_of(x0, x1);
#pragma unroll
    for (int o = 1; o < LPT; o *= 2) top = max(top, (uint32_t)__shfl_xor((int)top, o, LPT));
    const int kept = t & ((1 << cv.blk_shift) - 1);
    const int need = scale_exp(top), old = kept ? (int)*scale - 127 : need, e = max(old, need);
    if (old < e) {   // the block's earlier tokens move to the larger scale
        const float m = e - old > 120 ? 0.f : exp2_int(old - e);
        for (int i = 1; i <= kept; ++i) {
            uint4 *w = (uint4 *)(codes - (size_t)i * D + 16 * j);
            uint4 v = *w;
            v.x = rescale4(v.x, m);
            v.y = rescale4(v.y, m);
            v.z = rescale4(v.z, m);
            v.w = rescale4(v.w, m);
            *w = v;
        }
    }
    store_codes<D>(codes, p, x0, x1, e);
    if (j == 0 && (kept == 0 || e != old)) *scale = (uint8_t)(e + 127);
}

// A prefill call's sequences.  Workgroup: one scale block of tokens of one
// sequence (x), a slice of the heads (y); thread (head group, token, j), so
// that a head group's wavefronts hold every new token of the block and agree
// on its scale through LDS, once per pair of key and value heads.  Threads of
// the block's earlier tokens move those to a scale that grew.
template <int D>
__global__ __launch_bounds__(512) void k_append_seqs(QkvRows in, SeqTable seq, int nq, int nkv, RopeArgs rope,
                                                     uint16_t *__restrict__ q, long long ldq, CacheView cv, CacheLayer cl)
{
    constexpr int LPT = D / 16;
    const int blk = 1 << cv.blk_shift, tid = threadIdx.x;
    const int gt = blk * LPT, groups = blockDim.x / gt;      // threads of a head group
    const int hg = tid / gt, tok = tid % gt / LPT, j = tid % LPT;
    int i = 0;
    while (i + 1 < seq.n && seq.unit0[i + 1] <= (int)blockIdx.x) ++i;
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
    Pairs<D> p;
    p.init(rope, j, t);
    float x0[8], x1[8], y0[8], y1[8];
    // query heads of this slice
    const int ns = gridDim.y, sl = blockIdx.y;
    const int q_lo = (int)((long long)nq * sl / ns), q_hi = (int)((long long)nq * (sl + 1) / ns);
    if (fresh)
        for (int h = q_lo + hg; h < q_hi; h += groups) {
            load_pairs<D>(in, p, row, h, x0, x1);
            p.rotate(x0, x1, y0, y1);
            if (bad)
#pragma unroll
                for (int u = 0; u < 8; ++u) y0[u] = y1[u] = QNAN;
            store_bf16<D>(q + (size_t)row * ldq + (size_t)h * D, p, y0, y1);
        }
    if (bad) return;
    const int k_lo = (int)((long long)nkv * sl / ns), k_hi = (int)((long long)nkv * (sl + 1) / ns);
    if (!cv.e4m3) {
        if (fresh)
            for (int h = k_lo + hg; h < k_hi; h += groups) {
                const Place pl = place(cv, nkv, h, slot, page, t);
                load_pairs<D>(in, p, row, nq + h, x0, x1);
                p.rotate(x0, x1, y0, y1);
                store_bf16<D>((uint16_t *)cl.k + pl.row * D, p, y0, y1);
                load_pairs<D>(in, p, row, nq + nkv + h, x0, x1);
                store_bf16<D>((uint16_t *)cl.v + pl.row * D, p, x0, x1);
            }
        return;
    }
    __shared__ uint32_t tops[2][8][2];
    const int kept = max(0, start - t0);              // earlier tokens of the block
    const int wave = tid >> 6, gw = gt / 64;          // wavefronts of a head group
    const int per = (k_hi - k_lo + groups - 1) / groups;
    for (int it = 0; it < per; ++it) {
        const int h = k_lo + hg + it * groups;
        const bool on = h < k_hi;
        uint32_t tk = 0u, tv = 0u;
        if (on && fresh) {
            load_pairs<D>(in, p, row, nq + h, x0, x1);
            p.rotate_exact(x0, x1, y0, y1);
            load_pairs<D>(in, p, row, nq + nkv + h, x0, x1);
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
        __syncthreads();                              // the other buffer's readers passed the last one
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
                store_codes<D>(ck, p, y0, y1, ek);
                store_codes<D>(vk, p, x0, x1, ev);
            } else if (tok < kept) {
                auto move = [&](uint8_t *c, int old, int e) {
                    if (old >= e) return;
                    const float m = e - old > 120 ? 0.f : exp2_int(old - e);
                    uint4 v = *(uint4 *)(c + 16 * j);
                    v.x = rescale4(v.x, m);
                    v.y = rescale4(v.y, m);
                    v.z = rescale4(v.z, m);
                    v.w = rescale4(v.w, m);
                    *(uint4 *)(c + 16 * j) = v;
                };
                move(ck, ok, ek);
                move(vk, ov, ev);
            }
        }
        if (kept) __syncthreads();                    // every thread of a group has read the old scales (kept is uniform)
        if (on && tid % gt == 0) {
            cl.ks[pl.blk] = (uint8_t)(ek + 127);
            cl.vs[pl.blk] = (uint8_t)(ev + 127);
        }
    }
}

// ---------------------------------------------------------------------------
// Attention, one wavefront per (query, query head): 64 keys at a time, a key
// to a lane for the scores, then two dimensions to a lane for the values.
// ---------------------------------------------------------------------------
template <int D>
__device__ __forceinline__ void attend(const uint16_t *q, int n, int kvh, int nkv, int slot, const CacheView &cv,
                                       const CacheLayer &cl, uint16_t *out, bool bad)
{
    const int lane = threadIdx.x & 63;
    constexpr int E = D / 64;
    float qv[D];
#pragma unroll
    for (int i = 0; i < D; ++i) qv[i] = bf2f(q[i]);
    const float scale = 1.0f / sqrtf((float)D);
    float m = -INFINITY, l = 0.f, acc[E];
    for (int e = 0; e < E; ++e) acc[e] = 0.f;
    for (int b = 0; b < n && !bad; b += 64) {
        const int t = min(b + lane, n - 1);
        int page = 0;
        if (cv.kv.layout == 1) page = page_of(cv, slot, t);
        const bool lost = page < 0;
        const Place pl = place(cv, nkv, kvh, slot, max(page, 0), t);
        const uint8_t *k = (const uint8_t *)cl.k + pl.row * D;
        float sc = 0.f;
#pragma unroll
        for (int i = 0; i < D; i += 4) {
            const uint32_t w = *(const uint32_t *)(k + i);
            sc += qv[i] * __builtin_amdgcn_cvt_f32_fp8(w, 0);
            sc += qv[i + 1] * __builtin_amdgcn_cvt_f32_fp8(w, 1);
            sc += qv[i + 2] * __builtin_amdgcn_cvt_f32_fp8(w, 2);
            sc += qv[i + 3] * __builtin_amdgcn_cvt_f32_fp8(w, 3);
        }
        sc *= exp2_int((int)cl.ks[pl.blk] - 127) * scale;
        if (b + lane >= n) sc = -INFINITY;
        float mt = sc;
        for (int o = 32; o; o >>= 1) mt = fmaxf(mt, __shfl_xor(mt, o, 64));
        const float mn = fmaxf(m, mt);
        const float al = __expf(m - mn), pe = b + lane < n ? __expf(sc - mn) : 0.f;
        float ps = pe;
        for (int o = 32; o; o >>= 1) ps += __shfl_xor(ps, o, 64);
        l = l * al + ps;
        m = mn;
        for (int e = 0; e < E; ++e) acc[e] *= al;
        const float vsc = exp2_int((int)cl.vs[pl.blk] - 127);
        for (int i = 0; i < min(64, n - b); ++i) {
            const float pi = __shfl(pe, i, 64) * __shfl(vsc, i, 64);
            const size_t row = __shfl((unsigned long long)pl.row, i, 64);
            for (int e = 0; e < E; ++e) {
                const uint32_t c = ((const uint8_t *)cl.v)[row * D + E * lane + e];
                acc[e] += pi * __builtin_amdgcn_cvt_f32_fp8(c, 0);
            }
        }
        bad = __ballot(lost) != 0ull;
    }
    for (int e = 0; e < E; ++e) out[E * lane + e] = f2bf(bad ? QNAN : n > 0 ? acc[e] / l : 0.f);
}

template <int D>
__global__ __launch_bounds__(256) void k_attend_rows(const uint16_t *q, long long ldq, int rows, const uint8_t *valid,
                                                     const int32_t *lens, int plus_one, int nq, int nkv, CacheView cv,
                                                     CacheLayer cl, int max_len, uint16_t *out, long long ldo)
{
    const int u = blockIdx.x * 4 + (threadIdx.x >> 6), r = u / nq, h = u % nq;
    if (r >= rows) return;
    uint16_t *o = out + (size_t)r * ldo + (size_t)h * D;
    const bool live = valid == nullptr || valid[r];
    int n = live ? lens[r] : 0;
    bool bad = n < 0;
    if (live && !bad) {
        bad = n > max_len - plus_one;
        n += plus_one;
    }
    attend<D>(q + (size_t)r * ldq + (size_t)h * D, live ? n : 0, h / (nq / nkv), nkv, r, cv, cl, o, bad);
}

template <int D>
__global__ __launch_bounds__(256) void k_attend_seqs(const uint16_t *q, long long ldq, SeqTable seq, int nq, int nkv,
                                                     CacheView cv, CacheLayer cl, uint16_t *out, long long ldo)
{
    int i = 0;
    while (i + 1 < seq.n && seq.unit0[i + 1] <= (int)blockIdx.x) ++i;
    const int u = ((int)blockIdx.x - seq.unit0[i]) * 4 + (threadIdx.x >> 6), t = u / nq, h = u % nq;
    if (t >= seq.len[i]) return;
    const size_t r = (size_t)seq.row0[i] + t;
    attend<D>(q + r * ldq + (size_t)h * D, seq.start[i] + t + 1, h / (nq / nkv), nkv, seq.slot[i], cv, cl,
              out + r * ldo + (size_t)h * D, false);
}

}  // namespace

hipError_t launch_append_rows(const QkvRows &in, int rows, const uint8_t *valid, const int32_t *pos, int nq, int nkv,
                              int d, const RopeArgs &rope, uint16_t *q, long long ldq, const CacheView &cv,
                              const CacheLayer &cl, hipStream_t st)
{
    const long long threads = (long long)rows * (nq + 2 * nkv) * (d / 16);
    const dim3 grid((unsigned)((threads + 255) / 256));
    if (d == 128)
        KLAUNCH((k_append_rows<128>), grid, dim3(256), 0, st, in, rows, valid, pos, nq, nkv, rope, q, ldq, cv, cl);
    else if (d == 64)
        KLAUNCH((k_append_rows<64>), grid, dim3(256), 0, st, in, rows, valid, pos, nq, nkv, rope, q, ldq, cv, cl);
    else
        return hipErrorInvalidValue;
    return hipGetLastError();
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
    if (d == 128) KLAUNCH((k_append_seqs<128>), grid, block, 0, st, in, seq, nq, nkv, rope, q, ldq, cv, cl);
    else if (d == 64) KLAUNCH((k_append_seqs<64>), grid, block, 0, st, in, seq, nq, nkv, rope, q, ldq, cv, cl);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

hipError_t launch_attn8_rows(const uint16_t *q, long long ldq, int rows, const uint8_t *valid, const int32_t *lens,
                             int plus_one, int nq, int nkv, int d, const CacheView &cv, const CacheLayer &cl, int max_len,
                             uint16_t *out, long long ldo, hipStream_t st)
{
    const dim3 grid((unsigned)(((long long)rows * nq + 3) / 4));
    if (d == 128)
        KLAUNCH((k_attend_rows<128>), grid, dim3(256), 0, st, q, ldq, rows, valid, lens, plus_one, nq, nkv, cv, cl, max_len,
                out, ldo);
    else if (d == 64)
        KLAUNCH((k_attend_rows<64>), grid, dim3(256), 0, st, q, ldq, rows, valid, lens, plus_one, nq, nkv, cv, cl, max_len,
                out, ldo);
    else
        return hipErrorInvalidValue;
    return hipGetLastError();
}

hipError_t launch_attn8_seqs(const uint16_t *q, long long ldq, SeqTable &seq, int nq, int nkv, int d, const CacheView &cv,
                             const CacheLayer &cl, uint16_t *out, long long ldo, hipStream_t st)
{
    int units = 0;
    for (int i = 0; i < seq.n; ++i) {
        seq.unit0[i] = units;
        units += (seq.len[i] * nq + 3) / 4;
    }
    const dim3 grid(units);
    if (d == 128) KLAUNCH((k_attend_seqs<128>), grid, dim3(256), 0, st, q, ldq, seq, nq, nkv, cv, cl, out, ldo);
    else if (d == 64) KLAUNCH((k_attend_seqs<64>), grid, dim3(256), 0, st, q, ldq, seq, nq, nkv, cv, cl, out, ldo);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace corun
