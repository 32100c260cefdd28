// beam.hip -- beam search's selection (corun_beam_select): the best continuations
// of a group's rows by one token, of score s + l_v - log sum_u exp(l_u).
//
// Two launches.  k_beam_part reads the logits once, a part of a row to a
// workgroup, and leaves the part's maximum, its sum of exp(l - maximum) in 64
// bits, and its `keep` largest logits in order.  Within a row the order of the
// scores is that of the logits, so the best of a group are among these;
// k_beam_pick, a workgroup to a group, forms the rows' log-sums and scores in 64
// bits and sorts them out.
//
// Neither sorts what cannot be chosen.  A lower bound of the keep-th largest
// value comes from bisection over few values (the threads' maxima, or the
// lists' heads), some one to two times `keep` candidates reach it, and each finds
// its place by counting those before it.  Sums and places are in a fixed order,
// whatever the order in which candidates were noted.
//
// k_beam_part: 195 live rows of 151936 logits, 118 MB, in 37 us, 3.2 TB/s (a copy
// reaches 5.1).  Its vector arithmetic alone is some 25 us, most of it the exponentials
// in 64 bits (19 instructions for each logit); the rest is waiting for loads and for
// the part's other wavefronts.  Parts of 4096 columns came out the same (39 us), a
// workgroup that loads its next part while it works on this one slower (58 us for
// the whole call, 47 so): its registers leave fewer wavefronts.
// k_beam_pick: 7 us for 64 groups of 4 rows and 4 results, 11 for 4 groups of 32 rows
// and 64 results: a chain of dependent loads and barriers.  A lane's first five parts
// are read at once (75 parts to a row: 6.5 us, 8.1 with two at a time).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "device.h"
#include "groups.h"

namespace corun {
namespace {

// The workspace: of each part of each row its maximum, its sum, and its best
// logits and their columns (-1: none), [rows][parts][keep].
struct Best {
    double *sum;
    float *top;
    float *logit;
    int32_t *col;
};
constexpr int CAP = 1024;                              // candidates that a part sorts at once
constexpr int MOST = 4096;                             // the same of a group

// Rising unsigned keys of floating-point values that are no NaN, the same for both
// zeros, and back.
__device__ __forceinline__ uint32_t key32(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key32(uint32_t k)
{
    return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu));
}
__device__ __forceinline__ uint32_t key_high(double x)   // of the upper half: order kept, ties added; never 0
{
    const uint32_t u = (uint32_t)__double2hiint(x + 0.0);
    return max(u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u), 1u);
}

// exp(d) of d in [-700, 0], 64 bits, relative error below 1e-15 down to -40 and 1.1e-14
// down to -700, and exactly 1 at 0: 2^(n + f) with n the nearest whole number, 2^f by the
// polynomial of degree 10 that meets it at the Chebyshev points of [-1/2, 1/2], of which
// 0 is one (relative error 3.2e-16).  A row whose mask leaves one token so keeps its
// score to the bit, and its ties with finished rows.  Adding 1.5 2^52 leaves n in the
// low bits, so nothing but additions and multiplications is needed.
__device__ __forceinline__ double exp_neg(double d)
{
    const double magic = 6755399441055744.0, log2e = 1.4426950408889634074;
    const double z = __builtin_fma(d, log2e, magic);
    const double f = __builtin_fma(d, log2e, magic - z);
    double p = 7.0725859492692234e-09;
    p = __builtin_fma(p, f, 1.0208690299958306e-07);
    p = __builtin_fma(p, f, 1.3215442587921689e-06);
    p = __builtin_fma(p, f, 1.5252657260200837e-05);
    p = __builtin_fma(p, f, 1.5403530441736050e-04);
    p = __builtin_fma(p, f, 1.3333558230164974e-03);
    p = __builtin_fma(p, f, 9.6181291076068882e-03);
    p = __builtin_fma(p, f, 5.5504108664447722e-02);
    p = __builtin_fma(p, f, 2.4022650695910097e-01);
    p = __builtin_fma(p, f, 6.9314718055994995e-01);
    p = __builtin_fma(p, f, 1.0);
    return __hiloint2double(__double2hiint(p) + (__double2loint(z) << 20), __double2loint(p));
}
// exp(x - top), what is below exp(-700) as that
__device__ __forceinline__ double exp_under(float x, float top)
{
    return exp_neg(fmax((double)x - (double)top, -700.0));
}
// Lanes' places behind `base` where `on`, in lane order.
__device__ __forceinline__ int place_of(unsigned long long on, int base)
{
    return base + __builtin_amdgcn_mbcnt_hi((uint32_t)(on >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)on, 0));
}

// A wavefront's reduction by a commutative operation, the same bits in every lane:
// lanes' neighbours by data-parallel moves (pairs, quads, eights, sixteens), then
// the swaps of halves.
template <int CTRL>
__device__ __forceinline__ uint32_t moved(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, false);
}
template <int CTRL>
__device__ __forceinline__ float moved(float x) { return __uint_as_float(moved<CTRL>(__float_as_uint(x))); }
template <int CTRL>
__device__ __forceinline__ double moved(double x)
{
    return __hiloint2double((int)moved<CTRL>((uint32_t)__double2hiint(x)), (int)moved<CTRL>((uint32_t)__double2loint(x)));
}
// the value of the other half of 32 (HALF 16) or 64 lanes (HALF 32)
template <int HALF>
__device__ __forceinline__ uint32_t other(uint32_t x)
{
    const bool upper = threadIdx.x & HALF;
    if constexpr (HALF == 16) {
        const auto two = __builtin_amdgcn_permlane16_swap(x, x, false, false);
        return upper ? two[0] : two[1];
    } else {
        const auto two = __builtin_amdgcn_permlane32_swap(x, x, false, false);
        return upper ? two[0] : two[1];
    }
}
template <int HALF>
__device__ __forceinline__ float other(float x) { return __uint_as_float(other<HALF>(__float_as_uint(x))); }
template <int HALF>
__device__ __forceinline__ double other(double x)
{
    return __hiloint2double((int)other<HALF>((uint32_t)__double2hiint(x)), (int)other<HALF>((uint32_t)__double2loint(x)));
}
template <class T, class F>
__device__ __forceinline__ T over_wave(T x, F &&f)
{
    x = f(x, moved<0xB1>(x));                          // quad_perm [1, 0, 3, 2]
    x = f(x, moved<0x4E>(x));                          // quad_perm [2, 3, 0, 1]
    x = f(x, moved<0x141>(x));                         // row_half_mirror
    x = f(x, moved<0x140>(x));                         // row_mirror
    x = f(x, other<16>(x));
    return f(x, other<32>(x));
}
template <class T, class F>
__device__ __forceinline__ T over_row(T x, F &&f)          // of sixteen lanes
{
    x = f(x, moved<0xB1>(x));
    x = f(x, moved<0x4E>(x));
    x = f(x, moved<0x141>(x));
    return f(x, moved<0x140>(x));
}
template <class T>
__device__ __forceinline__ T wave_max(T x) { return over_wave(x, [](T a, T b) { return a > b ? a : b; }); }
template <class T>
__device__ __forceinline__ T wave_min(T x) { return over_wave(x, [](T a, T b) { return a < b ? a : b; }); }
__device__ __forceinline__ double wave_sum(double x) { return over_wave(x, [](double a, double b) { return a + b; }); }

enum { NONE = 0, LIVE, DONE };
__device__ __forceinline__ int row_kind(const BeamArgs &a, int r)
{
    const uint8_t *v = a.valid, *f = a.finished;       // both loads in flight together
    const int live = v == nullptr ? 1 : v[r], done = f == nullptr ? 0 : f[r];
    return live == 0 ? NONE : done != 0 ? DONE : LIVE;
}

// A part: 1024 J columns, 4 J to a thread, in registers.
template <int J>
__global__ __launch_bounds__(256) void k_beam_part(BeamArgs a, Best b, int parts)
{
    typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));
    __shared__ uint32_t maxima[256];
    __shared__ double wsum[4];
    __shared__ float wtop[4];
    __shared__ unsigned long long cand[CAP];           // key of the logit, then the column, lower ones larger
    __shared__ int count, wat[4];
    __shared__ float bound;
    const int part = blockIdx.x, r = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = a.keep;
    const float *row = a.logits + (size_t)r * a.ld;
    const int first = part * 1024 * J + 4 * tid;
    float x[4 * J];
    const auto load = [&]() {
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int c = first + 1024 * j;
            if (c + 4 <= a.vocab) {
                const f4u v = *(const f4u *)(row + c);
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * j + e] = v[e];
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[4 * j + e] = c + e < a.vocab ? row[c + e] : -INFINITY;
            }
        }
    };
    if (J == 2) load();                                // few workgroups: ahead of the row's flags
    if (row_kind(a, r) != LIVE) return;
    if (J != 2) load();
    float mine = x[0];
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 4 * J; i += 2) {
        mine = fmaxf(mine, fmaxf(x[i], x[i + 1]));
        nan |= __builtin_isunordered(x[i], x[i + 1]);
    }
    if (mine != mine) mine = -INFINITY;
    float top = wave_max(mine);
    if (lane == 0) wtop[wave] = top;
    maxima[tid] = key32(mine);
    if (tid == 0) count = 0;
    __syncthreads();
    top = fmaxf(fmaxf(wtop[0], wtop[1]), fmaxf(wtop[2], wtop[3]));

    // wavefront 0: a bound that at least K threads' maxima reach, and not many more
    if (wave == 0) {
        uint32_t m[4], lo = 0xffffffffu, hi;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            m[i] = maxima[64 * i + lane];
            lo = min(lo, m[i]);
        }
        lo = __builtin_amdgcn_readfirstlane(wave_min(lo));
        hi = __builtin_amdgcn_readfirstlane(key32(top)) + 1;
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            int n = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) n += __popcll(__ballot(m[i] >= mid));
            if (n >= K) lo = mid;
            else hi = mid;
            if (n >= K && n <= K + K / 2) break;
        }
        if (lane == 0) bound = fmaxf(of_key32(lo), -3.4028234663852886e38f);   // -inf is no candidate
    }
    // the others go on with the sum
    double s = 0;
    if (top > -INFINITY) {
#pragma unroll
        for (int i = 0; i < 4 * J; ++i) s += exp_under(x[i], top);
    }
    if (nan || top == INFINITY) s = __builtin_nan("");
    s = wave_sum(s);
    if (lane == 0) wsum[wave] = s;
    __syncthreads();
    const size_t at = (size_t)r * parts + part;
    if (tid == 0) {
        b.top[at] = top;
        b.sum[at] = wsum[0] + wsum[1] + wsum[2] + wsum[3];
    }
    // a wavefront's candidates are noted side by side
    const float least = bound;
    unsigned long long on[4 * J];
    int noted = 0;
#pragma unroll
    for (int i = 0; i < 4 * J; ++i) {
        on[i] = __ballot(x[i] >= least);
        noted += __popcll(on[i]);
    }
    int base = 0;
    if (lane == 0 && noted > 0) base = atomicAdd(&count, noted);
    base = __builtin_amdgcn_readfirstlane(base);
#pragma unroll
    for (int i = 0; i < 4 * J; ++i) {
        if (on[i] == 0) continue;
        const int n = place_of(on[i], base);
        if (x[i] >= least && n < CAP)
            cand[n] = (unsigned long long)key32(x[i]) << 32 | ~(uint32_t)(first + 1024 * (i / 4) + i % 4);
        base += __popcll(on[i]);
    }
    __syncthreads();
    const int n = count;
    float *logit = b.logit + at * K;
    int32_t *col = b.col + at * K;
    if (n <= CAP) {
        // 2^sub threads count for one candidate
        const int sub = n <= 32 ? 3 : n <= 64 ? 2 : n <= 128 ? 1 : 0;
        for (int i = tid >> sub; i < n; i += 256 >> sub) {
            const unsigned long long c = cand[i];
            int place = 0;
#pragma unroll 4
            for (int k = tid & ((1 << sub) - 1); k < n; k += 1 << sub) place += cand[k] > c;
            for (int o = 1; o < 1 << sub; o <<= 1) place += __shfl_xor(place, o, 64);
            if (place < K && (tid & ((1 << sub) - 1)) == 0) {
                logit[place] = of_key32((uint32_t)(c >> 32));
                col[place] = (int)~(uint32_t)c;
            }
        }
        for (int i = n + tid; i < K; i += 256) col[i] = -1;
        return;
    }
    // many equal ones: the largest behind the last, K times
    float last = INFINITY;
    int last_at = -1;
    for (int k = 0; k < K; ++k) {
        float v = -INFINITY;
        int c = INT32_MAX;
#pragma unroll
        for (int i = 0; i < 4 * J; ++i) {
            const int here = first + 1024 * (i / 4) + i % 4;
            if ((x[i] < last || (x[i] == last && here > last_at)) && x[i] > v) {
                v = x[i];
                c = here;
            }
        }
        for (int o = 32; o; o >>= 1) {
            const float w = __shfl_xor(v, o, 64);
            const int d = __shfl_xor(c, o, 64);
            if (w > v || (w == v && d < c)) {
                v = w;
                c = d;
            }
        }
        __syncthreads();
        if (lane == 0) {
            wtop[wave] = v;
            wat[wave] = c;
        }
        __syncthreads();
        for (int w = 0; w < 4; ++w)
            if (wtop[w] > v || (wtop[w] == v && wat[w] < c)) {
                v = wtop[w];
                c = wat[w];
            }
        if (tid == 0) {
            logit[k] = v;
            col[k] = c == INT32_MAX ? -1 : c;
        }
        last = v;
        last_at = c;
    }
}

// A candidate of a group: better(x, y) is the order of the results.
struct Candidate {
    double rank;
    int row;
    float logit;
    int col;
};
__device__ __forceinline__ bool better(const Candidate &x, const Candidate &y)
{
    if (x.rank != y.rank) return x.rank > y.rank;
    if (x.row != y.row) return x.row < y.row;
    if (x.logit != y.logit) return x.logit > y.logit;
    return x.col < y.col;
}

// One group.  Items are all of the group's entries, or where these are more than
// 4 T, its lists' heads; then the lists of those that reach the bound are read.
// The launch has few workgroups, and most of its time is waiting for loads that
// depend on one another and for instructions, so loops are left rolled.
template <int T>
__global__ __launch_bounds__(T) void k_beam_pick(BeamArgs a, Best b, int parts)
{
    constexpr int W = T / 64, LPT = 4, ROOM = MOST, NEAR = 8, HELD = 5;
    __shared__ double lse[MOST_BEAMS], score[MOST_BEAMS], weight[MOST_BEAMS];
    __shared__ int kind[MOST_BEAMS], wn[2][W], wi[W], count, selected, longer;
    __shared__ uint32_t wlo[W], whi[W];
    __shared__ double crank[ROOM], wr[W];
    __shared__ float clogit[ROOM];
    __shared__ int crow[ROOM], ccol[ROOM], sel[LPT * T], rest[LPT * T];
    const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = a.keep;
    if (tid == 0) count = selected = longer = 0;
    // the items' logits and columns, in flight while the rows' sums are formed
    const int lists = a.beams * parts;
    const bool all = lists * K <= LPT * T;
    const int items = all ? lists * K : lists;         // at most LPT T
    Candidate item[LPT];
#pragma unroll
    for (int m = 0; m < LPT; ++m) {
        const size_t i = min(tid + T * m, items - 1);
        const size_t at = (size_t)g * lists * K + (all ? i : i * K);
        item[m].logit = b.logit[at];
        item[m].col = b.col[at];
    }
    // rows' log-sums: sixteen lanes to a row
    for (int i = tid >> 4; i < a.beams; i += T / 16) {
        const int r = g * a.beams + i, l16 = tid & 15;
        const float *top = b.top + (size_t)r * parts;
        const double *sum = b.sum + (size_t)r * parts;
        int k = row_kind(a, r);
        const double w = a.weights == nullptr ? 1.0 : (double)a.weights[r];
        const float s = a.scores[r];
        float most = -INFINITY, t0[HELD];
        double x0[HELD];
#pragma unroll
        for (int j = 0; j < HELD; ++j) {
            const int p = l16 + 16 * j;
            t0[j] = -INFINITY;
            x0[j] = 0;
            if (p < parts) {
                t0[j] = top[p];
                x0[j] = sum[p];
            }
        }
#pragma unroll
        for (int j = 0; j < HELD; ++j) most = fmaxf(most, t0[j]);
        for (int p = l16 + 16 * HELD; p < parts; p += 16) most = fmaxf(most, top[p]);
        most = over_row(most, [](float x, float y) { return x > y ? x : y; });
        double total = 0;
#pragma unroll
        for (int j = 0; j < HELD; ++j)
            if (16 * j < parts) total += t0[j] > -INFINITY || x0[j] != x0[j] ? x0[j] * exp_under(t0[j], most) : 0.0;
#pragma unroll 2
        for (int p = l16 + 16 * HELD; p < parts; p += 16) {
            const float t = top[p];
            const double x = sum[p];
            total += t > -INFINITY || x != x ? x * exp_under(t, most) : 0.0;
        }
        total = over_row(total, [](double x, double y) { return x + y; });
        const double l = k == LIVE ? (double)most + log(total) : 0.0;
        // NaN or +inf among the logits, nothing but -inf, or a score or weight that is none
        if (!(w > 0 && w < INFINITY) || !(fabsf(s) < INFINITY) || !(fabs(l) < INFINITY)) k = NONE;
        if (l16 == 0) {
            lse[i] = l;
            score[i] = (double)s;
            weight[i] = w;
            kind[i] = k;
        }
    }
    __syncthreads();
    // completes a candidate, of which the logit and column are there: entry j of a list
    const auto complete = [&](int list, int j, Candidate &c) -> bool {
        const int i = list / parts;
        c.row = i;
        if (kind[i] == NONE) return false;
        double s = score[i];
        if (kind[i] == DONE) {
            if (j > 0 || list % parts > 0) return false;
            c.col = a.end_token;
            c.logit = 0.f;
        } else {
            if (c.col < 0) return false;
            s += (double)c.logit - lse[i];
        }
        c.rank = s * weight[i];
        return fabs(s) < INFINITY && fabs(c.rank) < INFINITY;
    };
    const auto entry = [&](int list, int j, Candidate &c) -> bool {
        const size_t at = ((size_t)g * lists + list) * K + j;
        c.logit = b.logit[at];
        c.col = b.col[at];
        return complete(list, j, c);
    };
    uint32_t key[LPT], lo = 0xffffffffu, hi = 0;
    int present = 0;
#pragma unroll
    for (int m = 0; m < LPT; ++m) {
        key[m] = 0u;
        if (T * m >= items) continue;
        const int i = tid + T * m;
        Candidate &c = item[m];
        const bool is = i < items && complete(all ? i / K : i, all ? i % K : 0, c);
        key[m] = is ? key_high(c.rank) : 0u;
        if (is) {
            lo = min(lo, key[m]);
            hi = max(hi, key[m]);
        }
        present += __popcll(__ballot(is));
    }
    lo = wave_min(lo);
    hi = wave_max(hi);
    if (lane == 0) {
        wlo[wave] = lo;
        whi[wave] = hi;
        wn[0][wave] = present;
    }
    __syncthreads();
    present = 0;
    for (int w = 0; w < W; ++w) {
        lo = min(lo, wlo[w]);
        hi = max(hi, whi[w]);
        present += wn[0][w];
    }
    if (present < K) lo = 1;                           // all of them
    else {
        ++hi;
#pragma unroll 1
        for (int step = 1; hi - lo > 1; ++step) {
            const uint32_t mid = lo + (hi - lo) / 2;
            int n = 0;
#pragma unroll
            for (int m = 0; m < LPT; ++m) n += __popcll(__ballot(key[m] >= mid));
            if (lane == 0) wn[step & 1][wave] = n;
            __syncthreads();
            n = 0;
            for (int w = 0; w < W; ++w) n += wn[step & 1][w];
            if (n >= K) lo = mid;
            else hi = mid;
            if (n >= K && n <= K + K / 2) break;
        }
    }
    const auto note = [&](const Candidate &c) {
        const int n = atomicAdd(&count, 1);
        if (n >= ROOM) return;
        crank[n] = c.rank;
        crow[n] = c.row;
        clogit[n] = c.logit;
        ccol[n] = c.col;
    };
#pragma unroll
    for (int m = 0; m < LPT; ++m) {
        if (key[m] < lo) continue;
        if (all) note(item[m]);
        else sel[atomicAdd(&selected, 1)] = tid + T * m;
    }
    __syncthreads();
    if (!all) {
        // the first entries of the lists whose heads reach the bound; where all of
        // these do, the others
        const int ns = selected;
#pragma unroll 1
        for (int i = tid; i < ns * NEAR; i += T) {
            const int j = i % NEAR, list = sel[i / NEAR];
            Candidate c;
            if (j >= K || !entry(list, j, c) || key_high(c.rank) < lo) continue;
            note(c);
            if (j == NEAR - 1) rest[atomicAdd(&longer, 1)] = list;
        }
        __syncthreads();
        const int nl = longer;
#pragma unroll 1
        for (int i = wave; i < nl; i += W) {
            const int j = NEAR + lane;
            Candidate c;
            if (j < K && entry(rest[i], j, c) && key_high(c.rank) >= lo) note(c);
        }
        __syncthreads();
    }
    const int n = count;
    const auto result = [&](int place, const Candidate &c, bool any) {
        const size_t o = (size_t)g * K + place;
        double s = 0;
        if (any) {
            s = score[c.row];
            if (kind[c.row] == LIVE) s += (double)c.logit - lse[c.row];
        }
        a.tokens[o] = any ? c.col : -1;
        a.parents[o] = any ? g * a.beams + c.row : -1;
        a.out_scores[o] = any ? (float)s : -INFINITY;
        if (a.out_finished != nullptr) a.out_finished[o] = any && (kind[c.row] == DONE || c.col == a.end_token);
    };
    if (n <= ROOM) {
        // 2^sub threads count for one candidate
        const int sub = n <= T / 16 ? 4 : n <= T / 8 ? 3 : n <= T / 4 ? 2 : 0, mine = tid & ((1 << sub) - 1);
#pragma unroll 1
        for (int i = tid >> sub; i < n; i += T >> sub) {
            const Candidate c{crank[i], crow[i], clogit[i], ccol[i]};
            int place = 0;
#pragma unroll 2
            for (int k = mine; k < n; k += 1 << sub) {
                const double x = crank[k];
                if (x > c.rank) ++place;
                else if (x == c.rank) place += better({x, crow[k], clogit[k], ccol[k]}, c);
            }
            for (int o = 1; o < 1 << sub; o <<= 1) place += __shfl_xor(place, o, 64);
            if (place < K && mine == 0) result(place, c, true);
        }
        for (int i = n + tid; i < K; i += T) result(i, {}, false);
        return;
    }
    // many equal ones: the best behind the last, K times, over all entries
    Candidate last{INFINITY, -1, INFINITY, -1};
#pragma unroll 1
    for (int k = 0; k < K; ++k) {
        Candidate best{-INFINITY, INT32_MAX, 0.f, INT32_MAX};
#pragma unroll 1
        for (int i = tid; i < lists; i += T) {
            Candidate c;
#pragma unroll 1
            for (int j = 0; j < K && entry(i, j, c); ++j)
                if (better(last, c)) {
                    if (better(c, best)) best = c;
                    break;                             // a list is in order
                }
        }
        for (int o = 32; o; o >>= 1) {
            const Candidate c{__shfl_xor(best.rank, o, 64), __shfl_xor(best.row, o, 64), __shfl_xor(best.logit, o, 64),
                              __shfl_xor(best.col, o, 64)};
            if (better(c, best)) best = c;
        }
        __syncthreads();
        if (lane == 0) {
            wr[wave] = best.rank;
            wi[wave] = best.row;
            clogit[wave] = best.logit;
            ccol[wave] = best.col;
        }
        __syncthreads();
        for (int w = 0; w < W; ++w) {
            const Candidate c{wr[w], wi[w], clogit[w], ccol[w]};
            if (better(c, best)) best = c;
        }
        if (tid == 0) result(k, best, best.row != INT32_MAX);
        last = best;
    }
}

// Columns of a part: 2048 where larger ones would leave workgroups for half of
// the chip only, 8192 else.
int columns(int vocab, int groups, int beams)
{
    const long long big = (vocab + 8191) / 8192, small = (vocab + 2047) / 2048;
    return big * groups * beams < 512 && small * beams <= 1024 ? 2048 : 8192;
}

}  // namespace

size_t beam_ws(int vocab, int groups, int beams, int keep)
{
    const int per = columns(vocab, groups, beams);
    const size_t n = (size_t)groups * beams * ((vocab + per - 1) / per);
    return n * 12 + n * keep * 8;
}

hipError_t launch_beam_select(const BeamArgs &a, void *ws, hipStream_t st)
{
    const int per = columns(a.vocab, a.groups, a.beams), parts = (a.vocab + per - 1) / per;
    const size_t n = (size_t)a.groups * a.beams * parts;
    Best b;
    b.sum = (double *)ws;
    b.top = (float *)(b.sum + n);
    b.logit = b.top + n;
    b.col = (int32_t *)(b.logit + n * a.keep);
    const dim3 grid(parts, a.groups * a.beams);
    if (per == 2048) KLAUNCH(k_beam_part<2>, grid, dim3(256), 0, st, a, b, parts);
    else KLAUNCH(k_beam_part<8>, grid, dim3(256), 0, st, a, b, parts);
    if (a.beams <= 8 && a.beams * parts <= 1024) KLAUNCH(k_beam_pick<256>, dim3(a.groups), dim3(256), 0, st, a, b, parts);
    else KLAUNCH(k_beam_pick<1024>, dim3(a.groups), dim3(1024), 0, st, a, b, parts);
    return hipGetLastError();
}

}  // namespace corun
