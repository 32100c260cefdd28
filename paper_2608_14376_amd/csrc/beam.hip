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

// Rising unsigned keys of floating-point values, the same for both zeros; NaN has none (0).
__device__ __forceinline__ uint32_t key32(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return x != x ? 0u : u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ uint32_t key_high(double x)   // of the upper half: order kept, ties added
{
    const uint32_t u = (uint32_t)__double2hiint(x + 0.0);
    return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

// exp(d) of d <= 0, 64 bits, relative error below 1e-12: 2^n times the series of
// exp to the tenth power on |x| <= ln(2) / 2 (next term 3e-13).
__device__ __forceinline__ double exp_neg(double d)
{
    const double t = fmax(d * 1.4426950408889634074, -1100.0), n = __builtin_rint(t);
    const double x = (t - n) * 0.69314718055994530942;
    double p = 1.0 / 3628800.0;
    p = __builtin_fma(p, x, 1.0 / 362880.0);
    p = __builtin_fma(p, x, 1.0 / 40320.0);
    p = __builtin_fma(p, x, 1.0 / 5040.0);
    p = __builtin_fma(p, x, 1.0 / 720.0);
    p = __builtin_fma(p, x, 1.0 / 120.0);
    p = __builtin_fma(p, x, 1.0 / 24.0);
    p = __builtin_fma(p, x, 1.0 / 6.0);
    p = __builtin_fma(p, x, 0.5);
    p = __builtin_fma(p, x, 1.0);
    p = __builtin_fma(p, x, 1.0);
    return ldexp(p, (int)n);
}

enum { NONE = 0, LIVE, DONE };
__device__ __forceinline__ int row_kind(const BeamArgs &a, int r)
{
    if (a.valid != nullptr && a.valid[r] == 0) return NONE;
    return a.finished != nullptr && a.finished[r] != 0 ? DONE : LIVE;
}

// A part: 1024 J columns, 4 J to a thread, in registers.
template <int J>
__global__ __launch_bounds__(256) void k_beam_part(BeamArgs a, Best b, int parts)
{
    typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));
    __shared__ uint32_t maxima[256];
    __shared__ double wsum[4];
    __shared__ float cl[CAP], wtop[4];
    __shared__ int cc[CAP];
    __shared__ int count, wat[4];
    __shared__ uint32_t bound;
    const int part = blockIdx.x, r = blockIdx.y, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = a.keep;
    if (row_kind(a, r) != LIVE) return;
    const float *row = a.logits + (size_t)r * a.ld;
    const int first = part * 1024 * J + 4 * tid;
    float x[4 * J];
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
    float mine = -INFINITY;
    bool bad = false;                                  // NaN or +inf: the row has no sum
#pragma unroll
    for (int i = 0; i < 4 * J; ++i) {
        mine = fmaxf(mine, x[i]);
        bad |= !(x[i] < INFINITY);
    }
    float top = mine;
    for (int o = 32; o; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
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
        for (int o = 32; o; o >>= 1) lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64));
        lo = __builtin_amdgcn_readfirstlane(lo);
        hi = __builtin_amdgcn_readfirstlane(key32(top)) + 1;
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            int n = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) n += __popcll(__ballot(m[i] >= mid));
            if (n >= K) lo = mid;
            else hi = mid;
            if (n >= K && n <= 2 * K) break;
        }
        if (lane == 0) bound = lo;
    }
    // the others go on with the sum
    double s = 0;
    if (top > -INFINITY) {
#pragma unroll
        for (int i = 0; i < 4 * J; ++i) s += exp_neg((double)x[i] - (double)top);
    }
    if (bad) s = __builtin_nan("");
    for (int o = 32; o; o >>= 1) s += __shfl_xor(s, o, 64);
    if (lane == 0) wsum[wave] = s;
    __syncthreads();
    const size_t at = (size_t)r * parts + part;
    if (tid == 0) {
        b.top[at] = top;
        b.sum[at] = wsum[0] + wsum[1] + wsum[2] + wsum[3];
    }
    const uint32_t least = max(bound, key32(-INFINITY) + 1);   // -inf is no candidate
#pragma unroll
    for (int i = 0; i < 4 * J; ++i) {
        if (key32(x[i]) >= least) {
            const int n = atomicAdd(&count, 1);
            if (n < CAP) {
                cl[n] = x[i];
                cc[n] = first + 1024 * (i / 4) + i % 4;
            }
        }
    }
    __syncthreads();
    const int n = count;
    float *logit = b.logit + at * K;
    int32_t *col = b.col + at * K;
    if (n <= CAP) {
        for (int i = tid; i < n; i += 256) {
            const float v = cl[i];
            const int c = cc[i];
            int place = 0;
            for (int k = 0; k < n; ++k) place += cl[k] > v || (cl[k] == v && cc[k] < c);
            if (place < K) {
                logit[place] = v;
                col[place] = c;
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
// 4 T, its lists' heads, whose lists are then walked as far as the bound.
template <int T>
__global__ __launch_bounds__(T) void k_beam_pick(BeamArgs a, Best b, int parts)
{
    constexpr int W = T / 64, LPT = 4, ROOM = MOST * T / 1024;
    __shared__ double lse[MOST_BEAMS], score[MOST_BEAMS], weight[MOST_BEAMS];
    __shared__ int kind[MOST_BEAMS], wn[2][W], wi[W], count;
    __shared__ uint32_t wlo[W], whi[W];
    __shared__ double crank[ROOM], wr[W];
    __shared__ float clogit[ROOM];
    __shared__ int crow[ROOM], ccol[ROOM];
    const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, K = a.keep;
    if (tid == 0) count = 0;
    for (int i = wave; i < a.beams; i += W) {
        const int r = g * a.beams + i;
        int k = row_kind(a, r);
        double w = a.weights == nullptr ? 1.0 : (double)a.weights[r], l = 0;
        const double s = a.scores[r];
        if (!(w > 0 && w < INFINITY) || !(fabs(s) < INFINITY)) k = NONE;
        if (k == LIVE) {
            float m = -INFINITY;
            for (int p = lane; p < parts; p += 64) m = fmaxf(m, b.top[(size_t)r * parts + p]);
            for (int o = 32; o; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
            double sum = 0;
            for (int p = lane; p < parts; p += 64) {
                const float t = b.top[(size_t)r * parts + p];
                const double ps = b.sum[(size_t)r * parts + p];
                sum += t > -INFINITY || ps != ps ? ps * exp_neg((double)t - (double)m) : 0.0;
            }
            for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o, 64);
            l = (double)m + log(sum);
            if (!(fabs(l) < INFINITY)) k = NONE;       // NaN or +inf among the logits, or nothing but -inf
        }
        if (lane == 0) {
            lse[i] = l;
            score[i] = s;
            weight[i] = w;
            kind[i] = k;
        }
    }
    __syncthreads();
    const int lists = a.beams * parts;
    const auto entry = [&](int list, int j, Candidate &c) -> bool {
        const int i = list / parts;
        c.row = i;
        if (kind[i] == NONE) return false;
        double s = score[i];
        if (kind[i] == DONE) {
            if (j > 0 || list % parts > 0) return false;
            c.col = a.end_token;
            c.logit = 0.f;
        } else {
            const size_t at = ((size_t)g * lists + list) * K + j;
            c.col = b.col[at];
            c.logit = b.logit[at];
            if (c.col < 0) return false;
            s += (double)c.logit - lse[i];
        }
        c.rank = s * weight[i];
        return fabs(s) < INFINITY && fabs(c.rank) < INFINITY;
    };
    const bool all = lists * K <= LPT * T;
    const int items = all ? lists * K : lists;         // at most LPT T: 64 beams of at most 64 parts
    uint32_t key[LPT], lo = 0xffffffffu, hi = 0;
    int present = 0;
#pragma unroll
    for (int m = 0; m < LPT; ++m) {
        const int i = tid + T * m;
        Candidate c;
        const bool is = i < items && (all ? entry(i / K, i % K, c) : entry(i, 0, c));
        key[m] = is ? max(key_high(c.rank), 1u) : 0u;
        if (is) {
            lo = min(lo, key[m]);
            hi = max(hi, key[m]);
        }
        present += __popcll(__ballot(is));
    }
    for (int o = 32; o; o >>= 1) {
        lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64));
        hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, 64));
    }
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
            if (n >= K && n <= 2 * K) break;
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
        const int i = tid + T * m;
        Candidate c;
        if (all) {
            if (entry(i / K, i % K, c)) note(c);
        } else {
            for (int j = 0; j < K; ++j) {
                if (!entry(i, j, c) || max(key_high(c.rank), 1u) < lo) break;
                note(c);
            }
        }
    }
    __syncthreads();
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
        for (int i = tid; i < n; i += T) {
            const Candidate c{crank[i], crow[i], clogit[i], ccol[i]};
            int place = 0;
            for (int k = 0; k < n; ++k) {
                const double x = crank[k];
                if (x > c.rank) ++place;
                else if (x == c.rank) place += better({x, crow[k], clogit[k], ccol[k]}, c);
            }
            if (place < K) result(place, c, true);
        }
        for (int i = n + tid; i < K; i += T) result(i, {}, false);
        return;
    }
    // many equal ones: the best behind the last, K times, over all entries
    Candidate last{INFINITY, -1, INFINITY, -1};
    for (int k = 0; k < K; ++k) {
        Candidate best{-INFINITY, INT32_MAX, 0.f, INT32_MAX};
        for (int i = tid; i < lists; i += T) {
            Candidate c;
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
    if (a.beams * parts * a.keep <= 1024) KLAUNCH(k_beam_pick<256>, dim3(a.groups), dim3(256), 0, st, a, b, parts);
    else KLAUNCH(k_beam_pick<1024>, dim3(a.groups), dim3(1024), 0, st, a, b, parts);
    return hipGetLastError();
}

}  // namespace corun
