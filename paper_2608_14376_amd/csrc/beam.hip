// beam.hip -- beam search's selection (corun_beam_select): the best continuations
// of a group's rows by one token.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "device.h"
#include "groups.h"

namespace corun {
namespace {

// The workspace: per row its log-sum, then its best logits and their columns.
struct Best {
    double *lse;                                       // [rows]
    float *logit;                                      // [rows][keep]
    int32_t *col;                                      // [rows][keep], -1: none
};

__device__ __forceinline__ bool row_live(const BeamArgs &a, int r) { return a.valid == nullptr || a.valid[r] != 0; }
__device__ __forceinline__ bool row_done(const BeamArgs &a, int r) { return a.finished != nullptr && a.finished[r] != 0; }

// The larger of (value, lower index) over the workgroup.
template <class T>
__device__ __forceinline__ void wg_best(T &v, int &i, T *lv, int *li)
{
    for (int o = 32; o; o >>= 1) {
        const T w = __shfl_xor(v, o, 64);
        const int j = __shfl_xor(i, o, 64);
        if (w > v || (w == v && j < i)) {
            v = w;
            i = j;
        }
    }
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    __syncthreads();
    if (lane == 0) {
        lv[wave] = v;
        li[wave] = i;
    }
    __syncthreads();
    for (int w = 0; w < 4; ++w)
        if (lv[w] > v || (lv[w] == v && li[w] < i)) {
            v = lv[w];
            i = li[w];
        }
}

__global__ __launch_bounds__(256) void k_beam_rows(BeamArgs a, Best b)
{
    __shared__ float lv[4];
    __shared__ int li[4];
    __shared__ double ls[4];
    const int r = blockIdx.x, tid = threadIdx.x;
    if (!row_live(a, r) || row_done(a, r)) return;
    const float *x = a.logits + (size_t)r * a.ld;
    float top = -INFINITY;
    int at = 0;
    for (int i = tid; i < a.vocab; i += 256) top = fmaxf(top, x[i]);
    wg_best(top, at, lv, li);
    double sum = 0;
    for (int i = tid; i < a.vocab; i += 256) sum += exp((double)x[i] - (double)top);
    for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o, 64);
    if ((tid & 63) == 0) ls[tid >> 6] = sum;
    __syncthreads();
    if (tid == 0) b.lse[r] = (double)top + log(ls[0] + ls[1] + ls[2] + ls[3]);
    float last = INFINITY;
    int last_at = -1;
    for (int k = 0; k < a.keep; ++k) {
        float v = -INFINITY;
        at = INT32_MAX;
        for (int i = tid; i < a.vocab; i += 256) {
            const float y = x[i];
            if ((y < last || (y == last && i > last_at)) && y > v) {
                v = y;
                at = i;
            }
        }
        wg_best(v, at, lv, li);
        if (tid == 0) {
            b.logit[(size_t)r * a.keep + k] = v;
            b.col[(size_t)r * a.keep + k] = at == INT32_MAX ? -1 : at;
        }
        last = v;
        last_at = at;
    }
}

__global__ __launch_bounds__(256) void k_beam_pick(BeamArgs a, Best b)
{
    __shared__ double lv[4];
    __shared__ int li[4];
    const int g = blockIdx.x, tid = threadIdx.x, n = a.beams * a.keep;
    double last = INFINITY;
    int last_at = -1;
    for (int k = 0; k < a.keep; ++k) {
        double best = -INFINITY, best_score = 0;
        int at = INT32_MAX, col = -1, done = 0;
        for (int i = tid; i < n; i += 256) {
            const int r = g * a.beams + i / a.keep, j = i % a.keep;
            if (!row_live(a, r)) continue;
            const double w = a.weights == nullptr ? 1.0 : (double)a.weights[r];
            if (!(w > 0) || isinf(w)) continue;
            double s = a.scores[r];
            int c = a.end_token;
            if (row_done(a, r)) {
                if (j > 0) continue;
            } else {
                c = b.col[(size_t)r * a.keep + j];
                if (c < 0) continue;
                s += (double)b.logit[(size_t)r * a.keep + j] - b.lse[r];
            }
            if (!isfinite(s)) continue;
            const double rank = s * w;
            if ((rank < last || (rank == last && i > last_at)) && rank > best) {
                best = rank;
                at = i;
            }
        }
        wg_best(best, at, lv, li);
        if (tid == 0) {
            const bool any = at != INT32_MAX;
            const int r = any ? g * a.beams + at / a.keep : -1;
            if (any) {
                done = row_done(a, r);
                col = done ? a.end_token : b.col[(size_t)r * a.keep + at % a.keep];
                best_score = (double)a.scores[r];
                if (!done) best_score += (double)b.logit[(size_t)r * a.keep + at % a.keep] - b.lse[r];
            }
            const size_t o = (size_t)g * a.keep + k;
            a.tokens[o] = col;
            a.parents[o] = r;
            a.out_scores[o] = any ? (float)best_score : -INFINITY;
            if (a.out_finished != nullptr) a.out_finished[o] = any && (done || col == a.end_token);
        }
        last = best;
        last_at = at;
    }
}

}  // namespace

size_t beam_ws(int vocab, int groups, int beams, int keep)
{
    const size_t rows = (size_t)groups * beams;
    return rows * 8 + rows * keep * 8;
}

hipError_t launch_beam_select(const BeamArgs &a, void *ws, hipStream_t st)
{
    const size_t rows = (size_t)a.groups * a.beams;
    Best b;
    b.lse = (double *)ws;
    b.logit = (float *)(b.lse + rows);
    b.col = (int32_t *)(b.logit + rows * a.keep);
    KLAUNCH(k_beam_rows, dim3((unsigned)rows), dim3(256), 0, st, a, b);
    KLAUNCH(k_beam_pick, dim3(a.groups), dim3(256), 0, st, a, b);
    return hipGetLastError();
}

}  // namespace corun
