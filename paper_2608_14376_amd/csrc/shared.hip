// shared.hip -- attention of a decode step whose rows share prefixes
// (corun_shared_attention).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "device.h"
#include "groups.h"

namespace corun {
namespace {

// What row r sees: n tokens, the first `prefix` of them of slot `slot`.  n < 0: the
// row's lengths are out of the launch's range.
struct Seen {
    int n, prefix, slot;
};
__device__ __forceinline__ int group_of(const GroupTable &g, int r)
{
    int lo = 0, hi = g.n - 1;                          // the last group whose first row is at or before r
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (g.row0[mid] <= r) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}
__device__ __forceinline__ Seen seen_by(const SharedArgs &a, const GroupTable &g, const CacheView &cv, int gi, int r)
{
    const int p = a.prefix_lens[gi], n = a.lens[r], slot = a.prefix_slots == nullptr ? g.row0[gi] : a.prefix_slots[gi];
    if (a.valid != nullptr && a.valid[r] == 0) return {0, 0, 0};
    const bool bad = p < 0 || p > a.max_prefix || (unsigned)slot >= (unsigned)cv.n_slots || n < p ||
                     (long long)n > (long long)p + a.max_suffix || n > cv.cap;
    return {bad ? -1 : n, p, slot};
}

// One wavefront to a (row, query head), 64 tokens at a time: a token to a lane
// for the scores, then D / 64 dimensions to a lane.
template <int D>
__global__ __launch_bounds__(64) void k_shared_rows(SharedArgs a, GroupTable gt, CacheView cv, CacheLayer cl)
{
    constexpr int E = D / 64;
    const int lane = threadIdx.x, h = blockIdx.x, r = blockIdx.y, nkv = a.nkv, kvh = h / (a.nq / nkv);
    const Seen s = seen_by(a, gt, cv, group_of(gt, r), r);
    uint16_t *out = a.out + (size_t)r * a.ldo + (size_t)h * D + E * lane;
    const uint16_t *q = a.q + (size_t)r * a.ldq + (size_t)h * D;
    if (s.n <= 0) {
        for (int e = 0; e < E; ++e) out[e] = s.n < 0 ? (uint16_t)0x7fc0 : (uint16_t)0;
        return;
    }
    const float scale = 1.0f / sqrtf((float)D);
    float m = -INFINITY, l = 0.f, acc[E] = {};
    bool lost = false;
    for (int b = 0; b < s.n; b += 64) {
        const int t = min(b + lane, s.n - 1), slot = t < s.prefix ? s.slot : r;
        size_t row, blk = 0;
        if (cv.kv.layout == 1) {
            const int ps = cv.kv.page_size;
            int page = cv.kv.page_table[(size_t)slot * cv.kv.max_pages_per_seq + t / ps];
            if ((unsigned)page >= (unsigned)cv.num_pages) {
                lost = true;
                page = 0;
            }
            const size_t head = (size_t)page * nkv + kvh;
            row = head * ps + t % ps;
            blk = head * (ps >> cv.blk_shift) + (t % ps >> cv.blk_shift);
        } else {
            const size_t head = (size_t)slot * nkv + kvh;
            row = head * cv.kv.max_seq_len + t;
            blk = head * (cv.kv.max_seq_len >> cv.blk_shift) + (t >> cv.blk_shift);
        }
        float ksc = 1.f, vsc = 1.f;
        if (cv.e4m3) {
            ksc = __uint_as_float((uint32_t)cl.ks[blk] << 23);
            vsc = __uint_as_float((uint32_t)cl.vs[blk] << 23);
        }
        const auto value = [&](const void *base, size_t i) {
            return cv.e4m3 ? __builtin_amdgcn_cvt_f32_fp8(((const uint8_t *)base)[i], 0) : bf2f(((const uint16_t *)base)[i]);
        };
        float sc = 0.f;
#pragma unroll 1
        for (int i = 0; i < D; ++i) sc += bf2f(q[i]) * value(cl.k, row * D + i);
        sc *= ksc * scale;
        const bool on = b + lane < s.n;
        float mt = on ? sc : -INFINITY;
        for (int o = 32; o; o >>= 1) mt = fmaxf(mt, __shfl_xor(mt, o, 64));
        const float mn = fmaxf(m, mt), off = mn == -INFINITY ? 0.f : mn;
        const float al = __expf(m - off), pe = on ? __expf(sc - off) : 0.f;
        float sum = pe;
        for (int o = 32; o; o >>= 1) sum += __shfl_xor(sum, o, 64);
        l = l * al + sum;
        m = mn;
        for (int e = 0; e < E; ++e) acc[e] *= al;
        for (int i = 0; i < min(64, s.n - b); ++i) {
            const float w = __shfl(pe, i, 64), vs = __shfl(vsc, i, 64);
            const size_t vr = __shfl((unsigned long long)row, i, 64);
            for (int e = 0; e < E; ++e) acc[e] += w * (value(cl.v, vr * D + E * lane + e) * vs);
        }
    }
    lost = __ballot(lost) != 0ull;
    for (int e = 0; e < E; ++e) out[e] = f2bf(lost ? __builtin_nanf("") : acc[e] / l);
}

}  // namespace

size_t shared_ws(const GroupTable &, int, int, int, int, int) { return 0; }

hipError_t launch_shared(const SharedArgs &a, const GroupTable &g, const CacheView &cv, const CacheLayer &cl, float *,
                         hipStream_t st)
{
    const dim3 grid(a.nq, g.row0[g.n]);
    if (a.d == 128) KLAUNCH(k_shared_rows<128>, grid, dim3(64), 0, st, a, g, cv, cl);
    else if (a.d == 64) KLAUNCH(k_shared_rows<64>, grid, dim3(64), 0, st, a, g, cv, cl);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}

}  // namespace corun
