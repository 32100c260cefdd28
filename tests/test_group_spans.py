"""Which tokens attention over shared prefixes reads, for every length, slot and
padding flag that a call may hold: the kernels' own functions, compiled for the
host."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

from paper_2608_14376_amd import build, corun
from tests.test_cache_ops import _i32, _kv

SOURCE = """#include "groups.h"
using namespace corun;
extern "C" void spans(int n, const int *in, int *out)
{
    for (int i = 0; i < n; ++i, in += 11, out += 8) {
        // valid, len, prefix, slot, max_prefix, max_suffix, cap, n_slots, chunk, split, row
        const Prefix p = prefix_within(in[2], in[3], in[4], in[7]);
        const int m = tokens_within(p, in[1], in[0], in[5], in[6]);
        const Span a = prefix_span(p, in[8], in[9]), b = own_span(p, in[10], m, in[8], in[9]);
        const int all[8] = {p.len, m, a.slot, a.t_lo, a.t_end, b.slot, b.t_lo, b.t_end};
        for (int k = 0; k < 8; ++k) out[k] = all[k];
    }
}
"""


@pytest.fixture(scope="module")
def spans(tmp_path_factory):
    where = tmp_path_factory.mktemp("spans")
    src, lib = where / "spans.cpp", where / "spans.so"
    src.write_text(SOURCE)
    subprocess.run([build.HIPCC, *build.FLAGS, "-shared", "-x", "hip", str(src), "-I", build.CSRC,
                    "-I", os.path.join(build.ROOT, "include"), "-o", str(lib)], check=True)
    call = ctypes.CDLL(str(lib)).spans

    def of(rows):
        x = np.ascontiguousarray(rows, np.int32)
        out = np.zeros((len(x), 8), np.int32)
        call(len(x), x.ctypes.data_as(ctypes.c_void_p), out.ctypes.data_as(ctypes.c_void_p))
        return out
    return of


FAR = (-(1 << 31), -(1 << 30), (1 << 31) - 1)


def grid(*axes):
    return np.stack([a.reshape(-1) for a in np.meshgrid(*axes, indexing="ij")], 1)


@pytest.mark.parametrize("cap,max_prefix,max_suffix,chunk", [(192, 192, 192, 128), (192, 100, 70, 128), (64, 1, 64, 32)])
def test_spans_stay_within_the_cache(spans, cap, max_prefix, max_suffix, chunk):
    slots = 3
    lens = [*range(-20, cap + 20, 3), 0, 1, cap - 1, cap, cap + 1, *FAR]
    prefix = [-17, -16, -15, -2, -1, 0, 1, 15, 16, 17, 31, 33, 63, 64, 99, 100, 101, cap - 1, cap, cap + 1, *FAR]
    splits = range(-(-(cap + 15) // chunk))
    x = grid([0, 1], lens, prefix, [-5, -1, 0, slots - 1, slots, *FAR], [max_prefix], [max_suffix], [cap], [slots], [chunk],
             splits, [2])
    p, n, ps, pa, pb, rs, ra, rb = spans(x).T
    valid, length, pre, slot = x[:, 0], x[:, 1], x[:, 2], x[:, 3]
    good = (pre >= 0) & (pre <= max_prefix) & (slot >= 0) & (slot < slots)
    assert np.array_equal(p, np.where(good, pre, -1))
    fits = good & (length >= pre) & (length.astype(np.int64) - pre <= max_suffix) & (length <= cap)
    assert np.array_equal(n, np.where(valid == 0, 0, np.where(fits, length, -1)))
    reads = pa < pb
    assert not (reads & ~good).any() and (pa[reads] >= 0).all() and (pb[reads] <= pre[reads]).all()
    assert (ps[reads] == slot[reads]).all() and (pb - pa)[reads].max() <= chunk
    reads = ra < rb
    assert not (reads & ~(good & fits & (valid != 0))).any(), x[reads & ~(good & fits & (valid != 0))][0]
    assert (ra[reads] >= pre[reads]).all() and (rb[reads] <= length[reads]).all() and (rs[reads] == 2).all()
    assert (rb - ra)[reads].max() <= chunk
    # over all splits every token once
    each = x[:, 9].max() + 1
    own = np.where(ra < rb, rb - ra, 0).reshape(-1, each).sum(1)
    first = slice(None, None, each)
    assert np.array_equal(own, np.where(good & fits & (valid != 0), length - pre, 0)[first])
    assert np.array_equal(np.where(pa < pb, pb - pa, 0).reshape(-1, each).sum(1), np.where(good, pre, 0)[first])


def test_spans_of_the_farthest_tokens(spans):
    """Lengths up to 2^30, splits of up to 2^30 tokens: no sum wraps."""
    cap = 1 << 30
    x = grid([1], [cap, cap - 1, cap - 16, 5], [cap, cap - 1, cap - 15, cap // 2 + 1, 3, 0], [0], [cap], [cap], [cap], [1],
             [1 << 30, (cap + 15 + 255) // 256 // 128 * 128 + 128], range(256), [0])
    far = x[:, 9].astype(np.int64) * x[:, 8] < cap + 15       # splits that a launch has
    x = x[far]
    p, n, ps, pa, pb, rs, ra, rb = spans(x).T
    t0 = x[:, 9].astype(np.int64) * x[:, 8]
    assert np.array_equal(np.where(pa < pb, pb - pa, 0), np.clip(p - t0, 0, x[:, 8]))
    base = (x[:, 2] & ~15) + t0
    want = np.where(n < 0, 0, np.clip(np.minimum(x[:, 1], base + x[:, 8]) - np.maximum(base, x[:, 2]), 0, None))
    assert np.array_equal(np.where(ra < rb, rb - ra, 0), want)


@pytest.mark.parametrize("groups", [(8, 16, 24, 32), (50, 60)])
@pytest.mark.parametrize("most", [15361, 16000, 20000, 29672, 32768, 65536, 100001, 1 << 20])
def test_prefixes_of_several_groups_take_sixteen_splits_at_most(groups, most):
    """The longest split of a prefix beside others is a fifteenth of it, rounded down: read off the workspace, whose parts
    are [splits][kv heads][blocks of 32 queries][32 (d + 2)] floats, one split of them for 16 tokens of a row's own."""
    nq, nkv, d = 64, 8, 128
    kv = _kv(n_slots=sum(groups), max_seq_len=1 << 20)
    size = corun.load().corun_shared_attention_workspace(ctypes.addressof(kv), nq, nkv, d, len(groups), _i32(*groups), most, 1)
    blocks = sum(-(-n * (nq // nkv) // 32) for n in groups)
    splits, rest = divmod(size, nkv * blocks * 32 * (d + 2) * 4)
    assert rest == 0 and 12 <= splits - 1 <= 16
