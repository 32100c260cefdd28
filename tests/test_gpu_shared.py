"""Attention over shared prefixes on the GPU against the 64-bit reference: head
layouts, caches, groups, prefixes and suffixes from nothing to long, padding,
what must not be seen, and calls out of range.

Tolerances: cache_reference.attention_bound with weights of at least 16 bits
(2^-14 leaves room for both halves' roundings), or, where a group has over 32
queries of a kv head on an e4m3 cache, of fp16: off by at most half a step, 2^-11,
and as much again as the others for what is far below the largest."""
import numpy as np
import pytest
import torch

from paper_2608_14376_amd import corun
from tests import cache_reference as ref
from tests import group_reference as gref
from tests.cache_reference import HostCache
from tests.test_gpu_cache_ops import rows_of, same

pytestmark = pytest.mark.gpu
DEV = "cuda"
U_WEIGHT = 2.0**-14


def u_weight(hc, q, groups):
    queries = max(groups) * (q.shape[1] // hc.d // hc.nkv)
    return U_WEIGHT + (2.0**-11 if hc.ks is not None and queries > 32 else 0.0)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def run(cache, q, groups, lens, prefix, slots=None, valid=None, most=(0, 0), ws=None, stream=None, out=None):
    nq = q.shape[1] // cache.head_dim
    if out is None:
        out = torch.full((q.shape[0], q.shape[1] + 8), 5.0, dtype=torch.bfloat16, device=DEV)[:, : q.shape[1]]
    if ws is None:
        ws = torch.full((corun.shared_attention_workspace(cache, groups, nq, *most),), 0xFF, dtype=torch.uint8, device=DEV)
    corun.shared_attention(cache, 0, q, groups, i32(lens), i32(prefix), out, ws,
                           prefix_slots=None if slots is None else i32(slots),
                           valid=None if valid is None else torch.tensor(valid, dtype=torch.uint8, device=DEV),
                           max_prefix=most[0], max_suffix=most[1], stream=stream)
    torch.cuda.synchronize()
    return out.cpu()


def check(hc, q, out, groups, lens, prefix, slots, valid=None, rows=None):
    d = hc.d
    of = np.repeat(np.arange(len(groups)), groups)
    for r in range(len(of)) if rows is None else rows:
        got = out[r].double().view(-1, d)
        if valid is not None and not valid[r]:
            assert (got == 0).all()
            continue
        want, pv, size = gref.shared_attention(hc, q[r].double().view(-1, d), r, slots[of[r]], prefix[of[r]], lens[r])
        tol = ref.attention_bound(want, pv, size, d, max(lens[r], 1), u_weight(hc, q, groups))
        err = (got - want).abs()
        assert (err <= tol).all(), (r, float((err / tol.clamp(min=1e-30)).max()), lens[r], prefix[of[r]])


def poison(hc, seen):
    """NaN wherever no row sees a token: seen[slot] = token ranges."""
    off = torch.ones((hc.k.shape[0], hc.k.shape[2]), dtype=torch.bool)
    for slot, spans in seen.items():
        for a, b in spans:
            for t in range(a, b):
                off[hc.at(slot, t)] = False
    for x in (hc.k, hc.v):
        x.transpose(1, 2)[off] = 0x7F if x.dtype == torch.uint8 else float("nan")


def case(groups, prefix, suffix, extra=True, seed=0):
    """(lens, prefix slots, number of slots): the prefixes in slots of their own behind the rows', or in the first rows'."""
    of = np.repeat(np.arange(len(groups)), groups)
    rows = len(of)
    rng = np.random.default_rng(seed)
    suf = [int(suffix[i % len(suffix)]) for i in rng.permutation(rows)]
    lens = [prefix[g] + s for g, s in zip(of, suf)]
    first = np.cumsum(groups) - groups
    slots = [rows + i for i in range(len(groups))] if extra else first.tolist()
    return lens, slots, rows + (len(groups) if extra else 0)


def ranges(groups, lens, prefix, slots):
    of = np.repeat(np.arange(len(groups)), groups)
    seen = {r: [(prefix[g], lens[r])] for r, g in enumerate(of)}
    for g, s in enumerate(slots):
        seen.setdefault(s, []).append((0, prefix[g]))
    return seen


GROUPS = [([1], [0]), ([1], [65]), ([4], [200]), ([3, 1, 9], [64, 0, 333]), ([40], [130]), ([5] * 7, [100, 0, 16, 17, 31, 255, 1]),
          ([100, 1, 30], [70, 500, 129])]


@pytest.mark.parametrize("dtype,blk,page", [("bf16", 16, 0), ("bf16", 16, 48), ("e4m3", 16, 16), ("e4m3", 64, 0), ("e4m3", 32, 96)])
@pytest.mark.parametrize("g", range(len(GROUPS)))
@pytest.mark.parametrize("heads", range(2))
def test_shared_attention(dtype, blk, page, g, heads):
    nq, nkv, d = [(4, 2, 64), (8, 2, 128), (2, 2, 128), (7, 1, 128), (16, 1, 64), (6, 2, 64)][(2 * g + 3 * heads + page + blk // 16) % 6]
    groups, prefix = GROUPS[g]
    lens, slots, n = case(groups, prefix, [0, 1, 15, 16, 17, 64, 100, 130])
    cap = -(-max(lens) // 192) * 192 + 192
    hc = HostCache(nkv, d, n, cap, blk, page, seed=g + d, dtype=dtype)
    poison(hc, ranges(groups, lens, prefix, slots))
    q, qd = rows_of(len(lens), nq, d, 5, 24)
    valid = None if g % 2 else [int(i % 5 != 3) for i in range(len(lens))]
    out = run(hc.device_cache(corun), qd, groups, lens, prefix, slots, valid)
    check(hc, q, out, groups, lens, prefix, slots, valid)


@pytest.mark.parametrize("dtype,blk,page", [("bf16", 16, 64), ("e4m3", 32, 32)])
@pytest.mark.parametrize("groups,prefix,suffix", [
    ([3], [6000], [0, 700, 40]), ([24, 2], [2500, 4100], [1, 300]), ([64], [3000], [5, 90]), ([1] * 6, [5000, 1, 0, 63, 2048, 4097], [3, 0]),
    ([260], [1500], [0, 2, 33])])
def test_long_prefixes(dtype, blk, page, groups, prefix, suffix):
    """Several splits of a prefix and of suffixes; the launch covers just what there is, or all of the capacity."""
    nq, nkv, d = 8, 2, 128
    lens, slots, n = case(groups, prefix, suffix)
    cap = -(-max(lens) // 64) * 64
    hc = HostCache(nkv, d, n, cap, blk, page, seed=3, dtype=dtype)
    cache = hc.device_cache(corun)
    q, qd = rows_of(len(lens), nq, d, 6)
    rows = sorted({0, 1, len(lens) // 2, len(lens) - 1} & set(range(len(lens))))
    for most in ((max(prefix), max(suffix)), (0, 0)):
        out = run(cache, qd, groups, lens, prefix, slots, most=most)
        check(hc, q, out, groups, lens, prefix, slots, rows=rows)
        assert not torch.isnan(out).any()


@pytest.mark.parametrize("dtype,nq,P,S,rows", [("bf16", 4, 70000, 50000, 2), ("e4m3", 8, 3, 100000, 1), ("e4m3", 16, 90000, 100, 8)])
def test_very_long(dtype, nq, P, S, rows):
    """More tokens than 256 splits of the shortest chunk hold, of prefixes and of a row's own."""
    d, nkv = 64, 1
    cap = -(-(P + S) // 16) * 16
    hc = HostCache(nkv, d, rows + 1, cap, 16, 0, seed=6, dtype=dtype)
    q, qd = rows_of(rows, nq, d, 14)
    lens = [P + S - 3 * r for r in range(rows)]
    out = run(hc.device_cache(corun), qd, [rows], lens, [P], [rows])
    check(hc, q, out, [rows], lens, [P], [rows], rows=sorted({0, rows - 1}))


@pytest.mark.parametrize("nq", [2, 16])
def test_the_most_rows_and_groups(nq):
    """65535 rows in 256 groups, of one query head to a kv head and of sixteen: every row against torch in fp32 (its sums of
    32 terms are off by under 2^-18 of the weighted sizes, beside the result's own rounding)."""
    nkv, d = (2, 64) if nq == 2 else (1, 64)
    groups = [256] * 255 + [255]
    rows = sum(groups)
    g = torch.Generator(device=DEV).manual_seed(1)
    k, v = (torch.randn((rows, nkv, 32, d), generator=g, device=DEV).bfloat16() for _ in range(2))
    cache = corun.KvCache([k], [v])
    q = torch.randn((rows, nq * d), generator=g, device=DEV).bfloat16()
    lens = torch.randint(16, 33, (rows,), generator=g, device=DEV, dtype=torch.int32)
    first = torch.arange(256, device=DEV, dtype=torch.int32) * 256
    ws = torch.empty(corun.shared_attention_workspace(cache, groups, nq), dtype=torch.uint8, device=DEV)
    out = torch.zeros_like(q)
    corun.shared_attention(cache, 0, q, groups, lens, torch.full_like(first, 16), out, ws, prefix_slots=first.flip(0).contiguous())
    of = torch.arange(rows, device=DEV) // 256
    at = first.flip(0).long()[of]
    kk, vv = (torch.cat([t[at][:, :, :16], t[:, :, 16:]], 2).float() for t in (k, v))
    s = (q.float().view(rows, nkv, nq // nkv, d) @ kk.transpose(2, 3).contiguous()) / 8.0
    s = s.masked_fill((torch.arange(32, device=DEV)[None, :] >= lens[:, None])[:, None, None], -float("inf"))
    p = torch.softmax(s, -1)
    want, pv = (p @ vv).view(rows, -1), (p @ vv.abs()).view(rows, -1)
    tol = ref.U_BF16 * (want.abs() + 2.0**-13 * pv) + (2.0**-13 + 2.0**-18) * pv
    assert ((out.float() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_prefix_in_the_first_rows_slot(dtype):
    groups, prefix = [3, 2], [90, 33]
    lens, slots, n = case(groups, prefix, [7, 1, 40], extra=False)
    hc = HostCache(2, 128, n, 192, 16, 0, seed=1, dtype=dtype)
    q, qd = rows_of(5, 8, 128, 7)
    out = run(hc.device_cache(corun), qd, groups, lens, prefix)
    check(hc, q, out, groups, lens, prefix, slots)


@pytest.mark.parametrize("dtype,page", [("bf16", 0), ("e4m3", 16)])
def test_calls_out_of_range_give_nan_and_touch_nothing_else(dtype, page):
    groups, cap = [2, 2, 2, 2, 1, 1], 192
    prefix = [100, 193, -1, 50, 60, 0]
    slots = [10, 10, 10, 12, 11, -5]
    lens = [120, 99, 200, 190, 10, 10, 80, 60, 192, 0]
    good = [0]                                         # row 1: shorter than its prefix; row 9: its prefix has no slot; row 8: a bad page, or fine
    hc = HostCache(2, 128, 12, cap, 16, page, seed=4, dtype=dtype)
    if page:
        hc.table[8, 11] = 9999
    else:
        good.append(8)
    q, qd = rows_of(10, 8, 128, 8)
    wide = torch.full((10, 8 * 128 + 16), 5.0, dtype=torch.bfloat16, device=DEV)
    out = run(hc.device_cache(corun), qd, groups, lens, prefix, slots, out=wide[:, : 8 * 128])
    of = np.repeat(np.arange(6), groups)
    for r in range(10):
        if r not in good:
            assert torch.isnan(out[r]).all(), r
    check(hc, q, out, groups, lens, [max(p, 0) for p in prefix], slots, rows=good)
    assert (wide[:, 8 * 128:] == 5.0).all()
    # lengths beyond the launch's
    out = run(hc.device_cache(corun), qd[:2], [2], [120, 190], [100], [10], most=(100, 89))
    assert not torch.isnan(out[0]).any() and torch.isnan(out[1]).all()
    out = run(hc.device_cache(corun), qd[:2], [2], [120, 180], [100], [10], most=(99, 192))
    assert torch.isnan(out).all()


@pytest.mark.parametrize("page", [16, 48])
@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
def test_bad_pages_reach_those_who_see_them(dtype, page):
    groups, prefix, cap = [20, 20], [100, 100], 192
    lens, slots, n = case(groups, prefix, [0, 10, 50])
    hc = HostCache(1, 128, n, cap, 16, page, seed=9, dtype=dtype)
    q, qd = rows_of(40, 4, 128, 9)
    want = run(hc.device_cache(corun), qd, groups, lens, prefix, slots)
    lost = [r for r in range(20) if lens[r] > 96 // page * page + page]
    hc.table[slots[1], 0] = -1                         # in the second group's prefix
    for r in range(20):
        hc.table[r, 96 // page + 1] = 1 << 30          # behind what some of the first group's rows see
        hc.table[r, 0] = -7                            # before it
    got = run(hc.device_cache(corun), qd, groups, lens, prefix, slots)
    assert torch.isnan(got[20:]).all()
    for r in range(20):
        if r in lost:
            assert torch.isnan(got[r]).all()
        else:
            assert same(got[r], want[r])
    assert 0 < len(lost) < 20


@pytest.mark.parametrize("dtype,blk,page", [("bf16", 16, 0), ("e4m3", 32, 64)])
@pytest.mark.parametrize("rows", [5, 70])
def test_rows_do_not_depend_on_their_place_or_neighbours(dtype, blk, page, rows):
    """Position invariance: the same bits at another row of the group, beside padding rows, or others of NaN."""
    nq, nkv, d, P = 8, 2, 128, 700
    hc = HostCache(nkv, d, rows + 1, 1024, blk, page, seed=2, dtype=dtype)
    q, qd = rows_of(rows, nq, d, 10)
    lens = [P + int(x) for x in np.random.default_rng(0).integers(0, 200, rows)]
    base = run(hc.device_cache(corun), qd, [rows], lens, [P], [rows])
    p = np.random.default_rng(1).permutation(rows)
    hp = HostCache(nkv, d, rows + 1, 1024, blk, page, seed=2, dtype=dtype)
    order = torch.from_numpy(np.append(p, rows))
    if page:
        hp.table = hc.table[order].clone()
    else:
        hp.k, hp.v = hc.k[order].clone(), hc.v[order].clone()
        if hc.ks is not None:
            hp.ks, hp.vs = hc.ks[order].clone(), hc.vs[order].clone()
    moved = run(hp.device_cache(corun), qd[torch.from_numpy(p).to(DEV)], [rows], [lens[i] for i in p], [P], [rows])
    assert same(moved, base[torch.from_numpy(p)])
    valid = [int(i % 2 == 0) for i in range(rows)]
    nan = qd.clone()
    nan[1::2] = float("nan")
    alone = run(hc.device_cache(corun), nan, [rows], lens, [P], [rows], valid=valid)
    assert same(alone[::2], base[::2]) and (alone[1::2] == 0).all()
    beside = run(hc.device_cache(corun), nan, [rows], lens, [P], [rows])
    assert same(beside[::2], base[::2]) and torch.isnan(beside[1::2]).all()


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("rows", [3, 50])
def test_scores_and_values_of_any_size(dtype, rows):
    """Scores up to some thousands, a key that takes all the weight, values that differ by 2^20 from token to token,
    and equal scores everywhere."""
    nq, nkv, d, P = 8, 2, 128, 300
    hc = HostCache(nkv, d, rows + 1, 384, 16, 0, seed=12, dtype=dtype)
    if dtype == "bf16":
        hc.v *= torch.exp2(torch.randint(-10, 11, (rows + 1, nkv, 384, 1), generator=torch.Generator().manual_seed(3)).float()).to(torch.bfloat16)
        hc.k[rows, :, 200] *= 30
    else:
        hc.vs += torch.randint(-10, 11, hc.vs.shape, generator=torch.Generator().manual_seed(3)).to(torch.uint8)
        hc.ks[rows, :, 12] += 5
    q, _ = rows_of(rows, nq, d, 13)
    q[0] *= 100
    q[1] = 0
    q[2] *= 1000
    lens = [P + 7 * (r % 9) for r in range(rows)]
    out = run(hc.device_cache(corun), q.to(DEV), [rows], lens, [P], [rows])
    check(hc, q, out, [rows], lens, [P], [rows])


@pytest.mark.parametrize("d,page", [(128, 0), (64, 32)])
@pytest.mark.parametrize("spread", [8, 24, 25, 60])
def test_scales_apart(d, page, spread):
    """Value scales of a prefix that are as far apart as one fp16 product takes, farther in one block of one split, and far
    apart everywhere; the weight goes to tokens of small scales, to those of large ones, and to all."""
    nq, nkv, rows, P, blk = 8, 2, 30, 1700, 16
    cap = -(-(P + 64) // 96) * 96 if page else 1792
    hc = HostCache(nkv, d, rows + 1, cap, blk, page, seed=30, dtype="e4m3")
    hc.vs[:] = 120
    at = [hc.at(rows, t) for t in range(0, P, blk)]
    rng = np.random.default_rng(spread)
    for i, (pg, t) in enumerate(at):
        near = min(spread, 24) if spread < 60 else 60
        up = 0 if i == 0 else int(rng.integers(-near, near + 1))
        if spread == 25 and i == 40:
            up = 25
        hc.vs[pg, :, t // blk] = 120 + up
    for i in (20, 41):                                 # keys that some queries meet
        pg, t = at[i]
        hc.ks[pg, :, t // blk] += 3
        hc.vs[pg, :, t // blk] = 120 + (8 if i == 20 else -8)
    q, _ = rows_of(rows, nq, d, 31)
    q[1] *= 8
    q[2] = 0
    lens = [P + r % 5 for r in range(rows)]
    out = run(hc.device_cache(corun), q.to(DEV), [rows], lens, [P], [rows])
    check(hc, q, out, [rows], lens, [P], [rows])


def test_cache_beyond_32_bits():
    """Rows and prefix behind 2^32 elements of a bf16 cache."""
    nkv, d, cap = 1, 128, 1 << 21
    k = torch.zeros((18, nkv, cap, d), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    g = torch.Generator(device=DEV).manual_seed(1)
    P, n, at = 40, 64, 17
    x = torch.randn((2, n, d), generator=g, device=DEV).bfloat16()
    k[at, 0, :n], v[at, 0, :n] = x[0], x[1]
    k[16, 0, :n], v[16, 0, :n] = x[1], x[0]
    cache = corun.KvCache([k], [v])
    q, qd = rows_of(18, 2, d, 3)
    lens = [P] * 16 + [n, n]
    ws = torch.empty(corun.shared_attention_workspace(cache, [18], 2, 64, 64), dtype=torch.uint8, device=DEV)
    out = run(cache, qd, [18], lens, [P], [at], most=(64, 64), ws=ws)
    kk, vv = x.double().cpu()
    for r, (a, b) in ((0, (kk[:P], vv[:P])), (17, (kk, vv)),
                      (16, (torch.cat([kk[:P], vv[P:]]), torch.cat([vv[:P], kk[P:]])))):
        want, pv, size = ref.attention(q[r].double().view(2, d), a[None], b[None], len(a))
        tol = ref.attention_bound(want, pv, size, d, n, U_WEIGHT)
        assert ((out[r].double().view(2, d) - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype,blk,page", [("bf16", 16, 16), ("e4m3", 16, 0)])
@pytest.mark.parametrize("rows,P", [(4, 900), (60, 700)])
def test_captured_attention_replays(dtype, blk, page, rows, P):
    """One capture, with lengths and prefixes that change between its replays: the eager bits each time."""
    nq, nkv, d, cap = 8, 2, 128, 1536
    hc = HostCache(nkv, d, rows + 1, cap, blk, page, seed=20, dtype=dtype)
    cache = hc.device_cache(corun)
    most = (1024, 256)
    size = corun.shared_attention_workspace(cache, [rows], nq, *most)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)
    qs = torch.zeros((rows, nq * d), dtype=torch.bfloat16, device=DEV)
    out = torch.zeros_like(qs)
    ln, pl, sl = i32([0] * rows), i32([0]), i32([rows])
    st, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=st):
        corun.shared_attention(cache, 0, qs, [rows], ln, pl, out, ws, prefix_slots=sl, max_prefix=most[0], max_suffix=most[1])
    for i in range(4):
        q, qd = rows_of(rows, nq, d, 30 + i)
        p = [P, 0, 1024, 31][i]
        lens = [p + (37 * r + i) % 250 for r in range(rows)]
        qs.copy_(qd)
        ln.copy_(i32(lens))
        pl.fill_(p)
        ws.fill_(0xFF)
        out.fill_(3.0)
        g.replay()
        torch.cuda.synchronize()
        assert same(out.cpu(), run(cache, qd, [rows], lens, [p], [rows], most=most).contiguous())
        check(hc, q, out.cpu(), [rows], lens, [p], [rows], rows=[0, rows - 1])


def test_two_streams_with_their_own_workspaces():
    nq, nkv, d, rows, P = 8, 2, 128, 20, 1300
    hc = HostCache(nkv, d, rows + 1, 1536, 16, 0, seed=21, dtype="bf16")
    cache = hc.device_cache(corun)
    lens = [P + 5 * r for r in range(rows)]
    q = [rows_of(rows, nq, d, 50 + i)[1].contiguous() for i in range(2)]
    want = [run(cache, x, [rows], lens, [P], [rows]) for x in q]
    size = corun.shared_attention_workspace(cache, [rows], nq)
    ws = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(2)]
    ln, pl, sl = i32(lens), i32([P]), i32([rows])
    out = [[torch.zeros_like(q[i]) for _ in range(15)] for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for j in range(15):
        for i in range(2):
            corun.shared_attention(cache, 0, q[i], [rows], ln, pl, out[i][j], ws[i], prefix_slots=sl, stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        for o in out[i]:
            assert same(o.cpu(), want[i].contiguous())


def test_python_refusals():
    hc = HostCache(2, 64, 5, 64, 16, 0, dtype="bf16")
    cache = hc.device_cache(corun)
    q = torch.zeros((4, 256), dtype=torch.bfloat16, device=DEV)
    ws = torch.zeros(max(16, corun.shared_attention_workspace(cache, [4], 4)), dtype=torch.uint8, device=DEV)
    ok = lambda **kw: corun.shared_attention(**{**dict(cache=cache, layer=0, q=q, group_rows=[4], lens=i32([0] * 4),
                                                       prefix_lens=i32([0]), out=torch.zeros_like(q), ws=ws), **kw})
    ok()
    for bad in (dict(layer=1), dict(q=q.float()), dict(q=q[:, :250]), dict(out=q[:3]), dict(group_rows=[3]), dict(group_rows=[2, 2]),
                dict(lens=i32([0] * 3)), dict(lens=i32([0] * 4).long()), dict(prefix_lens=i32([0, 0])), dict(prefix_slots=i32([0, 0])),
                dict(valid=i32([1] * 4)), dict(ws=ws.int()), dict(out=q.cpu())):
        with pytest.raises(ValueError):
            ok(**bad)
    with pytest.raises(corun.CorunError):
        ok(max_prefix=65)
    with pytest.raises(corun.CorunError):
        ok(group_rows=[4, 0], prefix_lens=i32([0, 0]))
    out = torch.full_like(q, 3.0)
    ok(out=out)
    torch.cuda.synchronize()
    assert (out == 0).all()
