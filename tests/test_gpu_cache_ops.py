"""The cache operators on the GPU against the 64-bit reference of
tests/cache_reference.py: rotary forms, appends, scales that grow, masks,
lengths from nothing to the capacity, pages, strides, and what must not be
touched."""
import numpy as np
import pytest
import torch

from paper_2608_14376_amd import corun
from tests import cache_reference as ref
from tests.cache_reference import HostCache

pytestmark = pytest.mark.gpu
DEV = "cuda"

ROPES = {
    "half": dict(theta=1e6),
    "interleaved": dict(theta=1e4, layout=corun.ROPE_INTERLEAVED),
    "half_part": dict(theta=1e4, rot_dim=32),
    "half_odd": dict(theta=1e4, rot_dim=22),
    "interleaved_part": dict(theta=1e4, rot_dim=10, layout=corun.ROPE_INTERLEAVED),
    "linear": dict(theta=1e4, scaling=corun.ROPE_LINEAR, factor=4.0),
    "bands": dict(theta=5e5, scaling=corun.ROPE_BANDS, factor=8.0, low=1.0, high=4.0, trained_len=8192, magnitude=1.25),
}


def make_rope(name, d):
    kw = ROPES[name]
    r = corun.rope(d, **kw)
    sc = {0: "none", 1: "linear", 2: "bands"}[kw.get("scaling", 0)]
    f = ref.freqs(kw["theta"], r.rot_dim, sc, kw.get("factor", 1.0), kw.get("low", 0.0), kw.get("high", 0.0),
                  kw.get("trained_len", 0))
    return r, lambda x, pos: ref.rotate(x, pos, f, r.rot_dim, bool(kw.get("layout", 0)), float(r.magnitude))


def rows_of(n, heads, d, seed, pad=0, loud=True):
    """bf16 [n, heads d] on the host, and the same on the device with `pad` further elements between rows."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, heads, d), generator=g)
    if loud:
        x[..., ::37] *= 6.0
    x = x.view(n, heads * d).to(torch.bfloat16)
    wide = torch.full((n, heads * d + pad), 7.0, dtype=torch.bfloat16)
    wide[:, : heads * d] = x
    return x, wide.to(DEV)[:, : heads * d]


def check_q(got, want, size):
    """q: one bf16 rounding of an fp32 rotation (products and sum: 4 roundings of the pair's size)."""
    tol = ref.U_BF16 * want.abs() + 4 * ref.U_F32 * size * 1.01
    bad = (got.double() - want).abs() > tol
    assert not bad.any(), (bad.nonzero()[:4], got.double()[bad][:4], want[bad][:4])


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# --------------------------------------------------------------------------
# Append
# --------------------------------------------------------------------------

@pytest.mark.parametrize("d,nkv,G", [(64, 2, 2), (128, 2, 4), (128, 1, 7), (64, 3, 1)])
@pytest.mark.parametrize("rope_name", list(ROPES))
@pytest.mark.parametrize("blk,page", [(16, 0), (32, 32), (16, 48), (64, 0)])
def test_decode_append(d, nkv, G, rope_name, blk, page):
    cap = 192
    pos = [0, 1, 15, 16, 17, 31, 63, 64, 100, cap - 1, 5, 40]
    valid = [1] * len(pos)
    valid[5] = valid[10] = 0
    pos[10] = -(2**31)                                # padding rows hold anything
    rows, nq = len(pos), nkv * G
    hc = HostCache(nkv, d, rows, cap, blk, page, seed=blk + page)
    cache = hc.device_cache(corun)
    rope, rot = make_rope(rope_name, d)
    pad = 24
    x, xd = rows_of(rows, nq + 2 * nkv, d, 3, pad)
    x[6, nq * d:] *= 40                               # tokens that need a larger scale than their block has
    x[8, nq * d:] *= 300
    x[4] = 0
    xd.copy_(x)
    q = torch.full((rows, nq * d + 8), 3.0, dtype=torch.bfloat16, device=DEV)
    corun.decode_append(cache, 0, xd, torch.tensor(pos, dtype=torch.int32, device=DEV), rope, q[:, : nq * d],
                        valid=torch.tensor(valid, dtype=torch.uint8, device=DEV))
    torch.cuda.synchronize()
    live = [r for r in range(rows) if valid[r]]
    x64 = x.double().view(rows, nq + 2 * nkv, d)
    y, size = rot(x64[:, : nq + nkv], torch.tensor([p if v else 0 for p, v in zip(pos, valid)]))
    qh = q.cpu()
    check_q(qh[live][:, : nq * d].view(len(live), nq, d), y[live][:, :nq], size[live][:, :nq])
    assert (qh[:, nq * d:] == 3.0).all() and (qh[[5, 10]] == 3.0).all()
    k = y[:, nq:]
    ref.check_append(hc, hc.after(), [(r, 1, pos[r], r) for r in live], k, x64[:, nq + nkv:])


@pytest.mark.parametrize("d,nkv,G", [(64, 2, 2), (128, 2, 3), (128, 8, 4)])
@pytest.mark.parametrize("rope_name", ["half", "interleaved_part", "half_odd", "bands"])
@pytest.mark.parametrize("blk,page", [(16, 16), (32, 0), (64, 64), (32, 96)])
def test_prefill_append(d, nkv, G, rope_name, blk, page):
    cap = 384 if page == 96 else 320
    lens, starts, slots = [1, 130, 33, 64, 7, 200], [0, 0, 5, 64, 63, 119], [3, 0, 5, 1, 7, 2]
    n, nq = sum(lens), nkv * G
    hc = HostCache(nkv, d, 8, cap, blk, page, seed=d + blk)
    cache = hc.device_cache(corun)
    rope, rot = make_rope(rope_name, d)
    x, xd = rows_of(n, nq + 2 * nkv, d, 4, 8)
    x[140:150, nq * d:] *= 50                         # in the sequence that starts inside a block
    xd.copy_(x)
    q = torch.full((n, nq * d), 3.0, dtype=torch.bfloat16, device=DEV)
    corun.prefill_append(cache, 0, xd, lens, starts, slots, rope, q)
    torch.cuda.synchronize()
    first = np.cumsum(lens) - lens
    p = torch.cat([torch.arange(s, s + m) for s, m in zip(starts, lens)])
    x64 = x.double().view(n, nq + 2 * nkv, d)
    y, size = rot(x64[:, : nq + nkv], p)
    check_q(q.cpu().view(n, nq, d), y[:, :nq], size[:, :nq])
    ref.check_append(hc, hc.after(), [(int(f), m, s, sl) for f, m, s, sl in zip(first, lens, starts, slots)],
                     y[:, nq:], x64[:, nq + nkv:])


@pytest.mark.parametrize("rope_name", ["half", "interleaved_part", "half_odd"])
@pytest.mark.parametrize("page", [0, 48])
def test_append_to_bf16_caches(rope_name, page):
    d, nkv, nq, cap = 128, 2, 6, 144
    hc = HostCache(nkv, d, 4, cap, 16, page, seed=5, dtype="bf16")
    cache = hc.device_cache(corun)
    rope, rot = make_rope(rope_name, d)
    lens, starts, slots = [20, 70], [3, 0], [2, 0]
    n = sum(lens)
    x, xd = rows_of(n + 4, nq + 2 * nkv, d, 6)
    q = torch.zeros((n + 4, nq * d), dtype=torch.bfloat16, device=DEV)
    corun.prefill_append(cache, 0, xd[:n], lens, starts, slots, rope, q[:n])
    pos = [70, 0, 23, 143]
    corun.decode_append(cache, 0, xd[n:], torch.tensor(pos, dtype=torch.int32, device=DEV), rope, q[n:])
    torch.cuda.synchronize()
    p = torch.cat([torch.arange(s, s + m) for s, m in zip(starts, lens)] + [torch.tensor(pos)])
    where = [(sl, t) for s, m, sl in zip(starts, lens, slots) for t in range(s, s + m)] + list(enumerate(pos))
    x64 = x.double().view(n + 4, nq + 2 * nkv, d)
    y, size = rot(x64[:, : nq + nkv], p)
    check_q(q.cpu().view(n + 4, nq, d), y[:, :nq], size[:, :nq])
    after = hc.after()
    k, v = hc.k.clone(), hc.v.clone()
    for r, (slot, t) in enumerate(where):
        a, b = hc.at(slot, t)
        check_q(after.k[a, :, b], y[r, nq:], size[r, nq:])
        k[a, :, b], v[a, :, b] = after.k[a, :, b], x.view(n + 4, nq + 2 * nkv, d)[r, nq + nkv:]
    assert same(after.k, k) and same(after.v, v)


def test_append_values_out_of_the_ordinary():
    """Zeros, subnormal and largest bf16 values, infinities and NaN, alone and beside ordinary ones."""
    d, nkv, nq, blk, cap = 64, 1, 1, 16, 64
    big, tiny = 3.3895313892515355e38, 2.0**-133
    rows = []
    for fill in (0.0, tiny, big, float("inf"), float("nan"), -float("inf"), 448.0, 450.0, 2.0**-100, 1.0):
        rows.append(torch.full((3 * d,), fill))
        mixed = torch.linspace(-2, 2, 3 * d)
        mixed[5::7] = fill
        rows.append(mixed)
    x = torch.stack(rows).to(torch.bfloat16)
    n = x.shape[0]
    hc = HostCache(nkv, d, n, cap, blk, seed=1)
    cache = hc.device_cache(corun)
    rope = corun.rope(d, 1e4, rot_dim=2)
    q = torch.zeros((n, d), dtype=torch.bfloat16, device=DEV)
    corun.decode_append(cache, 0, x.to(DEV), torch.zeros(n, dtype=torch.int32, device=DEV), rope, q)   # position 0: no turn
    torch.cuda.synchronize()
    x64 = x.double().view(n, 3, d)
    x64[:, :2, :2] = torch.where(torch.isfinite(x64[:, :2, :2]).all(-1, keepdim=True), x64[:, :2, :2],
                                 torch.full_like(x64[:, :2, :2], float("nan")))   # inf times a sine of 0
    ref.check_append(hc, hc.after(), [(r, 1, 0, r) for r in range(n)], x64[:, 1:2], x64[:, 2:], k_exact=True)


def test_append_one_by_one_matches_the_definition_at_every_step():
    """A block filled token by token, louder and quieter: its scale never falls and earlier codes follow it."""
    d, nkv, nq, blk = 128, 2, 2, 32
    for page in (0, 32):
        hc = HostCache(nkv, d, 2, 64, blk, page, seed=2)
        cache = hc.device_cache(corun)
        rope, rot = make_rope("half", d)
        q = torch.zeros((2, nq * d), dtype=torch.bfloat16, device=DEV)
        for t in range(40):
            x, xd = rows_of(2, nq + 2 * nkv, d, 100 + t)
            x *= 2.0 ** ((t * 7) % 11 - 5)
            xd.copy_(x)
            before = hc.after()
            corun.decode_append(cache, 0, xd, torch.tensor([t, t], dtype=torch.int32, device=DEV), rope, q)
            torch.cuda.synchronize()
            x64 = x.double().view(2, nq + 2 * nkv, d)
            y, _ = rot(x64[:, : nq + nkv], torch.tensor([t, t]))
            ref.check_append(before, hc.after(), [(0, 1, t, 0), (1, 1, t, 1)], y[:, nq:], x64[:, nq + nkv:])


def test_append_far_positions():
    """Angles of positions up to 2^31 - 1 (the rotation is of the position, whatever the cache holds)."""
    d, nkv, nq = 128, 1, 4
    rope, rot = make_rope("half", d)
    pos = [0, 131071, 1 << 20, (1 << 26) - 1]
    cap = 1 << 26
    # one page is every page: 2^22 pages of 16 tokens a slot, all the same one
    k = torch.zeros((2, nkv, 16, d), dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    table = torch.ones((4, cap // 16), dtype=torch.int32, device=DEV)
    cache = corun.KvCache([k], [v], page_table=table)
    x, xd = rows_of(4, nq + 2 * nkv, d, 9, loud=False)
    q = torch.zeros((4, nq * d), dtype=torch.bfloat16, device=DEV)
    for r, p in enumerate(pos):                       # one live row at a time: the slots share their page
        valid = torch.zeros(4, dtype=torch.uint8, device=DEV)
        valid[r] = 1
        corun.decode_append(cache, 0, xd, torch.tensor(pos, dtype=torch.int32, device=DEV), rope, q, valid=valid)
    y, size = rot(x.double().view(4, -1, d)[:, :nq], torch.tensor(pos))
    got = q.cpu().view(4, nq, d).double()
    # the reference's own angle p f is rounded: 2^-53 of up to 2^26 radians, 2^-27, against the rotation's size
    tol = ref.U_BF16 * y.abs() + (4 * ref.U_F32 + 2.0**-26) * size
    assert ((got - y).abs() <= tol).all()


def test_append_rows_outside_the_cache():
    """Positions and pages outside the cache: nothing appended, NaN queries, other rows untouched by it."""
    d, nkv, nq, blk, page, cap = 128, 2, 4, 16, 16, 64
    pos = [5, -1, cap, 2**31 - 1, -(2**31), 20, 33, 40]
    hc = HostCache(nkv, d, len(pos), cap, blk, page, seed=8)
    hc.table[5, 1], hc.table[6, 2] = -1, hc.k.shape[0]
    cache = hc.device_cache(corun)
    rope, rot = make_rope("half", d)
    x, xd = rows_of(len(pos), nq + 2 * nkv, d, 12)
    q = torch.zeros((len(pos), nq * d), dtype=torch.bfloat16, device=DEV)
    corun.decode_append(cache, 0, xd, torch.tensor(pos, dtype=torch.int32, device=DEV), rope, q)
    torch.cuda.synchronize()
    good = [0, 7]
    x64 = x.double().view(len(pos), -1, d)
    y, size = rot(x64[:, : nq + nkv], torch.tensor([5, 0, 0, 0, 0, 0, 0, 40]))
    qh = q.cpu().view(len(pos), nq, d)
    check_q(qh[good], y[good][:, :nq], size[good][:, :nq])
    assert torch.isnan(qh[1:7]).all()
    ref.check_append(hc, hc.after(), [(r, 1, pos[r], r) for r in good], y[:, nq:], x64[:, nq + nkv:])
    # a prompt that crosses the bad page of slot 5 (tokens 16 .. 31)
    hc2 = HostCache(nkv, d, len(pos), cap, blk, page, seed=8)
    hc2.table[5, 1] = hc2.k.shape[0] + 3
    cache = hc2.device_cache(corun)
    x, xd = rows_of(40, nq + 2 * nkv, d, 13)
    q = torch.zeros((40, nq * d), dtype=torch.bfloat16, device=DEV)
    corun.prefill_append(cache, 0, xd, [40], [4], [5], rope, q)
    torch.cuda.synchronize()
    x64 = x.double().view(40, -1, d)
    y, size = rot(x64[:, : nq + nkv], torch.arange(4, 44))
    qh = q.cpu().view(40, nq, d)
    ok = [t for t in range(40) if not 16 <= t + 4 < 32]
    check_q(qh[ok], y[ok][:, :nq], size[ok][:, :nq])
    assert torch.isnan(qh[12:28]).all()
    ref.check_append(hc2, hc2.after(), [(0, 12, 4, 5), (28, 12, 32, 5)], y[:, nq:], x64[:, nq + nkv:])


# --------------------------------------------------------------------------
# Decode attention
# --------------------------------------------------------------------------

def run_decode(cache, q, lens, valid=None, max_len=0, nq_d=None):
    rows = q.shape[0]
    out = torch.full_like(q, 5.0)
    nq = q.shape[1] // cache.head_dim
    ws = torch.full((corun.decode_attention_workspace(cache, rows, nq, max_len),), 255, dtype=torch.uint8, device=DEV)
    corun.decode_attention(cache, 0, q, torch.as_tensor(lens, dtype=torch.int32, device=DEV), out, ws,
                           valid=None if valid is None else torch.tensor(valid, dtype=torch.uint8, device=DEV),
                           max_len=max_len)
    torch.cuda.synchronize()
    return out.cpu()


def check_decode(hc, q, lens, rows, out, u_weight=2.0**-14):
    d = hc.d
    for r in rows:
        n = lens[r]
        if n == 0:
            assert (out[r] == 0).all()
            continue
        k, v = hc.values(r, n)
        o, pv, size = ref.attention(q[r].double().view(-1, d), k, v, n)
        got = out[r].double().view(-1, d)
        tol = ref.attention_bound(o, pv, size, d, n, u_weight)
        assert ((got - o).abs() <= tol).all(), (r, n, ((got - o).abs() / tol).max())


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 7, 8, 16])
@pytest.mark.parametrize("blk,page", [(16, 16), (32, 0), (64, 64), (16, 48)])
def test_decode_attention(d, G, blk, page):
    nkv, cap = 2, 768
    lens = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 255, 300, 511, 600, 767, 768]
    hc = HostCache(nkv, d, len(lens), cap, blk, page, seed=G)
    # stale tokens behind the last one: NaN codes and scales that nothing may see
    for r, n in enumerate(lens):
        for t in range(n, min(cap, n + 40)):
            a, b = hc.at(r, t)
            hc.k[a, :, b] = 0x7F
            hc.v[a, :, b] = 0xFF
    cache = hc.device_cache(corun)
    x, q = rows_of(len(lens), nkv * G, d, 21, pad=16, loud=False)
    out = run_decode(cache, q, lens)
    check_decode(hc, x, lens, range(len(lens)), out)


def test_decode_attention_padding_and_bad_rows():
    """Padding rows and empty ones are zero; lengths and pages outside the cache give NaN in that row alone."""
    d, nkv, G, blk, page, cap = 128, 2, 4, 16, 16, 256
    lens = [100, -(2**31), 256, 257, -1, 2**31 - 1, 0, 200, 90, 31]
    valid = [1, 0, 1, 1, 1, 1, 1, 1, 1, 0]
    hc = HostCache(nkv, d, len(lens), cap, blk, page, seed=4)
    hc.table[7, 11] = -5                              # tokens 176 .. 191
    hc.table[8, 6] = hc.k.shape[0]                    # behind the row's 90 tokens: not seen
    cache = hc.device_cache(corun)
    x, q = rows_of(len(lens), nkv * G, d, 22)
    out = run_decode(cache, q, lens, valid)
    check_decode(hc, x, lens, [0, 2, 8], out)
    for r in (1, 6, 9):
        assert (out[r] == 0).all()
    for r in (3, 4, 5, 7):
        assert torch.isnan(out[r]).all()
    # a bound below the capacity
    out = run_decode(cache, q, lens, valid, max_len=101)
    check_decode(hc, x, lens, [0, 8], out)
    assert torch.isnan(out[2]).all()


@pytest.mark.parametrize("page", [0, 16])
def test_decode_attention_is_position_invariant(page):
    """A row's bits do not depend on its slot, on the other rows or on what the workspace held."""
    d, nkv, G, blk, cap = 128, 2, 4, 16, 2048
    rows = 6
    lens = [700, 1, 2048, 1300, 64, 0]
    hc = HostCache(nkv, d, rows, cap, blk, page, seed=31)
    cache = hc.device_cache(corun)
    x, q = rows_of(rows, nkv * G, d, 23)
    base = run_decode(cache, q, lens)
    perm = [3, 5, 0, 1, 4, 2]
    hp = hc.after()
    if page:
        hp.table = hc.table[perm].clone()
    else:
        hp.k, hp.v, hp.ks, hp.vs = (t[perm].clone() for t in (hc.k, hc.v, hc.ks, hc.vs))
    moved = run_decode(hp.device_cache(corun), q[perm].contiguous(), [lens[i] for i in perm])
    assert same(moved, base[perm])
    for r in range(rows):
        others = [(lens[i] if i == r else (37 * i + 11) % cap) for i in range(rows)]
        valid = [1 if i == r or i % 2 else 0 for i in range(rows)]
        assert same(run_decode(cache, q, others, valid)[r], base[r])


def test_decode_attention_masked_scores_of_any_size():
    """Scores far apart (weights underflow), equal keys, and a NaN key of a visible token, which does give NaN."""
    d, nkv, G, blk, cap = 128, 1, 2, 16, 128
    hc = HostCache(nkv, d, 4, cap, blk, seed=3)
    hc.ks[0] = 140                                    # keys 2^19 times larger: one weight takes all
    hc.k[1] = 0x38                                    # every key alike: the mean of the values
    hc.k[2, 0, 9] = 0x7F
    cache = hc.device_cache(corun)
    x, q = rows_of(4, nkv * G, d, 24, loud=False)
    lens = [100, 77, 64, 9]
    out = run_decode(cache, q, lens)
    assert torch.isnan(out[2]).all()
    check_decode(hc, x, lens, [1, 3], out)
    # row 0: the largest score is ahead of the others by more than the fp32 error of scores of 2^19
    k, v = hc.values(0, 100)
    o, pv, _ = ref.attention(x[0].double().view(-1, d), k, v, 100)
    s = x[0].double().view(G, d) @ k[0].t() / d**0.5
    top = torch.topk(s, 2, -1).values
    assert (top[:, 0] - top[:, 1] > 200).all() and (s.abs().max() * 136 * ref.U_F32 < 50)
    assert ((out[0].double().view(G, d) - o).abs() <= ref.U_BF16 * o.abs() * 1.01 + 1e-6).all()


def test_decode_attention_beyond_32_bits():
    """Slots whose codes start more than 2^32 bytes into the cache."""
    d, nkv, G, blk, S = 128, 8, 1, 16, 1 << 21
    rows = 3                                          # slot 2 starts at 2^32
    k = torch.zeros((rows, nkv, S, d), dtype=torch.uint8, device=DEV)
    v = torch.zeros_like(k)
    ks = torch.full((rows, nkv, S // blk), 121, dtype=torch.uint8, device=DEV)
    vs = ks.clone()
    small = HostCache(nkv, d, rows, 64, blk, seed=6)
    k[:, :, :64], v[:, :, :64] = small.k.to(DEV), small.v.to(DEV)
    ks[:, :, :4], vs[:, :, :4] = small.ks.to(DEV), small.vs.to(DEV)
    cache = corun.KvCache([k], [v], [ks], [vs], blk)
    x, q = rows_of(rows, nkv * G, d, 25, loud=False)
    lens = [50, 3, 64]
    out = run_decode(cache, q, lens, max_len=64)
    check_decode(small, x, lens, range(rows), out)
    # append there, at the last position of the last slot, and read it back
    xq, xd = rows_of(rows, nkv * G + 2 * nkv, d, 26)
    valid = torch.tensor([0, 0, 1], dtype=torch.uint8, device=DEV)
    qo = torch.zeros((rows, nkv * G * d), dtype=torch.bfloat16, device=DEV)
    rope, rot = make_rope("half", d)
    corun.decode_append(cache, 0, xd, torch.tensor([0, 0, S - 1], dtype=torch.int32, device=DEV), rope, qo, valid=valid)
    torch.cuda.synchronize()
    want = xq.double().view(rows, -1, d)[2, nkv * G + nkv:]
    for h in range(nkv):
        ref.check_codes(v[2, h, S - 1].cpu(), int(vs[2, h, -1]) - 127, want[h], True)
    assert int(v[2, :, S - blk:S - 1].max()) == 0 and int(k[:2, :, 64:].amax()) == 0


# --------------------------------------------------------------------------
# Prefill attention
# --------------------------------------------------------------------------

def run_prefill(cache, q, lens, starts, slots):
    out = torch.full_like(q, 5.0)
    corun.prefill_attention(cache, 0, q, lens, starts, slots, out)
    torch.cuda.synchronize()
    return out.cpu()


def check_prefill(hc, x, out, seqs, every=1, u_weight=2.0**-8):
    d = hc.d
    for row, n, p0, slot in seqs:
        k, v = hc.values(slot, p0 + n)
        for t in sorted(set(range(0, n, every)) | {0, n - 1}):
            o, pv, size = ref.attention(x[row + t].double().view(-1, d), k, v, p0 + t + 1)
            got = out[row + t].double().view(-1, d)
            tol = ref.attention_bound(o, pv, size, d, p0 + t + 1, u_weight)
            assert ((got - o).abs() <= tol).all(), (slot, t, ((got - o).abs() / tol).max())


def seqs_of(lens, starts, slots):
    first = np.cumsum(lens) - lens
    return [(int(f), m, s, sl) for f, m, s, sl in zip(first, lens, starts, slots)]


@pytest.mark.parametrize("d,nkv,G", [(64, 2, 2), (128, 2, 1), (128, 2, 4), (64, 1, 3), (128, 1, 7), (128, 1, 16)])
@pytest.mark.parametrize("blk,page", [(16, 16), (32, 0), (64, 192)])
def test_prefill_attention(d, nkv, G, blk, page):
    lens, starts, slots = [1, 2, 31, 33, 64, 65, 129, 200], [0, 63, 0, 100, 64, 1, 300, 0], [7, 1, 2, 0, 4, 5, 3, 8]
    cap = 576
    hc = HostCache(nkv, d, 9, cap, blk, page, seed=40 + G)
    for m, s, sl in zip(lens, starts, slots):         # stale tokens behind each sequence
        for t in range(s + m, min(cap, s + m + 70)):
            a, b = hc.at(sl, t)
            hc.k[a, :, b] = 0xFF
            hc.v[a, :, b] = 0x7F
    cache = hc.device_cache(corun)
    x, q = rows_of(sum(lens), nkv * G, d, 41, pad=8, loud=False)
    out = run_prefill(cache, q, lens, starts, slots)
    check_prefill(hc, x, out, seqs_of(lens, starts, slots), every=3)


def test_prefill_attention_sequences_do_not_touch_each_other():
    """Bits of a sequence alone and beside others, and of a row in whole and last-row calls of its chunk sizes."""
    d, nkv, G, blk, cap = 128, 2, 4, 32, 512
    hc = HostCache(nkv, d, 4, cap, blk, seed=50)
    cache = hc.device_cache(corun)
    lens, starts, slots = [100, 257, 64, 1], [0, 40, 448, 511], [2, 0, 3, 1]
    x, q = rows_of(sum(lens), nkv * G, d, 51)
    out = run_prefill(cache, q, lens, starts, slots)
    for row, n, p0, slot in seqs_of(lens, starts, slots):
        alone = run_prefill(cache, q[row:row + n], [n], [p0], [slot])
        assert same(alone, out[row:row + n])


@pytest.mark.parametrize("d,page", [(128, 0), (64, 16)])
def test_prefill_attention_nan_reaches_only_those_who_see_it(d, page):
    """NaN keys make the queries from there on NaN; NaN values do so in their own dimension."""
    nkv, G, blk, cap = 2, 2, 16, 256
    hc = HostCache(nkv, d, 2, cap, blk, page, seed=55)
    for slot, h, t, e, what in [(0, 0, 40, 3, "v"), (0, 0, 63, 17, "v"), (0, 0, 64, d - 1, "v"), (0, 1, 129, 0, "v"),
                                (0, 1, 170, 5, "k"), (1, 0, 99, 31, "v"), (1, 1, 0, d // 2, "v")]:
        a, b = hc.at(slot, t)
        (hc.v if what == "v" else hc.k)[a, h, b, e] = 0xFF if t % 2 else 0x7F
    cache = hc.device_cache(corun)
    lens, starts, slots = [200, 61], [0, 40], [0, 1]
    x, q = rows_of(261, nkv * G, d, 56)
    out = run_prefill(cache, q, lens, starts, slots)
    for row, n, p0, slot in seqs_of(lens, starts, slots):
        k, v = hc.values(slot, p0 + n)
        for t in range(n):
            o, pv, size = ref.attention(x[row + t].double().view(-1, d), torch.nan_to_num(k), torch.nan_to_num(v), p0 + t + 1)
            o = o.view(nkv, G, d)
            seen = torch.isnan(v[:, : p0 + t + 1]).any(1)[:, None, :] | torch.isnan(k[:, : p0 + t + 1]).any(-1).any(-1)[:, None, None]
            got = out[row + t].double().view(nkv, G, d)
            assert torch.equal(torch.isnan(got), seen.expand_as(got)), (slot, t)
            tol = ref.attention_bound(o, pv.view(nkv, G, d), size, d, p0 + t + 1, 2.0**-8)
            fine = ~seen.expand_as(got)
            assert ((got - o).abs() <= tol)[fine].all(), (slot, t)


def test_prefill_attention_bad_pages():
    d, nkv, G, blk, page, cap = 128, 1, 2, 16, 16, 256
    hc = HostCache(nkv, d, 2, cap, blk, page, seed=60)
    good = hc.table.clone()
    hc.table[1, 5] = 1 << 30                          # tokens 80 .. 95
    cache = hc.device_cache(corun)
    lens, starts, slots = [150, 60], [0, 30], [0, 1]
    x, q = rows_of(210, nkv * G, d, 61)
    out = run_prefill(cache, q, lens, starts, slots)
    assert torch.isnan(out[150 + 50:]).all()          # positions 80 ..
    hc.table = good
    check_prefill(hc, x, out, [(0, 150, 0, 0), (150, 50, 30, 1)], every=7)


def test_prefill_attention_long():
    """A chunk deep in a long prompt, and more sequences than a tile's rows."""
    d, nkv, G, blk, page = 128, 2, 4, 16, 16
    cap = 5120
    hc = HostCache(nkv, d, 2, cap, blk, page, seed=70)
    cache = hc.device_cache(corun)
    x, q = rows_of(601, nkv * G, d, 71, loud=False)
    out = run_prefill(cache, q, [601], [4444], [1])
    check_prefill(hc, x, out, [(0, 601, 4444, 1)], every=60)
    lens = [1 + i % 5 for i in range(64)]
    hc = HostCache(nkv, d, 64, 64, blk, page, seed=72)
    cache = hc.device_cache(corun)
    x, q = rows_of(sum(lens), nkv * G, d, 73)
    starts, slots = [i % 17 for i in range(64)], [(i * 37) % 64 for i in range(64)]
    out = run_prefill(cache, q, lens, starts, slots)
    check_prefill(hc, x, out, seqs_of(lens, starts, slots))


@pytest.mark.parametrize("page", [0, 192])
def test_prefill_attention_of_many_rows_and_long_sequences(page):
    """Workgroups of eight wavefronts (over 2048 keys, more than 128 such workgroups); a sequence's bits alone,
    where there are few; rows before, around and behind a page that is none."""
    d, nkv, G, blk, cap = 128, 8, 16, 32, 2304
    hc = HostCache(nkv, d, 3, cap, blk, page, seed=74)
    a, b = hc.at(0, 2290)
    hc.v[a, 3, b, 7] = 0x7F
    cache = hc.device_cache(corun)
    lens, starts, slots = [1, 270, 40], [5, 2034, 2200], [1, 2, 0]
    x, q = rows_of(sum(lens), nkv * G, d, 75, pad=8, loud=False)
    out = run_prefill(cache, q, lens, starts, slots)
    check_prefill(hc, x, out, [(0, 1, 5, 1), (1, 270, 2034, 2)], every=45)
    check_prefill(hc, x, out, [(271, 40, 2200, 0)], every=80)
    for row, n, p0, slot in seqs_of(lens, starts, slots):
        if n < 270:
            assert same(run_prefill(cache, q[row:row + n], [n], [p0], [slot]), out[row:row + n])
    if page:
        hc.table[2, 11] = -1                          # tokens 2112 .., rows 78 .. of the second sequence
        bad = run_prefill(hc.device_cache(corun), q, lens, starts, slots)
        assert same(bad[:65], out[:65]) and same(bad[271:], out[271:])
        assert torch.isnan(bad[1 + 78:271]).all()
        hc.table[2, 11] = 0                           # any page: rows 64 .. 77 do not see it
        check_prefill(hc, x, bad, [(65, 14, 2098, 2)], every=6)



@pytest.mark.parametrize("d,nkv,G,n,start,blk,page", [
    (128, 2, 1, 1, 4990, 64, 0), (64, 1, 3, 70, 3001, 16, 48), (128, 8, 4, 33, 2047, 32, 32), (128, 1, 16, 100, 4000, 64, 192),
    (64, 4, 8, 129, 1100, 32, 0), (128, 4, 7, 31, 1025, 16, 16)])
def test_prefill_attention_of_few_rows_behind_many(d, nkv, G, n, start, blk, page):
    """Sequences that are split over their keys: alone, beside others, and with whatever was in the workspace."""
    cap = (start + n + 767) // 768 * 768
    hc = HostCache(nkv, d, 3, cap, blk, page, seed=76)
    cache = hc.device_cache(corun)
    lens, starts, slots = [40, n, 5], [0, start, 1600 if start > 2000 else 7], [1, 2, 0]
    x, q = rows_of(sum(lens), nkv * G, d, 77, pad=8, loud=False)
    need = corun.prefill_attention_workspace(cache, nkv * G, lens, starts)
    assert need >= corun.prefill_attention_workspace(cache, nkv * G, [n], [start]) > 0
    out = run_prefill(cache, q, lens, starts, slots)
    check_prefill(hc, x, out, seqs_of(lens, starts, slots), every=max(1, n // 5))
    alone = torch.full((n, nkv * G * d), 5.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device=DEV)     # NaN, were any of it read before it is written
    corun.prefill_attention(cache, 0, q[40:40 + n], [n], [start], [2], alone, ws=ws)
    torch.cuda.synchronize()
    assert same(alone.cpu(), out[40:40 + n])


@pytest.mark.parametrize("page", [0, 64])
def test_prefill_attention_split_rows_with_nan_and_bad_pages(page):
    """NaN values and a lost page inside a split: rows before them are as without, rows behind are NaN."""
    d, nkv, G, blk, n, start, cap = 128, 1, 2, 32, 300, 2000, 2304
    hc = HostCache(nkv, d, 1, cap, blk, page, seed=78)
    x, q = rows_of(n, nkv * G, d, 79, loud=False)
    assert corun.prefill_attention_workspace(hc.device_cache(corun), nkv * G, [n], [start]) > 0
    good = run_prefill(hc.device_cache(corun), q, [n], [start], [0])
    check_prefill(hc, x, good, [(0, n, start, 0)], every=60)
    a, b = hc.at(0, 2150)
    code = int(hc.v[a, 0, b, 11])
    hc.v[a, 0, b, 11] = 0x7F
    out = run_prefill(hc.device_cache(corun), q, [n], [start], [0])
    dims = torch.arange(nkv * G * d) % d == 11
    assert torch.equal(torch.isnan(out), (torch.arange(n) >= 150)[:, None] & dims[None])
    assert same(out[:96], good[:96])                  # units that take the tile of the NaN do their rows another way
    hc.v[a, 0, b, 11] = code
    check_prefill(hc, x, torch.where(dims[None], good, out), [(0, n, start, 0)], every=23)
    hc.v[a, 0, b, 11] = 0x7F
    if page:
        hc.table[0, 34] = hc.k.shape[0]               # tokens 2176 ..
        out = run_prefill(hc.device_cache(corun), q, [n], [start], [0])
        assert torch.isnan(out[176:]).all() and not torch.isnan(out[:150]).any() and same(out[:96], good[:96])


def test_prefill_attention_split_replays_from_a_graph():
    d, nkv, G, blk, n, start, cap = 128, 2, 4, 32, 50, 3000, 3136
    hc = HostCache(nkv, d, 2, cap, blk, seed=80)
    cache = hc.device_cache(corun)
    qs = [rows_of(n, nkv * G, d, 81 + i)[1] for i in range(3)]
    want = [run_prefill(cache, q, [n], [start], [1]) for q in qs]
    q, out = qs[0].clone(), torch.zeros_like(qs[0])
    ws = torch.zeros(corun.prefill_attention_workspace(cache, nkv * G, [n], [start]), dtype=torch.uint8, device=DEV)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        corun.prefill_attention(cache, 0, q, [n], [start], [1], out, ws=ws)
    for i in (1, 0, 2, 1):
        q.copy_(qs[i])
        out.zero_()
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        assert same(out.cpu(), want[i])



@pytest.mark.parametrize("d,G,page,start", [(128, 4, 0, 0), (64, 2, 48, 0), (128, 2, 16, 1000)])
def test_prefill_attention_values_of_any_size(d, G, page, start):
    """Blocks of values many powers of two apart, empty ones, and huge ones that a query does not see yet."""
    nkv, blk, n = 2, 16, 220
    cap = 1248 if start else 240
    hc = HostCache(nkv, d, 1, cap, blk, page, seed=90)
    first = start // blk
    for i, byte in ((0, 121), (1, 60), (2, 27), (3, 118), (4, 240), (5, 121), (6, 27), (7, 150), (8, 121), (9, 245), (10, 100)):
        a, b = hc.at(0, (first + i) * blk)
        hc.vs[a, i % 2, b // blk] = byte
        if i in (2, 6):
            hc.v[a, i % 2, b:b + blk] = 0             # what an append of zeros leaves
    x, q = rows_of(n, nkv * G, d, 91, loud=False)
    out = run_prefill(hc.device_cache(corun), q, [n], [start], [0])
    check_prefill(hc, x, out, [(0, n, start, 0)], every=3)



# --------------------------------------------------------------------------
# Together, as a layer calls them
# --------------------------------------------------------------------------

class Layer:
    """A prompt, then decode steps, through append and attention; the 64-bit
    reference reads what the device cache holds after each append."""

    def __init__(self, d=128, nkv=2, G=4, blk=16, page=16, rows=3, cap=160, rope="bands"):
        self.d, self.nkv, self.nq, self.rows = d, nkv, nkv * G, rows
        self.hc = HostCache(nkv, d, rows, cap, blk, page, seed=80)
        self.cache = self.hc.device_cache(corun)
        self.rope, self.rot = make_rope(rope, d)
        self.q = torch.zeros((256, self.nq * d), dtype=torch.bfloat16, device=DEV)
        self.out = torch.zeros_like(self.q)
        self.ws = torch.empty(max(16, corun.decode_attention_workspace(self.cache, rows, self.nq)), dtype=torch.uint8, device=DEV)

    def prompts(self, x, lens, slots):
        n = x.shape[0]
        corun.prefill_append(self.cache, 0, x, lens, None, slots, self.rope, self.q[:n])
        corun.prefill_attention(self.cache, 0, self.q[:n], lens, None, slots, self.out[:n])

    def step(self, x, pos, lens, valid):
        r = self.rows
        corun.decode_append(self.cache, 0, x, pos, self.rope, self.q[:r], valid=valid)
        corun.decode_attention(self.cache, 0, self.q[:r], lens, self.out[:r], self.ws, valid=valid)


@pytest.mark.parametrize("d,page", [(128, 16), (64, 0)])
def test_prompt_then_decode(d, page):
    lay = Layer(d=d, page=page)
    heads = lay.nq + 2 * lay.nkv
    lens = [37, 1, 80]
    x, xd = rows_of(sum(lens), heads, d, 81)
    lay.prompts(xd, lens, [2, 0, 1])
    torch.cuda.synchronize()
    hc = lay.hc.after()
    check_prefill(hc, lay.q[: sum(lens)].cpu(), lay.out[: sum(lens)].cpu(), [(0, 37, 0, 2), (37, 1, 0, 0), (38, 80, 0, 1)], every=5)
    pos = [1, 80, 37]
    for i in range(20):
        x, xd = rows_of(3, heads, d, 90 + i)
        valid = [1, 0 if i in (4, 5) else 1, 1]
        before = lay.hc.after()
        pd = torch.tensor(pos, dtype=torch.int32, device=DEV)
        lay.step(xd, pd, pd + 1, torch.tensor(valid, dtype=torch.uint8, device=DEV))
        torch.cuda.synchronize()
        after = lay.hc.after()
        x64 = x.double().view(3, heads, d)
        y, _ = lay.rot(x64[:, : lay.nq + lay.nkv], torch.tensor(pos))
        live = [r for r in range(3) if valid[r]]
        ref.check_append(before, after, [(r, 1, pos[r], r) for r in live], y[:, lay.nq:], x64[:, lay.nq + lay.nkv:])
        check_decode(after, lay.q[:3].cpu(), [p + 1 for p in pos], live, lay.out[:3].cpu())
        pos = [p + v for p, v in zip(pos, valid)]


def test_captured_step_replays():
    """A step captured once and replayed, with eager work between, gives the eager bits at every position."""
    a, b = Layer(), Layer()
    heads = a.nq + 2 * a.nkv
    x, xd = rows_of(3, heads, 128, 95)
    pos = torch.tensor([0, 40, 90], dtype=torch.int32, device=DEV)
    lens, valid = pos + 1, torch.tensor([1, 1, 0], dtype=torch.uint8, device=DEV)
    xs, ps, ls = xd.contiguous().clone(), pos.clone(), lens.clone()
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        a.step(xs, ps, ls, valid)
    for i in range(6):
        x, xd = rows_of(3, heads, 128, 96 + i)
        xs.copy_(xd)
        ps.copy_(pos + i)
        ls.copy_(lens + i)
        g.replay()
        b.step(xd, pos + i, lens + i, valid)
        torch.cuda.synchronize()
        assert same(a.out[:3], b.out[:3]) and same(a.q[:2], b.q[:2])
        for t, u in zip(a.hc.dev + a.hc.devs, b.hc.dev + b.hc.devs):
            assert same(t, u)


def test_two_streams_with_their_own_workspaces():
    lay = Layer(cap=160)
    q = [rows_of(3, lay.nq, 128, 200 + i)[1].contiguous() for i in range(2)]
    lens = torch.tensor([160, 77, 3], dtype=torch.int32, device=DEV)
    ws = [torch.empty_like(lay.ws) for _ in range(2)]
    want = [run_decode(lay.cache, qq, lens.cpu()) for qq in q]
    out = [torch.zeros_like(qq) for qq in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(20):
        for i in range(2):
            corun.decode_attention(lay.cache, 0, q[i], lens, out[i], ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert same(out[i].cpu(), want[i])


def test_python_refusals():
    lay = Layer()
    x = torch.zeros((3, (lay.nq + 2 * lay.nkv) * 128), dtype=torch.bfloat16, device=DEV)
    pos = torch.zeros(3, dtype=torch.int32, device=DEV)
    q = lay.q[:3]
    bad = [
        lambda: corun.decode_append(lay.cache, 1, x, pos, lay.rope, q),
        lambda: corun.decode_append(lay.cache, 0, x.float(), pos, lay.rope, q),
        lambda: corun.decode_append(lay.cache, 0, x, pos.long(), lay.rope, q),
        lambda: corun.decode_append(lay.cache, 0, x, pos.cpu(), lay.rope, q),
        lambda: corun.decode_append(lay.cache, 0, x, pos[:2], lay.rope, q),
        lambda: corun.decode_append(lay.cache, 0, x[:2], pos[:2], lay.rope, q),
        lambda: corun.decode_append(lay.cache, 0, x.t().contiguous().t(), pos, lay.rope, q),
        lambda: corun.decode_append(lay.cache, 0, x, pos, corun.rope(64), q),
        lambda: corun.prefill_append(lay.cache, 0, x, [1, 1], None, [0, 1], lay.rope, q),
        lambda: corun.prefill_append(lay.cache, 0, x, [1, 2], [0], [0, 1], lay.rope, q),
        lambda: corun.prefill_append(lay.cache, 0, x, [1, 2], None, [1, 1], lay.rope, q),
        lambda: corun.decode_attention(lay.cache, 0, q, pos, lay.out[:2], lay.ws),
        lambda: corun.decode_attention(lay.cache, 0, q, pos, lay.out[:3], lay.ws.view(torch.int8)),
        lambda: corun.prefill_attention(lay.cache, 0, q, [4], None, [0], lay.out[:3]),
    ]
    for f in bad:
        with pytest.raises((ValueError, corun.CorunError)):
            f()
    torch.cuda.synchronize()
