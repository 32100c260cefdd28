"""Prefill attention over e4m3 caches where scores and values range widely:
large values behind small weights, before and behind them, in one piece and
split over the keys.

The kernel's weights are fp16 of the softmax's weight times the largest scale
of the key's tile of 64, under a reference that is at most 2^4 above the
largest weight times scale (scales of a tile further apart than that are taken
singly).  Each is off by half a step, 2^-11 of itself, or, among the
subnormals, by 2^-25 where the largest is at least 2^(8 - 4); a code of at
most 448 multiplies it."""
import math

import numpy as np
import pytest
import torch

from paper_2608_14376_amd import corun
from tests import cache_reference as ref
from tests.cache_reference import HostCache
from tests.test_gpu_cache_ops import DEV, rows_of, run_prefill, seqs_of

pytestmark = pytest.mark.gpu
U_WEIGHT = 2.0**-11 + 2.0**-16   # fp16; fp32 roundings of scores moved by up to 90 (in base 2) for their scales: 2^-17.5, 2^-17


def lost(p, scale, n):
    """What n weights that fp16 cannot hold may add up to: p [.., n] of one row, scales 2^e of the keys."""
    return n * 2.0**-29 * 448 * (p * scale).max().item()


def check(hc, x, out, seqs, every):
    d, nkv, blk = hc.d, hc.nkv, hc.blk
    for row, n, p0, slot in seqs:
        k, v = hc.values(slot, p0 + n)
        for t in sorted(set(range(0, n, every)) | {0, n - 1}):
            m = p0 + t + 1
            q = x[row + t].double().view(-1, d)
            o, pv, size = ref.attention(q, k, v, m)
            got = out[row + t].double().view(-1, d)
            G = q.shape[0] // nkv
            s = torch.matmul(q.view(nkv, G, d), k[:, :m].transpose(1, 2).contiguous()) / math.sqrt(d)
            p = torch.softmax(s, -1)
            tol = ref.attention_bound(o, pv, size, d, m, U_WEIGHT).view(nkv, G, d)
            for h in range(nkv):
                sc = torch.stack([2.0 ** (hc.vs[hc.at(slot, i)[0], h, hc.at(slot, i)[1] // blk].double() - 127)
                                  for i in range(0, m, blk)]).repeat_interleave(blk)[:m]
                for g in range(G):
                    tol[h, g] += lost(p[h, g], sc, m)
            off = (got - o).abs() / tol.view(-1, d)
            assert (off <= 1).all(), (slot, t, off.max())


@pytest.mark.parametrize("start", [0, 2048])
@pytest.mark.parametrize("large_first", [False, True])
def test_one_large_value_behind_a_small_weight(start, large_first):
    """64 values of 1 at equal scores and one of 2^44 whose weight is 2^-36.7: a result of 3.4, not of 1."""
    d, blk, n, cap = 128, 64, 129, 2304
    hc = HostCache(1, d, 1, cap, blk, seed=1)
    hc.k[:], hc.v[:], hc.ks[:], hc.vs[:] = 0, 0x38, 127, 127        # scores of 0, values of 1
    hc.k[0, 0, :, 0] = 0xE0                                         # -32: no weight at all
    one = start + (0 if large_first else 128)                       # the tile of the large value, and that of the 64
    many = start + (64 if large_first else 0)
    hc.k[0, 0, many:many + 64, 0] = 0
    hc.k[0, 0, one, 0] = 0xD9                                       # -18: a score of -25.46, times log2 e -36.73
    hc.vs[0, 0, one // blk] = 127 + 36
    hc.v[0, 0, one // blk * blk:one // blk * blk + blk] = 0
    hc.v[0, 0, one] = 0x78                                          # 2^8
    x = torch.zeros((n, d), dtype=torch.bfloat16)
    x[:, 0] = 16
    out = run_prefill(hc.device_cache(corun), x.to(DEV), [n], [start], [0])
    got = out[128].double()
    want = 1 + 2.0**44 * math.exp(-18 * 16 / math.sqrt(d)) / 64
    assert ((got - want).abs() <= want * (2.0**-8 + 2.0**-10)).all(), (got[:4], want)
    check(hc, x, out, [(0, n, start, 0)], every=32)


@pytest.mark.parametrize("d,G,page,start,n", [(128, 2, 0, 0, 200), (64, 3, 48, 0, 200), (128, 2, 48, 1500, 60),
                                              (64, 2, 0, 2100, 33)])
@pytest.mark.parametrize("order", ["rising", "falling", "mixed"])
@pytest.mark.parametrize("spread", [20, 40, 60])
def test_values_as_large_as_their_weights_are_small(d, G, page, start, n, order, spread):
    """Blocks whose values are 2^L larger and whose weights 2^L smaller, L up to `spread`, so that all of them
    count.  With 60 the scales are further apart than one pass holds."""
    nkv, blk, cap = 2, 16, 2208
    hc = HostCache(nkv, d, 1, cap, blk, page, seed=spread + n)
    rng = np.random.default_rng(spread + start)
    blocks = cap // blk
    level = np.linspace(0, spread, blocks) if order != "mixed" else rng.uniform(0, spread, blocks)
    if order != "mixed" and start == 0:
        level = np.concatenate([np.linspace(0, spread, n // blk + 1), np.full(blocks - n // blk - 1, spread)])
    if order == "falling":
        level = spread - level
    hc.k[:] = 0
    for i in range(blocks):
        a, b = hc.at(0, i * blk)
        # the score of code c in dimension 0 under 2^0: 11.3125 c / sqrt(d), 16 / sqrt(d) or so in base 2
        want = -level[i] * math.log(2) * math.sqrt(d) / 11.3125
        codes = torch.tensor(want + rng.uniform(-2, 2, (nkv, blk))).float().to(torch.float8_e4m3fn)
        hc.k[a, :, b:b + blk, 0] = codes.view(torch.uint8)
        hc.ks[a, :, b // blk] = 127
        # where the code is rough, the value follows it
        got = codes.float().mean(1) * 11.3125 / math.sqrt(d) / math.log(2)
        sign = 1 if spread < 60 else 1.6
        hc.vs[a, :, b // blk] = (100 - sign * got + torch.tensor(rng.uniform(-3, 3, nkv))).clamp(27, 247).to(torch.uint8)
    x, _ = rows_of(n, nkv * G, d, 5, loud=False)
    x = (x.float() * 0).to(torch.bfloat16)
    x.view(n, nkv * G, d)[:, :, 0] = 11.3125
    out = run_prefill(hc.device_cache(corun), x.to(DEV), [n], [start], [0])
    check(hc, x, out, seqs_of([n], [start], [0]), every=max(1, n // 7))


@pytest.mark.parametrize("d,page", [(128, 0), (64, 16)])
def test_weights_keep_the_bits_of_fp16(d, page):
    """A few keys to a row, where a result is the small difference of large terms: weights of 8 bits would show."""
    nkv, G, blk, cap = 2, 2, 16, 64
    for seed in range(4):
        hc = HostCache(nkv, d, 1, cap, blk, page, seed=200 + seed)
        x, q = rows_of(24, nkv * G, d, 210 + seed, loud=False)
        out = run_prefill(hc.device_cache(corun), q, [24], [0], [0])
        check(hc, x, out, [(0, 24, 0, 0)], every=1)


@pytest.mark.parametrize("start", [0, 1024])
@pytest.mark.parametrize("d", [64, 128])
def test_a_lost_page_leaves_earlier_rows_alone(start, d):
    """Rows before a page that is none, in its tile: the same bits whatever stands in the cache's first page."""
    nkv, G, blk, page, n, cap = 1, 1, 16, 16, 64, 1152
    hc = HostCache(nkv, d, 2, cap, blk, page, seed=95)
    hc.table[hc.table == 0] = hc.k.shape[0] - 1       # no sequence has the first page
    x, q = rows_of(n, nkv * G, d, 96, loud=False)
    good = run_prefill(hc.device_cache(corun), q, [n], [start], [1])
    hc.table[1, (start + 48) // page] = -7            # tokens 48 .. 63 of the rows' tile
    outs = []
    for code, byte in ((0x38, 121), (0x7F, 121), (0x7E, 140), (0x7E, 247)):
        hc.v[0], hc.k[0], hc.vs[0] = code, code, byte
        outs.append(run_prefill(hc.device_cache(corun), q, [n], [start], [1]))
        assert torch.isnan(outs[-1][48:]).all() and not torch.isnan(outs[-1][:48]).any()
        assert torch.equal(outs[-1][:48].view(torch.uint8), outs[0][:48].view(torch.uint8)), (code, byte)
    check(hc, x, good, [(0, 40, start, 1)], every=9)
    hc.table[1, (start + 48) // page] = 0
    check(hc, x, outs[0], [(0, 48, start, 1)], every=9)


@pytest.mark.parametrize("d,page,start,n", [(128, 0, 0, 130), (64, 32, 0, 70), (128, 16, 1400, 40)])
@pytest.mark.parametrize("lo,hi", [(27, 52), (50, 75), (60, 90), (150, 165), (200, 240)])
def test_scales_at_both_ends(d, page, start, n, lo, hi):
    """Values of about 2^-95 up to 2^118: around the least and the largest scales of the fast pass, and beyond both."""
    nkv, G, blk, cap = 2, 2, 16, 1536
    hc = HostCache(nkv, d, 1, cap, blk, page, seed=lo)
    g = torch.Generator().manual_seed(hi)
    hc.vs = torch.randint(lo, hi + 1, hc.vs.shape, generator=g).to(torch.uint8)
    x, q = rows_of(n, nkv * G, d, 7, loud=False)
    out = run_prefill(hc.device_cache(corun), q, [n], [start], [0])
    check(hc, x, out, [(0, n, start, 0)], every=max(1, n // 5))
