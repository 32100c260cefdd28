"""Attention over shared prefixes where values range widely: blocks of an e4m3
prefix whose scales are far above or below the others', and values that only
small weights meet.

Every weight has at least 16 bits, however small, whatever the cache's type and
the number of queries: cache_reference.attention_bound with 2^-14, which leaves
room for both halves' roundings (2^-9 of 2^-8) and for fp32 sums."""
import pytest
import torch

from paper_2608_14376_amd import corun
from tests.cache_reference import HostCache
from tests.test_gpu_cache_ops import rows_of
from tests import cache_reference as ref
from tests import group_reference as gref
from tests.test_gpu_shared import DEV, U_WEIGHT, run

pytestmark = pytest.mark.gpu


def check(hc, q, out, rows, P, lens, slot):
    for r in rows:
        want, pv, size = gref.shared_attention(hc, q[r].double().view(-1, hc.d), r, slot, P, lens[r])
        tol = ref.attention_bound(want, pv, size, hc.d, lens[r], U_WEIGHT)
        err = (out[r].double().view(-1, hc.d) - want).abs()
        assert (err <= tol).all(), (r, float((err / tol.clamp(min=1e-300)).max()))


# 27 is the byte of a block whose values are all zero, as the append writes it
@pytest.mark.parametrize("byte", [27, 95, 96, 104, 136, 144, 145, 200])
@pytest.mark.parametrize("d,page,rows", [(128, 0, 30), (64, 48, 30), (128, 32, 3)])
def test_one_block_of_another_scale(d, page, rows, byte):
    """One block, not the first of its split, has another scale; its values are zero in all but one dimension, or in all."""
    nq, nkv, P, blk = 8, 2, 700, 16
    cap = -(-(P + 64) // 96) * 96 if page else 1792
    hc = HostCache(nkv, d, rows + 1, cap, blk, page, seed=40, dtype="e4m3")
    hc.vs[:] = 120
    pg, t = hc.at(rows, 400)
    codes = hc.v[pg, :, t:t + blk]
    codes[..., :5] = codes[..., 6:] = 0
    if byte == 27:
        codes[:] = 0
    hc.vs[pg, :, t // blk] = byte
    q, qd = rows_of(rows, nq, d, 41)
    lens = [P + r % 5 for r in range(rows)]
    out = run(hc.device_cache(corun), qd, [rows], lens, [P], [rows])
    check(hc, q, out, range(rows), P, lens, rows)


@pytest.mark.parametrize("dtype", ["bf16", "e4m3"])
@pytest.mark.parametrize("gap", [12, 24, 33, 50])
@pytest.mark.parametrize("groups", [[30], [3], [1, 40]])
def test_values_behind_small_weights(dtype, gap, groups):
    """One key has all but about 2^-gap of the weight, and values of zero in the upper half of the dimensions: what stands
    there comes from the others, of equal small weights."""
    nq, nkv, d, P, at = 8, 2, 128, 250, 100
    rows = sum(groups)
    hc = HostCache(nkv, d, rows + 1, 1536, 16, 0, seed=42, dtype=dtype)
    pg, t = hc.at(rows, at)
    hc.k[:], hc.v[pg, :, t, d // 2:] = 0, 0
    if dtype == "bf16":
        hc.k[pg, :, t, 0] = 1.0
    else:
        hc.ks[:] = 127
        hc.k[pg, :, t, 0] = 0x38                       # 1
    q = torch.zeros((rows, nq, d), dtype=torch.bfloat16)
    q[..., 0] = gap * 0.6931471805599453 * d**0.5      # the key's score, about gap in base 2
    q = q.view(rows, nq * d)
    lens = [P + r % 3 for r in range(rows)]
    out = run(hc.device_cache(corun), q.to(DEV), groups, lens, [P] * len(groups), [rows] * len(groups))
    check(hc, q, out, range(rows), P, lens, rows)


@pytest.mark.parametrize("heavy", [120, -8, 8])
def test_scales_apart_at_the_weights(heavy):
    """Scales of a prefix's blocks 24 above and 24 below each split's first, one 25 above and one 25 below in a later split;
    each is met by queries that give it most of their weight."""
    nq, nkv, d, rows, P, blk = 8, 2, 128, 40, 1500, 16
    hc = HostCache(nkv, d, rows + 1, 1792, blk, 0, seed=43, dtype="e4m3")
    hc.vs[:] = 120
    up = {3: 24, 9: -24, 35: 25, 60: -25, 80: 24}      # block: exponent; splits of 256 tokens start at 0, 16, 32 ..
    for b, e in up.items():
        hc.vs[rows, :, b] = 120 + e
    q, _ = rows_of(rows, nq, d, 44)
    if heavy < 100:
        for i, b in enumerate(up):                     # query row i: along the key of its block's third token
            key = hc.values(rows, P)[0][:, 16 * b + 2]
            along = key / key.norm(dim=-1, keepdim=True) * abs(heavy) * 2.0
            q[i] = (along if heavy > 0 else -along).repeat_interleave(nq // nkv, 0).reshape(-1).to(torch.bfloat16)
    lens = [P + r % 5 for r in range(rows)]
    out = run(hc.device_cache(corun), q.to(DEV), [rows], lens, [P], [rows])
    check(hc, q, out, range(rows), P, lens, rows)


@pytest.mark.parametrize("dtype,page", [("bf16", 0), ("bf16", 16), ("bf16", 48), ("e4m3", 0), ("e4m3", 16), ("e4m3", 48)])
@pytest.mark.parametrize("many", [1, 20])
@pytest.mark.parametrize("cap", [192, 1536])
def test_padding_rows_of_prefixes_out_of_range(dtype, page, many, cap):
    """Groups whose prefix has no length or no slot, that of row 0 among them: zeros for their padding rows, NaN for live
    ones, whether the call is one launch (cap 192, few rows) or split; rows of good groups beside them are right."""
    nq, nkv, d = 8, 2, 128
    groups = [2 * many, 2 * many, 2 * many, 2 * many, 2 * many, 2]
    rows = sum(groups)
    prefix, slots = [-1, cap + 1, 100, 33, 90, 100], [rows, rows, rows + 1, -5, -1, rows]
    hc = HostCache(nkv, d, rows + 1, cap, 16, page, seed=45, dtype=dtype)
    if page:
        hc.table[:5, 0] = 0                            # where reading before a page 0 would leave the cache
    of = [g for g, n in enumerate(groups) for _ in range(n)]
    valid = [int(r % 2) for r in range(rows)]
    lens = [[120, -1, 0, 150][(r // 2) % 4] if r < rows - 2 else 110 for r in range(rows)]
    valid[-2:] = 1, 1
    q, qd = rows_of(rows, nq, d, 46)
    out = torch.full((rows, nq * d), 5.0, dtype=torch.bfloat16, device=DEV)
    cache = hc.device_cache(corun)
    ws = torch.full((corun.shared_attention_workspace(cache, groups, nq),), 0xFF, dtype=torch.uint8, device=DEV)
    out = run(cache, qd, groups, lens, prefix, slots, valid, out=out, ws=ws)
    for r in range(rows - 2):
        assert (out[r] == 0).all() if not valid[r] else torch.isnan(out[r]).all(), (r, of[r])
    check(hc, q, out, [rows - 2, rows - 1], 100, lens, rows)
