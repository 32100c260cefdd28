"""Calls of the cache operators that use their workspaces: captured and
replayed, on two streams at once; and appends at the farthest positions."""
import numpy as np
import pytest
import torch

from paper_2608_14376_amd import corun
from tests import cache_reference as ref
from tests.cache_reference import HostCache
from tests.test_gpu_cache_ops import DEV, Layer, check_decode, make_rope, rows_of, run_decode, run_prefill, same

pytestmark = pytest.mark.gpu
CAP = 1536


@pytest.mark.parametrize("d,page", [(128, 16), (64, 0)])
def test_captured_step_of_several_splits_replays(d, page):
    """Append, attention over several splits and their merge, captured once: the eager bits at every replay, whatever
    the workspace holds."""
    a, b = Layer(d=d, page=page, cap=CAP), Layer(d=d, page=page, cap=CAP)
    assert corun.decode_attention_workspace(a.cache, 3, a.nq) > 0
    heads = a.nq + 2 * a.nkv
    pos = torch.tensor([126, 1270, 0], dtype=torch.int32, device=DEV)
    valid = torch.tensor([1, 1, 1], dtype=torch.uint8, device=DEV)
    xs = rows_of(3, heads, d, 95)[1].contiguous().clone()
    ps, ls = pos.clone(), pos + 1
    s, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=s):
        a.step(xs, ps, ls, valid)
    for i in range(6):                                # row 0 crosses from one split of 128 to two
        x, xd = rows_of(3, heads, d, 96 + i)
        xs.copy_(xd)
        ps.copy_(pos + i)
        ls.copy_(pos + i + 1)
        a.ws.fill_(0xFF)
        a.out.fill_(5.0)
        g.replay()
        b.step(xd, pos + i, pos + i + 1, valid)
        torch.cuda.synchronize()
        assert same(a.out[:3], b.out[:3]) and same(a.q[:3], b.q[:3])
        for t, u in zip(a.hc.dev + a.hc.devs, b.hc.dev + b.hc.devs):
            assert same(t, u)
        check_decode(b.hc.after(), b.q[:3].cpu(), (pos + i + 1).tolist(), range(3), b.out[:3].cpu())


def test_decode_on_two_streams_with_their_own_workspaces():
    lay = Layer(cap=CAP)
    size = corun.decode_attention_workspace(lay.cache, 3, lay.nq)
    assert size > 0
    q = [rows_of(3, lay.nq, 128, 200 + i)[1].contiguous() for i in range(2)]
    lens = torch.tensor([CAP, 777, 129], dtype=torch.int32, device=DEV)
    ws = [torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV) for _ in range(2)]
    want = [run_decode(lay.cache, qq, lens.cpu()) for qq in q]
    assert not same(want[0], want[1])
    out = [[torch.zeros_like(q[i]) for _ in range(20)] for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for n in range(20):
        for i in range(2):
            corun.decode_attention(lay.cache, 0, q[i], lens, out[i][n], ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        for o in out[i]:
            assert same(o.cpu(), want[i])


@pytest.mark.parametrize("own_ws", [True, False])
def test_prefill_on_two_streams_with_splits(own_ws):
    """Split prefill attention on two streams, with workspaces of the caller's or the allocator's."""
    d, nkv, G, blk, n, start = 128, 2, 4, 32, 40, 1400
    hc = HostCache(nkv, d, 2, CAP, blk, seed=82)
    cache = hc.device_cache(corun)
    size = corun.prefill_attention_workspace(cache, nkv * G, [n], [start])
    assert size > 0
    q = [rows_of(n, nkv * G, d, 300 + i)[1].contiguous() for i in range(2)]
    want = [run_prefill(cache, q[i], [n], [start], [i]) for i in range(2)]
    ws = [torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV) if own_ws else None for _ in range(2)]
    out = [[torch.zeros_like(q[i]) for _ in range(20)] for i in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for j in range(20):
        for i in range(2):
            corun.prefill_attention(cache, 0, q[i], [n], [start], [i], out[i][j], ws=ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        for o in out[i]:
            assert same(o.cpu(), want[i])


@pytest.mark.parametrize("e4m3", [False, True])
def test_append_at_the_farthest_positions(e4m3):
    """The last positions that a slot can have, 2^30 - 1, on one page of 2^20 tokens that is every page."""
    d, nkv, nq, page = 64, 1, 2, 1 << 20
    pos = [(1 << 30) - 1, (1 << 30) - (1 << 20) - 71, (1 << 29) + 5]   # blocks of their own in the page
    rope, _ = make_rope("half", d)
    table = torch.zeros((3, 1024), dtype=torch.int32, device=DEV)
    if e4m3:
        k, v = (torch.zeros((1, nkv, page, d), dtype=torch.uint8, device=DEV) for _ in range(2))
        ks, vs = (torch.full((1, nkv, page // 16), 27, dtype=torch.uint8, device=DEV) for _ in range(2))
        cache = corun.KvCache([k], [v], [ks], [vs], 16, table)
    else:
        k, v = (torch.zeros((1, nkv, page, d), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        cache = corun.KvCache([k], [v], page_table=table)
    x, xd = rows_of(3, nq + 2 * nkv, d, 9, loud=False)
    q = torch.zeros((3, nq * d), dtype=torch.bfloat16, device=DEV)
    corun.decode_append(cache, 0, xd, torch.tensor(pos, dtype=torch.int32, device=DEV), rope, q)
    # one beyond is outside the cache, as is the largest position
    q2 = torch.zeros_like(q)
    corun.decode_append(cache, 0, xd, torch.tensor([1 << 30, 2**31 - 1, -1], dtype=torch.int32, device=DEV), rope, q2)
    torch.cuda.synchronize()
    assert torch.isnan(q2).all()
    # turns of 2^30 positions by angles rounded to 64 bits: the kernel's turn count and the reference's angle are each
    # off by up to 2^-53 of 2^30 radians and a rounding more, together under 2^-21
    f = torch.tensor([rope.freq[i] for i in range(d // 2)], dtype=torch.float64)
    ang = torch.tensor(pos, dtype=torch.float64)[:, None] * f
    c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
    x64 = x.double().view(3, nq + 2 * nkv, d)
    u, w = x64[:, :nq + nkv, :d // 2], x64[:, :nq + nkv, d // 2:]
    y = torch.cat([u * c - w * s, w * c + u * s], -1)
    size = torch.cat([u.abs() + w.abs()] * 2, -1)
    tol = ref.U_BF16 * y.abs() + (4 * ref.U_F32 + 2.0**-21) * size
    assert ((q.cpu().double().view(3, nq, d) - y[:, :nq]).abs() <= tol[:, :nq]).all()
    for r, p in enumerate(pos):
        at = p % page
        for h, (cache_t, sc, want) in enumerate(((k, ks if e4m3 else None, y[r, nq:]),
                                                 (v, vs if e4m3 else None, x64[r, nq + nkv:]))):
            got = cache_t[0, :, at].cpu()
            if not e4m3:
                assert ((got.double() - want).abs() <= ref.U_BF16 * want.abs() + 2.0**-21 * size[r, nq:] * (1 - h)).all()
                continue
            e = int(sc[0, 0, at // 16]) - 127
            val = got.view(torch.float8_e4m3fn).float().double() * 2.0**e
            assert want.abs().max() <= 448 * 2.0**e * (1 + 1e-5) and want.abs().max() > 224 * 2.0**e * (1 - 1e-5)
            assert ((val - want).abs() <= torch.maximum(ref.U_E4M3 * want.abs(), torch.tensor(2.0**(e - 10), dtype=torch.float64))
                    + 2.0**-21 * size[r, nq:] * (1 - h)).all()


def test_one_row_whose_stride_is_no_multiple_of_8():
    """The distance to a row that is not there: a single row cut out of a wider buffer."""
    lay = Layer(cap=CAP, rows=1)
    heads = lay.nq + 2 * lay.nkv
    x = rows_of(1, heads, 128, 41)[1].contiguous()
    cut = lambda t: torch.cat([t, torch.zeros_like(t[:, :4])], 1).repeat(2, 1)[:1, : t.shape[1]]
    pos, live = torch.tensor([700], dtype=torch.int32, device=DEV), torch.ones(1, dtype=torch.uint8, device=DEV)
    lay.step(x, pos, pos + 1, live)
    q, out, xc = cut(lay.q[:1]), cut(lay.out[:1]), cut(x)
    assert xc.stride(0) % 8 == 4
    q.zero_(), out.zero_()
    corun.decode_append(lay.cache, 0, xc, pos, lay.rope, q, valid=live)
    corun.decode_attention(lay.cache, 0, q, pos + 1, out, lay.ws, valid=live)
    assert same(q, lay.q[:1]) and same(out, lay.out[:1])
    out.zero_()
    corun.prefill_attention(lay.cache, 0, q, [1], [700], [0], out)
    want = torch.zeros_like(lay.out[:1])
    corun.prefill_attention(lay.cache, 0, lay.q[:1], [1], [700], [0], want)
    torch.cuda.synchronize()
    assert same(out, want)
