"""Beam selection on the GPU against the 64-bit reference of
tests/group_reference.py.

Tokens, parents and flags are equal.  A score is the 64-bit one (reference and
kernel add the same terms in different orders: under vocab 2^-53 relative of the
sum, far below) rounded to fp32: half a step, 2^-24 relative."""
import numpy as np
import pytest
import torch

from paper_2608_14376_amd import corun
from tests import group_reference as gref

pytestmark = pytest.mark.gpu
DEV = "cuda"


def select(x, scores, beams, keep, valid=None, finished=None, weights=None, end=-1, pad=0, stream=None, ws=None):
    """Runs the operator on a device copy of numpy logits whose rows are `pad` elements apart (NaN between)."""
    rows, V = x.shape
    wide = torch.full((rows, V + pad), float("nan"), device=DEV)
    wide[:, :V] = torch.from_numpy(x).to(DEV)
    dev = lambda t, dt: None if t is None else torch.from_numpy(np.asarray(t)).to(DEV, dt)
    shape = (rows // beams, keep)
    tok, par = (torch.full(shape, 77, dtype=torch.int32, device=DEV) for _ in range(2))
    sc, fin = torch.full(shape, 7.0, device=DEV), torch.full(shape, 9, dtype=torch.uint8, device=DEV)
    if ws is None:
        ws = torch.full((corun.beam_select_workspace(V, shape[0], beams, keep),), 0xFF, dtype=torch.uint8, device=DEV)
    corun.beam_select(wide[:, :V], dev(scores, torch.float32), beams, tok, par, sc, ws, valid=dev(valid, torch.uint8),
                      finished=dev(finished, torch.uint8), weights=dev(weights, torch.float32), end_token=end,
                      out_finished=fin, stream=stream)
    torch.cuda.synchronize()
    return tok.cpu().numpy(), par.cpu().numpy(), sc.cpu().numpy(), fin.cpu().numpy()


def check(got, want):
    for a, b, name in zip(got, want, ("tokens", "parents", "scores", "finished")):
        if name == "scores":
            real = np.isfinite(b)
            assert np.array_equal(np.isneginf(a), ~real)
            assert (np.abs(a[real] - b[real]) <= 2.0**-24 * np.abs(b[real]) * (1 + 1e-6) + 2.0**-149).all()
        else:
            assert np.array_equal(a, b), (name, np.argwhere(a != b)[:4], a[a != b][:4], b[a != b][:4])


def logits_of(rows, V, seed, scale=2.0):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((rows, V)).astype(np.float32) * scale
    x[np.arange(rows)[:, None], rng.integers(0, V, (rows, 5))] += 6
    return x, -rng.exponential(4.0, rows).astype(np.float32)


@pytest.mark.parametrize("V", [1, 2, 31, 64, 257, 1024, 8191, 8193, 16384, 40001, 151936])
@pytest.mark.parametrize("groups,beams,keep,pad", [(1, 1, 1, 0), (3, 4, 8, 1), (2, 7, 5, 3), (1, 33, 64, 4)])
def test_select(V, groups, beams, keep, pad):
    x, s = logits_of(groups * beams, V, V + beams)
    check(select(x, s, beams, keep, pad=pad), gref.beam_select(x, s, beams, keep))


@pytest.mark.parametrize("V,beams,keep", [(1000, 5, 10), (9000, 3, 6), (20000, 64, 64)])
def test_padding_finished_rows_and_weights(V, beams, keep):
    groups = 3
    rows = groups * beams
    x, s = logits_of(rows, V, 3)
    rng = np.random.default_rng(5)
    valid, fin = (rng.random(rows) > 0.3).astype(np.uint8), (rng.random(rows) < 0.3).astype(np.uint8)
    w = rng.uniform(0.02, 0.1, rows).astype(np.float32)
    valid[:beams] = 0                                  # a group with nothing
    fin[beams:2 * beams] = 1                           # one where all are finished
    valid[beams] = 1
    x[(valid == 0) | (fin == 1)] = np.nan              # nothing of such rows' logits is used
    s[valid == 0] = np.nan
    end = int(np.argmax(np.nan_to_num(x[2 * beams:], nan=-9e9).max(0)))
    x[2 * beams:, end] += 20                           # some continuations end
    got = select(x, s, beams, keep, valid, fin, w, end, pad=2)
    want = gref.beam_select(x, s, beams, keep, valid, fin, w, end)
    check(got, want)
    assert (got[1][0] == -1).all() and (got[3][1][got[1][1] >= 0] == 1).all() and got[3][2].any()


@pytest.mark.parametrize("V", [100, 9000])
def test_weights_and_scores_out_of_range(V):
    x, s = logits_of(12, V, 8)
    w = np.ones(12, np.float32)
    w[:5] = [0.0, -1.0, np.inf, np.nan, 1e-38]
    s[5:9] = [-np.inf, np.nan, np.inf, -1e30]
    check(select(x, s, 6, 20, weights=w), gref.beam_select(x, s, 6, 20, weights=w))


@pytest.mark.parametrize("V", [3, 700, 8192, 30000])
def test_infinities_and_nan_among_the_logits(V):
    rows = 8
    x, s = logits_of(rows, V, 11)
    x[0, V // 2] = np.nan
    x[1, V - 1] = np.inf
    x[2] = -np.inf                                     # a mask that leaves nothing
    x[3, :] = -np.inf
    x[3, V // 3] = -5.0                                # ... one token
    x[4, ::2] = -np.inf
    x[5] = np.float32(-3.4028235e38)                   # the type's lowest value, and one token above it
    x[5, V - 1] = 1.0
    x[6, 0] = -np.float32(np.nan)
    check(select(x, s, 4, 8), gref.beam_select(x, s, 4, 8))


@pytest.mark.parametrize("V,step", [(5000, 0.5), (30000, 4.0), (9000, 1000.0), (151936, 1000.0)])
def test_ties_go_to_the_lower_row_and_token(V, step):
    """Equal logits within rows, and rows that are equal altogether; with a step of 1000 every logit is the same."""
    rng = np.random.default_rng(2)
    x = (np.round(rng.standard_normal((8, V)) * 2 / step) * step).astype(np.float32)
    x[3] = x[2]
    x[6] = x[7] = x[5]
    s = np.full(8, -2.5, np.float32)
    check(select(x, s, 4, 16), gref.beam_select(x, s, 4, 16))
    x = np.sort(x, 1)                                  # ascending and descending: the largest in one place
    check(select(x, s, 4, 16), gref.beam_select(x, s, 4, 16))
    x = np.ascontiguousarray(x[:, ::-1])
    check(select(x, s, 4, 16), gref.beam_select(x, s, 4, 16))


@pytest.mark.parametrize("V", [40, 9000])
def test_both_zeros_are_equal(V):
    x = -np.abs(logits_of(4, V, 9)[0])
    x[:, 3::7] = -0.0
    x[:, 5::14] = 0.0
    s = np.array([0.0, -0.0, -1.0, 0.0], np.float32)
    check(select(x, s, 4, 16), gref.beam_select(x, s, 4, 16))


@pytest.mark.parametrize("V,beams", [(30000, 64), (150, 64), (9000, 40)])
def test_wide_groups_of_equal_logits(V, beams):
    """All entries of all lists reach any bound: the slow paths of both launches."""
    x = np.zeros((beams, V), np.float32)
    s = -(np.arange(beams) // 2).astype(np.float32) * np.float32(0.25)
    check(select(x, s, beams, 64), gref.beam_select(x, s, beams, 64))
    s[:] = 0
    check(select(x, s, beams, 64), gref.beam_select(x, s, beams, 64))


def test_the_most_rows():
    rows, V = 65535, 5
    x = torch.randn((rows, V), generator=torch.Generator(device=DEV).manual_seed(2), device=DEV)
    tok, par = (torch.empty((rows, 2), dtype=torch.int32, device=DEV) for _ in range(2))
    sc = torch.empty((rows, 2), device=DEV)
    ws = torch.empty(corun.beam_select_workspace(V, rows, 1, 2), dtype=torch.uint8, device=DEV)
    corun.beam_select(x, torch.zeros(rows, device=DEV), 1, tok, par, sc, ws)
    top = x.topk(2, 1)
    lp = torch.log_softmax(x.double(), 1).gather(1, top.indices)
    assert torch.equal(tok.long(), top.indices) and torch.equal(par[:, 0], torch.arange(rows, dtype=torch.int32, device=DEV))
    assert ((sc.double() - lp).abs() <= 2.0**-24 * lp.abs() * (1 + 1e-6)).all()


def test_the_widest_vocabulary_and_group():
    V, beams = 1 << 19, 64
    x, s = logits_of(beams, V, 12)
    check(select(x, s, beams, 64), gref.beam_select(x, s, beams, 64))


def test_logits_of_any_size():
    rng = np.random.default_rng(4)
    x = rng.standard_normal((6, 12000)).astype(np.float32)
    x *= np.array([1e-30, 1e-3, 30, 1e4, 1e30, 3e37], np.float32)[:, None]
    s = np.zeros(6, np.float32)
    check(select(x, s, 1, 8), gref.beam_select(x, s, 1, 8))


def test_rows_do_not_depend_on_their_place():
    x, s = logits_of(12, 30011, 6)
    a = select(x, s, 1, 8)
    p = np.random.default_rng(1).permutation(12)
    b = select(x[p], s[p], 1, 8, pad=5)
    assert np.array_equal(a[0][p], b[0]) and np.array_equal(a[2][p].view(np.int32), b[2].view(np.int32))


def test_rows_beyond_32_bits_of_bytes():
    """A row that starts behind 2^32 bytes of logits."""
    V, ld, rows = 5000, 1 << 19, 2100
    x = torch.zeros((rows, ld), device=DEV)
    x[:, 4000] = 3.0
    x[rows - 1, 4999] = 9.0
    tok, par = (torch.empty((rows, 1), dtype=torch.int32, device=DEV) for _ in range(2))
    sc = torch.empty((rows, 1), device=DEV)
    ws = torch.empty(corun.beam_select_workspace(V, rows, 1, 1), dtype=torch.uint8, device=DEV)
    corun.beam_select(x[:, :V], torch.zeros(rows, device=DEV), 1, tok, par, sc, ws)
    want = torch.full((rows,), 4000, dtype=torch.int32)
    want[-1] = 4999
    assert torch.equal(tok[:, 0].cpu(), want) and torch.equal(par[:, 0].cpu(), torch.arange(rows, dtype=torch.int32))


def test_captured_selection_replays():
    V, beams, keep, groups = 20000, 4, 8, 2
    rows = groups * beams
    x, s = torch.zeros((rows, V), device=DEV), torch.zeros(rows, device=DEV)
    tok, par = (torch.empty((groups, keep), dtype=torch.int32, device=DEV) for _ in range(2))
    sc = torch.empty((groups, keep), device=DEV)
    ws = torch.empty(corun.beam_select_workspace(V, groups, beams, keep), dtype=torch.uint8, device=DEV)
    st, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=st):
        corun.beam_select(x, s, beams, tok, par, sc, ws)
    for i in range(4):
        hx, hs = logits_of(rows, V, 40 + i)
        x.copy_(torch.from_numpy(hx))
        s.copy_(torch.from_numpy(hs))
        ws.fill_(0xFF)
        g.replay()
        torch.cuda.synchronize()
        want = select(hx, hs, beams, keep)
        assert np.array_equal(tok.cpu().numpy(), want[0]) and np.array_equal(par.cpu().numpy(), want[1])
        assert np.array_equal(sc.cpu().numpy().view(np.int32), want[2].view(np.int32))


def test_two_streams_with_their_own_workspaces():
    V, beams, keep = 151936, 4, 8
    data = [logits_of(8, V, 60 + i) for i in range(2)]
    want = [select(x, s, beams, keep) for x, s in data]
    streams = [torch.cuda.Stream() for _ in range(2)]
    dev = [(torch.from_numpy(x).to(DEV), torch.from_numpy(s).to(DEV)) for x, s in data]
    outs = [[[torch.empty((2, keep), dtype=t, device=DEV) for t in (torch.int32, torch.int32, torch.float32)]
             for _ in range(10)] for _ in range(2)]
    ws = [torch.empty(corun.beam_select_workspace(V, 2, beams, keep), dtype=torch.uint8, device=DEV) for _ in range(2)]
    torch.cuda.synchronize()
    for n in range(10):
        for i in range(2):
            corun.beam_select(*dev[i], beams, *outs[i][n], ws[i], stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        for o in outs[i]:
            assert np.array_equal(o[0].cpu().numpy(), want[i][0]) and np.array_equal(o[1].cpu().numpy(), want[i][1])
            assert np.array_equal(o[2].cpu().numpy().view(np.int32), want[i][2].view(np.int32))


def test_python_refusals():
    x, s = torch.zeros((4, 100), device=DEV), torch.zeros(4, device=DEV)
    tok, par = (torch.zeros((2, 3), dtype=torch.int32, device=DEV) for _ in range(2))
    sc, ws = torch.zeros((2, 3), device=DEV), torch.zeros(1 << 16, dtype=torch.uint8, device=DEV)
    ok = lambda **kw: corun.beam_select(**{**dict(logits=x, scores=s, beams=2, tokens=tok, parents=par, out_scores=sc, ws=ws), **kw})
    ok()
    for bad in (dict(logits=x.double()), dict(logits=x.cpu()), dict(logits=x[:, ::2]), dict(logits=x[0]), dict(beams=3),
                dict(beams=0), dict(scores=s[:3]), dict(scores=s.double()), dict(tokens=tok.long()), dict(parents=par[:, :2]),
                dict(out_scores=sc.double()), dict(valid=torch.ones(3, dtype=torch.uint8, device=DEV)),
                dict(weights=torch.ones(4, dtype=torch.float64, device=DEV)), dict(ws=ws.int()), dict(ws=ws.cpu()),
                dict(out_finished=torch.zeros((2, 3), device=DEV))):
        with pytest.raises(ValueError):
            ok(**bad)
    with pytest.raises(corun.CorunError):
        ok(ws=ws[:16])
    with pytest.raises(corun.CorunError):
        ok(finished=torch.zeros(4, dtype=torch.uint8, device=DEV))
