"""Engines on e4m3 caches whose decode attention has several splits to a row,
and a mixture of experts on such a cache, against the float64 decoder of
tests/test_gpu_cache_engine.py, which reads the engine's own cache."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

import oracle
import tests.test_gpu_cache_engine as base
from paper_2608_14376_amd import corun
from paper_2608_14376_amd import workload as wl
from tests import cache_reference as ref
from tests.gpu_helpers import DEV, check_routing
from tests.test_gpu_cache_engine import B, TOL, Setup, _b, close, follow

pytestmark = pytest.mark.gpu


def start_rows(s, lens, seed=0):
    """Prompts of `lens` tokens in slots 0 ..: (tokens so far of each, next token of each)."""
    seqs = [list(wl.make_prompt(s.cfg["vocab"], n, seed=seed + i)) for i, n in enumerate(lens)]
    return seqs, np.array([s.eng.prefill(np.array(q, np.int32), i) for i, q in enumerate(seqs)], np.int32)


@pytest.mark.parametrize("name,blk,page,chunk,cap,lens", [
    ("small128", 32, 0, 64, 384, (63, 64, 65, 127, 128, 380)),
    ("tiny", 16, 48, 64, 384, (1, 62, 64, 126, 191, 192)),
    ("small128", 16, 32, 0, 1536, (127, 128, 129, 255, 256, 1100)),
    ("tiny", 64, 0, 0, 1536, (126, 1, 383, 384, 640, 1279)),
])
def test_decode_of_several_splits_against_the_reference(monkeypatch, name, blk, page, chunk, cap, lens):
    monkeypatch.setattr(base, "CAP", cap)
    s = Setup(name, blk, page, pf=max(lens), attn_chunk=chunk)
    plan = s.eng.plan()
    assert plan["attn_max_splits"] > 1 and max(lens) + 3 > 2 * plan["attn_chunk"]
    V_ = s.cfg["vocab"]
    seqs, toks = start_rows(s, lens)
    out = torch.empty((B, V_), dtype=torch.float32, device=DEV)
    for step in range(3):
        n = np.array([len(q) for q in seqs], np.int32)
        valid = np.ones(B, np.uint8)
        valid[step] = 0                               # another row is padding in each step
        nxt = s.eng.decode_step(toks, valid, n, out)
        for r in range(B):
            if valid[r]:
                close(out[r], follow(s, [int(toks[r])], len(seqs[r]), r))
                seqs[r].append(int(toks[r]))
                toks[r] = nxt[r]


@pytest.mark.parametrize("page,chunk,cap", [(0, 64, 384), (96, 64, 384), (32, 0, 1536)])
def test_position_invariance_of_several_splits(monkeypatch, page, chunk, cap):
    """Rows on both sides of split boundaries: the same bits in other slots, beside other rows, alone, eagerly."""
    monkeypatch.setattr(base, "CAP", cap)
    W = wl.make_weights(wl.config("small128"), seed=51)
    far = 128 if cap == 384 else 640
    prompts = [wl.make_prompt(2048, n, seed=20 + n) for n in (far - 2, 63, 5, 64)]
    first = None
    for slots_of, live, no_graph in (((0, 1, 2, 3), (0, 1, 2, 3), False), ((4, 0, 5, 2), (0, 1, 2, 3), False),
                                     ((3, 1, 2, 0), (0,), True), ((5, 4, 1, 3), (3, 0), True)):
        s = Setup(page=page, W=W, seed=100 + slots_of[0], pf=640, no_graph=no_graph, attn_chunk=chunk)
        assert s.eng.plan()["attn_max_splits"] > 1
        toks, valid, lens = np.full(B, -7, np.int32), np.zeros(B, np.uint8), np.full(B, 10**6, np.int32)
        for i in live:
            sl = slots_of[i]
            toks[sl], valid[sl], lens[sl] = s.eng.prefill(prompts[i], sl), 1, len(prompts[i])
        out = torch.empty((B, 2048), dtype=torch.float32, device=DEV)
        got = []
        for step in range(5):
            nxt = s.eng.decode_step(toks, valid, lens, out)
            got.append(out[slots_of[0]].clone())
            toks, lens = np.where(valid, nxt, toks).astype(np.int32), lens + valid
        bits = (got, s.bits(slots_of[0], far + 3))
        first = first or bits
        assert all(torch.equal(x, y) for x, y in zip(first[0], bits[0]))
        assert all(torch.equal(x, y) for p, q in zip(first[1], bits[1]) for x, y in zip(p, q))


@pytest.mark.parametrize("page", [0, 16])
def test_decode_run_of_several_splits(page):
    """A captured run whose rows cross split boundaries, and steps one by one."""
    s = Setup(page=page, blk=16, attn_chunk=64)
    s2 = Setup(page=page, blk=16, W=s.Wc, attn_chunk=64, no_graph=True)
    assert s.eng.plan()["attn_max_splits"] == 6
    lens = np.array([60, 64, 122, 1, 187, 250], np.int32)
    valid = np.ones(B, np.uint8)
    toks, again = start_rows(s, lens)[1], start_rows(s2, lens)[1]
    assert np.array_equal(toks, again)
    run = s.eng.decode_run(9, toks, valid, lens)
    t, n = toks.copy(), lens.copy()
    for i in range(9):
        t = s2.eng.decode_step(t, valid, n)
        assert np.array_equal(t, run[i])
        n = n + 1
    for r in range(B):
        assert all(torch.equal(x, y) for a, b in zip(s.bits(r, int(n[r])), s2.bits(r, int(n[r]))) for x, y in zip(a, b))
    assert s.eng.time_kernel(corun.K_ATTN_MERGE) > 0
    assert np.array_equal(s.eng.decode_step(t, valid, n), s2.eng.decode_step(t, valid, n))


def follow_moe(s, tokens, start, slot, rows, source):
    """follow() for a mixture of experts: float64 logits of the last of `tokens`, by the engine's choice of experts,
    which has to be the top k of router logits near the reference's."""
    cfg, W = s.cfg, s.Wc
    H, d, nq, nkv, eps = cfg["hidden"], cfg["head_dim"], cfg["n_heads"], cfg["n_kv_heads"], cfg["rms_eps"]
    Fe, k_, T = cfg["expert_ffn"], cfg["top_k"], len(tokens)
    sel, glog = s.eng.routing_trace(source)
    sel, glog = sel[:, rows], glog[:, rows]
    pos = torch.arange(start, start + T)
    x = W.embed[torch.as_tensor(np.asarray(tokens), dtype=torch.long)].double()
    allowed = torch.arange(start + T)[None, :] <= pos[:, None]
    rl, own = np.zeros(glog.shape), np.zeros(sel.shape, np.int32)
    for l in range(cfg["n_layers"]):
        h = _b(F.rms_norm(x, (H,), weight=W.attn_norm[l].double(), eps=eps))
        y = _b(h @ W.w_qkv[l].double().T).view(T, nq + 2 * nkv, d)
        qk, _ = s.rot(y[:, :nq + nkv], pos)
        q, K_new, V_new = _b(qk[:, :nq]), qk[:, nq:], y[:, nq + nkv:]
        K, V = s.values(l, slot, start + T)
        for got, want in ((K, K_new), (V, V_new)):
            new = got[:, start:].transpose(0, 1)
            half = torch.maximum(want.abs() * ref.U_E4M3, torch.full_like(want, 2.0**-10 * 2.0**-2))
            assert ((new - want).abs() <= half + TOL * want.abs().max()).all(), (l, (new - want).abs().max())
        o = F.scaled_dot_product_attention(q.transpose(0, 1), K.repeat_interleave(nq // nkv, 0),
                                           V.repeat_interleave(nq // nkv, 0), attn_mask=allowed)
        x = x + _b(o.transpose(0, 1).reshape(T, nq * d)) @ W.w_o[l].double().T
        h = _b(F.rms_norm(x, (H,), weight=W.mlp_norm[l].double(), eps=eps))
        router = h @ W.w_router[l].double().T
        rl[l] = router.numpy()
        y = torch.zeros_like(x)
        for t in range(T):
            own[l, t] = oracle.route(np.ascontiguousarray(rl[l, t]), k_)[0]
            w = torch.softmax(router[t, torch.as_tensor(sel[l, t], dtype=torch.long)], 0)
            for e, we in zip(sel[l, t], w):
                gu = h[t] @ W.w_exp_gate_up[l][int(e)].double().T
                a = _b(F.silu(_b(gu[:Fe])) * _b(gu[Fe:]))
                y[t] += we * (a @ W.w_exp_down[l][int(e)].double().T)
        x = x + y
    for t in range(T):
        check_routing(sel[:, t], glog[:, t], rl[:, t], own[:, t], (slot, start + t))
    return F.rms_norm(x[-1:], (H,), weight=W.final_norm.double(), eps=eps)[0] @ W.lm_head.double().T


@pytest.mark.parametrize("name,blk,page,chunk", [("small_moe", 32, 0, 0), ("tiny_moe", 16, 48, 64)])
def test_moe_against_the_reference(name, blk, page, chunk):
    s = Setup(name, blk, page, record_routing=True, attn_chunk=chunk)
    V_, slot = s.cfg["vocab"], 2
    lg = torch.empty(V_, dtype=torch.float32, device=DEV)
    seq = list(wl.make_prompt(V_, 70, seed=7))
    s.eng.prefill(np.array(seq, np.int32), slot, lg)
    close(lg, follow_moe(s, seq, 0, slot, slice(None), 1))
    more = list(wl.make_prompt(V_, 20, seed=8))
    nxt = s.eng.prefill_chunk(np.array(more, np.int32), len(seq), slot, lg)
    close(lg, follow_moe(s, more, len(seq), slot, slice(None), 1))
    seq += more
    other = s.eng.prefill(wl.make_prompt(V_, 5, seed=9), 4)
    toks, valid, lens = np.zeros(B, np.int32), np.zeros(B, np.uint8), np.zeros(B, np.int32)
    valid[[slot, 4]] = 1
    toks[slot], toks[4], lens[4] = nxt, other, 5
    out = torch.empty((B, V_), dtype=torch.float32, device=DEV)
    for _ in range(3):
        lens[slot] = len(seq)
        got = s.eng.decode_step(toks, valid, lens, out)
        close(out[slot], follow_moe(s, [int(toks[slot])], len(seq), slot, [slot], 0))
        seq.append(int(toks[slot]))
        toks[slot], toks[4], lens[4] = got[slot], got[4], lens[4] + 1


@pytest.mark.parametrize("e4m3", [True, False])
def test_no_rotary_table_where_no_kernel_reads_one(e4m3):
    """2^22 positions to a slot: a table of them would be 2 GiB at 64 pairs of 8 bytes."""
    cfg = wl.config("small128")
    W = base.to_device(wl.make_weights(cfg, seed=51))
    cap, dt = 1 << 22, torch.uint8 if e4m3 else torch.bfloat16
    k, v = ([torch.zeros((4, 2, 16, 128), dtype=dt, device=DEV) for _ in range(cfg["n_layers"])] for _ in range(2))
    kw = {}
    if e4m3:
        ks, vs = ([torch.full((4, 2, 1), 121, dtype=torch.uint8, device=DEV) for _ in range(cfg["n_layers"])] for _ in range(2))
        kw = dict(k_scale=ks, v_scale=vs, scale_block=16)
    table = torch.zeros((1, cap // 16), dtype=torch.int32, device=DEV)
    rope = None if e4m3 else corun.rope(128, layout=corun.ROPE_INTERLEAVED)
    torch.cuda.synchronize()
    before = torch.cuda.mem_get_info()[0]
    eng = corun.Engine(cfg, W, 1, k, v, layout=corun.KV_PAGED, page_size=16, page_table=table,
                       opt=corun.options(rope=rope), **kw)
    assert before - torch.cuda.mem_get_info()[0] < 1 << 30
    eng.close()
