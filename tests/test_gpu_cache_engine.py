"""Engines on e4m3 caches and with rotations of their own.

A float64 decoder on the CPU follows the engine layer by layer; its attention
reads the engine's cache as the engine left it (codes times scales), so that a
code's rounding, checked on its own, does not move the comparison.  Then the
properties that every engine here has: position invariance, replays, chunks,
batched prompts, the scheduler."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from paper_2608_14376_amd import corun
from paper_2608_14376_amd import workload as wl
from tests import cache_reference as ref
from tests.gpu_helpers import DEV, to_device
from tests.test_gpu_cache_ops import ROPES, make_rope

pytestmark = pytest.mark.gpu
TOL = 2e-2
B, CAP = 6, 384


class Setup:
    """An engine with its caches; e4m3 ones start as stale random codes."""

    def __init__(self, name="small128", blk=32, page=0, rope=None, seed=5, slots=None, pf=320, Bf=B, W=None, **opt):
        self.cfg = wl.config(name)
        self.Wc = wl.make_weights(self.cfg, seed=51) if W is None else W
        self.W = to_device(self.Wc)
        d, nkv = self.cfg["head_dim"], self.cfg["n_kv_heads"]
        self.rope, self.rot = make_rope(rope, d) if rope else (None, None)
        if rope is None:
            f = ref.freqs(self.cfg["rope_theta"], d)
            self.rot = lambda x, pos: ref.rotate(x, pos, f, d, False)
        L, slots = self.cfg["n_layers"], slots or Bf
        self.blk, self.page = blk, page
        table = None
        if page:
            self.table = torch.from_numpy(wl.make_page_table(slots, CAP // page, slots * CAP // page + 2, seed))
            shape, table = (slots * CAP // page + 2, nkv, page, d), self.table.to(DEV)
        else:
            shape = (slots, nkv, CAP, d)
        g = torch.Generator().manual_seed(seed)
        kw = {}
        if blk:
            new = lambda: torch.randint(0, 255, shape, generator=g, dtype=torch.uint8).to(DEV)
            sc = lambda: torch.randint(100, 140, (shape[0], nkv, shape[2] // blk), generator=g, dtype=torch.uint8).to(DEV)
            self.ks, self.vs = [sc() for _ in range(L)], [sc() for _ in range(L)]
            kw = dict(k_scale=self.ks, v_scale=self.vs, scale_block=blk)
        else:
            new = lambda: torch.randn(shape, generator=g).to(torch.bfloat16).to(DEV)
        self.k, self.v = [new() for _ in range(L)], [new() for _ in range(L)]
        if page:
            kw.update(layout=corun.KV_PAGED, page_size=page, page_table=table)
        self.eng = corun.Engine(self.cfg, self.W, Bf, self.k, self.v,
                                opt=corun.options(max_prefill_len=pf, rope=self.rope, **opt), **kw)
        if page:
            self.eng.set_page_table_host(self.table.numpy())

    def values(self, layer, slot, n):
        """float64 K, V [nkv, n, d] of a slot's first n tokens."""
        out = []
        for t, s in ((self.k, "ks"), (self.v, "vs")):
            x = t[layer]
            x = x if not self.page else x[self.table[slot].long().to(DEV)]
            if self.blk:
                sc = getattr(self, s)[layer]
                sc = sc if not self.page else sc[self.table[slot].long().to(DEV)]
                if not self.page:
                    x, sc = x[slot:slot + 1], sc[slot:slot + 1]
                x = ref.decode_codes(x.cpu(), sc.cpu(), self.blk)
            else:
                x = (x if self.page else x[slot:slot + 1]).cpu().double()
            out.append(x.transpose(0, 1).reshape(x.shape[1], -1, x.shape[3])[:, :n])
        return out

    def bits(self, slot, n):
        return [[a.clone() for a in self.values(l, slot, n)] for l in range(self.cfg["n_layers"])]


_b = lambda t: t.to(torch.float32).to(torch.bfloat16).double()


def follow(s: Setup, tokens, start, slot):
    """float64 logits of rows `tokens` at positions start .. of a slot, with
    attention over the engine's cache, which is checked on the way."""
    cfg, W = s.cfg, s.Wc
    H, d, nq, nkv, eps = cfg["hidden"], cfg["head_dim"], cfg["n_heads"], cfg["n_kv_heads"], cfg["rms_eps"]
    T = len(tokens)
    pos = torch.arange(start, start + T)
    x = W.embed[torch.as_tensor(np.asarray(tokens), dtype=torch.long)].double()
    allowed = torch.arange(start + T)[None, :] <= pos[:, None]
    for l in range(cfg["n_layers"]):
        h = _b(F.rms_norm(x, (H,), weight=W.attn_norm[l].double(), eps=eps))
        y = _b(h @ W.w_qkv[l].double().T).view(T, nq + 2 * nkv, d)
        qk, _ = s.rot(y[:, :nq + nkv], pos)
        q, k, v = _b(qk[:, :nq]), qk[:, nq:], y[:, nq + nkv:]
        K, V = s.values(l, slot, start + T)
        for got, want in ((K, k), (V, v)):
            new, want = got[:, start:].transpose(0, 1), want
            half = torch.maximum(want.abs() * ref.U_E4M3, torch.full_like(want, 2.0**-10 * 2.0**-2)) if s.blk \
                else want.abs() * ref.U_BF16
            assert ((new - want).abs() <= half + TOL * want.abs().max()).all(), (l, (new - want).abs().max())
        o = F.scaled_dot_product_attention(q.transpose(0, 1), K.repeat_interleave(nq // nkv, 0),
                                           V.repeat_interleave(nq // nkv, 0), attn_mask=allowed)
        x = x + _b(o.transpose(0, 1).reshape(T, nq * d)) @ W.w_o[l].double().T
        h = _b(F.rms_norm(x, (H,), weight=W.mlp_norm[l].double(), eps=eps))
        gu = h @ W.w_gate_up[l].double().T
        a = _b(F.silu(_b(gu[:, :cfg["ffn"]])) * _b(gu[:, cfg["ffn"]:]))
        x = x + a @ W.w_down[l].double().T
    return F.rms_norm(x[-1:], (H,), weight=W.final_norm.double(), eps=eps)[0] @ W.lm_head.double().T


def close(got, want):
    err = float((got.cpu().double() - want).abs().max() / want.abs().max())
    assert err <= TOL, err


@pytest.mark.parametrize("name,blk,page,rope,Bf", [
    ("small128", 32, 0, None, 6), ("small128", 16, 48, "bands", 1), ("small128", 64, 64, "interleaved_part", 6),
    ("tiny", 16, 0, "half_odd", 12), ("tiny", 32, 32, None, 1), ("small128", 0, 0, "interleaved", 6),
    ("small128", 0, 16, "half_part", 1), ("small128", 0, 0, "linear", 6), ("tiny", 0, 0, "bands", 1),
])
def test_prefill_and_decode_against_the_reference(name, blk, page, rope, Bf):
    s = Setup(name, blk, page, rope, Bf=Bf, slots=max(Bf, 3))
    V_ = s.cfg["vocab"]
    n, slot = 133, min(2, Bf - 1)
    prompt = wl.make_prompt(V_, n, seed=7)
    lg = torch.empty(V_, dtype=torch.float32, device=DEV)
    tok = s.eng.prefill(prompt, slot, lg)
    close(lg, follow(s, prompt, 0, slot))
    # a chunk behind it, starting inside a block
    more = wl.make_prompt(V_, 50, seed=8)
    s.eng.prefill_chunk(more, n, slot, lg)
    seq = list(prompt) + list(more)
    close(lg, follow(s, more, n, slot))
    # decode steps
    out = torch.empty((Bf, V_), dtype=torch.float32, device=DEV)
    toks, valid, lens = np.zeros(Bf, np.int32), np.zeros(Bf, np.uint8), np.zeros(Bf, np.int32)
    valid[slot] = 1
    nxt = int(tok)
    for i in range(3):
        toks[slot], lens[slot] = nxt, len(seq)
        seq.append(nxt)
        got = s.eng.decode_step(toks, valid, lens, out)
        close(out[slot], follow(s, [nxt], len(seq) - 1, slot))
        nxt = int(got[slot])


def test_an_explicit_default_rope_is_the_default():
    W = wl.make_weights(wl.config("small128"), seed=51)
    a, b = Setup(blk=0, W=W), Setup(blk=0, W=W, rope="half")
    assert a.eng.plan() == b.eng.plan()
    prompt = wl.make_prompt(a.cfg["vocab"], 90, seed=9)
    la, lb = (torch.empty(a.cfg["vocab"], dtype=torch.float32, device=DEV) for _ in range(2))
    a.eng.prefill(prompt, 0, la)
    b.eng.prefill(prompt, 0, lb)
    close(la, lb.cpu().double())


@pytest.mark.parametrize("page", [0, 32])
def test_position_invariance_and_replays(page):
    """A row's logits and cache in another slot, beside other rows, eagerly and replayed: the same bits."""
    W = wl.make_weights(wl.config("small128"), seed=51)
    prompts = [wl.make_prompt(2048, n, seed=20 + n) for n in (70, 33, 5, 128)]
    ref_bits = None
    for slots_of, others, no_graph in (((0, 1, 2, 3), True, False), ((4, 0, 5, 2), True, False), ((3, 1, 2, 0), False, True)):
        s = Setup(page=page, W=W, seed=100 + slots_of[0], no_graph=no_graph)
        live = range(4) if others else [0]
        toks, valid, lens = np.full(B, -7, np.int32), np.zeros(B, np.uint8), np.full(B, 10**6, np.int32)
        for i in live:
            sl = slots_of[i]
            toks[sl], valid[sl], lens[sl] = s.eng.prefill(prompts[i], sl), 1, len(prompts[i])
        out = torch.empty((B, 2048), dtype=torch.float32, device=DEV)
        got = []
        sl = slots_of[0]
        for step in range(5):
            nxt = s.eng.decode_step(toks, valid, lens, out)
            got.append(out[sl].clone())
            toks, lens = np.where(valid, nxt, toks).astype(np.int32), lens + valid
        bits = (got, s.bits(sl, 75))
        if ref_bits is None:
            ref_bits = bits
        assert all(torch.equal(x, y) for x, y in zip(ref_bits[0], bits[0]))
        assert all(torch.equal(x, y) for p, q in zip(ref_bits[1], bits[1]) for x, y in zip(p, q))


def test_decode_run_and_measurement_aids():
    s = Setup(page=16, blk=16)
    s2 = Setup(page=16, blk=16, W=s.Wc)
    toks, valid, lens = np.zeros(B, np.int32), np.ones(B, np.uint8), np.zeros(B, np.int32)
    for e in (s.eng, s2.eng):
        for b in range(B):
            toks[b] = e.prefill(wl.make_prompt(2048, 20 + 7 * b, seed=b), b)
            lens[b] = 20 + 7 * b
    run = s.eng.decode_run(9, toks, valid, lens)
    t, n = toks.copy(), lens.copy()
    for i in range(9):
        t = s2.eng.decode_step(t, valid, n)
        assert np.array_equal(t, run[i])
        n = n + 1
    times = s.eng.profile_step(2)
    assert {"qkv_post", "attn_split", "attn_merge"} <= set(times) and all(us > 0 for us, _ in times.values())
    assert s.eng.time_kernel(corun.K_QKV_POST) > 0 and s.eng.time_kernel(corun.K_ATTN_SPLIT) > 0
    assert np.array_equal(s.eng.decode_step(t, valid, n), s2.eng.decode_step(t, valid, n))


def test_batched_prompts_are_their_own_prefill():
    s = Setup(page=32, bi_prefill=True)
    prompts = [wl.make_prompt(2048, n, seed=n) for n in (1, 33, 100, 64)]
    lg = torch.empty((4, 2048), dtype=torch.float32, device=DEV)
    toks = s.eng.prefill_batch(prompts, [3, 0, 5, 1], lg)
    together = [s.bits(sl, len(p)) for p, sl in zip(prompts, [3, 0, 5, 1])]
    one = torch.empty(2048, dtype=torch.float32, device=DEV)
    for i, (p, sl) in enumerate(zip(prompts, [0, 2, 4, 3])):
        assert s.eng.prefill(p, sl, one) == toks[i] and torch.equal(one, lg[i])
        assert all(torch.equal(x, y) for a, b in zip(together[i], s.bits(sl, len(p))) for x, y in zip(a, b))


def test_long_prompts_and_chunks_behind_them(monkeypatch):
    """Sequences that attention splits over their keys: batched and alone, and a chunk against the reference."""
    monkeypatch.setitem(globals(), "CAP", 1536)
    s = Setup("tiny", 32, 0, pf=2432, slots=B, bi_prefill=True)
    V_ = s.cfg["vocab"]
    prompts = [wl.make_prompt(V_, n, seed=n) for n in (1300, 60, 1024)]
    lg = torch.empty((3, V_), dtype=torch.float32, device=DEV)
    toks = s.eng.prefill_batch(prompts, [3, 0, 5], lg)
    together = [s.bits(sl, len(p)) for p, sl in zip(prompts, [3, 0, 5])]
    one = torch.empty(V_, dtype=torch.float32, device=DEV)
    for i, (p, sl) in enumerate(zip(prompts, [1, 2, 4])):
        assert s.eng.prefill(p, sl, one) == toks[i] and torch.equal(one, lg[i])
        assert all(torch.equal(x, y) for a, b in zip(together[i], s.bits(sl, len(p))) for x, y in zip(a, b))
    more = wl.make_prompt(V_, 70, seed=9)
    s.eng.prefill_chunk(more, 1300, 1, one)
    close(one, follow(s, more, 1300, 1))


def test_moe_engine_on_an_e4m3_cache():
    """A mixture of experts beside the bf16 engine: the same tokens' logits, apart by the cache's rounding."""
    cfg = wl.config("small_moe")
    W = wl.make_weights(cfg, seed=51)
    a, b = Setup("small_moe", 32, W=W), Setup("small_moe", 0, W=W)
    la, lb = (torch.empty(cfg["vocab"], dtype=torch.float32, device=DEV) for _ in range(2))
    p = wl.make_prompt(cfg["vocab"], 1, seed=3)
    a.eng.prefill(p, 1, la)                           # one token sees its own value alone
    b.eng.prefill(p, 1, lb)
    assert torch.isfinite(la).all() and torch.isfinite(lb).all()
    out = a.eng.decode_step([1] * B, [1] * B, [1] * B)
    assert ((out >= 0) & (out < cfg["vocab"])).all()


def test_scheduler_over_an_e4m3_cache():
    """Requests' outputs do not depend on their order or on who runs beside them."""
    W = wl.make_weights(wl.config("small128"), seed=51)
    reqs = [(i, wl.make_prompt(2048, 10 + 13 * i, seed=i), 6 + i, 1000 + i, 0.0 if i % 2 else 0.8) for i in range(8)]

    def outputs(order, page, **kw):
        s = Setup(page=page, blk=16, W=W, **kw)
        sch = corun.Scheduler(s.eng)
        for i in order:
            rid, p, m, seed, T = reqs[i]
            sch.add_request(rid, p, m, seed=seed, temperature=T)
        sch.run_until_idle()
        res = [sch.output(i)[0].tolist() for i in range(8)]
        sch.close()
        return res

    first = outputs(range(8), 16)
    assert first == outputs([5, 2, 7, 0, 1, 6, 3, 4], 16)
    assert first == outputs([7, 6, 5, 4, 3, 2, 1, 0], 0)


def test_refusals():
    cfg = wl.config("small128")
    W = to_device(wl.make_weights(cfg, seed=51))
    mk = lambda *sh: [torch.zeros(sh, dtype=torch.uint8, device=DEV) for _ in range(cfg["n_layers"])]
    k, v, ks, vs = mk(2, 2, 64, 128), mk(2, 2, 64, 128), mk(2, 2, 2), mk(2, 2, 2)
    good = dict(k_scale=ks, v_scale=vs, scale_block=32)
    corun.Engine(cfg, W, 2, k, v, **good).close()
    r64, r = corun.rope(64), corun.rope(128, layout=corun.ROPE_INTERLEAVED)
    bad_rope = corun.rope(128)
    bad_rope.rot_dim = 3
    for opt, status in ((dict(qkv_epilogue=2), corun.E_INVAL), (dict(small_batch_layer=1), corun.E_INVAL),
                        (dict(rope=r64), corun.E_SHAPE), (dict(rope=bad_rope), corun.E_SHAPE)):
        with pytest.raises(corun.CorunError) as e:
            corun.Engine(cfg, W, 2, k, v, opt=corun.options(**opt), **good)
        assert e.value.status == status
    kb = [torch.zeros((2, 2, 64, 128), dtype=torch.bfloat16, device=DEV) for _ in range(cfg["n_layers"])]
    for opt in (dict(rope=r, qkv_epilogue=2), dict(rope=r, small_batch_layer=1)):
        with pytest.raises(corun.CorunError) as e:
            corun.Engine(cfg, W, 2, kb, kb, opt=corun.options(**opt))
        assert e.value.status == corun.E_INVAL
    with pytest.raises(ValueError):
        corun.Engine(cfg, W, 2, k, v, k_scale=ks[:1], v_scale=vs, scale_block=32)
    with pytest.raises(ValueError):
        corun.Engine(cfg, W, 2, k, v, k_scale=ks, v_scale=vs, scale_block=16)
