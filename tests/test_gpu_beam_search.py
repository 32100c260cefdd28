"""The operators for sequences that share a beginning, together, as a beam
search runs them: an engine's decode steps on a paged cache with selection and
pages between them, and a layer's append and attention over shared prefixes."""
import numpy as np
import pytest
import torch

from paper_2608_14376_amd import corun
from paper_2608_14376_amd import workload as wl
from tests import group_reference as gref
from tests.cache_reference import HostCache
from tests.gpu_helpers import DEV, to_device
from tests.test_gpu_cache_ops import make_rope, rows_of, same

pytestmark = pytest.mark.gpu


class Search:
    """Beam search over an engine: `searches` prompts of W beams each in the engine's slots, then one slot for each prompt."""

    def __init__(self, e4m3=False, W=4, searches=2, seed=0):
        self.cfg, self.W, self.n = wl.config("tiny"), W, searches
        cfg = self.cfg
        self.B = W * searches
        slots, ps, self.width, pages = self.B + searches, 16, 12, 120
        L, nkv, d = cfg["n_layers"], cfg["n_kv_heads"], cfg["head_dim"]
        dt = torch.uint8 if e4m3 else torch.bfloat16
        self.k, self.v = ([torch.zeros((pages, nkv, ps, d), dtype=dt, device=DEV) for _ in range(L)] for _ in range(2))
        scales = [[torch.full((pages, nkv, 1), 27, dtype=torch.uint8, device=DEV) for _ in range(L)] for _ in range(2)] \
            if e4m3 else (None, None)
        self.table = torch.zeros((slots, self.width), dtype=torch.int32, device=DEV)
        self.cache = corun.KvCache(self.k, self.v, *scales, 16, self.table) if e4m3 else \
            corun.KvCache(self.k, self.v, page_table=self.table)
        kw = dict(k_scale=scales[0], v_scale=scales[1], scale_block=16) if e4m3 else {}
        self.eng = corun.Engine(cfg, to_device(wl.make_weights(cfg, seed=seed)), self.B, self.k, self.v,
                                layout=corun.KV_PAGED, page_size=ps, page_table=self.table,
                                opt=corun.options(max_prefill_len=64), **kw)
        i32 = lambda n: torch.zeros(n, dtype=torch.int32, device=DEV)
        self.held, self.status, self.src, self.keep, self.hold = i32(slots), i32(1), i32(slots), i32(slots), i32(slots)
        self.ws = torch.empty(corun.pages_workspace(self.cache), dtype=torch.uint8, device=DEV)
        self.logits = torch.empty((self.B, cfg["vocab"]), device=DEV)

    def assign(self, src, keep, hold):
        for t, x in zip((self.src, self.keep, self.hold), (src, keep, hold)):
            t.copy_(torch.tensor(x, dtype=torch.int32))
        corun.pages_assign(self.cache, self.held, self.src, self.keep, self.status, self.ws, hold=self.hold)
        assert self.status.item() == 0

    def run(self, prompts, steps, end):
        """Returns (token lists of each beam behind its prompt, scores, finished), and every step's logits of live rows."""
        W, n, B = self.W, self.n, self.B
        at = [len(p) for p in prompts]
        self.assign([-1] * B + [B + i for i in range(n)], [0] * (B + n), [0] * B + at)
        first = torch.empty(self.cfg["vocab"], device=DEV)
        x = torch.empty((n, self.cfg["vocab"]), device=DEV)
        for i, p in enumerate(prompts):
            self.eng.prefill(p, slot=B + i, last_logits=first)
            x[i].copy_(first)
        tok, par = (torch.empty((n, W), dtype=torch.int32, device=DEV) for _ in range(2))
        sc, fin = torch.empty((n, W), device=DEV), torch.empty((n, W), dtype=torch.uint8, device=DEV)
        ws = torch.empty(corun.beam_select_workspace(self.cfg["vocab"], n, W, W), dtype=torch.uint8, device=DEV)
        corun.beam_select(x, torch.zeros(n, device=DEV), 1, tok, par, sc, ws, end_token=end, out_finished=fin)
        src = (par.flatten() + B).tolist()
        hist = [[t] for t in tok.flatten().tolist()]
        seen = [[(B + i // W, x[i // W].cpu().numpy())] for i in range(B)]
        lens = np.repeat(at, W)
        for _ in range(steps):
            keep = lens.tolist()
            self.assign(src + [B + i for i in range(n)], keep + at, [m + 1 for m in keep] + at)
            done = fin.flatten().cpu().numpy()
            live = (1 - done).astype(np.uint8)
            self.eng.decode_step(tok.flatten().cpu().numpy(), live, lens, self.logits)
            lens = lens + live
            host = self.logits.cpu().numpy()
            scores, was = sc.flatten().clone(), fin.flatten().clone()
            corun.beam_select(self.logits, scores, W, tok, par, sc, ws, finished=was, end_token=end, out_finished=fin)
            want = gref.beam_select(host, scores.cpu().numpy(), W, W, finished=done, end=end)
            assert np.array_equal(tok.cpu().numpy(), want[0]) and np.array_equal(par.cpu().numpy(), want[1])
            src = par.flatten().tolist()
            t = tok.flatten().tolist()
            seen = [seen[p] + ([] if done[p] else [(p, host[p])]) for p in src]
            hist = [hist[p] + ([] if done[p] else [t[i]]) for i, p in enumerate(src)]
            lens = lens[src]
        return hist, sc.flatten().tolist(), fin.flatten().tolist(), seen


@pytest.mark.parametrize("e4m3", [False, True])
def test_beam_search_on_an_engine(e4m3):
    """Each beam's logits are, bit for bit, those of its tokens decoded alone from the prompt in another slot: its
    pages held just its own past at every step.  Its score is the sum of its tokens' log-probabilities."""
    s = Search(e4m3)
    prompts = [wl.make_prompt(s.cfg["vocab"], 37, seed=5), wl.make_prompt(s.cfg["vocab"], 16, seed=6)]
    hist, scores, fin, seen = s.run(prompts, 21, end=int(3))
    assert len({tuple(h) for h in hist}) == s.B
    for b in range(s.B):
        other = Search(e4m3)
        W, B, n = other.W, other.B, other.n
        p = prompts[b // W]
        slot = (b * 5 + 2) % B
        own = [-1] * (B + n)
        own[slot] = slot
        hold = [0] * (B + n)
        hold[slot] = len(p) + len(hist[b]) + 1
        other.assign(own, [0] * (B + n), hold)
        first = torch.empty(s.cfg["vocab"], device=DEV)
        other.eng.prefill(p, slot=slot, last_logits=first)
        x, total = [first.cpu().numpy()], 0.0
        for i, t in enumerate(hist[b][:len(seen[b]) - 1]):
            toks, live, lens = np.zeros(B, np.int32), np.zeros(B, np.uint8), np.zeros(B, np.int32)
            toks[slot], live[slot], lens[slot] = t, 1, len(p) + i
            other.eng.decode_step(toks, live, lens, other.logits)
            x.append(other.logits[slot].cpu().numpy())
        for a, (_, l) in zip(x, seen[b]):
            assert np.array_equal(a.view(np.int32), l.view(np.int32))
        for a, t in zip(x, hist[b]):
            y = a.astype(np.float64)
            total += y[t] - (y.max() + np.log(np.exp(y - y.max()).sum()))
        # the score passes through fp32 at every step: half a step each
        assert abs(total - scores[b]) <= 2.0**-24 * abs(total) * (len(hist[b]) + 1)
        other.eng.close()


@pytest.mark.parametrize("dtype,blk", [("e4m3", 16), ("bf16", 16)])
def test_layer_of_beams_behind_a_shared_prompt(dtype, blk):
    """Append, reorder, shared attention over several steps: the results of a cache in which every row has all of its
    tokens, read by shared attention without any prefix and, from an 8-bit cache, by the decode attention that reads
    each row's whole slot."""
    nq, nkv, d, ps, W, P0 = 8, 2, 128, 16, 6, 203
    rope, _ = make_rope("half", d)
    hc = HostCache(nkv, d, W + 1, 320, blk, ps, seed=1, dtype=dtype, spare=60)
    cache = hc.device_cache(corun)
    pages = hc.k.shape[0]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=DEV)
    held, status = i32([0] * (W + 1)), i32([0])
    pws = torch.empty(corun.pages_workspace(cache), dtype=torch.uint8, device=DEV)
    give = lambda src, keep, hold: corun.pages_assign(cache, held, i32(src), i32(keep), status, pws, hold=i32(hold))
    give([-1] * W + [W], [0] * (W + 1), [0] * W + [P0])
    x, xd = rows_of(P0, nq + 2 * nkv, d, 3)
    q = torch.zeros((P0, nq * d), dtype=torch.bfloat16, device=DEV)
    corun.prefill_append(cache, 0, xd, [P0], None, [W], rope, q)
    shared = P0 // ps * ps                             # what the rows hold in common for good
    out = torch.zeros((W, nq * d), dtype=torch.bfloat16, device=DEV)
    most = (256, 64)
    ws = torch.empty(corun.shared_attention_workspace(cache, [W], nq, *most), dtype=torch.uint8, device=DEV)
    flat = HostCache(nkv, d, W, 320, blk, 0, seed=9, dtype=dtype)
    fcache = flat.device_cache(corun)
    fws = torch.empty(max(corun.shared_attention_workspace(fcache, [1] * W, nq), 16), dtype=torch.uint8, device=DEV)
    corun.prefill_append(fcache, 0, xd.repeat(W, 1), [P0] * W, None, list(range(W)), rope, q.repeat(W, 1))
    parents, n = [W] * W, P0
    rng = np.random.default_rng(0)
    for step in range(8):
        give(parents + [W], [n] * W + [P0], [n + 1] * W + [P0])
        if step:
            for t in flat.dev + (flat.devs or []):
                t.copy_(t[torch.tensor(parents, device=DEV)].clone())
        rows = rows_of(W, nq + 2 * nkv, d, 40 + step)[1]
        qs = torch.zeros((W, nq * d), dtype=torch.bfloat16, device=DEV)
        pos = i32([n] * W)
        corun.decode_append(cache, 0, rows, pos, rope, qs)
        corun.decode_append(fcache, 0, rows, pos, rope, qs)
        n += 1
        corun.shared_attention(cache, 0, qs, [W], i32([n] * W), i32([shared]), out, ws, prefix_slots=i32([W]),
                               max_prefix=most[0], max_suffix=most[1])
        want = torch.zeros_like(out)
        corun.shared_attention(fcache, 0, qs, [1] * W, i32([n] * W), i32([0] * W), want, fws)
        torch.cuda.synchronize()
        assert status.item() == 0
        # both are within 2^-14 in their weights of the same sums, and each is rounded to bf16 once
        a, b = out.double(), want.double()
        scale = flat.after().values(0, n)[1].abs().amax().item()
        assert ((a - b).abs() <= 2.0**-8 * (a.abs() + b.abs()) + 2.0**-12 * scale).all()
        if dtype == "e4m3":
            dec = torch.zeros_like(out)
            dws = torch.empty(corun.decode_attention_workspace(fcache, W, nq), dtype=torch.uint8, device=DEV)
            corun.decode_attention(fcache, 0, qs, i32([n] * W), dec, dws)
            assert ((dec.double() - b).abs() <= 2.0**-8 * (dec.double().abs() + b.abs()) + 2.0**-12 * scale).all()
        # the cache's own contents: what the rows see is bit for bit what the flat cache has
        h, f = hc.after(), flat.after()
        h.table = hc.devt.cpu()
        for r in (0, W - 1):
            assert all(same(s, t) for s, t in zip(gref.values(h, r, 0, n), gref.values(f, r, 0, n)))
        parents = rng.integers(0, W, W).tolist()
    used = i32([0])
    corun.pages_compact(cache, held, used, pws)
    want = out.clone()
    corun.shared_attention(cache, 0, qs, [W], i32([n] * W), i32([shared]), out, ws, prefix_slots=i32([W]),
                           max_prefix=most[0], max_suffix=most[1])
    torch.cuda.synchronize()
    assert same(out, want) and used.item() < pages and hc.devt[:W, : -(-n // ps)].max().item() < used.item()
