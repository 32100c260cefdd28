"""Operators for sequences that share a beginning, as measurable cases.

Three kinds that a beam search, or several samples of one prompt, run one after
another around a decode step:

``beam``     the best continuations over a group's beams and the vocabulary:
             log softmax of fp32 logits in 64 bits, added to the beams' scores;
             finished beams compete with the score they have;
``assign``   the pages of a paged cache after it: every slot takes the first
             tokens of some slot, whole pages shared, a part-filled one its
             own, pages for new tokens added, what no slot holds any more freed;
``compact``  pages in use moved to the lowest numbers, so that a pool can
             shrink;
``shared``   attention of one query token per row, where the rows of a group
             see a common prefix, read once for all of them, and each its own
             tokens behind it.

Caches are bf16, or e4m3 codes with a power-of-two scale byte for each block of
tokens of a KV head (code * 2^(byte - 127)), contiguous or paged.  Head shapes
and vocabularies are ``workload.CONFIGS``' where a comment names one.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"


def listed() -> list:
    return [
        # one user's beam search on an 8B-class model: four beams, eight candidates kept
        dict(name="beam_8b_w4", kind="beam", groups=1, beams=4, keep=8, vocab=151936, pad=0, done=0),
        # the package's headline batch as 64 searches, some beams finished, some rows padding
        dict(name="beam_8b_b256", kind="beam", groups=64, beams=4, keep=4, vocab=151936, pad=9, done=7),
        # wide searches on a 32B-class model, twice as many candidates as beams
        dict(name="beam_32b_wide", kind="beam", groups=4, beams=32, keep=64, vocab=152064, pad=0, done=11),
        # the step after it for one user: four beams on a bf16 cache
        dict(name="assign_8b_w4", kind="assign", dtype="bf16", layers=36, nkv=8, d=128, page=16, blk=0, groups=1,
             beams=4, lo=1003, hi=1003, own_pages=2, more=1),
        # sixteen searches at once on an 8-bit cache of the mixture of experts
        dict(name="assign_moe_16x4", kind="assign", dtype="e4m3", layers=48, nkv=4, d=128, page=32, blk=32, groups=16,
             beams=4, lo=100, hi=700, own_pages=2, more=1),
        # sixteen samples forked from one prompt on a 32B-class model, room for 64 tokens each
        dict(name="assign_32b_fork", kind="assign", dtype="e4m3", layers=64, nkv=8, d=128, page=64, blk=64, groups=1,
             beams=17, lo=1500, hi=1500, own_pages=0, more=64),
        # a small pool after a few requests have left
        dict(name="compact_tiny", kind="compact", dtype="bf16", layers=2, nkv=2, d=64, page=16, blk=0, slots=8,
             each=5, shared=2, pool=96),
        # a pool in pieces after many requests have left: half of its pages in use
        dict(name="compact_moe", kind="compact", dtype="e4m3", layers=48, nkv=4, d=128, page=32, blk=32, slots=24,
             each=12, shared=8, pool=592),
        # the smallest attention: four rows of the two-layer test model
        dict(name="shared_tiny_b4", kind="shared", dtype="bf16", nq=4, nkv=2, d=64, page=0, blk=0, groups=1,
             rlo=4, rhi=4, plo=100, phi=100, slo=0, shi=20, pad=0),
        # one user's eight beams over a long prompt
        dict(name="shared_8b_w8", kind="shared", dtype="e4m3", nq=32, nkv=8, d=128, page=16, blk=16, groups=1,
             rlo=8, rhi=8, plo=3000, phi=3000, slo=1, shi=100, pad=0),
        # a full batch behind one system prompt, bf16 cache, some rows padding
        dict(name="shared_8b_b256", kind="shared", dtype="bf16", nq=32, nkv=8, d=128, page=16, blk=0, groups=1,
             rlo=256, rhi=256, plo=6000, phi=6000, slo=16, shi=1024, pad=9),
        # four documents with several questions each on a 32B-class model, 8-bit cache
        dict(name="shared_32b_docs", kind="shared", dtype="e4m3", nq=64, nkv=8, d=128, page=64, blk=64, groups=4,
             rlo=8, rhi=32, plo=8000, phi=32768, slo=64, shi=2000, pad=0),
    ]


#: (query heads, KV heads, head size): the package's shapes, and generic ones with one, three and seven query heads to a KV head
HEADS = [(4, 2, 64), (8, 2, 128), (32, 8, 128), (64, 8, 128), (32, 4, 128), (16, 16, 64), (24, 8, 128), (28, 4, 128)]
LOGITS = 1 << 25      # logits of a drawn selection, at most
POOL = 3 << 27        # bytes of a drawn pool, at most
SCORES = 1 << 26      # query-key pairs x query heads of a drawn attention, at most


def _logint(rng, lo: int, hi: int) -> int:
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _draw_pages(rng) -> dict:
    nkv, d = rng.choice(HEADS)[1:]
    dtype = rng.choice(["bf16", "e4m3"])
    blk = rng.choice([16, 32, 64]) if dtype == "e4m3" else 0
    page = blk * rng.choice([1, 2, 4]) if blk else rng.choice([16, 32, 48, 64, 128])
    return dict(dtype=dtype, nkv=nkv, d=d, page=page, blk=blk)


def draw(rng) -> dict:
    kind = rng.choice(["beam", "beam", "assign", "assign", "compact", "shared", "shared", "shared"])
    if kind == "beam":
        vocab = rng.choice([_logint(rng, 16, 260000), 151936, 152064, 1024])
        beams = _logint(rng, 1, 64)
        return dict(kind=kind, groups=_logint(rng, 1, max(1, min(64, LOGITS // (vocab * beams)))), beams=beams,
                    keep=min(64, beams * rng.choice([1, 2])), vocab=vocab, pad=rng.choice([0, 5, 9]),
                    done=rng.choice([0, 7, 11]))
    if kind == "shared":
        nq, nkv, d = rng.choice(HEADS)
        dtype = rng.choice(["bf16", "e4m3"])
        blk = rng.choice([16, 32, 64]) if dtype == "e4m3" else 0
        rows = _logint(rng, 1, 192)
        groups = rng.choice([1, 1, rng.randint(1, max(1, min(16, rows)))])
        rhi = -(-rows // groups)
        phi = _logint(rng, 1, max(16, min(16384, SCORES // (nq * groups * rhi))))
        token = 4 * nkv * d                            # bytes of a token, in bf16
        shi = _logint(rng, 1, max(16, min(2048, SCORES // (nq * groups * rhi), POOL // (groups * rhi * token))))
        page = rng.choice([0, blk or 16, (blk or 16) * rng.choice([2, 3, 4])])
        if groups * (rhi + 1) * (phi + shi) * token > 2 * POOL:
            page = page or 64                          # a contiguous cache has room for the prefix in every slot
        return dict(kind=kind, dtype=dtype, nq=nq, nkv=nkv, d=d, blk=blk, page=page, groups=groups,
                    rlo=rng.choice([1, rhi]), rhi=rhi, plo=rng.choice([0, max(1, phi // 4), phi]), phi=phi,
                    slo=rng.choice([0, 1, shi]), shi=shi, pad=rng.choice([0, 0, 5]))
    c = dict(kind=kind, **_draw_pages(rng))
    if kind == "assign":
        beams = rng.randint(1, 16)
        c.update(groups=_logint(rng, 1, 32), beams=beams, lo=1, hi=_logint(rng, 16, 2000),
                 own_pages=rng.randint(0, 2), more=rng.choice([0, 1, 1, rng.randint(2, 150)]))
    else:
        c.update(slots=_logint(rng, 1, 64), each=_logint(rng, 1, 40), shared=rng.randint(0, 12))
        c["pool"] = (c["slots"] * c["each"] + c["shared"]) * rng.choice([1, 2, 3]) + rng.randint(0, 20)
    layers = POOL // (_pool_pages(c) * _page_bytes(c))
    if layers < 1:                                     # too many pages for one layer: fewer sequences
        c.update(dict(groups=1) if kind == "assign" else dict(slots=1, pool=3 * (c["each"] + c["shared"])))
        layers = max(1, POOL // (_pool_pages(c) * _page_bytes(c)))
    c["layers"] = min(layers, rng.choice([1, 2, 36, 48, 64]))
    return c


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------

def _spread(n: int, lo: int, hi: int) -> np.ndarray:
    """n whole numbers over [lo, hi], one from the middle of each of n equal
    parts of the range (of its logarithm where it spans more than 16); a range
    from 0 has one 0."""
    u = (np.arange(n) + 0.5) / n
    x = lo * (hi / lo) ** u if lo > 0 and hi > 16 * lo else lo + (hi - lo) * u
    if lo == 0 and n > 1:
        x[0] = 0
    return np.round(x).astype(np.int64)


def _gens(seed: int):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    return np.random.default_rng(seed), gen


def _i32(x):
    return torch.from_numpy(np.ascontiguousarray(x, np.int32)).to(DEV)


def prepare(case: dict, seed: int) -> dict:
    return {"beam": _prepare_beam, "assign": _prepare_assign, "compact": _prepare_compact,
            "shared": _prepare_shared}[case["kind"]](case, seed)


def _prepare_beam(c: dict, seed: int) -> dict:
    rng, gen = _gens(seed)
    rows, V = c["groups"] * c["beams"], c["vocab"]
    # a smooth bulk and a few tokens that stand out, as language models have them
    logits = torch.randn((rows, V), generator=gen, device=DEV) * 2.0
    n = min(V, 12)
    at = torch.randint(V, (rows, n), generator=gen, device=DEV)
    logits.scatter_add_(1, at, 6.0 + 3.0 * torch.randn((rows, n), generator=gen, device=DEV))
    spread = np.sort(rng.exponential(3.0, (c["groups"], c["beams"])), 1)
    scores = -(20.0 * rng.random((c["groups"], 1)) + spread)
    r = np.arange(rows)
    valid = np.ones(rows, np.uint8) if not c["pad"] else (r % c["pad"] != c["pad"] - 1).astype(np.uint8)
    done = np.zeros(rows, np.uint8) if not c["done"] else (r % c["done"] == c["done"] // 2).astype(np.uint8)
    weight = np.where(done, 1.0 / 30, 1.0 / 36)        # one over the length, finished beams being shorter
    st = dict(case=c, logits=logits, scores=torch.from_numpy(scores.reshape(-1).astype(np.float32)).to(DEV),
              valid=torch.from_numpy(valid).to(DEV), finished=torch.from_numpy(done).to(DEV),
              weight=torch.from_numpy(weight.astype(np.float32)).to(DEV), end=min(V - 1, 2))
    shape = (c["groups"], c["keep"])
    st["tokens"], st["parents"] = (torch.empty(shape, dtype=torch.int32, device=DEV) for _ in range(2))
    st["out_scores"] = torch.empty(shape, dtype=torch.float32, device=DEV)
    st["out_finished"] = torch.empty(shape, dtype=torch.uint8, device=DEV)
    if own:
        from paper_2608_14376_amd import corun
        st["ws"] = torch.empty(corun.beam_select_workspace(V, c["groups"], c["beams"], c["keep"]), dtype=torch.uint8,
                               device=DEV)
    return st


def _page_bytes(c: dict) -> int:
    """Of one page of one layer, keys and values with their scales."""
    e = c["page"] * c["d"] * (1 if c["blk"] else 2) + (c["page"] // c["blk"] if c["blk"] else 0)
    return 2 * c["nkv"] * e


def _lengths(c: dict) -> np.ndarray:
    """Tokens of each group of an assign case."""
    return _spread(c["groups"], c["lo"], c["hi"])


def _pool_pages(c: dict) -> int:
    if c["kind"] == "compact":
        return max(c["pool"], c["slots"] * c["each"] + c["shared"])
    n = _lengths(c)
    common = np.maximum(0, -(-n // c["page"]) - c["own_pages"] - 1)
    return int((common + c["beams"] * 2 * (c["own_pages"] + 2 + -(-c["more"] // c["page"]))).sum())


def _random_cache(c: dict, pages: int, gen):
    """Random elements of all layers, [layers, pages, ...]: codes and scales as their bits, none of them NaN."""
    shape = (c["layers"], pages, c["nkv"], c["page"], c["d"])
    out = {}
    for name in ("k", "v"):
        if c["blk"]:
            out[name] = torch.randint(0, 0x7f, shape, generator=gen, dtype=torch.uint8, device=DEV)
            out[name + "_scale"] = torch.randint(110, 125, (*shape[:3], c["page"] // c["blk"]), generator=gen,
                                                 dtype=torch.uint8, device=DEV)
        else:
            out[name] = torch.randint(0x3000, 0x4200, shape, generator=gen, dtype=torch.int16,
                                      device=DEV).view(torch.bfloat16)
    return out


def _own_cache(st: dict):
    from paper_2608_14376_amd import corun
    c = st["case"]
    if c["blk"]:
        return corun.KvCache(st["k"], st["v"], st["k_scale"], st["v_scale"], c["blk"], st["table"])
    return corun.KvCache(st["k"], st["v"], page_table=st["table"])


def _prepare_assign(c: dict, seed: int) -> dict:
    rng, gen = _gens(seed)
    W, ps = c["beams"], c["page"]
    pool, n = _pool_pages(c), _lengths(c)
    slots = c["groups"] * W
    width = int(-(-(n.max() + c["more"]) // ps)) + 1
    ids = rng.permutation(pool)
    table = np.zeros((slots, width), np.int32)
    held = np.zeros(slots, np.int32)
    src = np.zeros(slots, np.int32)
    at = 0
    for g in range(c["groups"]):
        total = int(-(-n[g] // ps))
        common = max(0, total - c["own_pages"]) if c["own_pages"] else total
        fork = c["own_pages"] == 0                     # samples of one prompt: slot 0 of the group has it, the others are empty
        first = ids[at:at + common]
        at += common
        for b in range(W):
            r = g * W + b
            if fork and b > 0:
                continue
            table[r, :common] = first
            table[r, common:total] = ids[at:at + total - common]
            at += total - common
            held[r] = total
        if fork:
            src[g * W:(g + 1) * W] = g * W
        else:                                          # the better half of the beams goes on, some of them twice
            best = rng.permutation(W)[:(W + 1) // 2]
            src[g * W:(g + 1) * W] = g * W + rng.permutation(np.resize(best, W))
    st = dict(case=c, pool=pool, **_random_cache(c, pool, gen), table=_i32(table), held=_i32(held), src=_i32(src),
              keep=_i32(np.repeat(n, W)), hold=_i32(np.repeat(n + c["more"], W)),
              status=torch.empty(1, dtype=torch.int32, device=DEV))
    if own:
        from paper_2608_14376_amd import corun
        st["cache"] = _own_cache(st)
        st["ws"] = torch.empty(corun.pages_workspace(st["cache"]), dtype=torch.uint8, device=DEV)
    return st


def _prepare_compact(c: dict, seed: int) -> dict:
    rng, gen = _gens(seed)
    pool, each = _pool_pages(c), c["each"]
    ids = rng.permutation(pool)
    table = np.zeros((c["slots"], c["shared"] + each), np.int32)
    table[:, :c["shared"]] = ids[:c["shared"]]         # a prompt that all slots share
    table[:, c["shared"]:] = ids[c["shared"]:c["shared"] + c["slots"] * each].reshape(c["slots"], each)
    held = np.full(c["slots"], c["shared"] + each)
    st = dict(case=c, pool=pool, **_random_cache(c, pool, gen), table=_i32(table), scattered=_i32(table),
              held=_i32(held), status=torch.empty(1, dtype=torch.int32, device=DEV))
    if own:
        from paper_2608_14376_amd import corun
        st["cache"] = _own_cache(st)
        st["ws"] = torch.empty(corun.pages_workspace(st["cache"]), dtype=torch.uint8, device=DEV)
    return st


def _groups(c: dict):
    """Rows and prefix length of each group."""
    return _spread(c["groups"], c["rlo"], c["rhi"]), _spread(c["groups"], c["plo"], c["phi"])


def _fill(shape, blk, gen):
    """Keys or values of normal size with a few loud dimensions: bf16, or codes with their scale bytes."""
    pages, nkv, tok, d = shape
    loud = torch.ones(d, device=DEV)
    loud[::37] = 6.0
    out = torch.empty(shape, dtype=torch.uint8 if blk else torch.bfloat16, device=DEV)
    scales = torch.empty((pages, nkv, tok // blk), dtype=torch.uint8, device=DEV) if blk else None
    step = max(1, (1 << 27) // (nkv * tok * d))
    for p in range(0, pages, step):
        m = min(step, pages - p)
        x = torch.randn((m, nkv, tok, d), generator=gen, device=DEV) * loud
        if not blk:
            out[p:p + m] = x.to(torch.bfloat16)
            continue
        x = x.view(m, nkv, tok // blk, blk, d)
        e = torch.ceil(torch.log2(x.abs().amax((3, 4), keepdim=True) / 448.0))
        scales[p:p + m] = (e + 127).to(torch.uint8).view(m, nkv, tok // blk)
        out[p:p + m] = torch.ldexp(x, -e).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).view(m, nkv, tok, d)
    return out, scales


def _prepare_shared(c: dict, seed: int) -> dict:
    rng, gen = _gens(seed)
    nq, nkv, d, page = c["nq"], c["nkv"], c["d"], c["page"]
    grows, prefix = _groups(c)
    rows = int(grows.sum())
    of = np.repeat(np.arange(c["groups"]), grows)
    suffix = rng.permutation(_spread(rows, c["slo"], c["shi"]))
    lens = prefix[of] + suffix
    slots = rows + c["groups"]                         # a slot for each row, then one that holds each prefix
    unit = page or c["blk"] or 16
    cap = -(-(int(lens.max()) + 64) // unit) * unit    # room to generate
    if page:
        table = np.zeros((slots, cap // page), np.int32)
        whole = prefix // page                         # pages that a row shares with its group's prefix
        need = np.concatenate([-(-(lens + 1) // page) - whole[of], -(-prefix // page)])
        first = np.cumsum(need) - need
        pool = int(need.sum())
        ids = rng.permutation(pool)
        for g in range(c["groups"]):
            i = rows + g
            table[i, :need[i]] = ids[first[i]:first[i] + need[i]]
        for r in range(rows):
            w = whole[of[r]]
            table[r, :w] = table[rows + of[r], :w]
            table[r, w:w + need[r]] = ids[first[r]:first[r] + need[r]]
        shape = (pool, nkv, page, d)
    else:
        table, shape = None, (slots, nkv, cap, d)
    st = dict(case=c, group_rows=grows.tolist(), table=None if table is None else _i32(table))
    st["k"], st["k_scale"] = _fill(shape, c["blk"], gen)
    st["v"], st["v_scale"] = _fill(shape, c["blk"], gen)
    live = np.ones(rows, np.uint8) if not c["pad"] else (np.arange(rows) % c["pad"] != c["pad"] - 1).astype(np.uint8)
    st["valid"], st["lens"] = torch.from_numpy(live).to(DEV), _i32(lens)
    st["prefix_slots"], st["prefix_lens"] = _i32(rows + np.arange(c["groups"])), _i32(prefix)
    st["prefix"], st["suffix_most"] = prefix.tolist(), int(suffix.max())
    st["q"] = torch.randn((rows, nq * d), generator=gen, device=DEV).to(torch.bfloat16)
    st["out"] = torch.zeros_like(st["q"])
    if own:
        from paper_2608_14376_amd import corun
        if c["blk"]:
            st["cache"] = corun.KvCache([st["k"]], [st["v"]], [st["k_scale"]], [st["v_scale"]], c["blk"], st["table"])
        else:
            st["cache"] = corun.KvCache([st["k"]], [st["v"]], page_table=st["table"])
        # what the step's launch covers: the longest of each, in steps that a program would round to
        st["most"] = (max(1, int(prefix.max())), -(-max(1, st["suffix_most"]) // 64) * 64)
        st["most"] = tuple(min(x, cap) for x in st["most"])
        st["ws"] = torch.empty(corun.shared_attention_workspace(st["cache"], st["group_rows"], nq, *st["most"]),
                               dtype=torch.uint8, device=DEV)
    return st


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------

def run(st: dict):
    c = st["case"]
    kind = c["kind"]
    if own:
        from paper_2608_14376_amd import corun
        if kind == "beam":
            corun.beam_select(st["logits"], st["scores"], c["beams"], st["tokens"], st["parents"], st["out_scores"],
                              st["ws"], valid=st["valid"], finished=st["finished"], weights=st["weight"],
                              end_token=st["end"], out_finished=st["out_finished"])
        elif kind == "assign":
            corun.pages_assign(st["cache"], st["held"], st["src"], st["keep"], st["status"], st["ws"], hold=st["hold"])
        elif kind == "compact":
            st["table"].copy_(st["scattered"])         # the pool as it was, so that every pass moves pages
            corun.pages_compact(st["cache"], st["held"], st["status"], st["ws"])
        else:
            corun.shared_attention(st["cache"], 0, st["q"], st["group_rows"], st["lens"], st["prefix_lens"], st["out"],
                                   st["ws"], prefix_slots=st["prefix_slots"], valid=st["valid"],
                                   max_prefix=st["most"][0], max_suffix=st["most"][1])
    elif kind == "beam":
        _plain_beam(st)
    elif kind == "assign":
        _plain_assign(st)
    elif kind == "compact":
        st["table"].copy_(st["scattered"])
        _plain_compact(st)
    else:
        st["out"] = _plain_shared(st)
    if kind == "beam":
        return {"tokens": st["tokens"], "parents": st["parents"], "scores": st["out_scores"],
                "finished": st["out_finished"]}
    if kind == "shared":
        return {"out": st["out"]}
    out = {"table": st["table"], "held": st["held"], "status": st["status"]}
    for n in ("k", "v"):
        out[n] = st[n].view(torch.float8_e4m3fn) if c["blk"] else st[n]
        if c["blk"]:
            out[n + "_scale"] = st[n + "_scale"].view(torch.float8_e8m0fnu)
    return out


def _plain_beam(st: dict):
    c = st["case"]
    W, k = c["beams"], c["keep"]
    x = st["logits"]
    rows, V = x.shape
    n = min(k, V)
    top = x.amax(1, keepdim=True).double()
    lse = top + torch.log(torch.exp(x.double() - top).sum(1, keepdim=True))
    l, tok = torch.sort(x, dim=1, descending=True, stable=True)      # equal logits: lower tokens first
    score = st["scores"].double()[:, None] + (l[:, :n].double() - lse)
    tok = tok[:, :n].int()
    done = st["finished"].bool()[:, None]
    only = torch.full_like(score, -math.inf)
    only[:, 0] = st["scores"].double()
    score = torch.where(done, only, score)
    tok = torch.where(done, torch.full_like(tok, st["end"]), tok)
    rank = score * st["weight"].double()[:, None]
    rank = torch.where(st["valid"].bool()[:, None] & score.isfinite(), rank, torch.full_like(rank, -math.inf))
    parent = torch.arange(rows, device=DEV, dtype=torch.int32)[:, None].expand(rows, n)
    rank, score, tok, parent, done = (t.reshape(-1, W * n) for t in (rank, score, tok, parent, done.expand(rows, n)))
    rank, at = torch.sort(rank, dim=1, descending=True, stable=True)
    m = min(k, W * n)
    real = rank[:, :m] > -math.inf
    at = at[:, :m]
    tok, parent = (torch.where(real, t.gather(1, at), -1) for t in (tok, parent))
    for name, t, rest in (("tokens", tok, -1), ("parents", parent, -1),
                          ("out_scores", torch.where(real, score.gather(1, at), -math.inf), -math.inf),
                          ("out_finished", real & (done.gather(1, at) | (tok == st["end"])), 0)):
        st[name].fill_(rest)
        st[name][:, :m] = t.to(st[name].dtype)


def _layers(st: dict):
    """Every layer's tensor of pages, and how many of its entries along the third dimension hold one block."""
    c = st["case"]
    for n in ("k", "v"):
        for t in st[n]:
            yield t, c["blk"] or 16
        for t in st.get(n + "_scale", []):
            yield t, 1


def _plain_assign(st: dict):
    c = st["case"]
    ps, pool, blk = c["page"], st["pool"], c["blk"] or 16
    old, held = st["table"].long(), st["held"].long()
    src, keep, hold = st["src"].long(), st["keep"].long(), st["hold"].long()
    slots, width = old.shape
    me, col = torch.arange(slots, device=DEV), torch.arange(width, device=DEV)
    keep, hold = (torch.where(src < 0, 0, t) for t in (keep, hold))
    taken = old[src.clamp(min=0)]
    nfull, rest, total = keep // ps, keep % ps, -(-hold // ps)
    full = col[None, :] < nfull[:, None]
    whole = torch.zeros(pool + 1, dtype=torch.bool, device=DEV)
    whole[torch.where(full, taken, pool)] = True
    whole[pool] = False
    tail = torch.where(rest > 0, taken.gather(1, nfull.clamp(max=width - 1)[:, None])[:, 0], pool)
    first = torch.full((pool + 1,), slots, device=DEV).scatter_reduce_(0, tail, me, "amin")
    stays = (rest > 0) & ~whole[tail] & (first[tail] == me)
    used = whole.clone()
    used[torch.where(stays, tail, pool)] = True
    free = torch.sort(used[:pool].int(), stable=True)[1]             # free pages first, ascending
    have = nfull + stays
    fresh = (total - have).clamp(min=0)
    missing = (fresh.sum() - (pool - used[:pool].sum())).clamp(min=0)
    at = (torch.cumsum(fresh, 0) - fresh)[:, None] + col[None, :] - have[:, None]
    new = torch.where(col[None, :] < nfull[:, None], taken, free[at.clamp(0, pool - 1)])
    new = torch.where((col[None, :] == nfull[:, None]) & stays[:, None], tail[:, None], new)
    new = torch.where(col[None, :] < total[:, None], new, old)
    done = missing == 0
    st["status"].copy_(missing)
    moved = torch.nonzero((rest > 0) & ~stays & done)[:, 0]
    a, b, n = tail[moved], new[moved, nfull[moved]], rest[moved]
    for t, unit in _layers(st):
        count = -(-n // blk) * unit
        here = (torch.arange(t.shape[2], device=DEV)[None, :] < count[:, None])[:, None, :]
        here = here[..., None] if t.dim() == 4 else here
        t[b] = torch.where(here, t[a], t[b])
    st["table"].copy_(torch.where(done, new, old))
    st["held"].copy_(torch.where(done, total, held))


def _plain_compact(st: dict):
    pool = st["pool"]
    old = st["table"].long()
    slots, width = old.shape
    inside = torch.arange(width, device=DEV)[None, :] < st["held"].long()[:, None]
    used = torch.zeros(pool + 1, dtype=torch.bool, device=DEV)
    used[torch.where(inside, old, pool)] = True
    used = used[:pool]
    n = used.sum()
    page = torch.arange(pool, device=DEV)
    a, b = torch.nonzero(used & (page >= n))[:, 0], torch.nonzero(~used & (page < n))[:, 0]
    name = page.clone()
    name[a] = b
    for t, _ in _layers(st):
        t[b] = t[a]
    st["table"].copy_(torch.where(inside, name[old], old))
    st["status"].copy_(n)


def _tokens(st: dict, name: str, slot, pos):
    """Keys or values in 32 bits at positions `pos` of slots `slot`: [..., nkv, d]."""
    c = st["case"]
    if c["page"]:
        slot, pos = st["table"][slot, pos // c["page"]].long(), pos % c["page"]
    x = st[name][slot, :, pos]
    if not c["blk"]:
        return x.float()
    e = st[name + "_scale"][slot, :, pos // c["blk"]]
    return x.view(torch.float8_e4m3fn).float() * torch.exp2(e.float() - 127)[..., None]


def _plain_shared(st: dict):
    c = st["case"]
    nq, nkv, d = c["nq"], c["nkv"], c["d"]
    G, S = nq // nkv, st["suffix_most"]
    out, r0 = [], 0
    for g, (R, P) in enumerate(zip(st["group_rows"], st["prefix"])):
        row = torch.arange(r0, r0 + R, device=DEV)
        q = st["q"][r0:r0 + R].float().view(R, nkv, G, d)
        slot = st["prefix_slots"][g].long().expand(P)
        at = torch.arange(P, device=DEV)
        k, v = (_tokens(st, n, slot, at).transpose(0, 1).contiguous() for n in ("k", "v"))       # [nkv, P, d]
        pos = P + torch.arange(S, device=DEV)
        n = st["lens"][r0:r0 + R].long()
        seen = pos[None, :] < n[:, None]
        pos = torch.minimum(pos[None, :].expand(R, S), (n - 1).clamp(min=0)[:, None])
        sk, sv = (_tokens(st, x, row[:, None].expand(R, S), pos).transpose(1, 2).contiguous() for x in ("k", "v"))
        a = (q.transpose(0, 1).reshape(nkv, R * G, d) @ k.transpose(1, 2)).view(nkv, R, G, P).transpose(0, 1)
        b = (q @ sk.transpose(2, 3)).masked_fill(~seen[:, None, None, :], -math.inf)
        s = torch.cat([a, b], -1) / math.sqrt(d)                                                 # [R, nkv, G, P + S]
        top = s.amax(-1, keepdim=True)
        p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
        p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
        o = (p[..., :P].transpose(0, 1).reshape(nkv, R * G, P) @ v).view(nkv, R, G, d).transpose(0, 1)
        o = o + p[..., P:].contiguous() @ sv
        out.append(torch.where(st["valid"][r0:r0 + R].bool()[:, None], o.reshape(R, nq * d), 0.0))
        r0 += R
    return torch.cat(out).to(torch.bfloat16)


# --------------------------------------------------------------------------
# What a pass cannot do without
# --------------------------------------------------------------------------

def work(case: dict) -> dict:
    """Logits once; moved tokens read and written, tables read and written;
    queries in and out and every token that some row sees once."""
    c = case
    if c["kind"] == "beam":
        rows = c["groups"] * c["beams"]
        r = np.arange(rows)
        used = np.ones(rows, bool)
        if c["pad"]:
            used &= r % c["pad"] != c["pad"] - 1
        if c["done"]:
            used &= r % c["done"] != c["done"] // 2
        n = int(used.sum()) * c["vocab"]
        return {"bytes": 4 * n + 13 * c["groups"] * c["keep"] + 10 * rows, "flops": 3 * n}
    if c["kind"] == "assign":
        n, W, ps, blk = _lengths(c), c["beams"], c["page"], c["blk"] or 16
        forks = W - 1 if c["own_pages"] == 0 else W // 2              # rows whose part-filled page is another's already
        tokens = (-(-(n % ps) // blk) * blk).sum() * forks
        tables = 4 * W * (-(-n // ps) + -(-(n + c["more"]) // ps)).sum()
        return {"bytes": float(2 * tokens * c["layers"] * _page_bytes(c) / ps + tables), "flops": 0}
    if c["kind"] == "compact":
        used, pool = c["slots"] * c["each"] + c["shared"], _pool_pages(c)
        entries = c["slots"] * (c["shared"] + c["each"])
        moves = used * (pool - used) / pool                          # on average over the seeds
        return {"bytes": 2 * moves * c["layers"] * _page_bytes(c) + 8 * entries, "flops": 0}
    grows, prefix = _groups(c)
    rows = int(grows.sum())
    suffix = _spread(rows, c["slo"], c["shi"])
    share = 1.0 if not c["pad"] else 1.0 - (rows // c["pad"]) / rows  # live rows
    tok = 2 * c["nkv"] * (c["d"] + 1 / c["blk"] if c["blk"] else 2 * c["d"])
    pairs = share * float((grows * prefix).sum() + suffix.sum())
    return {"bytes": float(share * rows * 4 * c["nq"] * c["d"] + tok * (prefix.sum() + share * suffix.sum())),
            "flops": 4 * c["nq"] * c["d"] * pairs}


# --------------------------------------------------------------------------
# The same results in 64 bits
# --------------------------------------------------------------------------

def exact(case: dict, seed: int):
    st = prepare(case, seed)
    return {"beam": _exact_beam, "assign": _exact_pages, "compact": _exact_pages,
            "shared": _exact_shared}[case["kind"]](st)


def _exact_beam(st: dict):
    c = st["case"]
    W, k, V = c["beams"], c["keep"], c["vocab"]
    host = {n: st[n].cpu().numpy() for n in ("scores", "valid", "finished", "weight")}
    out = {"tokens": np.full((c["groups"], k), -1), "parents": np.full((c["groups"], k), -1),
           "scores": np.full((c["groups"], k), -np.inf), "finished": np.zeros((c["groups"], k), np.int64)}
    for g in range(c["groups"]):
        found = []                                     # (-rank, row, place in the row, token, score, finished)
        for r in range(g * W, (g + 1) * W):
            s, w = float(host["scores"][r]), float(host["weight"][r])
            if not host["valid"][r]:
                continue
            if host["finished"][r]:
                found.append((-s * w, r, 0, st["end"], s, 1))
                continue
            x = st["logits"][r].cpu().numpy().astype(np.float64)
            lse = x.max() + math.log(math.fsum(np.exp(x - x.max())))
            some = np.argpartition(-x, min(k, V - 1))[:k] if k < V else np.arange(V)
            some = np.flatnonzero(x >= x[some].min())
            for i, v in enumerate(some[np.argsort(-x[some], kind="stable")][:k]):
                found.append((-(s + (x[v] - lse)) * w, r, i, int(v), s + (x[v] - lse), int(v == st["end"])))
        for i, (_, r, _, v, s, f) in enumerate(sorted(found)[:k]):
            out["tokens"][g, i], out["parents"][g, i], out["scores"][g, i], out["finished"][g, i] = v, r, s, f
    return {n: torch.from_numpy(x) for n, x in out.items()}


def _exact_pages(st: dict):
    """Tables page by page; elements are moved, not computed."""
    c = st["case"]
    ps, pool, blk = c["page"], st["pool"], c["blk"] or 16
    table, held = st["table"].cpu().numpy().astype(np.int64), st["held"].cpu().tolist()
    old = table.copy()
    moves = []                                         # from, to, tokens
    if c["kind"] == "compact":
        used = sorted({int(p) for r in range(len(held)) for p in old[r, :held[r]]})
        n = len(used)
        high, low = [p for p in used if p >= n], [p for p in range(n) if p not in set(used)]
        name = dict(zip(high, low))
        moves = [(a, b, ps) for a, b in name.items()]
        for r in range(len(held)):
            table[r, :held[r]] = [name.get(int(p), int(p)) for p in old[r, :held[r]]]
        status = n
    else:
        src, keep, hold = (st[x].cpu().tolist() for x in ("src", "keep", "hold"))
        rows = [(r, s, n, m) for r, (s, n, m) in enumerate(zip(src, keep, hold)) if s >= 0]
        whole = {int(old[s, i]) for _, s, n, _ in rows for i in range(n // ps)}
        owner = {}
        for r, s, n, _ in rows:
            if n % ps and int(old[s, n // ps]) not in whole:
                owner.setdefault(int(old[s, n // ps]), r)
        spare = iter([p for p in range(pool) if p not in whole and p not in owner])
        new_held = [0] * len(held)
        for r, s, n, m in rows:
            pages = [int(p) for p in old[s, :n // ps]]
            if n % ps:
                t = int(old[s, n // ps])
                if owner.get(t) != r:
                    p = next(spare)
                    moves.append((t, p, -(-(n % ps) // blk) * blk))
                    t = p
                pages.append(t)
            while len(pages) < -(-m // ps):
                pages.append(next(spare))
            table[r, :len(pages)] = pages
            new_held[r] = len(pages)
        held, status = new_held, 0
    for a, b, n in moves:
        for t, unit in _layers(st):
            t[b, :, :-(-n // blk) * unit] = t[a, :, :-(-n // blk) * unit]
    out = {"table": torch.from_numpy(table), "held": torch.tensor(held), "status": torch.tensor([status])}
    for x in ("k", "v"):
        out[x] = (st[x].view(torch.float8_e4m3fn) if c["blk"] else st[x]).double()
        if c["blk"]:
            out[x + "_scale"] = torch.exp2(st[x + "_scale"].double() - 127)
    return out


def _exact_shared(st: dict):
    c = st["case"]
    nq, nkv, d, page, blk = c["nq"], c["nkv"], c["d"], c["page"], c["blk"]
    G = nq // nkv
    q = st["q"].double().view(-1, nq, d)
    out = torch.zeros_like(q)
    table = None if st["table"] is None else st["table"].cpu().numpy()

    def span(name, slot, a, b):                        # tokens a .. b - 1 of a slot in 64 bits, [nkv, tokens, d]
        if b <= a:
            return torch.zeros((nkv, 0, d), dtype=torch.float64, device=DEV)
        if page:
            ids = torch.from_numpy(table[slot, a // page:-(-b // page)]).to(DEV).long()
            a0 = a // page * page
            w = st[name][ids].transpose(0, 1).reshape(nkv, -1, d)
            e = st[name + "_scale"][ids].transpose(0, 1).reshape(nkv, -1) if blk else None
        else:
            a0, w = 0, st[name][slot]
            e = st[name + "_scale"][slot] if blk else None
        if blk:
            w = w.contiguous().view(torch.float8_e4m3fn).double() * torch.exp2(e.double() - 127).repeat_interleave(blk, 1)[:, :, None]
        return w[:, a - a0:b - a0].double()

    live, lens = st["valid"].cpu().tolist(), st["lens"].cpu().tolist()
    r = 0
    for g, (R, P) in enumerate(zip(st["group_rows"], st["prefix"])):
        pk, pv = (span(n, sum(st["group_rows"]) + g, 0, P) for n in ("k", "v"))
        for r in range(r, r + R):
            if live[r] and lens[r] > 0:
                sk, sv = (span(n, r, P, lens[r]) for n in ("k", "v"))
                qr = q[r].view(nkv, G, d)
                s = torch.cat([qr @ pk.transpose(1, 2), qr @ sk.transpose(1, 2)], -1) / math.sqrt(d)
                w = torch.softmax(s, -1)
                out[r] = (w[..., :P] @ pv + w[..., P:] @ sv).reshape(nq, d)
        r += 1
    return {"out": out.view(-1, nq * d)}
