"""The attention operators of an 8-bit KV cache, as measurable cases.

Three operators that a decoder layer calls one after another once its QKV
projection has run:

``append``   rotary positions (half or interleaved pairs, on all of a head or
             its leading part, unscaled or scaled for long contexts) applied to
             the queries and keys of packed QKV rows, and the rotated keys and
             the values appended to a cache of e4m3 codes, whose power-of-two
             scales belong to one block of tokens of one KV head each;
``decode``   attention of one query token per row over that cache;
``prefill``  causal attention of whole prompts, or of chunks of long ones, over
             it.

An appended block's scale is the smallest power of two under which the largest
finite value among the new tokens is at most 448 and under which no earlier
token of the block is scaled up: where it grows, the earlier tokens' codes are
rounded to it.  Caches are contiguous (a slot's tokens in one piece) or paged.
Head shapes are ``workload.CONFIGS``' where a comment names one.

What is held in 8 bits comes back in its own type: codes as float8_e4m3fn,
scales as float8_e8m0fnu.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda"
NORM = 1.0   # standard deviation of queries, keys and values


def listed() -> list:
    return [
        # one user's next token on an 8B-class model: a few KB, launches count
        dict(name="append_8b_b1", kind="append", nq=32, nkv=8, d=128, rows=1, live=1, lo=3001, hi=3001, blk=32, page=0,
             layout="half", rot=128, scaling="none", theta=1e6),
        # a full decode step with padding rows, frequencies scaled by bands for long contexts
        dict(name="append_8b_b256", kind="append", nq=32, nkv=8, d=128, rows=256, live=162, lo=512, hi=4096, blk=32,
             page=0, layout="half", rot=128, scaling="bands", theta=5e5),
        # waiting prompts of ragged lengths on a paged cache; interleaved pairs on half of each head
        dict(name="append_moe_prompts", kind="append", nq=32, nkv=4, d=128, prompts=12, lo=100, hi=600, start=0, blk=16,
             page=16, layout="interleaved", rot=64, scaling="none", theta=1e4),
        # a whole long document on a 32B-class model, positions interpolated
        dict(name="append_32b_32768", kind="append", nq=64, nkv=8, d=128, prompts=1, lo=32768, hi=32768, start=0, blk=64,
             page=64, layout="half", rot=128, scaling="linear", theta=1e6),
        # the smallest attention: four slots of the two-layer test model, one with nothing cached
        dict(name="decode_tiny_b4", kind="decode", nq=4, nkv=2, d=64, rows=4, live=3, lo=0, hi=128, blk=16, page=0),
        # one user on an 8B-class model
        dict(name="decode_8b_b1", kind="decode", nq=32, nkv=8, d=128, rows=1, live=1, lo=4001, hi=4001, blk=32, page=0),
        # the package's headline batch, partly filled
        dict(name="decode_8b_b256", kind="decode", nq=32, nkv=8, d=128, rows=256, live=162, lo=512, hi=4096, blk=32,
             page=0),
        # long contexts on a 32B-class model with a paged cache
        dict(name="decode_32b_paged", kind="decode", nq=64, nkv=8, d=128, rows=32, live=32, lo=1024, hi=32768, blk=16,
             page=16),
        # an ordinary chat prompt
        dict(name="prefill_8b_600", kind="prefill", nq=32, nkv=8, d=128, prompts=1, lo=600, hi=600, start=0, blk=32,
             page=0),
        # waiting prompts of ragged lengths in one call, paged
        dict(name="prefill_8b_prompts", kind="prefill", nq=32, nkv=8, d=128, prompts=12, lo=100, hi=600, start=0, blk=16,
             page=16),
        # a whole document
        dict(name="prefill_8b_6000", kind="prefill", nq=32, nkv=8, d=128, prompts=1, lo=6000, hi=6000, start=0, blk=64,
             page=0),
        # one fixed-size chunk deep in a long prompt (chunked prefill), paged
        dict(name="prefill_8b_chunk", kind="prefill", nq=32, nkv=8, d=128, prompts=1, lo=2048, hi=2048, start=14336,
             blk=32, page=32),
    ]


#: (query heads, KV heads, head size): the package's shapes, and generic ones with one, three and seven query heads to a KV head
HEADS = [(4, 2, 64), (8, 2, 128), (32, 8, 128), (64, 8, 128), (32, 4, 128), (16, 16, 64), (24, 8, 128), (28, 4, 128)]
TOKENS = 1 << 19      # cached tokens x KV heads x head size / 1024 that a drawn decode batch reads at most
PAIRS = 1 << 30       # query-key pairs x query heads of a drawn prefill, at most


def _logint(rng, lo: int, hi: int) -> int:
    return int(min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng) -> dict:
    nq, nkv, d = rng.choice(HEADS)
    blk = rng.choice([16, 32, 64])
    page = rng.choice([0, 0, blk, blk * rng.choice([2, 3, 4])])
    c = dict(kind=rng.choice(["append", "append", "decode", "decode", "prefill"]), nq=nq, nkv=nkv, d=d, blk=blk, page=page)
    if c["kind"] == "append":
        c.update(layout=rng.choice(["half", "interleaved"]), rot=rng.choice([d, d, d // 2, 2 * rng.randint(1, d // 2)]),
                 scaling=rng.choice(["none", "linear", "bands"]), theta=rng.choice([1e4, 5e5, 1e6]))
    if c["kind"] == "decode" or (c["kind"] == "append" and rng.random() < 0.5):
        rows = _logint(rng, 1, 256)
        hi = _logint(rng, 16, max(16, min(65536, TOKENS * 1024 // (nkv * d * rows))))
        c.update(rows=rows, live=rng.randint((rows + 1) // 2, rows), lo=rng.choice([0, 1, hi // 8, hi]), hi=hi)
        return c
    n = rng.choice([1, 1, rng.randint(2, 24)])
    hi = _logint(rng, 1, 8192 // n)
    if c["kind"] == "append":
        start = rng.choice([0, 0, rng.randint(1, 16384)])
    else:
        while nq * n * hi * hi > 2 * PAIRS:
            hi = hi * 3 // 4
        start = rng.choice([0, 0, rng.randint(0, max(1, min(16384, PAIRS // (nq * n * hi) - hi)))])
    c.update(prompts=n, lo=rng.choice([max(1, hi // 8), hi]), hi=hi, start=start)
    return c


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------

def _lens(c: dict, n: int, seed: int) -> np.ndarray:
    """n lengths over [lo, hi] in a random order, one from each of n equal
    parts of the range (of its logarithm where it spans more than 16), so that
    every seed has the same total; a range from 0 has one length of 0."""
    lo, hi = c["lo"], c["hi"]
    u = (np.arange(n) + 0.5) / n
    x = lo * (hi / lo) ** u if lo > 0 and hi > 16 * lo else lo + (hi - lo) * u
    if lo == 0 and n > 1:
        x[0] = 0
    return np.random.default_rng(seed * 31 + 7).permutation(np.round(x).astype(np.int64))


def _rows_form(c: dict) -> bool:
    return "rows" in c


def _freqs(c: dict) -> list:
    """Radians per position of each rotated pair: theta^(-2 i / rot); linear:
    over the factor 4; bands: pairs that turn less than once over the trained
    8192 positions over the factor 8, more than four times as they are, a
    linear blend by turns between."""
    f = [c["theta"] ** (-2.0 * i / c["rot"]) for i in range(c["rot"] // 2)]
    if c["scaling"] == "linear":
        return [x / 4 for x in f]
    if c["scaling"] == "bands":
        keep = [min(1.0, max(0.0, (8192 * x / (2 * math.pi) - 1) / (4 - 1))) for x in f]
        return [x * (g + (1 - g) / 8) for x, g in zip(f, keep)]
    return f


def _magnitude(c: dict) -> float:
    return 1.25 if c["scaling"] == "bands" else 1.0   # a power-of-two fraction: the same in every type


def _heads_like(shape, gen, d):
    """Rows of heads: normal values with a few loud dimensions, as keys have."""
    x = torch.randn(shape, generator=gen, device=DEV) * NORM
    loud = torch.ones(d, device=DEV)
    loud[::37] = 6.0
    return (x.view(*shape[:-1], -1, d) * loud).view(shape)


def _fill(shape, blk, gen):
    """A cache's codes and scale bytes, quantised from normal values."""
    pages, nkv, tok, d = shape
    codes = torch.empty(shape, dtype=torch.uint8, device=DEV)
    scales = torch.empty((pages, nkv, tok // blk), dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 28) // (nkv * tok * d))
    for p in range(0, pages, step):
        m = min(step, pages - p)
        x = _heads_like((m, nkv, tok, d), gen, d).view(m, nkv, tok // blk, blk, d)
        e = torch.ceil(torch.log2(x.abs().amax((3, 4), keepdim=True) / 448.0))
        scales[p:p + m] = (e + 127).to(torch.uint8).view(m, nkv, tok // blk)
        codes[p:p + m] = torch.ldexp(x, -e).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).view(m, nkv, tok, d)
    return codes, scales


def prepare(case: dict, seed: int) -> dict:
    c = case
    nq, nkv, d, blk, page = c["nq"], c["nkv"], c["d"], c["blk"], c["page"]
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    st = dict(case=c)
    if _rows_form(c):
        n, live = c["rows"], c["live"]
        slots = n
        before = np.zeros(n, np.int64)
        before[:live] = _lens(c, live, seed)          # cached tokens
        after = before + 1
        st["valid"] = torch.from_numpy((np.arange(n) < live).astype(np.uint8)).to(DEV)
        st["lens"] = torch.from_numpy(before.astype(np.int32)).to(DEV)
        total = n
    else:
        n = c["prompts"]
        slots = n + 2
        lens = _lens(c, n, seed)
        after = lens + c["start"]
        st["lens"] = lens.astype(np.int32)
        st["starts"] = np.full(n, c["start"], np.int32)
        st["slots"] = rng.permutation(slots)[:n].astype(np.int32)
        total = int(lens.sum())
    st["longest"] = int(after.max())
    unit = page or blk
    cap = -(-(int(after.max()) + 64) // unit) * unit  # room to generate
    if page:
        need = -(-(after + 64) // page)
        at = np.cumsum(need) - need
        ids = rng.permutation(int(need.sum())).astype(np.int32)
        table = np.zeros((slots, cap // page), np.int32)
        where = np.arange(n) if _rows_form(c) else st["slots"]
        for i in range(n):
            table[where[i], :need[i]] = ids[at[i]:at[i] + need[i]]
        st["table"] = torch.from_numpy(table).to(DEV)
        shape = (ids.size, nkv, page, d)
    else:
        st["table"] = None
        shape = (slots, nkv, cap, d)
    st["k"], st["k_scale"] = _fill(shape, blk, gen)
    st["v"], st["v_scale"] = _fill(shape, blk, gen)
    if c["kind"] == "append":
        st["qkv"] = _heads_like((total, (nq + 2 * nkv) * d), gen, d).to(torch.bfloat16)
        st["q"] = torch.zeros((total, nq * d), dtype=torch.bfloat16, device=DEV)
    else:
        st["q"] = (torch.randn((total, nq * d), generator=gen, device=DEV) * NORM).to(torch.bfloat16)
        st["out"] = torch.zeros_like(st["q"])
    if own:
        from paper_2608_14376_amd import corun
        st["cache"] = corun.KvCache([st["k"]], [st["v"]], [st["k_scale"]], [st["v_scale"]], blk, st["table"])
        if c["kind"] == "append":
            st["rope"] = corun.rope(d, c["theta"], rot_dim=c["rot"],
                                    layout=corun.ROPE_HALF if c["layout"] == "half" else corun.ROPE_INTERLEAVED,
                                    scaling=dict(none=corun.ROPE_UNSCALED, linear=corun.ROPE_LINEAR,
                                                 bands=corun.ROPE_BANDS)[c["scaling"]],
                                    factor=dict(none=1.0, linear=4.0, bands=8.0)[c["scaling"]], low=1.0, high=4.0,
                                    trained_len=8192, magnitude=_magnitude(c))
        elif c["kind"] == "decode":
            st["ws"] = torch.empty(corun.decode_attention_workspace(st["cache"], c["rows"], nq), dtype=torch.uint8,
                                   device=DEV)
    else:
        _index(st)
    return st


def _index(st: dict):
    """Where the plain form's rows stand: sequence and position of each row,
    each sequence's slot and first new position, and the blocks that an append
    touches, so that a pass waits for nothing."""
    c = st["case"]
    if _rows_form(c):
        n = c["rows"]
        st["row_seq"] = torch.arange(c["live"], device=DEV)
        st["row_pos"] = st["lens"][:c["live"]].long()
        st["seq_slot"] = torch.arange(n, device=DEV)
        st["seq_start"] = st["lens"].long()
    else:
        lens = torch.from_numpy(st["lens"]).to(DEV).long()
        st["row_seq"] = torch.repeat_interleave(torch.arange(c["prompts"], device=DEV), lens)
        first = torch.cumsum(lens, 0) - lens
        st["seq_start"] = torch.from_numpy(st["starts"]).to(DEV).long()
        st["row_at"] = torch.arange(int(lens.sum()), device=DEV) - first[st["row_seq"]]
        st["row_pos"] = st["row_at"] + st["seq_start"][st["row_seq"]]
        st["seq_slot"] = torch.from_numpy(st["slots"]).to(DEV).long()
    if c["kind"] == "append":
        st["freqs"] = torch.tensor(_freqs(c), dtype=torch.float64, device=DEV)
        span = st["longest"] // c["blk"] + 2
        blocks, st["row_block"] = torch.unique(st["row_seq"] * span + st["row_pos"] // c["blk"], return_inverse=True)
        st["block_seq"], st["block_at"] = blocks // span, blocks % span


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------

def run(st: dict):
    c = st["case"]
    if own:
        from paper_2608_14376_amd import corun
        if c["kind"] == "append" and _rows_form(c):
            corun.decode_append(st["cache"], 0, st["qkv"], st["lens"], st["rope"], st["q"], valid=st["valid"])
        elif c["kind"] == "append":
            corun.prefill_append(st["cache"], 0, st["qkv"], st["lens"], st["starts"], st["slots"], st["rope"], st["q"])
        elif c["kind"] == "decode":
            corun.decode_attention(st["cache"], 0, st["q"], st["lens"], st["out"], st["ws"], valid=st["valid"])
        else:
            corun.prefill_attention(st["cache"], 0, st["q"], st["lens"], st["starts"], st["slots"], st["out"])
    elif c["kind"] == "append":
        _plain_append(st)
    elif c["kind"] == "decode":
        st["out"] = _plain_decode(st)
    else:
        st["out"] = _plain_prefill(st)
    if c["kind"] == "append":
        return {"q": st["q"], "k": st["k"].view(torch.float8_e4m3fn), "v": st["v"].view(torch.float8_e4m3fn),
                "k_scale": st["k_scale"].view(torch.float8_e8m0fnu), "v_scale": st["v_scale"].view(torch.float8_e8m0fnu)}
    return {"out": st["out"]}


def _place(st: dict, seq, pos):
    """Index into the cache's first dimension, and position within its third, of positions `pos` of sequences `seq`."""
    slot = st["seq_slot"][seq]
    if st["table"] is None:
        return slot, pos
    page = st["case"]["page"]
    return st["table"][slot, pos // page].long(), pos % page


def _rotate(x, st: dict):
    """x [rows, heads, d] in 32 bits, rotated; angles in 64."""
    c = st["case"]
    rot, h = c["rot"], c["rot"] // 2
    a = st["row_pos"].double()[:, None] * st["freqs"][None, :]
    cs, sn = ((t * _magnitude(c)).float()[:, None, :] for t in (torch.cos(a), torch.sin(a)))
    if c["layout"] == "half":
        u, w = x[..., :h], x[..., h:rot]
        return torch.cat([u * cs - w * sn, w * cs + u * sn, x[..., rot:]], -1)
    u, w = x[..., :rot:2], x[..., 1:rot:2]
    y = torch.stack([u * cs - w * sn, w * cs + u * sn], -1).flatten(-2)
    return torch.cat([y, x[..., rot:]], -1)


def _plain_append(st: dict):
    c = st["case"]
    nq, nkv, d = c["nq"], c["nkv"], c["d"]
    rows = st["row_pos"].numel()                       # live rows come first
    x = st["qkv"][:rows].view(-1, nq + 2 * nkv, d).float()
    st["q"][:rows] = _rotate(x[:, :nq], st).to(torch.bfloat16).view(-1, nq * d)
    _plain_quantise(st, st["k"], st["k_scale"], _rotate(x[:, nq:nq + nkv], st))
    _plain_quantise(st, st["v"], st["v_scale"], x[:, nq + nkv:])


def _plain_quantise(st: dict, codes, scales, x):
    """Appends x [rows, nkv, d] in 32 bits."""
    c = st["case"]
    blk, nkv = c["blk"], c["nkv"]
    of_row, useq, ublk = st["row_block"], st["block_seq"], st["block_at"]
    top = torch.where(x.isfinite(), x.abs(), torch.zeros_like(x)).amax(-1)
    top = torch.zeros((useq.numel(), nkv), device=x.device).scatter_reduce(0, of_row[:, None].expand(-1, nkv), top, "amax")
    m, e = torch.frexp(top)                            # top = m 2^e, 1/2 <= m < 1; 448 = (7/8) 2^9
    need = torch.where(top > 0, e - 9 + (m > 0.875).int(), torch.full_like(e, -100)).clamp(min=-100)
    sp, sb = _place(st, useq, ublk * blk)
    sb = sb // blk
    old = scales[sp, :, sb].int() - 127
    kept = (st["seq_start"][useq] - ublk * blk).clamp(0, blk)    # earlier tokens of the block
    new = torch.where(kept[:, None] > 0, torch.maximum(old, need), need)
    scales[sp, :, sb] = (new + 127).to(torch.uint8)
    # earlier tokens, rounded to a scale that grew
    j = torch.arange(blk, device=x.device)
    at = (sb * blk)[:, None] + j[None, :]
    was = codes[sp[:, None], :, at]                    # [blocks, blk, nkv, d]
    moved = torch.ldexp(was.view(torch.float8_e4m3fn).float(), (old - new)[:, None, :, None])
    moved = moved.to(torch.float8_e4m3fn).view(torch.uint8)
    earlier = (j[None, :] < kept[:, None])[:, :, None, None]
    codes[sp[:, None], :, at] = torch.where(earlier, moved, was)
    y = torch.ldexp(x, -new[of_row][:, :, None])
    y = torch.where(y.isfinite(), y, torch.full_like(y, math.nan)).to(torch.float8_e4m3fn).view(torch.uint8)
    rp, rt = _place(st, st["row_seq"], st["row_pos"])
    codes[rp, :, rt] = y


def _cached(st: dict, codes, scales, n: int):
    """Positions 0 .. n - 1 of every sequence in 32 bits: [sequences, nkv, n, d]."""
    c = st["case"]
    blk, page, d = c["blk"], c["page"], c["d"]
    slot = st["seq_slot"]
    if st["table"] is None:
        q, s = codes[slot, :, :n], scales[slot, :, :-(-n // blk)]
    else:
        pages = st["table"][slot, :-(-n // page)].long()                # [sequences, pages]
        q = codes[pages].transpose(1, 2).flatten(2, 3)[:, :, :n]
        s = scales[pages].transpose(1, 2).flatten(2, 3)[:, :, :-(-n // blk)]
    s = torch.exp2(s.float() - 127).repeat_interleave(blk, 2)[:, :, :n, None]
    return q.contiguous().view(torch.float8_e4m3fn).float() * s


def _softmax_pv(s, v):
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
    return (p @ v) / p.sum(-1, keepdim=True).clamp(min=1e-30)


def _plain_decode(st: dict):
    c = st["case"]
    nq, nkv, d, rows = c["nq"], c["nkv"], c["d"], c["rows"]
    n = st["longest"]
    k, v = _cached(st, st["k"], st["k_scale"], n), _cached(st, st["v"], st["v_scale"], n)
    s = (st["q"].float().view(rows, nkv, nq // nkv, d) @ k.transpose(2, 3)) / math.sqrt(d)
    seen = torch.arange(n, device=DEV)[None, :] < (st["lens"].long() * st["valid"].long())[:, None]
    s = s.masked_fill(~seen[:, None, None, :], -math.inf)
    return _softmax_pv(s, v).view(rows, nq * d).to(torch.bfloat16)


def _plain_prefill(st: dict):
    c = st["case"]
    nq, nkv, d, n, L = c["nq"], c["nkv"], c["d"], c["prompts"], st["longest"]
    m = L - c["start"]
    k, v = _cached(st, st["k"], st["k_scale"], L), _cached(st, st["v"], st["v_scale"], L)
    q = torch.zeros((n, m, nq, d), device=DEV)         # prompts padded to the longest
    q[st["row_seq"], st["row_at"]] = st["q"].float().view(-1, nq, d)
    q = q.view(n, m, nkv, nq // nkv, d).permute(0, 2, 3, 1, 4).reshape(n, nkv, nq // nkv * m, d)
    s = ((q @ k.transpose(2, 3)) / math.sqrt(d)).view(n, nkv, nq // nkv, m, L)
    at = c["start"] + torch.arange(m, device=DEV)
    s = s.masked_fill(torch.arange(L, device=DEV)[None, :] > at[:, None], -math.inf)
    o = _softmax_pv(s.view(n, nkv, -1, L), v).view(n, nq, m, d).transpose(1, 2)
    return o[st["row_seq"], st["row_at"]].reshape(-1, nq * d).to(torch.bfloat16)


# --------------------------------------------------------------------------
# What a pass cannot do without
# --------------------------------------------------------------------------

def work(case: dict) -> dict:
    """Queries in and out, the appended tokens or the cached tokens that some
    query sees, with their scales, each once."""
    c = case
    nq, nkv, d, blk = c["nq"], c["nkv"], c["d"], c["blk"]
    tok = 2 * nkv * (d + 1 / blk)                      # bytes of a cached token's keys and values
    lens = _lens(c, c["live"] if _rows_form(c) else c["prompts"], 0)
    if c["kind"] == "append":
        T = c["live"] if _rows_form(c) else int(lens.sum())
        return {"bytes": T * ((2 * nq + 2 * nkv) * d * 2 + 2 * nkv * d + 4) + 2 * nkv * T / blk,
                "flops": T * (3 * (nq + nkv) * c["rot"] + 3 * 2 * nkv * d)}
    if c["kind"] == "decode":
        T, cached, pairs = c["live"], int(lens.sum()), int(lens.sum())
    else:
        T, cached = int(lens.sum()), int((lens + c["start"]).sum())
        pairs = int((lens * c["start"] + lens * (lens + 1) // 2).sum())
    return {"bytes": T * 2 * nq * d * 2 + cached * tok, "flops": 4 * nq * d * pairs}


# --------------------------------------------------------------------------
# The same results in 64 bits
# --------------------------------------------------------------------------

def _seqs(st: dict) -> list:
    """(first row, rows, first position, slot) of every live sequence."""
    c = st["case"]
    if _rows_form(c):
        return [(r, 1, int(p), r) for r, p in enumerate(st["lens"].tolist()) if r < c["live"]]
    out, row = [], 0
    for n, s, slot in zip(st["lens"].tolist(), st["starts"].tolist(), st["slots"].tolist()):
        out.append((row, n, s, slot))
        row += n
    return out


def _spot(st: dict, slot: int, t: int):
    page = st["case"]["page"]
    return (slot, t) if not page else (int(st["table_host"][slot, t // page]), t % page)


def _e4m3(y):
    """The nearest e4m3 value, ties to even; what is not finite is NaN."""
    a = y.abs()
    e = torch.where(a > 0, torch.floor(torch.log2(a.clamp(min=1e-300))), torch.zeros_like(a)).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.where(y.isfinite(), torch.round(y / step) * step, torch.full_like(y, math.nan))


def _exact_append(st: dict):
    c = st["case"]
    nq, nkv, d, blk, rot = c["nq"], c["nkv"], c["d"], c["blk"], c["rot"]
    f = torch.tensor(_freqs(c), dtype=torch.float64, device=DEV)
    x = st["qkv"].double().view(-1, nq + 2 * nkv, d)
    vals = {"k": st["k"].view(torch.float8_e4m3fn).double(), "v": st["v"].view(torch.float8_e4m3fn).double()}
    exps = {n: st[n + "_scale"].double() - 127 for n in ("k", "v")}
    q = st["q"].double().view(-1, nq, d)
    i = torch.arange(rot // 2, device=DEV)
    lo, hi = (i, i + rot // 2) if c["layout"] == "half" else (2 * i, 2 * i + 1)
    for row, n, p0, slot in _seqs(st):
        y = x[row:row + n].clone()
        z = torch.polar(torch.full((n, rot // 2), _magnitude(c), dtype=torch.float64, device=DEV),
                        torch.arange(p0, p0 + n, device=DEV).double()[:, None] * f)[:, None, :]
        z = torch.complex(y[:, :nq + nkv][..., lo], y[:, :nq + nkv][..., hi]) * z
        y[:, :nq + nkv, lo], y[:, :nq + nkv, hi] = z.real, z.imag
        q[row:row + n] = y[:, :nq]
        t = p0
        while t < p0 + n:
            b0 = t // blk * blk
            m = min(b0 + blk, p0 + n) - t
            pg, at = _spot(st, slot, b0)
            for name, part in (("k", y[:, nq:nq + nkv]), ("v", y[:, nq + nkv:])):
                new = part[t - p0:t - p0 + m].transpose(0, 1)          # [nkv, m, d]
                top = torch.where(new.isfinite(), new.abs(), torch.zeros_like(new)).amax((1, 2))
                need = torch.where(top > 0, torch.ceil(torch.log2(top.clamp(min=1e-300) / 448)),
                                   torch.full_like(top, -100)).clamp(min=-100)
                old = exps[name][pg, :, at // blk].clone()
                e = torch.maximum(old, need) if t > b0 else need
                exps[name][pg, :, at // blk] = e
                if t > b0:
                    was = vals[name][pg, :, at:at + t - b0]
                    vals[name][pg, :, at:at + t - b0] = _e4m3(was * torch.exp2(old - e)[:, None, None])
                vals[name][pg, :, at + t - b0:at + t - b0 + m] = _e4m3(new * torch.exp2(-e)[:, None, None])
            t += m
    return {"q": q.view(-1, nq * d), "k": vals["k"], "v": vals["v"], "k_scale": torch.exp2(exps["k"]),
            "v_scale": torch.exp2(exps["v"])}


def _exact_attention(st: dict):
    c = st["case"]
    nq, nkv, d, blk, page = c["nq"], c["nkv"], c["d"], c["blk"], c["page"]
    G = nq // nkv
    q = st["q"].double().view(-1, nq, d)
    out = torch.zeros_like(q)
    for row, n, p0, slot in _seqs(st):
        L = p0 if c["kind"] == "decode" else p0 + n    # a decode row sees its cached tokens
        if L == 0:
            continue
        kv = []
        for name in ("k", "v"):
            if page:
                ids = torch.from_numpy(st["table_host"][slot, :-(-L // page)]).to(DEV).long()
                w, s = st[name][ids], st[name + "_scale"][ids]
                w, s = w.transpose(0, 1).reshape(nkv, -1, d), s.transpose(0, 1).reshape(nkv, -1)
            else:
                w, s = st[name][slot], st[name + "_scale"][slot]
            w = w[:, :L].contiguous().view(torch.float8_e4m3fn).double()
            kv.append(w * torch.exp2(s.double() - 127).repeat_interleave(blk, 1)[:, :L, None])
        for r in range(0, n, 512):
            m = min(512, n - r)
            for g in range(nkv):
                s = torch.einsum("mgd,ld->mgl", q[row + r:row + r + m, g * G:(g + 1) * G], kv[0][g]) / math.sqrt(d)
                if c["kind"] == "prefill":
                    last = torch.arange(p0 + r, p0 + r + m, device=DEV)
                    s.masked_fill_(torch.arange(L, device=DEV)[None, None, :] > last[:, None, None], -math.inf)
                out[row + r:row + r + m, g * G:(g + 1) * G] = torch.einsum("mgl,ld->mgd", torch.softmax(s, -1), kv[1][g])
    return {"out": out.view(-1, nq * d)}


def exact(case: dict, seed: int):
    st = prepare(case, seed)
    if st["table"] is not None:
        st["table_host"] = st["table"].cpu().numpy()
    return _exact_append(st) if case["kind"] == "append" else _exact_attention(st)
