"""Plain references of the operators for sequences that share a beginning: beam
selection and attention in 64 bits, pages by lists."""
from __future__ import annotations

import math

import numpy as np
import torch

from tests import cache_reference as ref


def beam_select(logits, scores, beams, keep, valid=None, finished=None, weights=None, end=-1):
    """numpy fp32 logits [rows, vocab] -> (tokens, parents, scores in 64 bits, finished) [groups, keep]."""
    rows, V = logits.shape
    groups = rows // beams
    out = (np.full((groups, keep), -1), np.full((groups, keep), -1), np.full((groups, keep), -np.inf),
           np.zeros((groups, keep), np.int64))
    for g in range(groups):
        found = []
        for r in range(g * beams, (g + 1) * beams):
            s, w = float(scores[r]), 1.0 if weights is None else float(weights[r])
            if (valid is not None and not valid[r]) or not (math.isfinite(w) and w > 0) or not math.isfinite(s):
                continue
            if finished is not None and finished[r]:
                found.append((-s * w, r, 0, end, s, 1))
                continue
            x = logits[r].astype(np.float64)
            if np.isnan(x).any() or np.isposinf(x).any() or np.isneginf(x).all():
                continue
            lse = x.max() + math.log(math.fsum(np.exp(x - x.max()).tolist()))
            order = np.argsort(-x, kind="stable")[:keep]
            for i, v in enumerate(order):
                if np.isfinite(x[v]):
                    found.append((-(s + (x[v] - lse)) * w, r, i, int(v), s + (x[v] - lse), int(v == end)))
        for i, (_, r, _, v, s, f) in enumerate(sorted(found)[:keep]):
            out[0][g, i], out[1][g, i], out[2][g, i], out[3][g, i] = v, r, s, f
    return out


class Pages:
    """A paged cache's table and counts as lists, and what every token of a page holds: (page, token) -> a label."""

    def __init__(self, table, held, pages, page_size, block):
        self.table, self.held = [list(map(int, t)) for t in table], list(map(int, held))
        self.pages, self.ps, self.block = pages, page_size, block
        self.width = len(self.table[0])

    def assign(self, src, keep, hold):
        """Returns (status, moves): moves are (from, to, tokens); nothing changes unless the status is 0."""
        rows = []
        for r, s in enumerate(src):
            if s == -1:
                continue
            if not 0 <= s < len(self.held):
                return -1, []
            n, m, has = keep[r], hold[r], self.held[s]
            if not 0 <= has <= self.width or not 0 <= n <= has * self.ps or not n <= m <= self.width * self.ps:
                return -1, []
            taken = self.table[s][:-(-n // self.ps)]
            if any(not 0 <= p < self.pages for p in taken):
                return -1, []
            rows.append((r, taken, n, m))
        whole = {p for _, taken, n, _ in rows for p in taken[:n // self.ps]}
        owner = {}
        for r, taken, n, _ in rows:
            if n % self.ps and taken[-1] not in whole:
                owner.setdefault(taken[-1], r)
        free = [p for p in range(self.pages) if p not in whole and p not in owner]
        new, moves, used = {}, [], 0
        for r, taken, n, m in rows:
            pages = taken[:n // self.ps]
            if n % self.ps:
                t = taken[-1]
                if owner.get(t) == r:
                    pages.append(t)
                else:
                    moves.append((t, len(pages), r, -(-(n % self.ps) // self.block) * self.block))
            new[r] = (pages, -(-m // self.ps))
        final = {}
        for r in sorted(new):
            pages, total = new[r]
            n = total - len(pages)
            final[r] = pages + [free[i] if i < len(free) else None for i in range(used, used + n)]
            used += n
        if used > len(free):
            return used - len(free), []
        for r in range(len(self.held)):
            pages = final.get(r, [])
            self.table[r][:len(pages)] = pages
            self.held[r] = len(pages)
        return 0, [(t, final[r][i], n) for t, i, r, n in moves]

    def compact(self):
        for r, n in enumerate(self.held):
            if not 0 <= n <= self.width or any(not 0 <= p < self.pages for p in self.table[r][:n]):
                return -1, []
        used = sorted({p for t, n in zip(self.table, self.held) for p in t[:n]})
        n = len(used)
        name = dict(zip([p for p in used if p >= n], [p for p in range(n) if p not in set(used)]))
        for t, h in zip(self.table, self.held):
            t[:h] = [name.get(p, p) for p in t[:h]]
        return n, [(a, b, self.ps) for a, b in name.items()]


def move(tensors, moves, block):
    """Carries out moves on [pages, nkv, tokens or blocks, ...] tensors; the block counts of scale tensors follow from
    their third dimension."""
    for t, per in tensors:
        for a, b, n in moves:
            t[b, :, : n // block * per] = t[a, :, : n // block * per]


def values(hc: ref.HostCache, slot, a, b):
    """float64 K, V [nkv, b - a, d] of tokens a .. b - 1, from nothing but their pages or their slot."""
    out = []
    for codes, sc in ((hc.k, hc.ks), (hc.v, hc.vs)):
        if hc.page:
            a0 = a // hc.page * hc.page
            ids = hc.table[slot, a // hc.page:-(-b // hc.page)].long()
            flat = lambda t: t[ids].transpose(0, 1).reshape(hc.nkv, -1, *t.shape[3:])
        else:
            a0, flat = 0, lambda t: t[slot]
        val = ref.decode_codes(flat(codes), flat(sc), hc.blk) if sc is not None else flat(codes).double()
        out.append(val[:, a - a0:b - a0])
    return out


def shared_values(hc: ref.HostCache, slot, prefix_slot, prefix, n):
    """float64 K, V [nkv, n, d] that a row of n tokens sees."""
    parts = [values(hc, s, a, b) for s, a, b in ((prefix_slot, 0, prefix), (slot, prefix, n)) if b > a]
    return [torch.cat(x, 1) for x in zip(*parts)] if parts else [torch.zeros((hc.nkv, 0, hc.d), dtype=torch.float64)] * 2


def shared_attention(hc: ref.HostCache, q, slot, prefix_slot, prefix, n):
    """As cache_reference.attention, of one row q float64 [nq, d]."""
    k, v = shared_values(hc, slot, prefix_slot, prefix, n)
    return ref.attention(q, k, v, n)
