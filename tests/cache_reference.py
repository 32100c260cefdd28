"""Plain 64-bit reference of the cache operators, and the bounds their results
have to keep.

Rounding to t is off by at most half a step: U[t] = eps / 2 relative (bf16
2^-8, e4m3 2^-4; e4m3 values below 2^-6 by 2^-10).  fp32 arithmetic adds
2^-24 for each operation, the device's exp 2^-21."""
from __future__ import annotations

import math

import numpy as np
import torch

U_BF16, U_E4M3, U_F32 = 2.0**-8, 2.0**-4, 2.0**-24


def freqs(theta, rot, scaling="none", factor=1.0, low=0.0, high=0.0, trained=0):
    f = [theta ** (-2.0 * i / rot) for i in range(rot // 2)]
    if scaling == "linear":
        return [x / factor for x in f]
    if scaling == "bands":
        out = []
        for x in f:
            n = trained * x / (2 * math.pi)
            g = 0.0 if n <= low else 1.0 if n >= high else (n - low) / (high - low)
            out.append(g * x + (1 - g) * x / factor)
        return out
    return f


def rotate(x, pos, f, rot, interleaved, mag=1.0):
    """x float64 [n, heads, d] at positions pos; also sum |x| mag of each pair, the scale of fp32 errors."""
    y, size = x.clone(), x.abs().clone()
    for i in range(rot // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
        ang = pos.double() * f[i]
        c, s = (torch.cos(ang) * mag)[:, None], (torch.sin(ang) * mag)[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., b] * c + x[..., a] * s
        size[..., a] = size[..., b] = (x[..., a].abs() + x[..., b].abs()) * mag
    return y, size


def decode_codes(codes, scale_bytes, blk):
    """float64 values of codes [.., tokens, d] under scale bytes [.., tokens / blk]."""
    v = codes.view(torch.float8_e4m3fn).to(torch.float32).double()
    return v * torch.exp2(scale_bytes.double() - 127).repeat_interleave(blk, -1).unsqueeze(-1)


def need_exp(amax):
    """Smallest e >= -100 with amax <= 448 2^e."""
    e = -100
    while amax > 448.0 * 2.0**e:
        e += 1
    return e


def check_codes(codes, e, values, exact):
    """codes (uint8 [.., d]) are the nearest e4m3 values to values / 2^e; 64-bit
    values computed another way may sit 1e-7 (relative) over a tie."""
    got = codes.view(torch.float8_e4m3fn).to(torch.float32).double()
    x = values * 2.0 ** (-e)
    fin = torch.isfinite(x)
    assert torch.equal(torch.isnan(got), ~fin)
    x, got = x[fin], got[fin]
    half = torch.maximum(x.abs() * U_E4M3, torch.full_like(x, 2.0**-10))
    assert (torch.abs(got - x) <= half * (1 + 1e-6) + (0 if exact else 1e-7) * x.abs()).all()


def attention(q, k, v, n_keys):
    """q float64 [nq, d], k, v float64 [nkv, L, d] -> (out, sum p |v|, largest
    sum |q k| / sqrt d) of one query over the first n_keys keys."""
    nq, d = q.shape
    nkv = k.shape[0]
    G = nq // nkv
    if n_keys == 0:
        return torch.zeros_like(q), torch.zeros_like(q), 0.0
    qq = q.view(nkv, G, d)
    kk, vv = k[:, :n_keys], v[:, :n_keys]
    s = torch.matmul(qq, kk.transpose(1, 2).contiguous()) / math.sqrt(d)
    size = (torch.matmul(qq.abs(), kk.abs().transpose(1, 2).contiguous()) / math.sqrt(d)).max().item()
    p = torch.softmax(s, -1)
    return torch.matmul(p, vv).reshape(nq, d), torch.matmul(p, vv.abs()).reshape(nq, d), size


def attention_bound(out, pv, size, d, n_keys, u_weight):
    """How far a bf16 result may be from `out`: its rounding, the weights'
    (u_weight each), twice the scores' error (a weight and the sum both carry
    it), exp, and the fp32 sums over keys."""
    ds = (d + 8) * U_F32 * size
    rel = u_weight + 2 * ds + 2.0**-20 + 2 * (64 + math.sqrt(n_keys)) * U_F32
    return U_BF16 * (out.abs() + rel * pv) + rel * pv


class HostCache:
    """An e4m3 (or bf16) cache on the host side of a test: random contents,
    contiguous or paged, and where a token of a slot stands."""

    def __init__(self, nkv, d, slots, cap, blk, page=0, seed=0, spare=3, dtype="e4m3", stale_nan=False):
        g = torch.Generator().manual_seed(seed)
        self.nkv, self.d, self.slots, self.cap, self.blk, self.page = nkv, d, slots, cap, blk, page
        if page:
            per = cap // page
            ids = torch.randperm(slots * per + spare, generator=g)[: slots * per]
            self.table = ids.view(slots, per).to(torch.int32)
            shape = (slots * per + spare, nkv, page, d)
        else:
            self.table = None
            shape = (slots, nkv, cap, d)
        x = torch.randn(shape, generator=g)
        if dtype == "bf16":
            self.k, self.v = x.to(torch.bfloat16), torch.randn(shape, generator=g).to(torch.bfloat16)
            self.ks = self.vs = None
            return
        self.k = (x * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        self.v = (torch.randn(shape, generator=g) * 60).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        s = (shape[0], nkv, shape[2] // blk)
        # values of about 1: codes of about 60 under 2^-6, some blocks louder or quieter
        self.ks = (121 + torch.randint(-2, 3, s, generator=g)).to(torch.uint8)
        self.vs = (121 + torch.randint(-2, 3, s, generator=g)).to(torch.uint8)

    def tensors(self):
        return [t for t in (self.k, self.v, self.ks, self.vs, self.table) if t is not None]

    def at(self, slot, t):
        """(index of the first dimension, token within the third)."""
        return (slot, t) if not self.page else (int(self.table[slot, t // self.page]), t % self.page)

    def values(self, slot, n):
        """float64 K, V [nkv, n, d] of the first n tokens."""
        out = []
        for codes, sc in ((self.k, self.ks), (self.v, self.vs)):
            val = decode_codes(codes, sc, self.blk) if sc is not None else codes.double()
            if self.page:
                ids = self.table[slot, : -(-n // self.page)].long()
                val = val[ids].transpose(0, 1).reshape(self.nkv, -1, self.d)[:, :n]
            else:
                val = val[slot, :, :n]
            out.append(val)
        return out

    def device_cache(self, corun, dev="cuda"):
        self.dev = [t.to(dev) for t in (self.k, self.v)]
        self.devs = [t.to(dev) for t in (self.ks, self.vs)] if self.ks is not None else None
        self.devt = self.table.to(dev) if self.table is not None else None
        if self.devs is None:
            return corun.KvCache([self.dev[0]], [self.dev[1]], page_table=self.devt)
        return corun.KvCache([self.dev[0]], [self.dev[1]], [self.devs[0]], [self.devs[1]], self.blk, self.devt)

    def after(self):
        """The device's contents as a HostCache of their own."""
        h = object.__new__(HostCache)
        h.__dict__.update(self.__dict__)
        h.k, h.v = (t.cpu() for t in self.dev)
        if self.devs is not None:
            h.ks, h.vs = (t.cpu() for t in self.devs)
        return h


def check_append(before: HostCache, after: HostCache, seqs, k, v, k_exact=False):
    """after = before with tokens appended: seqs = [(first row, rows, first
    position, slot)], k and v float64 [rows, nkv, d] (k rotated).  Every byte
    outside the appended tokens and their blocks' earlier tokens is as it was."""
    want_same = {n: torch.ones(getattr(before, n).shape[:3], dtype=torch.bool) for n in ("k", "v")}
    sc_same = {n: torch.ones(before.ks.shape, dtype=torch.bool) for n in ("ks", "vs")}
    blk = before.blk
    for row, n, p0, slot in seqs:
        t = p0
        while t < p0 + n:
            b0 = t // blk * blk
            m = min(b0 + blk, p0 + n) - t
            pg, at = before.at(slot, b0)
            for name, scn, x, exact in (("k", "ks", k, k_exact), ("v", "vs", v, True)):
                for h in range(before.nkv):
                    new = x[row + t - p0:row + t - p0 + m, h]
                    fin = new[torch.isfinite(new)]
                    amax = fin.abs().max().item() if fin.numel() else 0.0
                    sc_same[scn][pg, h, at // blk] = False
                    e = int(getattr(after, scn)[pg, h, at // blk]) - 127
                    old = int(getattr(before, scn)[pg, h, at // blk]) - 127
                    tol = 0.0 if exact else 1e-9
                    lo, hi = need_exp(amax * (1 - tol)), need_exp(amax * (1 + tol))
                    if t > b0:
                        lo, hi = max(lo, old), max(hi, old)
                    assert lo <= e <= hi, (name, slot, t, h, e, lo, hi)
                    got = getattr(after, name)[pg, h]
                    check_codes(got[at + t - b0:at + t - b0 + m], e, new, exact)
                    was = getattr(before, name)[pg, h, at:at + t - b0]
                    moved = (was.view(torch.float8_e4m3fn).float() * 2.0 ** (old - e)).to(torch.float8_e4m3fn)
                    if t > b0:
                        a, b = got[at:at + t - b0].view(torch.float8_e4m3fn).float(), moved.float()
                        assert torch.equal(torch.nan_to_num(a, nan=1e9), torch.nan_to_num(b, nan=1e9))
                want_same[name][pg, :, at:at + t - b0 + m] = False
            t += m
    for n in ("k", "v"):
        assert torch.equal(getattr(before, n)[want_same[n]], getattr(after, n)[want_same[n]])
    for n in ("ks", "vs"):
        assert torch.equal(getattr(before, n)[sc_same[n]], getattr(after, n)[sc_same[n]])
