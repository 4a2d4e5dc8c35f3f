"""Plain 64-bit forms of the paged-cache calls, on CPU tensors, and the page layouts of
spade.h as index formulas. A sequence's tokens are [L, H, d]; nothing here knows tiles,
splits or lists of pages beyond their definition."""
from __future__ import annotations

import math

import torch

from paper_2608_03335_amd import spade as S

E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], dtype=torch.float64)
BF16_HALF = 2.0 ** -8   # one rounding to bf16, relative
FP32_HALF = 2.0 ** -24


def bf16(x):
    return x.float().to(torch.bfloat16)


# ------------------------------------------------------------------ layout

def k_place(P, d, fp4):
    """Flat place of (token, channel) inside one page's K: elements, or nibbles."""
    t, c = torch.arange(P)[:, None], torch.arange(d)[None]
    if not fp4:
        return ((((t // 16) * (d // 32) + c // 32) * 4 + c % 32 // 8) * 16 + t % 16) * 8 + c % 8
    w = d // 4
    return (((t // 16) * 4 + c // w) * 16 + t % 16) * w + c % w


def v_place(P, d, fp4):
    t, c = torch.arange(P)[:, None], torch.arange(d)[None]
    j = (t % 32 // 16) * 4 + t % 4
    g = t % 16 // 4
    if not fp4:
        return ((((t // 32) * (d // 16) + c // 16) * 4 + g) * 16 + c % 16) * 8 + j
    return (((((t // 32) * (d // 64) + c // 64) * 4 + g) * 16 + c % 16) * 4 + c % 64 // 16) * 8 + j


def k_scale_place(P, d):
    t, r = torch.arange(P)[:, None], torch.arange(d // 32)[None]
    return ((t // 16) * (d // 32) + r) * 16 + t % 16


def v_scale_place(P, d):
    t, r = torch.arange(P)[:, None], torch.arange(d // 32)[None]
    return (((t // 32) * 4 + t % 16 // 4) * (d // 32) + r) * 8 + (t % 32 // 16) * 4 + t % 4


def _nibbles(x):
    return torch.stack((x & 15, x >> 4), -1).flatten(-2)


def unpack(buf, scale, P, d, fp4, side):
    """One side's page buffer [n, H, ...] -> stored values fp64 [n, H, P, d]."""
    place = (k_place if side == "k" else v_place)(P, d, fp4)
    n, H = buf.shape[:2]
    if not fp4:
        return buf.reshape(n, H, P * d)[:, :, place.flatten()].view(n, H, P, d).double()
    code = _nibbles(buf.reshape(n, H, -1))[:, :, place.flatten()].view(n, H, P, d).long()
    sp = (k_scale_place if side == "k" else v_scale_place)(P, d)
    s = scale.reshape(n, H, -1)[:, :, sp.flatten()].view(n, H, P, d // 32).long()
    two = torch.where(s == 255, torch.tensor(float("nan"), dtype=torch.float64), 2.0 ** (s.double() - 127))
    val = E2M1[code & 7] * torch.where(code > 7, -1.0, 1.0).double()
    return (val.unflatten(-1, (-1, 32)) * two[..., None]).flatten(-2)


def pack(values, P, d, fp4, side, out, out_scale):
    """Inverse of unpack for values already representable (fp64 [n, H, P, d]), into CPU buffers."""
    n, H = values.shape[:2]
    place = (k_place if side == "k" else v_place)(P, d, fp4).flatten()
    if not fp4:
        flat = out.view(n, H, P * d)
        flat[:, :, place] = values.reshape(n, H, P * d).to(torch.bfloat16)
        return
    code, scale = quantise_codes(values)
    nib = torch.zeros(n, H, P * d, dtype=torch.uint8)
    nib[:, :, place] = code.reshape(n, H, P * d)
    out.view(n, H, -1)[:] = nib[..., 0::2] | (nib[..., 1::2] << 4)
    sp = (k_scale_place if side == "k" else v_scale_place)(P, d).flatten()
    out_scale.view(n, H, -1)[:, :, sp] = scale.reshape(n, H, -1)


# ------------------------------------------------------------------ definitions

def quantise_codes(x):
    """fp64 [..., d] of bf16 values -> (codes uint8 [..., d], scale bytes [..., d / 32])."""
    g = x.double().unflatten(-1, (-1, 32))
    fine = torch.isfinite(g).all(-1)
    top = torch.where(fine[..., None], g.abs(), 0.0).amax(-1)
    e = torch.full_like(top, -126.0)
    for _ in range(253):  # the least exponent with top <= 7 * 2^e, step by step
        e = torch.where(top > 7.0 * 2.0 ** e, e + 1, e)
    a = g.abs() / (2.0 ** e)[..., None]
    dist = (a[..., None] - E2M1).abs()
    best = dist.min(-1, keepdim=True)[0]
    near = dist == best
    even = near & (torch.arange(8) % 2 == 0)                    # ties: the even code
    code = torch.where(even.any(-1), even.int().argmax(-1), near.int().argmax(-1))
    code = torch.where((e == 126)[..., None], code.clamp(max=5), code)
    code = torch.where((g < 0) & (code > 0), code + 8, code)
    code = torch.where(fine[..., None], code, 0)
    scale = torch.where(fine, e + 127, torch.tensor(255.0, dtype=torch.float64))
    return code.flatten(-2).to(torch.uint8), scale.to(torch.uint8)


def stored(x, fp4):
    """What the cache holds for bf16 tokens x: fp64 values."""
    if not fp4:
        return x.double()
    code, s = quantise_codes(x.double())
    two = torch.where(s == 255, torch.tensor(float("nan"), dtype=torch.float64), 2.0 ** (s.double() - 127))
    val = E2M1[(code & 7).long()] * torch.where(code > 7, -1.0, 1.0).double()
    return (val.unflatten(-1, (-1, 32)) * two[..., None]).flatten(-2)


def rotate(x, cos, sin, interleaved):
    """x bf16 [n, heads, d], cos / sin fp32 [n, rot / 2]: elementary fp32 operations, one by one."""
    half = cos.shape[1]
    y = x.float().clone()
    a = y[..., 0:2 * half:2] if interleaved else y[..., :half]
    b = y[..., 1:2 * half:2] if interleaved else y[..., half:2 * half]
    c, s = cos[:, None], sin[:, None]
    ra, rb = a * c - b * s, a * s + b * c
    if interleaved:
        y[..., 0:2 * half:2], y[..., 1:2 * half:2] = ra, rb
    else:
        y[..., :half], y[..., half:2 * half] = ra, rb
    return y.to(torch.bfloat16)


def page_means(keys, P):
    """Stored keys fp64 [L, H, d] -> bf16 [pages, H, d]."""
    return torch.stack([bf16(p.mean(0)) for p in keys.split(P)]) if len(keys) else (
        torch.zeros(0, *keys.shape[1:], dtype=torch.bfloat16))


def seen_by(L, n, causal):
    return [max(L - n + i + 1, 0) if causal else L for i in range(n)]


def select(q, mean, seen, P, topk, sink, local):
    """q bf16 [n, Hq, d], mean bf16 [pages, H, d] -> list of page lists, row (token, head)."""
    n, Hq, d = q.shape
    H = mean.shape[1] if len(mean) else 1
    rows = []
    for i in range(n):
        vis = -(-seen[i] // P)
        for h in range(H):
            qs = q[i].double().view(H, -1, d)[h].sum(0)
            score = (mean[:vis, h].double() * qs).sum(-1).tolist()
            forced = [j for j in range(vis) if j < sink or j >= vis - local]
            rest = [j for j in range(vis) if j not in forced]
            rest.sort(key=lambda j: (math.isnan(score[j]), -score[j] if score[j] == score[j] else 0, j))
            take = min(topk, vis) - len(forced)
            rows.append(sorted(forced + rest[:max(take, 0)]))
    return rows


def attend(q, k, v, seen, lists, P, scale):
    """q bf16 [n, Hq, d]; k, v stored fp64 [L, H, d]; lists: sets of pages a row, or None.
    Returns o, lse (fp64) and the error allowances of a kernel that keeps scores and sums in
    fp32 and rounds P and O to bf16 once each:
      a logit's error dl <= (d + 8) 2^-24 (scale sum|q||k| + |logit|) + 2^-24 (sum of d fp32
      products, the scaling, the subtraction of the maximum, the exponential);
      |o - exact| <= 2^-8 |o| + (2^-8 + 2 dl + (n + 8) 2^-24) sum w |v|;
      |lse - exact| <= dl + (n + 16) 2^-24 + 2^-23 |lse|."""
    n, Hq, d = q.shape
    L, H = k.shape[:2]
    o = torch.zeros(n, Hq, d, dtype=torch.float64)
    lse = torch.full((n, Hq), float("-inf"), dtype=torch.float64)
    o_tol, l_tol = torch.zeros_like(o), torch.zeros_like(lse)
    for i in range(n):
        for h in range(H):
            keys = torch.arange(min(seen[i], L))
            if lists is not None:
                inside = torch.zeros(-(-max(L, 1) // P), dtype=torch.bool)
                for j in lists[i * H + h]:
                    if 0 <= j < -(-seen[i] // P):
                        inside[j] = True
                keys = keys[inside[keys // P]]
            if len(keys) == 0:
                continue
            G = Hq // H
            for hq in range(h * G, (h + 1) * G):
                x = q[i, hq].double()
                s = (k[keys, h] * x).sum(-1) * scale
                size = (k[keys, h].abs() * x.abs()).sum(-1) * scale
                dl = float(((d + 8) * FP32_HALF * (size + s.abs()) + FP32_HALF).max())
                top = s.max()
                w = torch.exp(s - top)
                total = w.sum()
                w = w / total
                o[i, hq] = (w[:, None] * v[keys, h]).sum(0)
                lse[i, hq] = top + torch.log(total)
                room = (w[:, None] * v[keys, h].abs()).sum(0)
                o_tol[i, hq] = BF16_HALF * o[i, hq].abs() + (
                    BF16_HALF + 2 * dl + (len(keys) + 8) * FP32_HALF) * room
                l_tol[i, hq] = dl + (len(keys) + 16) * FP32_HALF + 2 * FP32_HALF * lse[i, hq].abs()
    return o, lse, o_tol, l_tol


# ------------------------------------------------------------------ a batch in hand

class Batch:
    """Sequences with tokens on the CPU and a cache on `dev` that holds them: random pages out
    of a larger pool, all bytes of it filled with `fill` first."""

    def __init__(self, lens, news, Hq, H, d, P, fp4, seed=0, dev="cuda", held=None, spare=3,
                 width=None, fill=None, gain=1.0):
        self.lens, self.news, self.Hq, self.H, self.d, self.P, self.fp4 = lens, news, Hq, H, d, P, fp4
        self.dev = dev
        gen = torch.Generator().manual_seed(seed)
        rand = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
        self.k = [bf16(rand(L, H, d) * gain) for L in lens]
        self.v = [bf16(rand(L, H, d)) for L in lens]
        self.n = sum(news)
        self.q = bf16(rand(self.n, Hq, d) * gain)
        pages = [-(-L // P) for L in lens]
        self.width = max(pages + [1]) if width is None else width
        self.n_pages = sum(pages) + spare
        perm = torch.randperm(self.n_pages, generator=gen).int()
        self.table = torch.full((len(lens), self.width), -1, dtype=torch.int32)
        used = 0
        for b, m in enumerate(pages):
            self.table[b, :m] = perm[used:used + m]
            used += m
        self.cu = torch.tensor([0] + torch.tensor(news).cumsum(0).tolist() if news else [0],
                               dtype=torch.int32)
        shape = (self.n_pages, H, P, d // 2 if fp4 else d)
        dt = torch.uint8 if fp4 else torch.bfloat16
        self.buf = {x: torch.zeros(shape, dtype=dt) for x in ("k", "v")}
        for x in ("k_scale", "v_scale"):
            self.buf[x] = torch.zeros(self.n_pages, H, P, d // 32, dtype=torch.uint8) if fp4 else None
        self.buf["k_mean"] = torch.zeros(self.n_pages, H, d, dtype=torch.bfloat16)
        if fill is not None:
            for t in self.buf.values():
                if t is not None:
                    t.fill_(255 if t.dtype == torch.uint8 else fill)
        self.hold([L for L in lens] if held is None else held)

    def hold(self, held):
        """The cache holds the first held[b] tokens of every sequence, as they are."""
        P, d, H = self.P, self.d, self.H
        for b, L in enumerate(held):
            mean = page_means(stored(self.k[b][:L], self.fp4), P)
            for j in range(-(-L // P)):
                page = int(self.table[b, j])
                for x, y in (("k", self.k[b]), ("v", self.v[b])):
                    old = unpack(self.buf[x][page:page + 1], None if not self.fp4 else
                                 self.buf[x + "_scale"][page:page + 1], P, d, self.fp4, x)
                    part = stored(y[j * P:min((j + 1) * P, L)], self.fp4)
                    old[0, :, :len(part)] = part.transpose(0, 1)
                    keep_scale = self.buf[x + "_scale"][page:page + 1] if self.fp4 else None
                    pack(old, P, d, self.fp4, x, self.buf[x][page:page + 1], keep_scale)
                self.buf["k_mean"][page] = mean[j]

    def to_device(self, n_tokens=None):
        dev = self.dev
        self.g = {x: None if t is None else t.to(dev).clone() for x, t in self.buf.items()}
        fmt = S.SPADE_CACHE_FP4 if self.fp4 else S.SPADE_CACHE_BF16
        self.c = S.cache(fmt, self.H, self.d, self.P, self.g["k"], self.g["v"], self.g["k_mean"],
                         self.g["k_scale"], self.g["v_scale"])
        self.lens_t = torch.tensor(self.lens, dtype=torch.int32).to(dev)
        self.b = S.batch(self.table.to(dev), self.lens_t, self.cu.to(dev),
                         self.n if n_tokens is None else n_tokens)
        return self

    def new(self, x):
        """The new tokens of k or v, packed."""
        return torch.cat([t[L - n:] for t, L, n in zip(x, self.lens, self.news)] or [])

    def rows(self):
        """(sequence, its first row, its new tokens) of every sequence."""
        c = self.cu.tolist()
        return [(b, c[b], c[b + 1] - c[b]) for b in range(len(self.lens))]

    def workspace(self, topk=0):
        need = max(S.spade_cache_attn_workspace_bytes(self.c, self.b, self.Hq, topk),
                   S.spade_cache_select_workspace_bytes(self.c, self.b, self.Hq, topk) if topk else 0)
        return torch.empty(max(need, 16), dtype=torch.uint8, device=self.dev)

    def ref_select(self, q, causal, topk, sink, local, keys=None):
        rows = []
        for b, t0, n in self.rows():
            k = stored(self.k[b], self.fp4) if keys is None else keys[b]
            rows += select(q[t0:t0 + n], page_means(k, self.P), seen_by(self.lens[b], n, causal),
                           self.P, topk, sink, local) if self.lens[b] else [[]] * (n * self.H)
        return rows

    def ref_attend(self, q, causal, lists, scale, keys=None, values=None):
        out = []
        for b, t0, n in self.rows():
            k = stored(self.k[b], self.fp4) if keys is None else keys[b]
            v = stored(self.v[b], self.fp4) if values is None else values[b]
            part = None if lists is None else lists[t0 * self.H:(t0 + n) * self.H]
            out.append(attend(q[t0:t0 + n], k, v, seen_by(self.lens[b], n, causal), part, self.P, scale))
        return [torch.cat(x) for x in zip(*out)]

    def lists_to(self, lists, topk, junk=-7):
        """Page lists as the calls take them."""
        counts = torch.tensor([len(r) for r in lists], dtype=torch.int32).view(self.n, self.H)
        idx = torch.full((self.n * self.H, topk), junk, dtype=torch.int32)
        for r, row in enumerate(lists):
            idx[r, :len(row)] = torch.tensor(row, dtype=torch.int32)
        return counts.to(self.dev), idx.view(self.n, self.H, topk).to(self.dev)
