"""Measured cases of the paged key/value cache: append, page selection, attention, read-back.

A stream of tokens (frames of a video generated chunk by chunk, or a text generated
token by token) keeps its keys and values in pages. Each call of a layer appends the
new tokens, picks pages for every new query and attends to them. A case is one such
call, or one of its operators, over a batch of sequences of different lengths.

`run` computes the plain form (elementary torch operations) or, with `own` set, makes
the framework's calls. Both start from the same buffers in the cache's page layout.

Page layout (P tokens a page; a tile is 16 tokens, d channels a head):
  bf16 k     [page, head, P/16, d/32, 4, 16, 8]: token = (tile, m), channel = (s, g, j)
  bf16 v     [page, head, P/32, d/16, 4, 16, 2, 4]: token = (kb, jt, g, jj), channel = (ct, m)
  4-bit k    [page, head, P/16, 4, 16, d/8] bytes: token = (tile, m), channel = (g, byte, nibble)
  4-bit v    [page, head, P/32, d/64, 4, 16, 4, 4] bytes: token = (kb, jt, g, jj) with the key's
             nibble 4 jt + jj, channel = (half, ct, m)
  k scales   [page, head, P/16, d/32, 16] bytes, v scales [page, head, P/32, 4, d/32, 2, 4]
  mean keys  [page, head, d] bf16
"""
import math

import torch

own = False

E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---------------------------------------------------------------- cases

def _case(kind, fmt, B, hq, h, d, page, lens, new, topk=0, causal=True, sink=1, local=2, rot=None,
          interleaved=False, grid_h=0, grid_w=0, name=None):
    c = dict(kind=kind, fmt=fmt, B=B, hq=hq, h=h, d=d, page=page, len_min=lens[0], len_max=lens[1],
             new_min=new[0], new_max=new[1], topk=topk, causal=causal, sink=sink, local=local,
             rot=d if rot is None else rot, interleaved=interleaved, grid_h=grid_h, grid_w=grid_w)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token for each of a serving batch: latency of the append
        _case("append", "bf16", 32, 32, 8, 128, 64, (300, 8000), (1, 1), name="append_step"),
        # three latent frames of 30 x 52 tokens enter the cache, rotated by their (t, y, x)
        _case("append", "bf16", 1, 12, 12, 128, 64, (14040, 14040), (4680, 4680), interleaved=True,
              grid_h=30, grid_w=52, name="append_frames"),
        # ragged prompts into 4-bit pages, and what the cache then holds, as raster tensors
        _case("append_read", "fp4", 7, 16, 4, 64, 32, (501, 5003), (37, 3001), rot=32,
              name="append_read_4bit"),
        # a long prompt into 4-bit pages and back
        _case("append_read", "fp4", 2, 32, 8, 128, 128, (9001, 16384), (9001, 16384),
              name="append_read_long"),
        # page choice of a token-by-token batch with long contexts
        _case("select", "bf16", 16, 32, 8, 128, 64, (2000, 65536), (1, 1), topk=32,
              name="select_step"),
        # page choice for every token of a chunk of a prompt
        _case("select", "bf16", 2, 16, 2, 64, 32, (9000, 16411), (1501, 2003), topk=24,
              name="select_chunk"),
        # one query, a short context: the smallest attention
        _case("attend", "bf16", 1, 16, 4, 128, 64, (8000, 8000), (1, 1), topk=16,
              name="attend_single"),
        # a serving batch over whole 4-bit contexts
        _case("attend", "fp4", 64, 32, 8, 128, 64, (700, 16384), (1, 1), name="attend_step_4bit"),
        # two very long contexts, whole, in bf16
        _case("attend", "bf16", 2, 32, 4, 128, 128, (100001, 131072), (1, 1),
              name="attend_long"),
        # new frames over the pages of all frames of a 21 x 30 x 52 video, no causal mask
        _case("attend", "bf16", 1, 12, 12, 128, 64, (32760, 32760), (4680, 4680), topk=40,
              causal=False, name="attend_frames"),
        # chunks of a prompt over selected 4-bit pages
        _case("attend", "fp4", 3, 32, 4, 64, 32, (4001, 12007), (300, 1777), topk=32,
              name="attend_chunk_4bit"),
        # the whole layer call of a serving batch: append, select, attend
        _case("step", "fp4", 24, 32, 8, 128, 64, (900, 32768), (1, 1), topk=32,
              name="layer_step_4bit"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append_read", "select", "attend", "attend", "step"])
    d = rng.choice([64, 128])
    h = rng.choice([1, 2, 3, 4, 5, 8, 12])
    g = rng.choice([1, 2, 3, 4, 5, 7, 8, 16]) if h <= 4 else rng.choice([1, 2, 4])
    page = rng.choice([32, 64, 64, 96, 128, 160, 256])
    fmt = rng.choice(["bf16", "fp4"])
    single = rng.random() < 0.5
    if single:
        B = _log(rng, 1, 48)
        hi = _log(rng, 40, max(64, min(131072, 900000 // (B * max(h, 4)) * 4)))
        new = (1, rng.choice([1, 1, 2, 5]))
    else:
        B = _log(rng, 1, 6)
        hi = _log(rng, 100, 16384 // B + 400)
        most = _log(rng, 2, min(hi, 2500 // B + 2))
        new = (rng.randint(0, most), most)
    lo = max(rng.randint(1, hi), new[1])
    hi = max(hi, lo)
    topk = _log(rng, 4, 64)
    if kind == "select":  # contexts of more pages than are kept
        hi = max(hi, 24 * page)
    if kind == "attend" and rng.random() < 0.4:
        topk = 0
    if kind in ("append", "append_read"):
        topk = 0
        if fmt == "fp4":
            kind = "append_read"
    case = _case(kind, fmt, B, h * g, h, d, page, (lo, hi), new, topk=topk,
                 causal=rng.random() < 0.6, sink=rng.randint(0, 1), local=rng.randint(1, 3),
                 rot=rng.choice([d, d, d // 2, 0]), interleaved=rng.random() < 0.5)
    most = [max(work(c)[x] for c in listed() if c["kind"] == kind) for x in ("bytes", "flops")]
    while any(work(case)[x] > m for x, m in zip(("bytes", "flops"), most)):
        for x in ("len_min", "len_max", "new_min", "new_max"):  # no dearer than the listed ones
            case[x] = max(case[x] * 3 // 4, 0 if x == "new_min" else 1)
    if kind == "select":
        case["topk"] = min(topk, max(5, case["len_max"] // page // 3))
    return case


def _spread(lo, hi, i, n, turn):
    """Value i of n between lo and hi; the last one is hi."""
    if i == n - 1:
        return hi
    return lo + int((hi - lo) * ((i * 0.6180339887 + turn) % 1.0))


def _sizes(case):
    """Tokens in the cache (new ones among them) and new tokens, for each sequence."""
    B = case["B"]
    lens = [_spread(case["len_min"], case["len_max"], b, B, 0.31) for b in range(B)]
    new = [min(_spread(case["new_min"], case["new_max"], b, B, 0.77), lens[b]) for b in range(B)]
    return lens, new


def _visible(case, length, n):
    """Visible tokens of each of a sequence's n queries."""
    return [length - n + 1 + i if case["causal"] else length for i in range(n)]


def work(case):
    lens, news = _sizes(case)
    hq, h, d, P = case["hq"], case["h"], case["d"], case["page"]
    n = sum(news)
    token = 2 * h * (2 * d if case["fmt"] == "bf16" else d // 2 + d // 32)  # K and V of one token
    by = fl = 0
    kind = case["kind"]
    if kind in ("append", "append_read", "step"):
        by += n * (hq + 2 * h) * d * 2 + n * token + n * case["rot"] * 4
        by += n * hq * d * 2 if kind != "step" else 0
        fl += 3 * n * (hq + h) * case["rot"]
        by += sum(-(-m // P) + 1 for m in news if m) * h * d * 2
    if kind == "append_read":
        by += sum(lens) * (token + 4 * h * d)
    for length, m in zip(lens, news):
        pages = -(-length // P)
        if kind in ("select", "step") and m:
            by += pages * h * d * 2 + (m * hq * d * 2 if kind == "select" else 0)
            by += m * h * (case["topk"] + 1) * 4 if kind == "select" else 0
            fl += sum(2 * (-(-v // P)) * h * d for v in _visible(case, length, m)) + m * hq * d
        if kind in ("attend", "step") and m:
            if case["topk"]:
                kept = [min(v, case["topk"] * P) for v in _visible(case, length, m)]
                by += min(sum(kept), length) * token
                by += m * h * (case["topk"] + 1) * 4 if kind == "attend" else 0
            else:
                kept = _visible(case, length, m)
                by += length * token
            by += m * hq * (d * 2 + 4) + (m * hq * d * 2 if kind == "attend" else 0)
            fl += 4 * sum(kept) * hq * d
    return {"bytes": by, "flops": fl}


# ---------------------------------------------------------------- inputs

def _inputs(case, seed):
    """Sequence data as plain token tensors (bf16, on the GPU), from the seed alone.

    Keys drift smoothly along a sequence (frames of one scene, paragraphs of one
    subject) with noise on top; a query resembles keys around an anchor that moves
    slowly with the query's position, so neighbouring queries want similar pages."""
    lens, news = _sizes(case)
    hq, h, d = case["hq"], case["h"], case["d"]
    G = hq // h
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 1000003 + 17)
    rand = lambda *s: torch.randn(*s, generator=gen, device=dev)  # noqa: E731
    ks, vs, qs = [], [], []
    for L, n in zip(lens, news):
        knots = rand(L // 150 + 2, h, d)
        at = torch.arange(L, device=dev, dtype=torch.float32) / 150.0
        i0 = at.long()
        f = (at - i0.float()).view(L, 1, 1)
        base = knots[i0] * (1 - f) + knots[i0 + 1] * f
        ks.append((base + 0.5 * rand(L, h, d)).bfloat16())
        vs.append(rand(L, h, d).bfloat16())
        if n:
            start = torch.rand(1, generator=gen, device=dev)
            i = torch.arange(n, device=dev, dtype=torch.float32)
            anchor = ((start + 0.4 * i / max(n, 200)) % 1.0 * (L - 1)).long()
            like = base[anchor].view(n, h, 1, d) + 0.5 * base[L - n:].view(n, h, 1, d)
            qs.append((0.8 * like + 0.7 * rand(n, h, G, d)).reshape(n, hq, d).bfloat16())
    n_pages = sum(-(-L // case["page"]) for L in lens)
    perm = torch.randperm(n_pages + 3, generator=gen, device=dev)
    width = max(-(-L // case["page"]) for L in lens)
    table = torch.zeros(case["B"], width, dtype=torch.int32, device=dev)
    used = 0
    for b, L in enumerate(lens):
        m = -(-L // case["page"])
        table[b, :m] = perm[used:used + m].int()
        used += m
    q = torch.cat(qs) if qs else torch.zeros(0, hq, d, dtype=torch.bfloat16, device=dev)
    return dict(lens=lens, news=news, k=ks, v=vs, q=q, table=table, n_pages=n_pages + 3)


def _angles(case, lens, news):
    """fp64 angles of every table row, and the table row of each new token (or None:
    the token's place in its sequence)."""
    half = case["rot"] // 2
    gh, gw = case["grid_h"], case["grid_w"]
    if not gh:
        inv = 10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))
        return torch.arange(max(lens), dtype=torch.float64)[:, None] * inv, None
    t = -(-max(lens) // (gh * gw))
    n = torch.arange(t * gh * gw)
    place = (n // (gh * gw), n // gw % gh, n % gw)
    part = (half - 2 * (half // 3), half // 3, half // 3)
    rows = torch.cat([p[:, None].double() * 10000.0 ** (-torch.arange(m, dtype=torch.float64) / m)
                      for p, m in zip(place, part)], 1)
    pos = torch.cat([torch.arange(L - n, L) for L, n in zip(lens, news)])
    return rows, pos


# ---------------------------------------------------------------- plain form

def _new_cache(case, n_pages):
    h, d, P, dev = case["h"], case["d"], case["page"], "cuda"
    c = dict(k_mean=torch.zeros(n_pages, h, d, dtype=torch.bfloat16, device=dev))
    if case["fmt"] == "bf16":
        c["k"] = torch.zeros(n_pages, h, P, d, dtype=torch.bfloat16, device=dev)
        c["v"] = torch.zeros(n_pages, h, P, d, dtype=torch.bfloat16, device=dev)
        c["k_scale"] = c["v_scale"] = None
    else:
        for x in ("k", "v"):
            c[x] = torch.zeros(n_pages, h, P, d // 2, dtype=torch.uint8, device=dev)
            c[x + "_scale"] = torch.ones(n_pages, h, P, d // 32, dtype=torch.uint8, device=dev)
    return c


def _views(case, c):
    """Views of the page buffers with the token's indexes first (see the module's text)."""
    h, d, P = case["h"], case["d"], case["page"]
    n = c["k"].shape[0]
    if case["fmt"] == "bf16":
        return dict(k=c["k"].view(n, h, P // 16, d // 32, 4, 16, 8).permute(0, 2, 5, 1, 3, 4, 6),
                    v=c["v"].view(n, h, P // 32, d // 16, 4, 16, 2, 4).permute(0, 2, 6, 4, 7, 1, 3, 5))
    return dict(k=c["k"].view(n, h, P // 16, 4, 16, d // 8).permute(0, 2, 4, 1, 3, 5),
                v=c["v"].view(n, h, P // 32, d // 64, 4, 16, 4, 4),
                ks=c["k_scale"].view(n, h, P // 16, d // 32, 16).permute(0, 2, 4, 1, 3),
                vs=c["v_scale"].view(n, h, P // 32, 4, d // 32, 2, 4).permute(0, 2, 5, 3, 6, 1, 4))


def _two(e):
    """2^e in fp32, for whole numbers e in [-126, 127]."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """x [..., d] bf16 -> 4-bit codes [..., d] and group scales [..., d/32], as bytes."""
    g = x.float().unflatten(-1, (-1, 32))
    top = g.abs().amax(-1)
    e = torch.frexp(top)[1] - 3                  # top in [4, 8) * 2^e: 7 * 2^e may be enough
    e = torch.where(top > 0, e, -126).clamp(min=-126)
    e = torch.where(top > 7.0 * _two(e), e + 1, e)
    a = g.abs() * _two(-e)[..., None]
    code = ((a > 0.25).byte() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5)
            + (a > 5.0))
    code = torch.where((g < 0) & (code > 0), code + 8, code)
    return code.flatten(-2).byte(), (e + 127).byte()


def _values(code, scale):
    """fp32 values of 4-bit codes [..., d] with group scales [..., d/32]."""
    mag = torch.tensor(E2M1 + tuple(-x for x in E2M1), device=code.device)[code.long()]
    return (mag.unflatten(-1, (-1, 32)) * _two(scale.int() - 127)[..., None]).flatten(-2)


def _v_codes(raw, d):
    """Packed V pages [n, h, P/32, d/64, 4, 16, 4, 4] -> codes [n, h, P, d]."""
    c = torch.stack((raw & 15, raw >> 4), -1).flatten(-2)            # nibbles 0..7 of a dword
    c = c.unflatten(-1, (2, 4))                                      # (jt, jj)
    c = c.permute(0, 1, 2, 7, 4, 8, 3, 6, 5)                         # n h kb jt g jj half ct m
    return c.reshape(c.shape[0], c.shape[1], -1, d)


def _v_pack(code):
    """Inverse of _v_codes."""
    n, h, P, d = code.shape
    c = code.view(n, h, P // 32, 2, 4, 4, d // 64, 4, 16).permute(0, 1, 2, 6, 4, 8, 7, 3, 5)
    c = c.reshape(n, h, P // 32, d // 64, 4, 16, 4, 4, 2)
    return c[..., 0] | (c[..., 1] << 4)


def _pages(case, c, ids):
    """Stored tokens of pages `ids` as fp32 [len(ids), P, h, d] keys and values."""
    w, d = _views(case, c), case["d"]
    h, P = case["h"], case["page"]
    m = ids.numel()
    if case["fmt"] == "bf16":
        k = w["k"][ids].reshape(m, P, h, d).float()
        v = w["v"][ids].reshape(m, P, h, d).float()
        return k, v
    raw = w["k"][ids].reshape(m, P, h, d // 2)
    k = torch.stack((raw & 15, raw >> 4), -1).flatten(-2)
    v = _v_codes(w["v"][ids], d).transpose(1, 2)
    return (_values(k, w["ks"][ids].reshape(m, P, h, d // 32)),
            _values(v, w["vs"][ids].reshape(m, P, h, d // 32)))


def _store(case, c, page, slot, k, v):
    """Writes tokens k, v [n, h, d] at slots of physical pages."""
    w, h, d = _views(case, c), case["h"], case["d"]
    n = page.numel()
    tile, m, kb, r = slot // 16, slot % 16, slot // 32, slot % 32
    at = (page, kb, r // 16, r % 16 // 4, r % 4)
    if case["fmt"] == "bf16":
        w["k"][page, tile, m] = k.view(n, h, d // 32, 4, 8)
        w["v"][at] = v.view(n, h, d // 16, 16)
        return
    code, scale = _quantise(k)
    w["k"][page, tile, m] = (code[..., 0::2] | (code[..., 1::2] << 4)).view(n, h, 4, d // 8)
    w["ks"][page, tile, m] = scale
    code, scale = _quantise(v)
    w["vs"][at] = scale
    ids, where = torch.unique(page, return_inverse=True)
    old = _v_codes(w["v"][ids], d).transpose(1, 2).contiguous()
    old[where, slot] = code
    w["v"][ids] = _v_pack(old.transpose(1, 2))


def _means(case, c, ids, fill):
    """Mean stored key of the first `fill` tokens of pages `ids`."""
    k, _ = _pages(case, c, ids)
    P = case["page"]
    live = torch.arange(P, device="cuda")[None, :] < fill[:, None]
    total = (k.double() * live[:, :, None, None]).sum(1)
    c["k_mean"][ids] = (total / fill.double()[:, None, None]).float().bfloat16()


def _places(case, st, first, last):
    """Physical page and slot of tokens first[b]..last[b]-1, and the touched pages with
    their fill, over all sequences."""
    P = case["page"]
    page, slot, ids, fill = [], [], [], []
    for b, (lo, hi) in enumerate(zip(first, last)):
        if hi <= lo:
            continue
        t = torch.arange(lo, hi, device="cuda")
        page.append(st["table"][b].long()[t // P])
        slot.append(t % P)
        j = torch.arange(lo // P, (hi - 1) // P + 1, device="cuda")
        ids.append(st["table"][b].long()[j])
        fill.append((hi - j * P).clamp(max=P))
    return torch.cat(page), torch.cat(slot), torch.cat(ids), torch.cat(fill)


def _rotate(case, st, x):
    """x [n, heads, d] bf16, rotated by its tokens' table rows: fp32, rounded once."""
    rot = case["rot"]
    if rot == 0:
        return x.clone()
    y = x.float()
    cos, sin = st["cos"][st["row"]][:, None], st["sin"][st["row"]][:, None]
    if case["interleaved"]:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
    a, b = a * cos - b * sin, a * sin + b * cos
    if case["interleaved"]:
        turned = torch.stack((a, b), -1).flatten(-2)
    else:
        turned = torch.cat((a, b), -1)
    return torch.cat((turned, y[..., rot:]), -1).bfloat16()


def _plain_append(case, st):
    q = _rotate(case, st, st["q"])
    c = st["cache"]
    _store(case, c, st["page"], st["slot"], _rotate(case, st, st["k_new"]), st["v_new"])
    _means(case, c, st["ids"], st["fill"])
    return q


def _plain_read(case, st):
    P = case["page"]
    for b, L in enumerate(st["lens_host"]):
        k, v = _pages(case, st["cache"], st["table"][b].long()[:-(-L // P)])
        for out, x in ((st["k_read"], k), (st["v_read"], v)):
            out[b, :, :L] = x.flatten(0, 1)[:L].transpose(0, 1).bfloat16()


def _plain_select(case, st, q):
    h, d, P, K = case["h"], case["d"], case["page"], case["topk"]
    t0 = 0
    for b, (L, n) in enumerate(zip(st["lens_host"], st["new_host"])):
        pages = -(-L // P)
        mean = st["cache"]["k_mean"][st["table"][b].long()[:pages]].double()  # [pages, h, d]
        mean = mean.permute(1, 2, 0).contiguous()
        step = max(1, (1 << 26) // (h * pages))
        for i0 in range(0, n, step):
            m = min(step, n - i0)
            qs = q[t0 + i0:t0 + i0 + m].double().view(m, h, -1, d).sum(2).transpose(0, 1)
            score = torch.matmul(qs.contiguous(), mean).transpose(0, 1)       # [m, h, pages]
            at = torch.arange(i0, i0 + m, device="cuda")
            seen = L - n + 1 + at if case["causal"] else torch.full_like(at, L)
            vis = (seen + P - 1) // P
            j = torch.arange(pages, device="cuda")
            forced = (j[None] < case["sink"]) | (j[None] >= vis[:, None] - case["local"])
            hidden = j[None] >= vis[:, None]
            score = score.masked_fill(forced[:, None], float("inf"))
            score = score.masked_fill(hidden[:, None], float("-inf"))
            kk = min(K, pages)
            best = torch.sort(score, stable=True, dim=-1, descending=True)[1][..., :kk]
            count = vis.clamp(max=K)
            best = best.masked_fill(torch.arange(kk, device="cuda") >= count[:, None, None], 1 << 30)
            best = torch.sort(best, -1)[0]
            best = best.masked_fill(best == 1 << 30, -1)
            st["indices"][t0 + i0:t0 + i0 + m, :, :kk] = best.int()
            st["counts"][t0 + i0:t0 + i0 + m] = count[:, None].int()
        t0 += n


def _plain_attend(case, st, q):
    hq, h, d, P = case["hq"], case["h"], case["d"], case["page"]
    G = hq // h
    t0 = 0
    for b, (L, n) in enumerate(zip(st["lens_host"], st["new_host"])):
        if n == 0:
            continue
        pages = -(-L // P)
        k, v = _pages(case, st["cache"], st["table"][b].long()[:pages])
        k = k.flatten(0, 1)[:L].permute(1, 2, 0).contiguous()             # [h, d, L]
        v = v.flatten(0, 1)[:L].transpose(0, 1).contiguous()              # [h, L, d]
        step = max(1, (1 << 28) // (hq * L))
        for i0 in range(0, n, step):
            m = min(step, n - i0)
            rows = slice(t0 + i0, t0 + i0 + m)
            x = q[rows].float().view(m, h, G, d).transpose(0, 1).reshape(h, m * G, d).contiguous()
            s = (torch.matmul(x, k) * st["scale"]).view(h, m, G, L)
            at = torch.arange(i0, i0 + m, device="cuda")
            seen = L - n + 1 + at if case["causal"] else torch.full_like(at, L)
            live = (torch.arange(L, device="cuda")[None] < seen[:, None])[None]   # [1, m, L]
            if case["topk"]:
                member = torch.zeros(m, h, pages + 1, dtype=torch.bool, device="cuda")
                width = min(case["topk"], st["indices"].shape[-1])
                idx = st["indices"][rows][..., :width].long()
                ok = torch.arange(width, device="cuda") < st["counts"][rows][..., None]
                member.scatter_(2, torch.where(ok, idx, pages), True)
                live = live & member[:, :, :pages].transpose(0, 1).repeat_interleave(P, -1)[..., :L]
            s.masked_fill_(~live[:, :, None], float("-inf"))
            top = s.amax(-1, keepdim=True)
            p = torch.exp(s - top)
            total = p.sum(-1, keepdim=True)
            o = torch.matmul(p.view(h, m * G, L), v).view(h, m, G, d) / total
            st["o"][rows] = o.transpose(0, 1).reshape(m, hq, d).bfloat16()
            st["lse"][rows] = (top + torch.log(total)).squeeze(-1).transpose(0, 1).reshape(m, hq)
        t0 += n


# ---------------------------------------------------------------- preparation and passes

def prepare(case, seed):
    x = _inputs(case, seed)
    lens, news, n = x["lens"], x["news"], sum(x["news"])
    hq, h, d, K = case["hq"], case["h"], case["d"], case["topk"]
    dev = "cuda"
    st = dict(case=case, lens_host=lens, new_host=news, table=x["table"], q=x["q"],
              scale=1.0 / math.sqrt(d), cache=_new_cache(case, x["n_pages"]))
    kind = case["kind"]
    adds = kind in ("append", "append_read", "step")
    first = [0] * case["B"]
    held = [L - m if adds else L for L, m in zip(lens, news)]
    if sum(held):
        page, slot, ids, fill = _places(case, st, first, held)
        _store(case, st["cache"], page, slot, torch.cat([k[:a] for k, a in zip(x["k"], held)]),
               torch.cat([v[:a] for v, a in zip(x["v"], held)]))
        _means(case, st["cache"], ids, fill)
    st["k_new"] = torch.cat([k[L - m:] for k, L, m in zip(x["k"], lens, news)])
    st["v_new"] = torch.cat([v[L - m:] for v, L, m in zip(x["v"], lens, news)])
    st["lens"] = torch.tensor(lens, dtype=torch.int32, device=dev)
    cu = [0]
    for m in news:
        cu.append(cu[-1] + m)
    st["cu"] = torch.tensor(cu, dtype=torch.int32, device=dev)
    if adds:
        rows, pos = _angles(case, lens, news)
        st["cos"], st["sin"] = rows.cos().float().to(dev), rows.sin().float().to(dev)
        st["pos"] = None if pos is None else pos.int().to(dev)
        if n:
            place = torch.cat([torch.arange(L - m, L) for L, m in zip(lens, news)])
            st["row"] = (place if pos is None else pos).to(dev)
            st["page"], st["slot"], st["ids"], st["fill"] = _places(case, st, [L - m for L, m in
                                                                               zip(lens, news)], lens)
        st["q_out"] = torch.zeros_like(st["q"])
    if kind == "append_read":
        shape = (case["B"], h, max(lens), d)
        st["k_read"] = torch.zeros(shape, dtype=torch.bfloat16, device=dev)
        st["v_read"] = torch.zeros(shape, dtype=torch.bfloat16, device=dev)
    if K:
        st["counts"] = torch.zeros(n, h, dtype=torch.int32, device=dev)
        st["indices"] = torch.full((n, h, K), -1, dtype=torch.int32, device=dev)
    if kind in ("attend", "step"):
        st["o"] = torch.zeros(n, hq, d, dtype=torch.bfloat16, device=dev)
        st["lse"] = torch.zeros(n, hq, dtype=torch.float32, device=dev)
        if kind == "attend" and K:
            _plain_select(case, st, st["q"])
    if own:
        from paper_2608_03335_amd import spade as S
        c = st["cache"]
        fmt = S.SPADE_CACHE_BF16 if case["fmt"] == "bf16" else S.SPADE_CACHE_FP4
        st["c"] = S.cache(fmt, h, d, case["page"], c["k"], c["v"], c["k_mean"], c["k_scale"],
                          c["v_scale"])
        st["b"] = S.batch(st["table"], st["lens"], st["cu"], n)
        if adds and case["rot"]:
            st["rope"] = S.rope(st["cos"], st["sin"], st["pos"], interleaved=case["interleaved"])
        need = max(S.spade_cache_select_workspace_bytes(st["c"], st["b"], hq, K) if K else 0,
                   S.spade_cache_attn_workspace_bytes(st["c"], st["b"], hq, K))
        st["workspace"] = torch.empty(max(need, 16), dtype=torch.uint8, device=dev)
    return st


def _outputs(st):
    kind, c = st["case"]["kind"], st["cache"]
    if kind == "append":
        return [st["q_out"], c["k"], c["v"], c["k_mean"]]
    if kind == "append_read":
        return [st["q_out"], st["k_read"], st["v_read"], c["k_mean"]]
    if kind == "select":
        return [st["counts"], st["indices"]]
    if kind == "attend":
        return [st["o"], st["lse"]]
    return [st["q_out"], st["counts"], st["indices"], st["o"], st["lse"], c["k_mean"]]


def run(st):
    case = st["case"]
    kind = case["kind"]
    q = st["q"]
    if own:
        from paper_2608_03335_amd import spade as S
        c, b, ws = st["c"], st["b"], st["workspace"]
        if kind in ("append", "append_read", "step"):
            S.spade_cache_append(c, b, st["k_new"], st["v_new"], q, st["q_out"], st.get("rope"))
            q = st["q_out"]
        if kind == "append_read":
            S.spade_cache_read(c, b, st["k_read"], st["v_read"])
        if kind in ("select", "step"):
            S.spade_cache_select(c, b, q, case["topk"], st["counts"], st["indices"],
                                 causal=case["causal"], sink=case["sink"], local=case["local"],
                                 workspace=ws)
        if kind in ("attend", "step"):
            S.spade_cache_attn(c, b, q, st["scale"], st["o"], st["lse"], st.get("counts"),
                               st.get("indices"), causal=case["causal"], workspace=ws)
        return _outputs(st)
    if kind in ("append", "append_read", "step") and q.shape[0]:
        st["q_out"].copy_(_plain_append(case, st))
        q = st["q_out"]
    if kind == "append_read":
        _plain_read(case, st)
    if kind in ("select", "step"):
        _plain_select(case, st, q)
    if kind in ("attend", "step"):
        _plain_attend(case, st, q)
    return _outputs(st)


# ---------------------------------------------------------------- 64-bit results

def _exact_rotate(case, x, turn):
    """x [n, heads, d] as complex pairs times the unit numbers `turn`, fp64."""
    rot = case["rot"]
    y = x.double()
    if rot == 0:
        return y
    head = y[..., :rot]
    if case["interleaved"]:
        z = torch.complex(head[..., 0::2].contiguous(), head[..., 1::2].contiguous())
    else:
        z = torch.complex(*(p.contiguous() for p in head.chunk(2, -1)))
    z = z * turn[:, None]
    out = torch.stack((z.real, z.imag), -2 if not case["interleaved"] else -1).flatten(-2)
    return torch.cat((out, y[..., rot:]), -1)


def _exact_stored(case, x):
    """What the cache holds for x [..., d]: bf16 values, or the nearest 4-bit values."""
    x = x.float().bfloat16().double()
    if case["fmt"] == "bf16":
        return x
    g = x.unflatten(-1, (-1, 32))
    top = g.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(top.clamp(min=1e-300) / 7.0))
    e = torch.where(torch.exp2(e - 1) * 7 >= top, e - 1, e)
    e = torch.where(torch.exp2(e) * 7 < top, e + 1, e).clamp(-126, 127)
    a = g.abs() * torch.exp2(-e)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    near = (torch.round(a / step) * step).clamp(max=6.0)      # torch.round: ties to even
    return (torch.sign(g) * near * torch.exp2(e)).flatten(-2)


def _exact_pages(case, x):
    """Stored tokens [L, h, d] -> mean of each page [pages, h, d]."""
    return torch.stack([p.mean(0) for p in x.split(case["page"])])


def _layout(case, x, table, n_pages):
    """Token tensors of all sequences -> a page buffer (bf16 layout), zero elsewhere."""
    h, d, P = case["h"], case["d"], case["page"]
    plain = torch.zeros(2, n_pages, P, h, d, dtype=torch.float64, device="cuda")
    for b, (k, v) in enumerate(x):
        for side, y in ((0, k), (1, v)):
            for j, part in enumerate(y.split(P)):
                plain[side, int(table[b, j]), :part.shape[0]] = part
    k = plain[0].view(n_pages, P // 16, 16, h, d // 32, 4, 8).permute(0, 3, 1, 4, 5, 2, 6)
    v = plain[1].view(n_pages, P // 32, 2, 4, 4, h, d // 16, 16).permute(0, 5, 1, 6, 3, 7, 2, 4)
    return k.reshape(n_pages, h, P, d), v.reshape(n_pages, h, P, d)


def _exact_lists(case, q, mean, vis):
    """q [n, hq, d], mean [pages, h, d] (bf16 values) -> page lists, one list a row."""
    n, h = q.shape[0], case["h"]
    qs = q.double().view(n, h, -1, case["d"]).sum(2)
    out = []
    score = torch.stack([qs[:, a] @ mean[:, a].T.contiguous() for a in range(h)], 1).cpu().numpy()
    for i in range(n):
        forced = [j for j in range(vis[i]) if j < case["sink"] or j >= vis[i] - case["local"]]
        rest = slice(min(case["sink"], vis[i]), max(min(case["sink"], vis[i]), vis[i] - case["local"]))
        for a in range(h):
            free = max(min(case["topk"], vis[i]) - len(forced), 0)
            order = (-score[i, a, rest]).argsort(kind="stable")[:free] + rest.start
            out.append(sorted(set(forced) | set(int(j) for j in order)))
    return out


def _exact_attend(case, q, k, v, seen, lists):
    """Softmax attention, one K/V head at a time, fp64. lists: one per (query, head) or None."""
    n, hq, d = q.shape
    h, P = case["h"], case["page"]
    G, L = hq // h, k.shape[0]
    o = torch.empty(n, hq, d, dtype=torch.float64, device="cuda")
    lse = torch.empty(n, hq, dtype=torch.float64, device="cuda")
    key = torch.arange(L, device="cuda")
    step = max(1, (1 << 27) // (G * L))
    for i0 in range(0, n, step):
        m = min(step, n - i0)
        see = torch.tensor(seen[i0:i0 + m], device="cuda")
        for a in range(h):
            bias = torch.zeros(m, L, dtype=torch.float64, device="cuda")
            if lists is not None:
                bias += float("-inf")
                rows = [lists[(i0 + i) * h + a] for i in range(m)]
                r = torch.tensor([i for i, x in enumerate(rows) for _ in x], device="cuda")
                p = torch.tensor([j for x in rows for j in x], device="cuda")
                keep = torch.zeros(m, -(-L // P), dtype=torch.bool, device="cuda")
                keep[r, p] = True
                bias[keep.repeat_interleave(P, 1)[:, :L]] = 0.0
            bias[key[None] >= see[:, None]] = float("-inf")
            x = q[i0:i0 + m, a * G:(a + 1) * G].double().reshape(m * G, d)
            s = (x @ k[:, a].T.contiguous()) / math.sqrt(d)
            s = s.view(m, G, L) + bias[:, None]
            lse[i0:i0 + m, a * G:(a + 1) * G] = torch.logsumexp(s, -1)
            w = torch.softmax(s, -1).view(m * G, L)
            o[i0:i0 + m, a * G:(a + 1) * G] = (w @ v[:, a].contiguous()).view(m, G, d)
    return o, lse


def exact(case, seed):
    x = _inputs(case, seed)
    lens, news, kind, P = x["lens"], x["news"], case["kind"], case["page"]
    adds = kind in ("append", "append_read", "step")
    rows, pos = _angles(case, lens, news) if adds else (None, None)
    q_out, stored, lists, counts, os, ls = [], [], [], [], [], []
    t0 = 0
    if kind in ("select", "step") and sum(news) * case["h"] > 60000:
        return None  # the lists are sorted row by row
    for b, (L, n) in enumerate(zip(lens, news)):
        q, k, v = x["q"][t0:t0 + n], x["k"][b], x["v"][b]
        keys = k.double()
        if adds and n:
            at = torch.arange(L - n, L) if pos is None else pos[t0:t0 + n]
            angle = rows[at]                              # the tables hold fp32 values
            turn = torch.complex(*(f.float().double() for f in (angle.cos(), angle.sin()))).to("cuda")
            keys = torch.cat((keys[:L - n], _exact_rotate(case, k[L - n:], turn)))
            qr = _exact_rotate(case, q, turn)
        else:
            qr = q.double()
        if kind in ("append", "append_read", "step"):
            q_out.append(qr)
        held = (_exact_stored(case, keys), _exact_stored(case, v.double()))
        stored.append(held)
        q16 = qr.float().bfloat16()
        seen = _visible(case, L, n)
        vis = [-(-s // P) for s in seen]
        if case["topk"] and n:
            mean = _exact_pages(case, held[0]).float().bfloat16().double()
            if kind == "attend":  # the lists are this case's input
                one = dict(lens_host=[L], new_host=[n], table=torch.arange(
                    mean.shape[0], device="cuda")[None], cache=dict(k_mean=mean.bfloat16()),
                    counts=torch.zeros(n, case["h"], dtype=torch.int32, device="cuda"),
                    indices=torch.full((n, case["h"], case["topk"]), -1, dtype=torch.int32,
                                       device="cuda"))
                _plain_select(case, one, q16)
                part = [[j for j in r if j >= 0] for r in one["indices"].flatten(0, 1).tolist()]
            else:
                part = _exact_lists(case, q16, mean, vis)
            lists += part
            counts += [len(r) for r in part]
        else:
            part = None
        if kind in ("attend", "step") and n:
            o, lse = _exact_attend(case, q16, held[0], held[1], seen, part)
            os.append(o)
            ls.append(lse)
        t0 += n
    n, h, K = sum(news), case["h"], case["topk"]
    if K:
        idx = torch.full((n * h, K), -1, dtype=torch.int32)
        for r, row in enumerate(lists):
            idx[r, :len(row)] = torch.tensor(row, dtype=torch.int32)
        picked = [torch.tensor(counts, dtype=torch.int32).view(n, h).to("cuda"),
                  idx.view(n, h, K).to("cuda")]
    if kind == "select":
        return picked
    if kind == "attend":
        return [torch.cat(os), torch.cat(ls)]
    mean = torch.zeros(x["n_pages"], h, case["d"], dtype=torch.float64, device="cuda")
    for b, (k, _) in enumerate(stored):
        for j, m in enumerate(_exact_pages(case, k)):
            mean[int(x["table"][b, j])] = m
    turned = torch.cat(q_out)
    if kind == "append":
        return [turned, *_layout(case, stored, x["table"], x["n_pages"]), mean]
    if kind == "append_read":
        reads = []
        for side in (0, 1):
            out = torch.zeros(case["B"], h, max(lens), case["d"], dtype=torch.float64, device="cuda")
            for b, held in enumerate(stored):
                out[b, :, :lens[b]] = held[side].transpose(0, 1)
            reads.append(out)
        return [turned, *reads, mean]
    return [turned, *picked, torch.cat(os), torch.cat(ls), mean]
