"""spade_cache_attn with many new tokens a sequence (tiles of 128 rows that share their keys):
the 64-bit definition on some K/V heads, and what must never reach a result. Enough heads and
rows that the call takes that kernel."""
import math

import pytest
import torch

from paper_2608_03335_amd import spade as S

from . import _cache as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _say(*a):
    print(*a, flush=True)


def _lists(x, causal, topk, gen, near):
    """Page lists of every (token, head): pages near the token's place, and random ones."""
    rows = []
    for b, t0, n in x.rows():
        for i, s in enumerate(C.seen_by(x.lens[b], n, causal)):
            vis = -(-s // x.P)
            for _ in range(x.H):
                k = min(topk, vis)
                if near:
                    first = max(0, vis - k - i // 40)
                    row = set(range(first, min(first + k - k // 3, vis)))
                else:
                    row = set()
                for j in torch.randperm(vis, generator=gen).tolist():
                    if len(row) >= k:
                        break
                    row.add(j)
                rows.append(sorted(row))
    return rows


def _run(x, causal, lists, topk, scale):
    o = torch.full((x.n, x.Hq, x.d), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((x.n, x.Hq), 7.0, dtype=torch.float32, device=DEV)
    counts = idx = None
    if lists is not None:
        counts, idx = x.lists_to(lists, topk)
    assert S.spade_cache_attn_workspace_bytes(x.c, x.b, x.Hq, topk) == 0
    S.spade_cache_attn(x.c, x.b, x.q.to(DEV), scale, o, lse, counts, idx, causal=causal)
    torch.cuda.synchronize()
    return o.cpu(), lse.cpu()


def _compare(x, got, causal, lists, scale, heads, tokens=None):
    G = x.Hq // x.H
    tokens = range(x.n) if tokens is None else tokens
    for b, t0, n in x.rows():
        seen = C.seen_by(x.lens[b], n, causal)
        mine = [i for i in range(n) if t0 + i in tokens]
        for h in heads:
            q = x.q[t0:t0 + n, h * G:(h + 1) * G][mine]
            part = None if lists is None else [lists[(t0 + i) * x.H + h] for i in mine]
            ro, rl, ot, lt = C.attend(q, C.stored(x.k[b][:, h:h + 1], x.fp4), C.stored(x.v[b][:, h:h + 1], x.fp4),
                                      [seen[i] for i in mine], part, x.P, scale)
            rows = [t0 + i for i in mine]
            o, lse = got[0][rows, h * G:(h + 1) * G].double(), got[1][rows, h * G:(h + 1) * G].double()
            empty = torch.isinf(rl)
            assert torch.equal(torch.isinf(lse) & (lse < 0), empty), (b, h)
            assert bool(((o - ro).abs() <= ot).all()), (b, h, float(((o - ro).abs() - ot).max()))
            assert bool(((lse - rl).abs() <= lt)[~empty].all()), (b, h)


CASES = [  # lens, news, Hq, H, d, P, causal, topk, near
    ([300, 290], [150, 107], 64, 64, 64, 32, True, 3, True),
    ([300, 290], [150, 107], 64, 64, 128, 32, False, 0, True),
    ([260], [260], 64, 64, 128, 96, True, 0, True),
    ([700, 33, 0, 150], [200, 33, 0, 150], 160, 32, 64, 64, True, 5, False),
    ([2000], [130], 128, 32, 128, 32, True, 20, True),
    ([900, 800], [70, 64], 128, 16, 64, 32, False, 9, False),
    ([500], [260], 70, 10, 128, 160, True, 2, True),
    ([400], [130], 128, 4, 64, 256, True, 0, False),
    ([17500], [520], 32, 32, 64, 32, True, 40, False),
]


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}x{c[3]}-d{c[4]}-P{c[5]}-c{int(c[6])}-k{c[7]}")
def test_chunk(case, fp4):
    lens, news, Hq, H, d, P, causal, topk, near = case
    _say("chunk", case, fp4)
    small = sum(-(-L // P) for L in lens) < 200
    x = C.Batch(lens, news, Hq, H, d, P, fp4, seed=31, fill=float("nan") if small else None).to_device()
    lists = _lists(x, causal, topk, torch.Generator().manual_seed(7), near) if topk else None
    scale = 1 / math.sqrt(d)
    got = _run(x, causal, lists, topk, scale)
    picked = None if small else set(range(0, x.n, 13)) | {x.n - 1}
    _compare(x, got, causal, lists, scale, (0, H // 2, H - 1), picked)


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("-inf")])
@pytest.mark.parametrize("side", ["k", "v"])
def test_hidden_tokens_never_reach_a_result(fp4, bad, side):
    """As in the test of few tokens: rows that do not see the bad tokens are bit for bit as if
    they were not there, rows that do are not finite."""
    H, d, P, n, L = 64, 64, 32, 256, 400
    made = []
    for dirty in (False, True):
        x = C.Batch([L], [n], H, H, d, P, fp4, seed=33, held=[0])
        if dirty:
            toks = x.k if side == "k" else x.v
            toks[0][L - n + 100] = bad      # a new token: hidden from new tokens 0..99
            toks[0][70] = bad               # page 2: hidden by lists
        x.hold([L])
        made.append(x.to_device())
    clean, x = made
    _say("hidden", fp4, bad, side)
    lists = [[0, 1, 3, 7, 11] if i % 2 else [0, 2, 3, 7, 11] for i in range(n) for _ in range(H)]
    lists = [[j for j in r if j * P <= L - n + i // H] for i, r in enumerate(lists)]
    at = (L - n + 100) // P
    for topk, rows in ((5, lists), (0, None)):
        want, got = _run(clean, True, rows, topk, 0.125), _run(x, True, rows, topk, 0.125)
        for i in range(n):
            new = i >= 100 and (topk == 0 or at in rows[i * H])
            sees = new or topk == 0 or i % 2 == 0
            if not sees:
                assert torch.equal(got[0][i], want[0][i]) and torch.equal(got[1][i], want[1][i]), (topk, i)
            elif side == "v" or bad != bad:
                assert bool(torch.isnan(got[0][i].float()).any() | torch.isinf(got[0][i].float()).any()), (topk, i)


def test_few_and_many_tokens_agree():
    """The same queries in one call of many tokens and one by one (the other kernel): both
    within their allowance of the same values."""
    x = C.Batch([600], [256], 64, 64, 64, 64, False, seed=35).to_device()
    many = _run(x, True, None, 0, 0.125)
    for i in (0, 31, 32, 127, 128, 255):
        lens = torch.tensor([600 - 255 + i], dtype=torch.int32, device=DEV)
        b = S.batch(x.table.to(DEV), lens, torch.tensor([0, 1], dtype=torch.int32, device=DEV), 1)
        o = torch.empty(1, 64, 64, dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(max(S.spade_cache_attn_workspace_bytes(x.c, b, 64), 16), dtype=torch.uint8, device=DEV)
        S.spade_cache_attn(x.c, b, x.q[i:i + 1].to(DEV), 0.125, o, workspace=ws)
        torch.cuda.synchronize()
        ro, _, ot, _ = C.attend(x.q[i:i + 1], x.k[0].double(), x.v[0].double(), [600 - 255 + i], None, 64, 0.125)
        assert bool(((o.cpu().double() - ro).abs() <= ot).all())
        assert bool(((many[0][i:i + 1].double() - ro).abs() <= ot).all())


def test_damaged_offsets_cannot_fault():
    x = C.Batch([300, 290], [150, 107], 64, 64, 64, 32, True, seed=36).to_device()
    q = x.q.to(DEV)
    o = torch.empty(x.n, 64, 64, dtype=torch.bfloat16, device=DEV)
    idx = torch.randint(-2 ** 31, 2 ** 31 - 1, (x.n, 64, 3), dtype=torch.int64).to(torch.int32).to(DEV)
    counts = torch.randint(-5, 100, (x.n, 64), dtype=torch.int32).to(DEV)
    table = x.table.clone()
    table[0, 2], table[1, 1] = -1, 10 ** 6
    for lens, cu in (([10 ** 9, -4], [0, 100, 257]), ([300, 290], [250, 2, -3]), ([-2 ** 31, 2 ** 31 - 1], [0, 257, 257]),
                     ([300, 290], [3, 150, 250])):
        b = S.batch(table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
                    torch.tensor(cu, dtype=torch.int32, device=DEV), x.n)
        o.fill_(7.0)
        S.spade_cache_attn(x.c, b, q, 0.125, o, counts=counts, indices=idx)
        S.spade_cache_attn(x.c, b, q, 0.125, o)
        torch.cuda.synchronize()
    assert bool((o[:3] == 7).all()) and bool((o[250:] == 7).all())
