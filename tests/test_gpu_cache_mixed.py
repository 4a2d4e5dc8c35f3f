"""Attention of batches whose sequences differ much (a chunk of a prompt beside single tokens over
longer contexts, with and without lists), and of groups of more than 32 query heads with many
tokens."""
import math

import pytest
import torch

from paper_2608_03335_amd import spade as S

from . import _cache as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


CASES = [  # lens, news, Hq, H, d, P
    ([6000] + [300 + 41 * i for i in range(16)], [1] + [700 if i == 7 else 1 for i in range(16)], 32, 8, 128, 64),
    ([2500, 9000, 40, 0, 700], [1, 1, 1, 0, 640], 16, 4, 64, 32),
    ([900, 500], [300, 1], 64, 1, 128, 64),
    ([700], [257], 128, 1, 64, 32),
    ([1200, 1100], [130, 3], 96, 2, 64, 96),
]


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("topk", [0, 4])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}-{max(c[1])}-{c[2]}x{c[3]}-d{c[4]}-P{c[5]}")
def test_mixed(case, topk, fp4):
    lens, news, Hq, H, d, P = case
    print("mixed", case, topk, fp4, flush=True)
    x = C.Batch(lens, news, Hq, H, d, P, fp4, seed=81).to_device()
    gen = torch.Generator().manual_seed(3)
    lists = counts = idx = None
    if topk:
        lists = []
        for b, t0, n in x.rows():
            for s in C.seen_by(lens[b], n, True):
                lists += [sorted(torch.randperm(-(-s // P), generator=gen)[:topk].tolist()) for _ in range(H)]
        counts, idx = x.lists_to(lists, topk)
    scale = 1 / math.sqrt(d)
    o = torch.full((x.n, Hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((x.n, Hq), 7.0, dtype=torch.float32, device=DEV)
    ws = x.workspace(topk)
    ws.fill_(255)
    S.spade_cache_attn(x.c, x.b, x.q.to(DEV), scale, o, lse, counts, idx, workspace=ws)
    torch.cuda.synchronize()
    o, lse, G = o.cpu().double(), lse.cpu().double(), Hq // H
    for b, t0, n in x.rows():
        pick = sorted({i for i in (0, n // 3, n // 2, n - 1) if 0 <= i < n})
        if not pick:
            continue
        seen = C.seen_by(lens[b], n, True)
        rows = [t0 + i for i in pick]
        for h in {0, H - 1}:
            part = None if lists is None else [lists[t * H + h] for t in rows]
            heads = slice(h * G, (h + 1) * G)
            ro, rl, ot, lt = C.attend(x.q[rows, heads], C.stored(x.k[b][:, h:h + 1], fp4),
                                      C.stored(x.v[b][:, h:h + 1], fp4), [seen[i] for i in pick], part, P, scale)
            assert bool(((o[rows, heads] - ro).abs() <= ot).all()), (b, h)
            empty = torch.isinf(rl)   # more new tokens than the sequence holds: the first see nothing
            assert torch.equal(torch.isinf(lse[rows, heads]), empty), (b, h)
            assert bool(((lse[rows, heads] - rl).abs() <= lt)[~empty].all()), (b, h)
