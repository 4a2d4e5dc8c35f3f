"""spade_cache_select where sums cancel: inputs so far apart in size that an fp64 sum depends on
its order. Scores closer than the sums' rounding may rank either way, but the same on
every call; everything else is ranked by the exact scores, and pages with equal means tie."""
from fractions import Fraction

import pytest
import torch

from paper_2608_03335_amd import spade as S

from . import _cache as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("pages,n,G", [(70, 1, 1), (300, 3, 2), (1500, 2, 4)])
def test_sums_that_cancel(pages, n, G):
    P, d, topk = 32, 64, 25
    gen = torch.Generator().manual_seed(pages)
    mean = torch.randn(pages, 1, d, generator=gen)
    big = 2.0 ** torch.randint(40, 62, (pages,), generator=gen).float()
    at = torch.stack([torch.randperm(d, generator=gen)[:2] for _ in range(pages)])
    mean[torch.arange(pages), 0, at[:, 0]] = big
    mean[torch.arange(pages), 0, at[:, 1]] = -big
    mean[:, 0, 0] += 2.0 ** torch.randint(0, 40, (pages,), generator=gen).float()
    mean[1::7] = mean[1].clone()                       # pages alike
    mean = mean.to(torch.bfloat16)
    q = torch.ones(n, G, d)
    q[:, :, 1::3] = 2.0 ** -20
    q = (q * (1 + torch.randint(0, 4, (n, G, 1), generator=gen))).to(torch.bfloat16)
    print("cancel", pages, n, G, flush=True)
    kv = torch.empty(pages, 1, P, d, dtype=torch.bfloat16, device=DEV)
    c = S.cache(S.SPADE_CACHE_BF16, 1, d, P, kv, kv, mean.to(DEV))
    b = S.batch(torch.arange(pages, dtype=torch.int32, device=DEV)[None],
                torch.tensor([P * pages], dtype=torch.int32, device=DEV),
                torch.tensor([0, n], dtype=torch.int32, device=DEV), n)
    ws = torch.empty(S.spade_cache_select_workspace_bytes(c, b, G, topk), dtype=torch.uint8, device=DEV)

    def call():
        counts = torch.zeros(n, 1, dtype=torch.int32, device=DEV)
        idx = torch.full((n, 1, topk), -1, dtype=torch.int32, device=DEV)
        S.spade_cache_select(c, b, q.to(DEV), topk, counts, idx, causal=False, local=0, workspace=ws)
        assert bool((counts == topk).all())
        return idx.cpu()

    idx = call()
    for _ in range(3):
        assert torch.equal(call(), idx)
    frac = lambda t: [Fraction(x) for x in t.double().tolist()]  # noqa: E731
    rows = [frac(mean[j, 0]) for j in range(pages)]
    for i in range(n):
        qs = [sum(col) for col in zip(*(frac(q[i, g]) for g in range(G)))]
        qa = [sum(abs(v) for v in col) for col in zip(*(frac(q[i, g]) for g in range(G)))]
        score = [sum(a * m for a, m in zip(qs, r)) for r in rows]
        # G - 1 and d - 1 sums and a product, each off by 2^-53 of at most the sum of sizes
        room = [Fraction(G + d, 2 ** 53) * sum(a * abs(m) for a, m in zip(qa, r)) for r in rows]
        kept = idx[i, 0].tolist()
        left = [j for j in range(pages) if j not in kept]
        assert kept == sorted(set(kept))
        assert all(score[a] + room[a] >= score[z] - room[z] for a in kept for z in left), i
        alike = [j for j in range(1, pages, 7)]
        ins = [j in kept for j in alike]
        assert ins == sorted(ins, reverse=True), i      # of pages alike the first ones
