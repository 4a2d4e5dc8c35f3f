"""Tokens that have no place: behind the end of a sequence's table, and before its start."""
import pytest
import torch

from paper_2608_03335_amd import spade as S

from . import _cache as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens,news", [([70, 33], [10, 3]), ([200, 64], [5, 2]), ([6, 40], [9, 1]),
                                       ([-3, 40], [4, 1]), ([3000, 50], [2990, 7])])
def test_tokens_without_a_place(lens, news, causal, fp4):
    """Tables of two pages of 32. Token i of n lies at lens - n + i and is kept where that is in
    0..63; its query sees the tokens up to its place that are kept, or all of them."""
    P, H, Hq, d, room = 32, 2, 4, 64, 64
    print("ends", lens, news, causal, fp4, flush=True)
    held = [min(max(L - n, 0), room) for L, n in zip(lens, news)]
    x = C.Batch([room] * 2, [0, 0], Hq, H, d, P, fp4, seed=13, held=held, fill=float("nan")).to_device()
    n = sum(news)
    gen = torch.Generator().manual_seed(2)
    q, k, v = (torch.randn(n, h, d, generator=gen).to(torch.bfloat16) for h in (Hq, H, H))
    cu = [0, news[0], n]
    b = S.batch(x.table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
                torch.tensor(cu, dtype=torch.int32, device=DEV), n)
    q_out = torch.zeros(n, Hq, d, dtype=torch.bfloat16, device=DEV)
    S.spade_cache_append(x.c, b, k.to(DEV), v.to(DEV), q.to(DEV), q_out)
    counts = torch.zeros(n, H, dtype=torch.int32, device=DEV)
    idx = torch.full((n, H, 1), -1, dtype=torch.int32, device=DEV)
    ws = torch.empty(max(S.spade_cache_select_workspace_bytes(x.c, b, Hq, 1),
                         S.spade_cache_attn_workspace_bytes(x.c, b, Hq), 16), dtype=torch.uint8, device=DEV)
    S.spade_cache_select(x.c, b, q_out, 1, counts, idx, causal=causal, workspace=ws)
    o = torch.full_like(q_out, 7.0)
    lse = torch.zeros(n, Hq, dtype=torch.float32, device=DEV)
    S.spade_cache_attn(x.c, b, q_out, 0.125, o, lse, causal=causal, workspace=ws)
    rk, rv = (torch.full((2, H, 70, d), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    S.spade_cache_read(x.c, b, rk, rv)
    torch.cuda.synchronize()
    assert torch.equal(q_out.cpu(), q)
    for s, (L, m) in enumerate(zip(lens, news)):
        place = torch.arange(L - m, L)
        kept = (place >= 0) & (place < room)
        have = min(max(L, 0), room)
        keys, values = x.k[s].clone(), x.v[s].clone()
        rows = slice(cu[s], cu[s] + m)
        keys[place[kept]], values[place[kept]] = k[rows][kept], v[rows][kept]
        keys, values = C.stored(keys[:have], fp4), C.stored(values[:have], fp4)
        for got, want in ((rk, keys), (rv, values)):
            assert torch.equal(got[s, :, :have].cpu().double(), want.transpose(0, 1))
            assert bool((got[s, :, have:] == 9).all())
        pick = sorted({0, m // 2, m - 1, max(m - 6, 0), min(3, m - 1)})
        seen = [min(max(L - m + i + 1, 0), have) if causal else have for i in pick]
        at = [cu[s] + i for i in pick]
        for i, t in zip(seen, at):
            pages = -(-i // P)
            assert counts[t].tolist() == [min(pages, 1)] * H
            assert idx[t].flatten().tolist() == [pages - 1] * H   # local: the last visible page
        ro, rl, ot, lt = C.attend(q[at], keys, values, seen, None, P, 0.125)
        empty = torch.isinf(rl)
        assert bool(((o[at].cpu().double() - ro).abs() <= ot).all())
        assert torch.equal(torch.isinf(lse[at].cpu()), empty)
        assert bool(((lse[at].cpu().double() - rl).abs() <= lt)[~empty].all())
