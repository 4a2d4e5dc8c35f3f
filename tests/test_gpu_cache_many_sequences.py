"""Cache calls of up to 2^20 sequences, the limit: the sequence of a workgroup's tokens is found
among all of them in a few steps, and sequences without new tokens cost little."""
import pytest
import torch

from paper_2608_03335_amd import spade as S

from . import _cache as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _say(*a):
    print(*a, flush=True)


def test_one_token_each():
    """Attention to one token gives its value, whatever its score."""
    B, P, d = 2 ** 20, 32, 64
    _say("one token each of", B)
    gen = torch.Generator(device=DEV).manual_seed(1)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV).to(torch.bfloat16)  # noqa: E731
    pk, pv = (torch.empty(B, 1, P, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    mean = torch.empty(B, 1, d, dtype=torch.bfloat16, device=DEV)
    c = S.cache(S.SPADE_CACHE_BF16, 1, d, P, pk, pv, mean)
    table = torch.randperm(B, generator=gen, device=DEV).int()[:, None].contiguous()
    k, v, q = rand(B, 1, d), rand(B, 1, d), rand(B, 1, d)
    b = S.batch(table, torch.ones(B, dtype=torch.int32, device=DEV),
                torch.arange(B + 1, dtype=torch.int32, device=DEV), B)
    q_out = torch.zeros_like(q)
    S.spade_cache_append(c, b, k, v, q, q_out)
    counts = torch.zeros(B, 1, dtype=torch.int32, device=DEV)
    idx = torch.full((B, 1, 2), -1, dtype=torch.int32, device=DEV)
    ws = torch.empty(max(S.spade_cache_select_workspace_bytes(c, b, 1, 2),
                         S.spade_cache_attn_workspace_bytes(c, b, 1), 16), dtype=torch.uint8, device=DEV)
    S.spade_cache_select(c, b, q, 2, counts, idx, workspace=ws)
    o, o2 = torch.zeros_like(q), torch.zeros_like(q)
    S.spade_cache_attn(c, b, q, 0.125, o, workspace=ws)
    ws = torch.empty(max(S.spade_cache_attn_workspace_bytes(c, b, 1, 2), 16), dtype=torch.uint8, device=DEV)
    S.spade_cache_attn(c, b, q, 0.125, o2, counts=counts, indices=idx, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(q_out, q) and torch.equal(mean[table[:, 0].long()], k)
    assert bool((counts == 1).all()) and bool((idx[..., 0] == 0).all()) and bool((idx[..., 1] == -1).all())
    assert torch.equal(o, v) and torch.equal(o2, v)


@pytest.mark.parametrize("at", [0, 150001, 2 ** 18 - 1])
def test_one_token_among_many_sequences(at):
    """A long context whose sequence alone has a new token."""
    B, H, Hq, P, d, L = 2 ** 18, 8, 32, 64, 64, 20000
    _say("one token among", B, at)
    x = C.Batch([L], [1], Hq, H, d, P, False, seed=3, held=[L - 1]).to_device()
    table = torch.full((B, x.width), -1, dtype=torch.int32, device=DEV)
    table[at] = x.table[0].to(DEV)
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    lens[at] = L
    cu = torch.zeros(B + 1, dtype=torch.int32, device=DEV)
    cu[at + 1:] = 1
    b = S.batch(table, lens, cu, 1)
    q, q_out = x.q.to(DEV), torch.zeros(1, Hq, d, dtype=torch.bfloat16, device=DEV)
    S.spade_cache_append(x.c, b, x.new(x.k).to(DEV), x.new(x.v).to(DEV), q, q_out)
    counts = torch.zeros(1, H, dtype=torch.int32, device=DEV)
    idx = torch.full((1, H, 9), -1, dtype=torch.int32, device=DEV)
    ws = torch.empty(max(S.spade_cache_select_workspace_bytes(x.c, b, Hq, 9),
                         S.spade_cache_attn_workspace_bytes(x.c, b, Hq), 16), dtype=torch.uint8, device=DEV)
    S.spade_cache_select(x.c, b, q_out, 9, counts, idx, workspace=ws)
    o = torch.zeros_like(q_out)
    lse = torch.zeros(1, Hq, dtype=torch.float32, device=DEV)
    S.spade_cache_attn(x.c, b, q_out, 0.125, o, lse, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(q_out, q)
    lists = x.ref_select(x.q, True, 9, 0, 1)
    assert idx[0].tolist() == lists
    ro, rl, ot, lt = C.attend(x.q, x.k[0].double(), x.v[0].double(), [L], None, P, 0.125)
    assert bool(((o.cpu().double() - ro).abs() <= ot).all())
    assert bool(((lse.cpu().double() - rl).abs() <= lt).all())


def test_selection_in_slabs():
    """More scores than are kept at once: tokens of a sequence on both sides of a cut."""
    B, H, P, d, width = 1500, 4, 32, 64, 16384
    news = [1 + b % 3 for b in range(B)]          # 2999 tokens; a slab holds 2^26 / (4 * 16384) = 1024
    lens = [40 + (37 * b) % 90 + n for b, n in enumerate(news)]
    x = C.Batch(lens, news, H, H, d, P, False, seed=5, width=width)
    x.to_device()
    counts = torch.zeros(x.n, H, dtype=torch.int32, device=DEV)
    idx = torch.full((x.n, H, 2), -1, dtype=torch.int32, device=DEV)
    S.spade_cache_select(x.c, x.b, x.q.to(DEV), 2, counts, idx, workspace=x.workspace(2))
    torch.cuda.synchronize()
    want = x.ref_select(x.q, True, 2, 0, 1)
    assert counts.flatten().tolist() == [len(r) for r in want]
    got = idx.cpu().view(-1, 2).tolist()
    assert [g[:len(w)] for g, w in zip(got, want)] == want


def test_damaged_offsets_of_many_sequences_cannot_fault():
    """Offsets in any order lead to some sequence or to none, never outside."""
    B, H, P, d = 3000, 2, 32, 64
    news = [b % 2 for b in range(B)]
    x = C.Batch([5] * B, news, H, H, d, P, False, seed=7).to_device()
    gen = torch.Generator().manual_seed(8)
    cu = torch.randint(-2 ** 31, 2 ** 31 - 1, (B + 1,), generator=gen, dtype=torch.int64)
    k, v, q = x.new(x.k).to(DEV), x.new(x.v).to(DEV), x.q.to(DEV)
    counts = torch.zeros(x.n, H, dtype=torch.int32, device=DEV)
    idx = torch.zeros(x.n, H, 2, dtype=torch.int32, device=DEV)
    ws, o = x.workspace(2), torch.empty_like(q)
    for bad in (cu, cu % (2 * x.n), cu.sort(descending=True)[0]):
        b = S.batch(x.table.to(DEV), x.lens_t, bad.int().to(DEV), x.n)
        S.spade_cache_append(x.c, b, k, v, q, torch.empty_like(q))
        S.spade_cache_select(x.c, b, q, 2, counts, idx, workspace=ws)
        S.spade_cache_attn(x.c, b, q, 0.125, o, counts=counts, indices=idx, workspace=ws)
        S.spade_cache_attn(x.c, b, q, 0.125, o, workspace=x.workspace())
        torch.cuda.synchronize()
