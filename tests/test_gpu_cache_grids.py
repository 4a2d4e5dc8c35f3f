"""Cache calls of more workgroups than one launch takes (2^24 of 256 threads): the last sequence
of such a call is served like the first. Nearly all workgroups find nothing to do."""
import pytest
import torch

from paper_2608_03335_amd import spade as S

pytestmark = pytest.mark.gpu
DEV = "cuda"
LAUNCH = 2 ** 32 // 256


def _say(*a):
    print(*a, flush=True)


def _pool(n_pages, H, P, d, gen):
    k, v = (torch.zeros(n_pages, H, P, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    mean = torch.zeros(n_pages, H, d, dtype=torch.bfloat16, device=DEV)
    return S.cache(S.SPADE_CACHE_BF16, H, d, P, k, v, mean), mean


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def test_read_of_a_large_table():
    B, H, P, d, width = 256, 8, 32, 64, 4096
    assert B * width * H * 2 >= LAUNCH
    _say("read", B, width, H)
    gen = torch.Generator().manual_seed(1)
    c, _ = _pool(8, H, P, d, gen)
    table = torch.full((B, width), -1, dtype=torch.int32)
    table[0, :2] = torch.tensor([1, 2])
    table[255, 4095] = 3
    # what the pages hold goes in through two short sequences with the same pages
    k, v = (torch.randn(40 + 32, H, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(2))
    short = S.batch(_i32([[1, 2], [3, 4]]), _i32([40, 32]), _i32([0, 40, 72]), 72)
    S.spade_cache_append(c, short, k, v)
    lens = torch.zeros(B, dtype=torch.int32)
    lens[0], lens[255] = 40, width * P
    N = width * P
    rk, rv = (torch.empty(B, H, N, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    for r in (rk, rv):
        r[0, :, :64], r[1, :, :64], r[255, :, -64:] = 9.0, 9.0, 9.0
    S.spade_cache_read(c, S.batch(table.to(DEV), lens.to(DEV), _i32([0] * (B + 1)), 0), rk, rv)
    torch.cuda.synchronize()
    for r, x in ((rk, k), (rv, v)):
        assert torch.equal(r[0, :, :40], x[:40].transpose(0, 1)) and bool((r[0, :, 40:64] == 9).all())
        assert torch.equal(r[255, :, -32:], x[40:].transpose(0, 1)) and bool((r[255, :, -64:-32] == 9).all())
        assert bool((r[1, :, :64] == 9).all())


def test_read_of_a_large_table_for_few_tokens():
    """The grid counts the pages that N tokens take, not the table's."""
    B, H, P, d, width = 1024, 8, 32, 64, 16384
    c, _ = _pool(2, H, P, d, None)
    k, v = (torch.randn(33, H, d, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16).to(DEV)
            for _ in range(2))
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    table[B - 1, :2] = _i32([1, 0])
    S.spade_cache_append(c, S.batch(_i32([[1, 0]]), _i32([33]), _i32([0, 33]), 33), k, v)
    lens = torch.full((B,), 33, dtype=torch.int32, device=DEV)
    rk, rv = (torch.full((B, H, 33, d), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    S.spade_cache_read(c, S.batch(table, lens, _i32([0] * (B + 1)), 0), rk, rv)
    torch.cuda.synchronize()
    for r, x in ((rk, k), (rv, v)):
        assert torch.equal(r[B - 1], x.transpose(0, 1)) and bool((r[:B - 1] == 9).all())


def test_append_to_many_pages():
    B, H, P, d = 420, 4096, 256, 64
    assert (B // P + 2 * B) * H * 5 >= LAUNCH
    _say("append", B, H)
    gen = torch.Generator().manual_seed(2)
    c, mean = _pool(4, H, P, d, gen)
    table = torch.full((B, 1), -1, dtype=torch.int32)
    table[0], table[B - 1] = 2, 1
    k, v, q = (torch.randn(B, H, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(3))
    q_out = torch.zeros_like(q)
    b = S.batch(table.to(DEV), _i32([1] * B), _i32(list(range(B + 1))), B)
    S.spade_cache_append(c, b, k, v, q, q_out)
    rk, rv = (torch.full((B, H, 1, d), 9.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    S.spade_cache_read(c, b, rk, rv)
    torch.cuda.synchronize()
    assert torch.equal(q_out, q)
    for r, x in ((rk, k), (rv, v)):
        assert torch.equal(r[[0, B - 1], :, 0], x[[0, B - 1]]) and bool((r[1:B - 1] == 9).all())
    assert torch.equal(mean[[2, 1]], k[[0, B - 1]]) and not bool(mean[[0, 3]].any())


def test_attention_of_many_tiles():
    B, H, P, d = 4096, 4096, 32, 64
    assert (B // 16 + B) * H >= LAUNCH
    _say("attention", B, H)
    gen = torch.Generator().manual_seed(4)
    c, _ = _pool(3, H, P, d, gen)
    k, v = (torch.randn(2, H, d, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(2))
    S.spade_cache_append(c, S.batch(_i32([[2], [1]]), _i32([1, 1]), _i32([0, 1, 2]), 2), k, v)
    table = torch.full((B, 1), -1, dtype=torch.int32)
    table[0], table[B - 1] = 2, 1
    q = torch.ones(B, H, d, dtype=torch.bfloat16, device=DEV)
    o = torch.full_like(q, 7.0)
    b = S.batch(table.to(DEV), _i32([1] * B), _i32(list(range(B + 1))), B)
    assert S.spade_cache_attn_workspace_bytes(c, b, H) == 0
    S.spade_cache_attn(c, b, q, 0.125, o)
    torch.cuda.synchronize()
    assert torch.equal(o[[0, B - 1]], v)   # of one token: its value
    assert not bool(o[1:B - 1].any())
