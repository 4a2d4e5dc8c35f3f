"""Tokens written over others: the cache and its means hold what was written last, in bf16 and
in 4 bits, wherever in a page the rewind ends; and CachePath after rewinds and releases
against the same stream in 64 bits."""
import pytest
import torch

from paper_2608_03335_amd import spade as S
from paper_2608_03335_amd.pipeline import CachePath, grid_rope

from . import _cache as C
from .test_gpu_cache_append import _check
from .test_gpu_cache_path import Mirror

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("P,d", [(64, 128), (32, 64), (96, 64), (256, 128)])
@pytest.mark.parametrize("back", [1, 5, 17, 32, 40, 99])
def test_other_tokens_are_overwritten(back, P, d, fp4):
    """150 tokens of which the last `back` are others at first, up to 100 times as large, then the
    right ones in two pieces."""
    L, H = 150, 2
    print("rewind", back, P, d, fp4, flush=True)
    x = C.Batch([L], [L], 2, H, d, P, fp4, seed=71, held=[0])
    x.to_device()
    gen = torch.Generator().manual_seed(back)
    grow = 100.0 ** torch.rand(L, H, 1, generator=gen)
    other = [(torch.randn(L, H, d, generator=gen) * grow).to(torch.bfloat16) for _ in range(2)]
    at = L - back

    def put(lo, hi, k, v):
        b = S.batch(x.table.to(DEV), torch.tensor([hi], dtype=torch.int32, device=DEV),
                    torch.tensor([0, hi - lo], dtype=torch.int32, device=DEV), hi - lo)
        S.spade_cache_append(x.c, b, k[lo:hi].to(DEV), v[lo:hi].to(DEV))

    put(0, at, x.k[0], x.v[0])
    put(at, L, *other)
    mid = at + back // 3
    if mid > at:
        put(at, mid, x.k[0], x.v[0])
        torch.cuda.synchronize()
        x.lens = [mid]   # the page's mean no longer counts the tokens behind
        _check(x, x.k, "first piece")
    put(mid, L, x.k[0], x.v[0])
    torch.cuda.synchronize()
    x.lens = [L]
    _check(x, x.k, "whole")


@pytest.mark.parametrize("fp4,topk", [(False, 3), (True, 3), (False, 0), (True, 0)])
def test_stream_with_rewinds_and_releases(fp4, topk):
    B, Hq, H, d, page = 3, 4, 2, 64, 32
    print("stream with rewinds", fp4, topk, flush=True)
    cos, sin = grid_rope(6, 7, 9, d, device="cpu")
    p = CachePath(B, Hq, H, d, n_pages=11, max_pages=7, max_tokens=220, page=page, fp4=fp4, topk=topk,
                  sink=1, local=1, rope=(cos.to(DEV), sin.to(DEV)), device=DEV)
    ref = Mirror(p, cos, sin, fp4)
    gen = torch.Generator().manual_seed(1)

    def rewind(b, L):
        p.rewind(b, L)
        ref.k[b], ref.v[b] = ref.k[b][:L], ref.v[b][:L]

    def release(b):
        p.release(b)
        ref.k[b], ref.v[b] = ref.k[b][:0], ref.v[b][:0]

    steps = [([70, 100, 40], []), ([1, 2, 1], []),
             ([30, 1, 60], [lambda: rewind(0, 45), lambda: rewind(2, 3)]),      # inside a page
             ([0, 5, 1], [lambda: rewind(1, 64)]),                              # at a page's end
             ([90, 1, 1], [lambda: release(1)]),                                # its pages go to 0
             ([1, 40, 0], [lambda: rewind(0, 100), lambda: release(2)]),
             ([1, 1, 33], [lambda: rewind(1, 0)])]
    for new, changes in steps:
        for change in changes:
            change()
        n = sum(new)
        q, k, v = (torch.randn(n, h, d, generator=gen).to(torch.bfloat16) for h in (Hq, H, H))
        p.plan(new)
        lse = torch.empty(n, Hq, dtype=torch.float32, device=DEV)
        o = p.run(q.to(DEV), k.to(DEV), v.to(DEV), lse=lse)
        torch.cuda.synchronize()
        ro, rl, ot, lt = ref.step(new, q, k, v)
        assert bool(((o.cpu().double() - ro).abs() <= ot).all()), new
        assert bool(((lse.cpu().double() - rl).abs() <= lt).all()), new
        rk, rv = p.read()
        for b in range(B):
            L = p.length[b]
            assert L == len(ref.k[b])
            assert torch.equal(rk[b, :, :L].cpu().double(), ref.k[b].transpose(0, 1))
            assert torch.equal(rv[b, :, :L].cpu().double(), ref.v[b].transpose(0, 1))
            assert not bool(rk[b, :, L:].any()) and not bool(rv[b, :, L:].any())
