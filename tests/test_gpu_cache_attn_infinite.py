"""spade_cache_attn where every score that a query sees is -inf: as if it saw nothing, in the
tiles of few and of many rows, split and not; with one finite score, that token's value."""
import pytest
import torch

from paper_2608_03335_amd import spade as S

from . import _cache as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("L,n,H", [(90, 1, 2), (90, 7, 1), (4000, 2, 1), (400, 256, 64), (4200, 300, 8)])
def test_scores_of_minus_infinity(L, n, H):
    print("minus infinity", L, n, H, flush=True)
    x = C.Batch([L], [n], H, H, 64, 32, False, seed=91, held=[0])
    x.k[0][:, :, 3] = float("-inf")
    x.q[:, :, 3] = 1.0
    one = L - n + n // 2                 # seen by the queries from n // 2 on
    x.k[0][one, H - 1, 3] = 0.5
    x.hold([L])
    x.to_device()
    o = torch.full((n, H, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((n, H), 7.0, dtype=torch.float32, device=DEV)
    S.spade_cache_attn(x.c, x.b, x.q.to(DEV), 0.125, o, lse, workspace=x.workspace())
    torch.cuda.synchronize()
    o, lse = o.cpu(), lse.cpu()
    sees = torch.zeros(n, H, dtype=torch.bool)
    sees[n // 2:, H - 1] = True
    assert torch.equal(lse == float("-inf"), ~sees) and not bool(o[~sees].any())
    assert torch.equal(o[sees], x.v[0][one, H - 1].expand(n - n // 2, 64))
    score = (x.q[n // 2:, H - 1].double() * x.k[0][one, H - 1].double()).sum(-1) * 0.125
    room = (x.q[n // 2:, H - 1].double() * x.k[0][one, H - 1].double()).abs().sum(-1) * 0.125
    # 64 products, the scaling, the logarithm and its sum: fp32 roundings of at most the sizes
    assert bool(((lse[n // 2:, H - 1].double() - score).abs() <= 96 * C.FP32_HALF * (room + 8)).all())
