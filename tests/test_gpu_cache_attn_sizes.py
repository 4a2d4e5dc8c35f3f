"""spade_cache_attn on values near the ends of bf16: weights that grow along the walk must not
carry them past the largest fp32 number, since the weighted mean itself does not leave
their range."""
import pytest
import torch

from paper_2608_03335_amd import spade as S

from . import _cache as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _rising(L, n, H, P, fp4, size):
    """Scores that are about 0 on the first 32 keys and about 5.2 (2^7.5) above behind them; values
    up to `size`."""
    x = C.Batch([L], [n], H, H, 64, P, fp4, seed=61, held=[0])
    gen = torch.Generator().manual_seed(5)
    x.k[0] = (x.k[0].float() * 0.01).to(torch.bfloat16)
    x.k[0][:, :, 0] = 8.0
    x.k[0][:32, :, 0] = 0.0
    x.q[:, :, 0] = 1.0
    x.v[0] = ((2 * torch.rand(L, H, 64, generator=gen, dtype=torch.float64) - 1) * size).to(torch.bfloat16)
    x.hold([L])
    return x.to_device()


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("L,n,H", [(500, 1, 2), (500, 5, 1), (3000, 1, 1), (600, 256, 64), (2500, 300, 8)])
def test_large_values(L, n, H, fp4):
    # 3000 keys of weight 1 at most: the sums stay below 3000 * 2^115 < 2^127
    size = 2.0 ** (122 if L < 1000 else 115)
    print("large values", L, n, H, fp4, flush=True)
    x = _rising(L, n, H, 32, fp4, size)
    o = torch.empty(n, H, 64, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(n, H, dtype=torch.float32, device=DEV)
    S.spade_cache_attn(x.c, x.b, x.q.to(DEV), 0.65, o, lse, workspace=x.workspace())
    torch.cuda.synchronize()
    pick, heads = sorted({0, n // 3, n - 1}), sorted({0, H - 1})
    seen = C.seen_by(L, n, True)
    for h in heads:
        ro, rl, ot, lt = C.attend(x.q[pick][:, h:h + 1], C.stored(x.k[0][:, h:h + 1], fp4),
                                  C.stored(x.v[0][:, h:h + 1], fp4), [seen[i] for i in pick], None, 32, 0.65)
        assert bool(((o.cpu()[pick][:, h:h + 1].double() - ro).abs() <= ot).all()), h
        assert bool(((lse.cpu()[pick][:, h:h + 1].double() - rl).abs() <= lt).all()), h


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("L,n,H", [(500, 1, 2), (3000, 1, 1), (600, 256, 64)])
def test_small_values(L, n, H, fp4):
    """Values down to 2^-110: every one between that and 2^-104."""
    print("small values", L, n, H, fp4, flush=True)
    x = _rising(L, n, H, 32, fp4, 1.0)
    gen = torch.Generator().manual_seed(6)
    size = 2.0 ** (-110 + 6 * torch.rand(L, H, 64, generator=gen, dtype=torch.float64))
    x.v[0] = (size * (1 - 2 * torch.randint(0, 2, size.shape, generator=gen))).to(torch.bfloat16)
    x.hold([L])
    x.to_device()
    o = torch.empty(n, H, 64, dtype=torch.bfloat16, device=DEV)
    S.spade_cache_attn(x.c, x.b, x.q.to(DEV), 0.65, o, workspace=x.workspace())
    torch.cuda.synchronize()
    pick = sorted({0, n // 3, n - 1})
    seen = C.seen_by(L, n, True)
    for h in {0, H - 1}:
        ro, _, ot, _ = C.attend(x.q[pick][:, h:h + 1], C.stored(x.k[0][:, h:h + 1], fp4),
                                C.stored(x.v[0][:, h:h + 1], fp4), [seen[i] for i in pick], None, 32, 0.65)
        assert bool(((o.cpu()[pick][:, h:h + 1].double() - ro).abs() <= ot).all()), h
