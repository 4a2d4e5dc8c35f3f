"""spade_cache_attn with many new tokens a sequence and few heads: tiles of 128 rows whose pages
are shared between workgroups and joined. The 64-bit definition, and what must never reach a
result."""
import math

import pytest
import torch

from paper_2608_03335_amd import spade as S

from . import _cache as C
from .test_gpu_cache_chunk import _compare

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _say(*a):
    print(*a, flush=True)


def _call(x):
    o = torch.full((x.n, x.Hq, x.d), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((x.n, x.Hq), 7.0, dtype=torch.float32, device=DEV)
    ws = x.workspace()
    # partial results of 128 rows: the tiles of the rows that share keys, and more than one of each
    assert ws.numel() >= 2 * 128 * (x.d + 2) * 4
    ws.fill_(255)  # what the workspace holds does not matter
    return x.q.to(DEV), o, lse, ws


def _run(x, causal, scale):
    q, o, lse, ws = _call(x)
    S.spade_cache_attn(x.c, x.b, q, scale, o, lse, causal=causal, workspace=ws)
    torch.cuda.synchronize()
    return o.cpu(), lse.cpu()


CASES = [  # lens, news, Hq, H, d, P, causal
    ([5000], [500], 16, 4, 128, 64, True),
    ([4100], [200], 32, 8, 64, 32, True),
    ([9000], [300], 8, 1, 128, 96, False),
    ([6000, 0, 40, 3500], [260, 0, 40, 129], 24, 8, 128, 32, True),
    ([4500], [300], 32, 1, 128, 256, True),
    ([6000, 2100], [250, 130], 9, 3, 64, 32, False),
    ([33000], [140], 14, 2, 64, 160, True),
    ([3000], [1100], 12, 12, 64, 32, True),
]


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}x{c[3]}-d{c[4]}-P{c[5]}-c{int(c[6])}")
def test_split_chunk(case, fp4):
    lens, news, Hq, H, d, P, causal = case
    _say("split chunk", case, fp4)
    x = C.Batch(lens, news, Hq, H, d, P, fp4, seed=51).to_device()
    scale = 1 / math.sqrt(d)
    got = _run(x, causal, scale)
    _compare(x, got, causal, None, scale, {0, H - 1}, set(range(0, x.n, 11)) | {x.n - 1})


def test_more_new_tokens_than_the_context_holds():
    """Rows that see nothing are zero with a logsumexp of -inf, whichever split walks for them."""
    x = C.Batch([5000], [500], 16, 4, 128, 64, False, seed=53).to_device()
    lens = torch.tensor([470], dtype=torch.int32, device=DEV)
    b = S.batch(x.table.to(DEV), lens, torch.tensor([0, 500], dtype=torch.int32, device=DEV), 500)
    q, o, lse, ws = _call(x)
    S.spade_cache_attn(x.c, b, q, 0.09, o, lse, causal=True, workspace=ws)
    torch.cuda.synchronize()
    assert not bool(o[:30].any()) and bool((lse[:30] == float("-inf")).all())
    pick = [30, 31, 157, 158, 499]
    ro, rl, ot, lt = C.attend(x.q[pick, :4], x.k[0][:470, :1].double(), x.v[0][:470, :1].double(),
                              [i - 29 for i in pick], None, 64, 0.09)
    assert bool(((o.cpu()[pick, :4].double() - ro).abs() <= ot).all())
    assert bool(((lse.cpu()[pick, :4].double() - rl).abs() <= lt).all())


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("side", ["k", "v"])
def test_hidden_tokens_never_reach_a_result(fp4, side):
    """A new token that holds NaN: the tokens before it are bit for bit as if it were not there,
    it and those behind it are not finite."""
    H, d, P, n, L = 16, 64, 32, 300, 4200
    made = []
    for dirty in (False, True):
        x = C.Batch([L], [n], H, H, d, P, fp4, seed=57, held=[0])
        if dirty:
            (x.k if side == "k" else x.v)[0][L - n + 100] = float("nan")
        x.hold([L])
        made.append(x.to_device())
    _say("hidden, split", fp4, side)
    (o0, l0), (o1, l1) = [_run(x, True, 0.125) for x in made]
    assert torch.equal(o0[:100], o1[:100]) and torch.equal(l0[:100], l1[:100])
    assert bool(torch.isfinite(o0.float()).all()) and not bool(torch.isfinite(o1[100:].float()).any())


def test_captured_and_replayed():
    """Replays, with eager calls between them, equal these, bit for bit."""
    x = C.Batch([5000], [500], 16, 4, 128, 64, False, seed=59).to_device()
    q, o, lse, ws = _call(x)
    o2, lse2 = o.clone(), lse.clone()
    graph = torch.cuda.CUDAGraph()
    S.spade_cache_attn(x.c, x.b, q, 0.09, o, lse, causal=True, workspace=ws)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        S.spade_cache_attn(x.c, x.b, q, 0.09, o, lse, causal=True, workspace=ws)
    for _ in range(3):
        o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        ws.fill_(255)
        S.spade_cache_attn(x.c, x.b, q, 0.09, o2, lse2, causal=True, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
