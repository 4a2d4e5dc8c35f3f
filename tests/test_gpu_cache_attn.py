"""spade_cache_attn against its definition in 64 bits, within the allowance that
_cache.attend derives for each value; and what must never reach a result."""
import math

import pytest
import torch

from paper_2608_03335_amd import spade as S

from . import _cache as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _say(*a):
    print(*a, flush=True)


def _run(x, causal, lists=None, topk=0, scale=None, junk=None):
    scale = 1 / math.sqrt(x.d) if scale is None else scale
    o = torch.full((x.n, x.Hq, x.d), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((x.n, x.Hq), 7.0, dtype=torch.float32, device=DEV)
    counts = idx = None
    if lists is not None:
        counts, idx = x.lists_to(lists, topk, **({} if junk is None else dict(junk=junk)))
    ws = x.workspace(topk)
    ws.fill_(255)  # what the workspace holds does not matter
    S.spade_cache_attn(x.c, x.b, x.q.to(DEV), scale, o, lse, counts, idx, causal=causal, workspace=ws)
    torch.cuda.synchronize()
    return o.cpu(), lse.cpu(), scale


def _compare(x, got, want):
    o, lse, _ = got
    ro, rl, o_tol, l_tol = want
    empty = torch.isinf(rl)
    assert torch.equal(torch.isinf(lse) & (lse < 0), empty)
    assert bool((o[empty] == 0).all())
    err = (o.double() - ro).abs()
    assert bool((err <= o_tol).all()), float((err - o_tol).max())
    err = (lse.double() - rl).abs()[~empty]
    assert bool((err <= l_tol[~empty]).all()), float((err - l_tol[~empty]).max())


def _random_lists(x, causal, topk, seed=0):
    gen = torch.Generator().manual_seed(seed)
    rows = []
    for b, t0, n in x.rows():
        for s in C.seen_by(x.lens[b], n, causal):
            vis = -(-s // x.P)
            for _ in range(x.H):
                k = min(topk, vis)
                rows.append(sorted(torch.randperm(vis, generator=gen)[:k].tolist()))
    return rows


CASES = [  # lens, news, Hq, H, d, P, causal
    ([1], [1], 1, 1, 64, 32, True),
    ([17], [1], 4, 2, 128, 64, True),
    ([33, 0, 1, 64], [1, 0, 1, 1], 4, 4, 64, 32, False),
    ([100, 31], [37, 31], 2, 2, 64, 32, True),
    ([100, 31], [37, 31], 2, 2, 128, 32, False),
    ([700, 65, 128], [1, 1, 1], 16, 2, 128, 64, True),
    ([513], [5], 20, 1, 64, 128, True),
    ([400], [3], 40, 1, 128, 96, True),
    ([300, 290], [9, 4], 5, 1, 128, 160, True),
    ([2100], [2], 6, 2, 64, 256, False),
    ([5000], [1], 3, 1, 128, 64, True),
    ([260], [16], 14, 2, 128, 32, True),
]
ids = lambda c: f"{c[0]}-{c[1]}-{c[2]}x{c[3]}-d{c[4]}-P{c[5]}-c{int(c[6])}"  # noqa: E731


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("case", CASES, ids=ids)
def test_all_visible_tokens(case, fp4):
    lens, news, Hq, H, d, P, causal = case
    _say("attend, all", case, fp4)
    x = C.Batch(lens, news, Hq, H, d, P, fp4, seed=21, fill=float("nan")).to_device()
    got = _run(x, causal)
    _compare(x, got, x.ref_attend(x.q, causal, None, got[2]))


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("case", CASES, ids=ids)
@pytest.mark.parametrize("topk", [1, 3, 40])
def test_listed_pages(case, fp4, topk):
    lens, news, Hq, H, d, P, causal = case
    _say("attend, lists", case, fp4, topk)
    x = C.Batch(lens, news, Hq, H, d, P, fp4, seed=22, fill=float("nan")).to_device()
    lists = _random_lists(x, causal, topk)
    got = _run(x, causal, lists, topk)
    _compare(x, got, x.ref_attend(x.q, causal, lists, got[2]))


def test_large_logits_and_other_scales():
    x = C.Batch([500, 90], [2, 5], 4, 2, 128, 64, False, seed=23, gain=6.0).to_device()
    for scale in (0.02, 0.3, 1.0):
        got = _run(x, True, scale=scale)
        _compare(x, got, x.ref_attend(x.q, True, None, scale))


def test_lists_are_sets_of_visible_pages():
    """Any order, entries listed twice, invisible and absurd entries, counts out of range."""
    x = C.Batch([300, 200, 90], [3, 1, 20], 4, 2, 64, 32, False, seed=24, fill=float("nan")).to_device()
    clean, given = [], []
    gen = torch.Generator().manual_seed(2)
    for b, t0, n in x.rows():
        for s in C.seen_by(x.lens[b], n, True):
            vis = -(-s // x.P)
            for _ in range(x.H):
                row = torch.randint(0, vis, (6,), generator=gen).tolist()
                clean.append(sorted(set(row)))
                row += [row[0], -1, vis, vis + 3, 2 ** 31 - 1, -2 ** 31]
                given.append([row[i] for i in torch.randperm(12, generator=gen).tolist()])
    got = _run(x, True, given, 12)
    _compare(x, got, x.ref_attend(x.q, True, clean, got[2]))
    counts, idx = x.lists_to(given, 12)
    counts[0], counts[1] = 10 ** 9, -4      # all 12 entries; none
    clean[2 * 1], clean[2 * 1 + 1] = [], []
    o = torch.empty(x.n, 4, 64, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(x.n, 4, dtype=torch.float32, device=DEV)
    S.spade_cache_attn(x.c, x.b, x.q.to(DEV), got[2], o, lse, counts, idx, workspace=x.workspace(12))
    torch.cuda.synchronize()
    _compare(x, (o.cpu(), lse.cpu(), got[2]), x.ref_attend(x.q, True, clean, got[2]))


def test_rows_with_empty_lists():
    x = C.Batch([100, 40], [3, 17], 2, 1, 128, 32, True, seed=25).to_device()
    lists = [[] if i % 3 else [0] for i in range(x.n)]
    got = _run(x, True, lists, 2)
    _compare(x, got, x.ref_attend(x.q, True, lists, got[2]))
    got = _run(x, True, [[] for _ in range(x.n)], 2)
    assert bool((got[0] == 0).all()) and bool((got[1] == float("-inf")).all())


def test_more_new_tokens_than_the_context_holds():
    """lens below the new tokens: the first ones see nothing."""
    x = C.Batch([40], [40], 2, 2, 64, 32, False, seed=26).to_device()
    b = S.batch(x.table.to(DEV), torch.tensor([12], dtype=torch.int32, device=DEV), x.cu.to(DEV), 40)
    o = torch.full((40, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.empty(40, 2, dtype=torch.float32, device=DEV)
    S.spade_cache_attn(x.c, b, x.q.to(DEV), 0.1, o, lse, workspace=x.workspace())
    torch.cuda.synchronize()
    x.lens = [12]
    want = C.attend(x.q, x.k[0][:12].double(), x.v[0][:12].double(), C.seen_by(12, 40, True), None, 32, 0.1)
    _compare(x, (o.cpu(), lse.cpu(), 0.1), want)
    assert bool((o[:28] == 0).all()) and bool((o[28:] != 0).any())


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("side", ["k", "v"])
def test_hidden_tokens_never_reach_a_result(fp4, bad, side):
    """Tokens with NaN or infinities that some queries of a tile see and their neighbours do
    not (causal order, pages of other lists): the others are as if they were not there."""
    Hq, H, d, P = 2, 1, 64, 32
    clean = C.Batch([200], [20], Hq, H, d, P, fp4, seed=27)
    x = C.Batch([200], [20], Hq, H, d, P, fp4, seed=27)
    toks = x.k if side == "k" else x.v
    toks[0][190] = bad                # the new token 10: hidden from new tokens 0..9
    toks[0][70] = bad                 # page 2: hidden by lists
    x.hold([200])
    clean.to_device(), x.to_device()
    lists = [[0, 1, 5, 6] if i % 2 else [0, 2, 5, 6] for i in range(20)]
    _say("hidden", fp4, bad, side)
    for topk, rows in ((0, None), (4, lists)):
        want, got = _run(clean, True, rows, topk), _run(x, True, rows, topk)
        for i in range(20):
            sees = i >= 10 or topk == 0 or i % 2 == 0
            if not sees:
                assert torch.equal(got[0][i], want[0][i]) and torch.equal(got[1][i], want[1][i]), i
            else:
                wo = C.attend(x.q[i:i + 1], C.stored(x.k[0], fp4), C.stored(x.v[0], fp4), [181 + i],
                              None if rows is None else [rows[i]], P, got[2])[0]
                assert torch.equal(torch.isnan(got[0][i].double()), torch.isnan(wo[0])), i


def test_rows_of_no_sequence_and_bad_pages():
    x = C.Batch([100, 90], [2, 3], 2, 2, 64, 32, False, seed=28, fill=float("nan"))
    x.cu = torch.tensor([3, 5, 8], dtype=torch.int32)
    x.table[1, 1] = x.n_pages + 2                 # tokens 32..63 of sequence 1 are nowhere
    x.to_device(n_tokens=10)
    q = torch.randn(10, 2, 64, generator=torch.Generator().manual_seed(3)).to(torch.bfloat16)
    o = torch.full((10, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.full((10, 2), 7.0, dtype=torch.float32, device=DEV)
    ws = x.workspace()
    S.spade_cache_attn(x.c, x.b, q.to(DEV), 0.125, o, lse, workspace=ws)
    torch.cuda.synchronize()
    for rows in (slice(0, 3), slice(8, 10)):
        assert bool((o[rows] == 7).all()) and bool((lse[rows] == 7).all())
    every = [[0, 1, 2, 3]] * 4 + [[0, 2]] * 6     # (token, head) rows
    want = [C.attend(q[t0:t0 + n], x.k[b].double(), x.v[b].double(), C.seen_by(x.lens[b], n, True),
                     every[2 * (t0 - 3):2 * (t0 - 3 + n)], 32, 0.125) for b, t0, n in x.rows()]
    _compare(x, (o[3:8].cpu(), lse[3:8].cpu(), 0.125), [torch.cat(w) for w in zip(*want)])
    for lens, cu in (([10 ** 9, -4], [0, 5, 9]), ([100, 90], [7, 2, -3]), ([-2 ** 31, 2 ** 31 - 1], [0, 9, 9])):
        b = S.batch(x.table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
                    torch.tensor(cu, dtype=torch.int32, device=DEV), 10)
        S.spade_cache_attn(x.c, b, q.to(DEV), 0.125, o, lse, workspace=ws)
    torch.cuda.synchronize()


def test_same_call_same_bits():
    """Split over the chip (one token, a long context) and not: every run gives the same bits."""
    for lens, news in (([6000], [1]), ([900] * 40, [9] * 40)):
        x = C.Batch(lens, news, 4, 2, 128, 64, True, seed=29).to_device()
        first = _run(x, True)
        for _ in range(3):
            again = _run(x, True)
            assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_without_lse():
    x = C.Batch([300], [3], 4, 2, 64, 64, False, seed=30).to_device()
    o = torch.empty(3, 4, 64, dtype=torch.bfloat16, device=DEV)
    S.spade_cache_attn(x.c, x.b, x.q.to(DEV), 0.125, o, workspace=x.workspace())
    torch.cuda.synchronize()
    assert torch.equal(o.cpu(), _run(x, True, scale=0.125)[0])
