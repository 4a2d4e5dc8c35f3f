"""spade_cache_select against its definition: counts and page lists are equal."""
import pytest
import torch

from paper_2608_03335_amd import spade as S

from . import _cache as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _say(*a):
    print(*a, flush=True)


def _run(x, q, topk, sink, local, causal, junk=-5):
    counts = torch.full((x.n, x.H), junk, dtype=torch.int32, device=DEV)
    idx = torch.full((x.n, x.H, topk), junk, dtype=torch.int32, device=DEV)
    S.spade_cache_select(x.c, x.b, q.to(DEV), topk, counts, idx, causal=causal, sink=sink,
                         local=local, workspace=x.workspace(topk))
    torch.cuda.synchronize()
    counts, idx = counts.cpu().flatten(), idx.cpu().view(-1, topk)
    assert all(bool((idx[r, n:] == junk).all()) for r, n in enumerate(counts.tolist()))
    return [idx[r, :n].tolist() for r, n in enumerate(counts.tolist())]


CASES = [  # lens, news, Hq, H, d, P, topk, sink, local, causal
    ([1], [1], 1, 1, 64, 32, 1, 0, 1, True),
    ([5, 0, 700], [5, 0, 3], 4, 2, 128, 32, 4, 1, 1, True),
    ([5, 0, 700], [5, 0, 3], 4, 2, 128, 32, 4, 1, 1, False),
    ([3000], [1], 8, 8, 64, 32, 7, 0, 0, False),
    ([2049, 2048, 2047], [1, 1, 1], 14, 2, 128, 64, 9, 2, 3, True),
    ([900, 31], [40, 31], 6, 3, 64, 32, 6, 0, 2, True),
    ([9000], [2], 16, 1, 128, 32, 200, 1, 1, True),
    ([40000], [3], 5, 1, 64, 32, 33, 0, 2, True),
    ([1500], [9], 32, 1, 128, 96, 5, 1, 2, False),
    ([1200], [30], 3, 3, 128, 256, 64, 2, 2, True),
]


@pytest.mark.parametrize("fp4", [False, True])
@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}-{c[2]}x{c[3]}-d{c[4]}-P{c[5]}-k{c[6]}-c{int(c[9])}")
def test_select(case, fp4):
    lens, news, Hq, H, d, P, topk, sink, local, causal = case
    _say("select", case, fp4)
    x = C.Batch(lens, news, Hq, H, d, P, fp4, seed=11).to_device()
    got = _run(x, x.q, topk, sink, local, causal)
    assert got == x.ref_select(x.q, causal, topk, sink, local)


def test_ties_go_to_the_lowest_page():
    P, d, pages = 32, 64, 100
    x = C.Batch([P * pages], [2], 2, 1, d, P, False, seed=3)
    x.k[0][:] = x.k[0][:P].repeat(pages, 1, 1)          # every page alike
    x.k[0][P * 40:P * 41] += 1.0                         # but one
    x.q[1] = 0                                           # all scores 0, of either sign
    x.hold([P * pages])
    x.to_device()
    got = _run(x, x.q, 10, 0, 1, True)
    assert got == x.ref_select(x.q, True, 10, 0, 1)
    assert got[1] == list(range(9)) + [99]


def test_scores_that_differ_in_the_last_place():
    """Page scores that only fp64 tells apart: q . mean with differences of 2^-30 of the sum."""
    P, d, pages = 32, 128, 64
    x = C.Batch([P * pages], [1], 1, 1, d, P, False, seed=3)
    x.q[0, 0] = 1.0
    x.q[0, 0, 0] = 2.0 ** -20
    x.hold([P * pages])
    mean = torch.full((pages, 1, d), 1.0)
    mean[:, 0, 0] = torch.tensor([((37 * j) % 64) / 64.0 for j in range(pages)])  # times 2^-20
    for j in range(pages):
        x.buf["k_mean"][int(x.table[0, j])] = mean[j].to(torch.bfloat16)
    x.to_device()
    got = _run(x, x.q, 20, 0, 0, False)
    assert got == C.select(x.q, mean.to(torch.bfloat16), [P * pages], P, 20, 0, 0)


@pytest.mark.parametrize("topk,local", [(12, 1), (58, 2)])
def test_scores_that_are_not_finite(topk, local):
    """NaN scores rank last, infinities at the ends; forced pages stay whatever they score."""
    P, d, pages = 32, 64, 60
    x = C.Batch([P * pages], [1], 2, 1, d, P, False, seed=5)
    x.hold([P * pages])
    bad = {0: float("nan"), 3: float("inf"), 4: float("-inf"), 17: float("nan"), 58: float("inf"), 59: float("nan")}
    mean = torch.stack([x.buf["k_mean"][int(x.table[0, j])] for j in range(pages)])
    for j, val in bad.items():
        mean[j, 0, 5] = val
        x.buf["k_mean"][int(x.table[0, j])] = mean[j]
    x.q[0, :, 5] = 1.0
    x.to_device()
    want = C.select(x.q, mean, [P * pages], P, topk, 1, local)
    assert _run(x, x.q, topk, 1, local, False) == want
    x.q[0, :, 7] = float("nan")                          # every score NaN: index order
    want = C.select(x.q, mean, [P * pages], P, topk, 1, local)
    assert _run(x, x.q, topk, 1, local, False) == want
    assert want[0] == list(range(topk - local)) + list(range(pages - local, pages))


def test_rows_of_no_sequence_stay_and_bad_tables_cannot_fault():
    x = C.Batch([400, 300], [3, 2], 2, 2, 64, 32, False, seed=6)
    x.cu = torch.tensor([1, 4, 6], dtype=torch.int32)
    x.table[1, 3] = -9
    x.table[1, 5] = 2 ** 31 - 1
    x.to_device(n_tokens=9)
    gen = torch.Generator().manual_seed(1)
    q = torch.randn(9, 2, 64, generator=gen).to(torch.bfloat16)
    counts = torch.full((9, 2), -5, dtype=torch.int32, device=DEV)
    idx = torch.full((9, 2, 6), -5, dtype=torch.int32, device=DEV)
    ws = x.workspace(6)
    S.spade_cache_select(x.c, x.b, q.to(DEV), 6, counts, idx, workspace=ws)
    torch.cuda.synchronize()
    for rows in (slice(0, 1), slice(6, 9)):
        assert bool((counts[rows] == -5).all()) and bool((idx[rows] == -5).all())
    mean = C.page_means(x.k[0].double(), 32)
    want = C.select(q[1:4], mean, C.seen_by(400, 3, True), 32, 6, 0, 1)
    assert idx[1:4].cpu().view(-1, 6).tolist() == want
    for lens, cu in (([10 ** 9, -4], [0, 5, 9]), ([400, 300], [7, 2, -3]), ([0, 1], [0, 9, 9])):
        b = S.batch(x.table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV),
                    torch.tensor(cu, dtype=torch.int32, device=DEV), 9)
        S.spade_cache_select(x.c, b, q.to(DEV), 6, counts, idx, workspace=ws)
    torch.cuda.synchronize()


def test_the_longest_table():
    """16384 pages, the limit, and a topk of more than all of them."""
    P, d, L = 32, 64, 16384 * 32
    gen = torch.Generator().manual_seed(9)
    mean = torch.randn(16384, 1, d, generator=gen).to(torch.bfloat16)
    q = torch.randn(1, 2, d, generator=gen).to(torch.bfloat16)
    kv = torch.empty(16384, 1, P, d, dtype=torch.bfloat16, device=DEV)
    c = S.cache(S.SPADE_CACHE_BF16, 1, d, P, kv, kv, mean.to(DEV))
    table = torch.arange(16384, dtype=torch.int32, device=DEV)[None]
    b = S.batch(table, torch.tensor([L], dtype=torch.int32, device=DEV),
                torch.tensor([0, 1], dtype=torch.int32, device=DEV), 1)
    score = (mean[:, 0].double() * q[0].double().sum(0)).sum(-1)
    order = torch.sort(score, stable=True, descending=True)[1]
    for topk in (1, 100, 16383, 20000):
        counts = torch.zeros(1, 1, dtype=torch.int32, device=DEV)
        idx = torch.full((1, 1, topk), -1, dtype=torch.int32, device=DEV)
        ws = torch.empty(max(S.spade_cache_select_workspace_bytes(c, b, 2, topk), 16),
                         dtype=torch.uint8, device=DEV)
        S.spade_cache_select(c, b, q.to(DEV), topk, counts, idx, causal=False, local=0, workspace=ws)
        n = min(topk, 16384)
        assert int(counts) == n
        assert torch.equal(idx[0, 0, :n].cpu().long(), torch.sort(order[:n])[0])


@pytest.mark.parametrize("size", [1e-38, 1e-30, 1e30, 2e37])
def test_very_small_and_very_large_scores(size):
    """Sizes at which fp32 scores underflow or overflow: fp64 still ranks."""
    P, d, pages = 32, 64, 80
    x = C.Batch([P * pages], [2], 4, 2, d, P, False, seed=6)
    x.q = (x.q.double() * size).to(torch.bfloat16)
    x.hold([P * pages])
    x.to_device()
    assert _run(x, x.q, 20, 1, 2, True) == x.ref_select(x.q, True, 20, 1, 2)


@pytest.mark.parametrize("pages", [255, 257, 1023, 1025, 4095, 4097])
def test_page_counts_at_the_edges_of_the_row_kernels(pages):
    """One wave, four and sixteen a row; few rows and many; more kept than 64 pages in doubt."""
    P, d = 32, 64
    gen = torch.Generator().manual_seed(pages)
    mean = torch.randn(pages, 2, d, generator=gen).to(torch.bfloat16)
    mean[10:100] = mean[10]                       # ninety pages alike
    kv = torch.empty(pages, 2, P, d, dtype=torch.bfloat16, device=DEV)
    c = S.cache(S.SPADE_CACHE_BF16, 2, d, P, kv, kv, mean.to(DEV))
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None]
    for n in (3, 1100):
        q = torch.randn(n, 2, d, generator=gen).to(torch.bfloat16)
        q[0, 0] = mean[10, 0]                     # the alike pages lead this row
        b = S.batch(table, torch.tensor([P * pages - 5], dtype=torch.int32, device=DEV),
                    torch.tensor([0, n], dtype=torch.int32, device=DEV), n)
        for topk in (40, 150):
            counts = torch.zeros(n, 2, dtype=torch.int32, device=DEV)
            idx = torch.full((n, 2, topk), -1, dtype=torch.int32, device=DEV)
            ws = torch.empty(S.spade_cache_select_workspace_bytes(c, b, 2, topk), dtype=torch.uint8, device=DEV)
            S.spade_cache_select(c, b, q.to(DEV), topk, counts, idx, causal=False, local=1, workspace=ws)
            score = torch.einsum("nhc,jhc->nhj", q.double(), mean.double())
            score[..., pages - 1] = float("inf")
            order = torch.sort(score, dim=-1, stable=True, descending=True)[1][..., :topk]
            assert bool((counts == min(topk, pages)).all())
            assert torch.equal(idx[..., :min(topk, pages)].cpu().long(), torch.sort(order, -1)[0]), (n, topk)
