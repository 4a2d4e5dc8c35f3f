"""spade_cache_append and spade_cache_read against their definitions: every stored bit, the
rotated queries, the page means, and the bytes that must stay as they were. Rotation,
rounding, the 4-bit codes and the means have one right answer, so nothing here has a tolerance."""
import pytest
import torch

from paper_2608_03335_amd import spade as S

from . import _cache as C

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _say(*a):
    print(*a, flush=True)


def _tables(n_pos, rot, seed=3):
    gen = torch.Generator().manual_seed(seed)
    a = torch.rand(n_pos, rot // 2, generator=gen, dtype=torch.float64) * 1e4
    return a.cos().float(), a.sin().float()


def _check(x, keys, what=""):
    """The device cache holds keys (bf16 token tensors) and x.v, and their pages' means."""
    P, d = x.P, x.d
    got = {s: C.unpack(x.g[s].cpu(), None if not x.fp4 else x.g[s + "_scale"].cpu(), P, d, x.fp4, s)
           for s in ("k", "v")}
    mean = x.g["k_mean"].cpu()
    for b, L in enumerate(x.lens):
        want_mean = C.page_means(C.stored(keys[b][:L], x.fp4), P)
        for j in range(-(-L // P)):
            page = int(x.table[b, j])
            n = min(P, L - j * P)
            for s, y in (("k", keys[b]), ("v", x.v[b])):
                want = C.stored(y[j * P:j * P + n], x.fp4).transpose(0, 1)
                assert torch.equal(torch.nan_to_num(got[s][page, :, :n], nan=123.0),
                                   torch.nan_to_num(want, nan=123.0)), (what, s, b, j)
            assert torch.equal(torch.nan_to_num(mean[page].float(), nan=123.0),
                               torch.nan_to_num(want_mean[j].float(), nan=123.0)), (what, "mean", b, j)


CASES = [  # lens, news, Hq, H, d, P, fp4, rot, interleaved
    ([1], [1], 1, 1, 64, 32, False, 64, False),
    ([1], [1], 4, 2, 128, 64, True, 128, True),
    ([31, 32, 33, 64, 65], [1, 1, 1, 1, 1], 8, 2, 128, 32, False, 128, False),
    ([31, 32, 33, 64, 65], [2, 32, 33, 1, 34], 6, 3, 64, 32, True, 32, False),
    ([200, 0, 77], [150, 0, 77], 5, 5, 128, 96, False, 96, True),
    ([300, 129, 5], [299, 1, 0], 16, 2, 64, 128, True, 64, True),
    ([513], [513], 3, 1, 128, 256, False, 16, True),
    ([257, 700], [257, 411], 4, 4, 128, 256, True, 0, False),
    ([160, 161, 159], [3, 3, 160 - 1], 2, 2, 64, 160, False, 48, False),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{c[0]}-{c[1]}-d{c[4]}-P{c[5]}-{'fp4' if c[6] else 'bf16'}")
@pytest.mark.parametrize("strided", [False, True])
def test_append(case, strided):
    lens, news, Hq, H, d, P, fp4, rot, inter = case
    _say("append", case, strided)
    x = C.Batch(lens, news, Hq, H, d, P, fp4, seed=1, held=[L - n for L, n in zip(lens, news)])
    before = {s: None if t is None else t.clone() for s, t in x.buf.items()}
    x.to_device()
    cos, sin = _tables(max(lens) + 1, rot) if rot else (None, None)
    k_new, v_new = x.new(x.k), x.new(x.v)
    if strided:  # slices of one fused projection
        fused = torch.cat([x.q.flatten(1), k_new.flatten(1), v_new.flatten(1)], 1).to(DEV)
        q = fused[:, :Hq * d].view(-1, Hq, d)
        k = fused[:, Hq * d:(Hq + H) * d].view(-1, H, d)
        v = fused[:, (Hq + H) * d:].view(-1, H, d)
    else:
        q, k, v = x.q.to(DEV), k_new.to(DEV), v_new.to(DEV)
    q_out = torch.full((x.n, Hq, d), 7.0, dtype=torch.bfloat16, device=DEV)
    rope = S.rope(cos.to(DEV), sin.to(DEV), interleaved=inter) if rot else None
    S.spade_cache_append(x.c, x.b, k, v, q, q_out, rope)
    torch.cuda.synchronize()
    keys, want_q = [], []
    for b, t0, n in x.rows():
        L = lens[b]
        if rot and n:
            turn = (cos[L - n:L], sin[L - n:L], inter)
            keys.append(torch.cat([x.k[b][:L - n], C.rotate(x.k[b][L - n:], *turn)]))
            want_q.append(C.rotate(x.q[t0:t0 + n], *turn))
        else:
            keys.append(x.k[b])
            want_q.append(x.q[t0:t0 + n])
    assert torch.equal(q_out.cpu().view(torch.int16), torch.cat(want_q).view(torch.int16))
    _check(x, keys)
    # pages of no sequence, and places behind a sequence, keep their bytes
    used = set(x.table[x.table >= 0].tolist())
    for s, t in before.items():
        if t is not None:
            for page in range(x.n_pages):
                if page not in used:
                    assert torch.equal(x.g[s][page].cpu(), t[page])


@pytest.mark.parametrize("fp4", [False, True])
def test_one_by_one_chunks_and_rewritten_tokens_agree(fp4):
    L, P, d, H = 150, 64, 128, 2
    _say("append in pieces", fp4)
    whole = C.Batch([L], [L], 2, H, d, P, fp4, seed=5, held=[0])
    whole.to_device()
    k, v = whole.k[0].to(DEV), whole.v[0].to(DEV)
    S.spade_cache_append(whole.c, whole.b, k, v)
    for pieces in ([1] * L, [7] * 21 + [3], [100, -60, 70, 40]):
        x = C.Batch([L], [L], 2, H, d, P, fp4, seed=5, held=[0])
        x.to_device()
        at = 0
        for n in pieces:
            if n < 0:  # the last tokens are taken back; garbage was written meanwhile
                at += n
                continue
            cu = torch.tensor([0, n], dtype=torch.int32, device=DEV)
            lens = torch.tensor([at + n], dtype=torch.int32, device=DEV)
            b = S.batch(x.table.to(DEV), lens, cu, n)
            S.spade_cache_append(x.c, b, k[at:at + n], v[at:at + n])
            at += n
        torch.cuda.synchronize()
        assert at == L
        for s in ("k", "v", "k_mean", "k_scale", "v_scale"):
            if x.g[s] is not None:
                assert torch.equal(x.g[s].cpu().view(torch.uint8), whole.g[s].cpu().view(torch.uint8)), (s, pieces[:3])


@pytest.mark.parametrize("fp4", [False, True])
def test_partial_writes_keep_the_neighbours(fp4):
    """New tokens in the middle of a page: bytes of later slots (garbage of the pool) stay."""
    x = C.Batch([45], [6], 1, 2, 64, 64, fp4, seed=2, held=[39], fill=3.0)
    x.to_device()
    old = {s: x.g[s].clone() for s in ("k", "v")}
    S.spade_cache_append(x.c, x.b, x.new(x.k).to(DEV), x.new(x.v).to(DEV))
    torch.cuda.synchronize()
    page = int(x.table[0, 0])
    for s, place in (("k", C.k_place), ("v", C.v_place)):
        at = place(64, 64, fp4)[45:].flatten()
        a, b = x.g[s][page].cpu().view(2, -1), old[s][page].cpu().view(2, -1)
        if fp4:
            a, b = C._nibbles(a), C._nibbles(b)
        assert torch.equal(a[:, at], b[:, at])
    _check(x, x.k)


def test_given_positions_and_positions_outside_the_tables():
    rot, d = 64, 64
    x = C.Batch([40, 8], [5, 8], 4, 2, d, 32, False, seed=4, held=[35, 0]).to_device()
    cos, sin = _tables(20, rot)
    pos = torch.tensor([0, 19, 20, -1, 7, 3, 3, 2 ** 31 - 1, -2 ** 31, 0, 1, 18, 19], dtype=torch.int32)
    q_out = torch.empty(13, 4, d, dtype=torch.bfloat16, device=DEV)
    S.spade_cache_append(x.c, x.b, x.new(x.k).to(DEV), x.new(x.v).to(DEV), x.q.to(DEV), q_out,
                         S.rope(cos.to(DEV), sin.to(DEV), pos.to(DEV)))
    torch.cuda.synchronize()
    ok = (pos >= 0) & (pos < 20)
    row = torch.where(ok, pos, 0).long()
    turn = lambda t: torch.where(ok[:, None, None], C.rotate(t, cos[row], sin[row], False), t)  # noqa: E731
    assert torch.equal(q_out.cpu().view(torch.int16), turn(x.q).view(torch.int16))
    new = turn(x.new(x.k))
    _check(x, [torch.cat([x.k[0][:35], new[:5]]), new[5:]])


def test_values_at_the_ends_of_four_bits():
    """Ties, the 7 * 2^e border, zeros, subnormals, the largest bf16, infinities and NaN."""
    d, H = 64, 1
    rows = torch.zeros(12, d)
    rows[0, :9] = torch.tensor([7.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0])
    rows[1, :9] = torch.tensor([7.0625, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, -5.0])
    rows[2, :4] = torch.tensor([2.0 ** -130, 2.0 ** -127, -2.0 ** -126, 2.0 ** -133])
    rows[3, 0] = 3.3895313892515355e38
    rows[3, 1:4] = torch.tensor([3e38, -2.9e38, 1e38])
    rows[4, 3], rows[4, 40] = float("inf"), 1.0
    rows[5, 33], rows[5, 2] = float("nan"), 2.0
    rows[6, 5] = float("-inf")
    rows[7] = torch.linspace(-8, 8, d)
    rows[8] = torch.linspace(0, 1e-3, d)
    rows[9, 10] = -0.0
    rows[10] = 1.0
    rows[11] = -6.0
    tok = rows.to(torch.bfloat16)[:, None]
    x = C.Batch([12], [12], 1, H, d, 32, True, held=[0])
    x.k[0] = x.v[0] = tok
    x.to_device()
    S.spade_cache_append(x.c, x.b, tok.to(DEV), tok.to(DEV))
    k = torch.zeros(1, H, 12, d, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    S.spade_cache_read(x.c, x.b, k, v)
    torch.cuda.synchronize()
    _check(x, x.k)
    want = torch.nan_to_num(C.stored(tok, True)[:, 0], nan=123.0)
    for got in (k, v):
        assert torch.equal(torch.nan_to_num(got[0, 0].cpu().double(), nan=123.0), want)


def test_rows_of_no_sequence_and_bad_pages_stay():
    """Rows before cu[0] and behind cu[B], and tokens whose page is outside the pool."""
    x = C.Batch([70, 40], [4, 3], 2, 2, 64, 32, False, seed=6, held=[66, 37])
    x.cu = torch.tensor([2, 6, 9], dtype=torch.int32)
    x.table[1, 1] = x.n_pages + 5
    x.to_device(n_tokens=12)
    old = {s: x.g[s].clone() for s in ("k", "v", "k_mean")}
    gen = torch.Generator().manual_seed(1)
    t = lambda h: torch.randn(12, h, 64, generator=gen).to(torch.bfloat16).to(DEV)  # noqa: E731
    k, v, q = t(2), t(2), t(2)
    q_out = torch.full((12, 2, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    S.spade_cache_append(x.c, x.b, k, v, q, q_out)
    torch.cuda.synchronize()
    assert torch.equal(q_out[2:9], q[2:9])
    assert bool((q_out[:2] == 7).all()) and bool((q_out[9:] == 7).all())
    x.k[0][66:], x.v[0][66:] = k[2:6].cpu(), v[2:6].cpu()
    x.lens = [70, 32]  # tokens 37..39 went nowhere: page 1 of sequence 1 is outside
    for s in ("k", "v"):
        page = int(x.table[1, 0])
        assert torch.equal(x.g[s][page], old[s][page])
    x.lens, x.table = [70], x.table[:1]
    _check(x, x.k)


def test_offsets_beyond_a_batch_cannot_lead_outside():
    """Lengths above the table, below the new tokens, and offsets that do not ascend: no
    fault, and sequences that keep the rules are served."""
    x = C.Batch([64, 64, 64], [2, 2, 2], 1, 1, 64, 32, False, seed=7, held=[62, 62, 62])
    x.to_device()
    lens = torch.tensor([64, 1, 10 ** 9], dtype=torch.int32, device=DEV)
    b = S.batch(x.table.to(DEV), lens, x.cu.to(DEV), 6)
    S.spade_cache_append(x.c, b, x.new(x.k).to(DEV), x.new(x.v).to(DEV))
    torch.cuda.synchronize()
    x.lens, x.table, keep = [64], x.table[:1], x.table
    _check(x, x.k)
    for cu in ([0, 4, 2, 6], [5, 3, -9, 100], [-2 ** 31, 2 ** 31 - 1, 0, 6]):
        b = S.batch(keep.to(DEV), lens, torch.tensor(cu, dtype=torch.int32, device=DEV), 6)
        q = torch.zeros(6, 1, 64, dtype=torch.bfloat16, device=DEV)
        S.spade_cache_append(x.c, b, x.new(x.k).to(DEV)[:2].repeat(3, 1, 1),
                             x.new(x.v).to(DEV)[:2].repeat(3, 1, 1), q, torch.empty_like(q))
    torch.cuda.synchronize()


@pytest.mark.parametrize("d,P,fp4", [(64, 32, False), (128, 96, True), (128, 256, False), (64, 160, True)])
def test_read(d, P, fp4):
    lens = [0, 1, P - 1, P, P + 1, 3 * P + 17]
    _say("read", d, P, fp4)
    x = C.Batch(lens, [0] * 6, 1, 3, d, P, fp4, seed=8, fill=float("nan")).to_device()
    N = 3 * P + 5  # shorter than the longest sequence
    k = torch.full((6, 3, N, d), 9.0, dtype=torch.bfloat16, device=DEV)
    v = torch.full_like(k, 9.0)
    S.spade_cache_read(x.c, x.b, k, v)
    torch.cuda.synchronize()
    for b, L in enumerate(lens):
        n = min(L, N)
        for got, toks in ((k, x.k), (v, x.v)):
            want = C.stored(toks[b][:n], fp4).transpose(0, 1)
            assert torch.equal(got[b, :, :n].cpu().double(), want)
            assert bool((got[b, :, n:] == 9).all())


def test_offsets_past_32_bits():
    """A pool of more than 2^31 elements a side: the last pages are written and read."""
    n_pages, P, d = 70000, 256, 128
    k = torch.empty(n_pages, 1, P, d, dtype=torch.bfloat16, device=DEV)
    v = torch.empty_like(k)
    assert k.numel() > 2 ** 31
    mean = torch.empty(n_pages, 1, d, dtype=torch.bfloat16, device=DEV)
    c = S.cache(S.SPADE_CACHE_BF16, 1, d, P, k, v, mean)
    table = torch.tensor([[n_pages - 1, n_pages - 3]], dtype=torch.int32, device=DEV)
    L = 300
    b = S.batch(table, torch.tensor([L], dtype=torch.int32, device=DEV),
                torch.tensor([0, L], dtype=torch.int32, device=DEV), L)
    gen = torch.Generator().manual_seed(0)
    tk, tv, q = (torch.randn(L, 1, d, generator=gen).to(torch.bfloat16) for _ in range(3))
    S.spade_cache_append(c, b, tk.to(DEV), tv.to(DEV))
    rk = torch.zeros(1, 1, L, d, dtype=torch.bfloat16, device=DEV)
    rv = torch.zeros_like(rk)
    S.spade_cache_read(c, b, rk, rv)
    o = torch.empty(L, 1, d, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(max(S.spade_cache_attn_workspace_bytes(c, b, 1), 16), dtype=torch.uint8, device=DEV)
    S.spade_cache_attn(c, b, q.to(DEV), 0.1, o, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(rk[0, 0].cpu(), tk[:, 0]) and torch.equal(rv[0, 0].cpu(), tv[:, 0])
    want, _, tol, _ = C.attend(q, tk.double(), tv.double(), C.seen_by(L, L, True), None, P, 0.1)
    assert bool(((o.cpu().double() - want).abs() <= tol).all())
