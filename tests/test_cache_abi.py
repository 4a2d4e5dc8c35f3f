"""Refusals of the paged-cache calls, through the C ABI and the binding: all come before
any launch, so these run without a GPU."""
import ctypes

import pytest
import torch

from paper_2608_03335_amd import spade as S

NULL = None
FAKE = 0x1000       # aligned, never dereferenced
MISALIGNED = 0x1008
INV, UNS, WS, OK = (S.SPADE_ERR_INVALID_ARG, S.SPADE_ERR_UNSUPPORTED, S.SPADE_ERR_WORKSPACE,
                    S.SPADE_OK)


def _cache(**kw):
    f = dict(format=0, H=2, d=128, page=64, n_pages=10, k=FAKE, v=FAKE, k_mean=FAKE, k_scale=FAKE,
             v_scale=FAKE)
    f.update(kw)
    return S.spade_cache(*[f[k] for k, _ in S.spade_cache._fields_])


def _batch(**kw):
    f = dict(B=2, max_pages=5, n_tokens=4, table=FAKE, lens=FAKE, cu=FAKE)
    f.update(kw)
    return S.spade_batch(*[f[k] for k, _ in S.spade_batch._fields_])


def _rope(**kw):
    f = dict(n_pos=100, rot=128, interleaved=0, cos=FAKE, sin=FAKE, pos=NULL)
    f.update(kw)
    return S.spade_rope(*[f[k] for k, _ in S.spade_rope._fields_])


def _append(c=None, b=None, k=FAKE, ks=256, v=FAKE, vs=256, q=FAKE, qs=1024, Hq=8, out=0x2000,
            rope=None):
    r = lambda x: None if x is None else ctypes.byref(x)  # noqa: E731
    return S.lib().spade_cache_append(r(c or _cache()), r(b or _batch()), k, ks, v, vs, q, qs, Hq,
                                      out, r(rope), None)


def _select(c=None, b=None, q=FAKE, Hq=8, topk=4, sink=1, local=1, causal=1, counts=FAKE,
            indices=FAKE, ws=FAKE, n=1 << 40):
    return S.lib().spade_cache_select(ctypes.byref(c or _cache()), ctypes.byref(b or _batch()), q,
                                      Hq, topk, sink, local, causal, counts, indices, ws, n, None)


def _attn(c=None, b=None, q=FAKE, Hq=8, counts=FAKE, indices=FAKE, topk=4, causal=1, scale=0.1,
          o=0x2000, lse=NULL, ws=FAKE, n=1 << 40):
    return S.lib().spade_cache_attn(ctypes.byref(c or _cache()), ctypes.byref(b or _batch()), q, Hq,
                                    counts, indices, topk, causal, scale, o, lse, ws, n, None)


def _read(c=None, b=None, N=100, k=FAKE, v=0x2000):
    return S.lib().spade_cache_read(ctypes.byref(c or _cache()), ctypes.byref(b or _batch()), N, k,
                                    v, None)


ALL = (_append, _select, _attn, _read)


@pytest.mark.parametrize("kw,expect", [
    (dict(format=2), INV), (dict(format=-1), INV), (dict(H=0), INV), (dict(n_pages=0), INV),
    (dict(d=96), UNS), (dict(page=16), UNS), (dict(page=48), UNS), (dict(page=288), UNS),
    (dict(H=4097), UNS), (dict(n_pages=1 << 26), UNS)])
def test_cache_sizes(kw, expect):
    for call in ALL:
        assert call(c=_cache(**kw)) == expect
        assert S.lib().spade_last_error()


@pytest.mark.parametrize("kw,expect", [
    (dict(B=-1), INV), (dict(n_tokens=-1), INV), (dict(max_pages=0), INV),
    (dict(B=(1 << 20) + 1), UNS), (dict(n_tokens=(1 << 28) + 1), UNS),
    (dict(max_pages=(1 << 23) + 1), UNS)])
def test_batch_sizes(kw, expect):
    for call in ALL:
        assert call(b=_batch(**kw)) == expect


def test_null_structs():
    L = S.lib()
    c, b = ctypes.byref(_cache()), ctypes.byref(_batch())
    assert L.spade_cache_append(None, b, FAKE, 256, FAKE, 256, None, 0, 0, None, None, None) == INV
    assert L.spade_cache_append(c, None, FAKE, 256, FAKE, 256, None, 0, 0, None, None, None) == INV
    assert L.spade_cache_read(None, b, 1, FAKE, 0x2000, None) == INV
    assert L.spade_cache_select(c, None, FAKE, 8, 4, 0, 1, 1, FAKE, FAKE, None, 0, None) == INV
    assert L.spade_cache_attn(None, b, FAKE, 8, None, None, 0, 1, 0.1, FAKE, None, None, 0, None) == INV
    assert L.spade_cache_attn_workspace_bytes(None, b, 8, 0) == 0
    assert L.spade_cache_select_workspace_bytes(c, None, 8, 4) == 0


@pytest.mark.parametrize("kw,expect", [
    (dict(q=NULL), INV), (dict(out=NULL), INV), (dict(q=NULL, out=NULL), INV),   # Hq without q
    (dict(Hq=7), INV), (dict(Hq=0), INV), (dict(Hq=2 * 129, qs=1 << 20), UNS),
    (dict(k=NULL), INV), (dict(v=NULL), INV), (dict(k=MISALIGNED), INV), (dict(q=MISALIGNED), INV),
    (dict(ks=248), INV), (dict(vs=257), INV), (dict(qs=1016), INV), (dict(ks=1 << 33), UNS),
    (dict(out=FAKE, qs=2048), INV),
    (dict(rope=_rope(rot=8)), INV), (dict(rope=_rope(rot=144)), INV), (dict(rope=_rope(rot=-16)), INV),
    (dict(rope=_rope(n_pos=-1)), INV), (dict(rope=_rope(interleaved=2)), INV),
    (dict(rope=_rope(cos=NULL)), INV), (dict(rope=_rope(sin=MISALIGNED)), INV),
    (dict(c=_cache(k=NULL)), INV), (dict(c=_cache(k_mean=NULL)), INV),
    (dict(c=_cache(format=1, v_scale=NULL)), INV), (dict(c=_cache(v=MISALIGNED)), INV),
    (dict(b=_batch(table=NULL)), INV), (dict(b=_batch(lens=NULL)), INV), (dict(b=_batch(cu=NULL)), INV)])
def test_append_refusals(kw, expect):
    assert _append(**kw) == expect, S.lib().spade_last_error()


@pytest.mark.parametrize("kw,expect", [
    (dict(topk=0), INV), (dict(sink=-1), INV), (dict(local=-1), INV), (dict(sink=3, local=2), INV),
    (dict(local=0), INV), (dict(causal=2), INV), (dict(Hq=9), INV), (dict(Hq=258), UNS),
    (dict(b=_batch(max_pages=16385)), UNS), (dict(q=NULL), INV), (dict(q=MISALIGNED), INV),
    (dict(counts=NULL), INV), (dict(indices=NULL), INV), (dict(c=_cache(k_mean=NULL)), INV),
    (dict(sink=1 << 30, local=1 << 30, topk=1 << 30), INV)])
def test_select_refusals(kw, expect):
    assert _select(**kw) == expect


@pytest.mark.parametrize("kw,expect", [
    (dict(counts=NULL), INV), (dict(indices=NULL), INV), (dict(topk=0), INV), (dict(topk=-1), INV),
    (dict(counts=NULL, indices=NULL), INV), (dict(causal=-1), INV), (dict(scale=0.0), INV),
    (dict(scale=float("nan")), INV), (dict(scale=float("inf")), INV), (dict(scale=-1.0), INV),
    (dict(scale=1e39), INV), (dict(Hq=9), INV), (dict(b=_batch(max_pages=16385)), UNS),
    (dict(b=_batch(max_pages=1 << 23), c=_cache(page=256), counts=NULL, indices=NULL, topk=0), UNS),
    (dict(q=NULL), INV), (dict(o=NULL), INV), (dict(o=MISALIGNED), INV), (dict(o=FAKE), INV),
    (dict(c=_cache(v=NULL)), INV), (dict(c=_cache(format=1, k_scale=NULL)), INV)])
def test_attn_refusals(kw, expect):
    assert _attn(**kw) == expect


@pytest.mark.parametrize("kw,expect", [
    (dict(N=-1), INV), (dict(k=NULL), INV), (dict(v=FAKE), INV), (dict(v=MISALIGNED), INV),
    (dict(c=_cache(k=NULL)), INV), (dict(b=_batch(lens=NULL)), INV),
    (dict(b=_batch(B=1 << 20, max_pages=1 << 20)), UNS)])
def test_read_refusals(kw, expect):
    assert _read(**kw) == expect


def test_workspace_is_asked_for():
    L = S.lib()
    c, b = _cache(), _batch(n_tokens=2, max_pages=2000)
    need = L.spade_cache_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(b), 8, 0)
    assert need > 0   # two tokens over long contexts: split over the chip
    kw = dict(c=c, b=b, counts=NULL, indices=NULL, topk=0)
    assert _attn(**kw, n=need - 1) == WS
    assert _attn(**kw, n=need, ws=NULL) == WS
    assert _attn(**kw, n=need, ws=MISALIGNED) == WS


def test_empty_problems_launch_nothing():
    for b in (_batch(B=0, table=NULL, lens=NULL, cu=NULL), _batch(n_tokens=0, table=NULL, lens=NULL, cu=NULL)):
        c = _cache(k=NULL, v=NULL, k_mean=NULL)
        assert _append(c=c, b=b, k=NULL, v=NULL) == OK
        assert _select(c=c, b=b, q=NULL, counts=NULL, indices=NULL, ws=NULL, n=0) == OK
        assert _attn(c=c, b=b, q=NULL, o=NULL, counts=NULL, indices=NULL, topk=0, ws=NULL, n=0) == OK
        assert S.lib().spade_cache_attn_workspace_bytes(ctypes.byref(c), ctypes.byref(b), 8, 0) == 0
    assert _read(b=_batch(B=0, table=NULL, lens=NULL), k=NULL, v=NULL) == OK
    assert _read(N=0, k=NULL, v=NULL) == OK


# ------------------------------------------------------------------ the binding's own checks

def _raises(match, fn, *a, **kw):
    with pytest.raises(S.SpadeError, match=match) as e:
        fn(*a, **kw)
    assert e.value.status == INV


def test_binding_builders():
    k = torch.zeros(3, 2, 64, 128, dtype=torch.bfloat16)
    _raises("unknown cache format", S.cache, 5, 2, 128, 64, k, k)
    _raises("v must be torch.bfloat16", S.cache, 0, 2, 128, 64, k, k.float())
    _raises("v holds", S.cache, 0, 2, 128, 64, k, k[:2])
    _raises("k_mean holds", S.cache, 0, 2, 128, 64, k, k, k[0, 0, :5])
    _raises("k must be torch.uint8", S.cache, 1, 2, 128, 64, k, k, None, k, k)
    _raises("needs k_scale", S.cache, 1, 2, 128, 64, k, k)
    u = torch.zeros(3, 2, 64, 64, dtype=torch.uint8)
    _raises("v_scale holds", S.cache, 1, 2, 128, 64, u, u, None, u, u[:1, :1, :, :2].contiguous())
    _raises("GPU tensor", S.cache, 0, 2, 128, 64, k, k)
    t = torch.zeros(2, 4, dtype=torch.int32)
    _raises("table must be a", S.batch, t[0], t[0], t[0], 1)
    _raises("lens must be torch.int32", S.batch, t, t[:, 0].long(), t[0], 1)
    _raises("cu holds", S.batch, t, t[0], t[0, :2].contiguous(), 1)
    _raises("table must be contiguous", S.batch, t.t(), t[0], t[0], 1)
    _raises("GPU tensor", S.batch, t, t[0], t[0], 1)
    f = torch.zeros(10, 32)
    _raises("sin holds", S.rope, f, f[:9])
    _raises("pos must be torch.int32", S.rope, f, f, torch.zeros(4))
    _raises("cos must be a", S.rope, f[0], f)


def _structs():
    c = S.spade_cache(0, 2, 128, 64, 10, FAKE, FAKE, FAKE, None, None)
    b = S.spade_batch(2, 5, 4, FAKE, FAKE, FAKE)
    c.device = b.device = torch.device("cpu")
    return c, b


def test_binding_calls():
    c, b = _structs()
    kv = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    q = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    _raises("must come from", S.spade_cache_append, None, b, kv, kv)
    _raises("k must be torch.bfloat16", S.spade_cache_append, c, b, kv.float(), kv)
    _raises(r"v must be \[4, 2, 128\]", S.spade_cache_append, c, b, kv, kv[:3])
    _raises("heads must be contiguous", S.spade_cache_append, c, b, kv.transpose(1, 2).contiguous().transpose(1, 2), kv)
    _raises("come together", S.spade_cache_append, c, b, kv, kv, q)
    _raises("q_out must be contiguous", S.spade_cache_append, c, b, kv, kv, q,
            torch.zeros(4, 128, 8, dtype=torch.bfloat16).transpose(1, 2))
    _raises("rope must come from", S.spade_cache_append, c, b, kv, kv, q, q, 3)
    _raises("GPU tensor", S.spade_cache_append, c, b, kv, kv)
    i32 = torch.zeros(8, dtype=torch.int32)
    _raises("q must be", S.spade_cache_select, c, b, q[:3], 2, i32, i32)
    _raises("indices holds", S.spade_cache_select, c, b, q, 2, i32, i32)
    _raises("come together", S.spade_cache_attn, c, b, q, 0.1, q, None, i32)
    _raises("indices must be", S.spade_cache_attn, c, b, q, 0.1, q, None, i32, i32)
    _raises("lse holds", S.spade_cache_attn, c, b, q, 0.1, q, torch.zeros(31))
    _raises("GPU tensor", S.spade_cache_attn, c, b, q, 0.1, q)
    out = torch.zeros(2, 2, 9, 128, dtype=torch.bfloat16)
    _raises("k must be", S.spade_cache_read, c, b, out[:1], out)
    _raises("v holds", S.spade_cache_read, c, b, out, out[:1])
    m = torch.zeros(4, 8, 128, dtype=torch.bfloat16, device="meta")
    _raises("other arguments on", S.spade_cache_attn, c, b, m, 0.1, q)
