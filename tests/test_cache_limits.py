"""Sizes at which a cache call is refused for its number of workgroups (2^31 and more): told on
the host, before any launch."""
import ctypes

import pytest

from paper_2608_03335_amd import spade as S

FAKE = 0x1000  # aligned, never dereferenced


def _structs(B, max_pages, n_tokens, H=8, page=64):
    return (S.spade_cache(S.SPADE_CACHE_BF16, H, 128, page, 10, FAKE, FAKE, FAKE, None, None),
            S.spade_batch(B, max_pages, n_tokens, FAKE, FAKE, FAKE))


def _refused(status, word):
    return status == S.SPADE_ERR_UNSUPPORTED and word in S.lib().spade_last_error()


@pytest.mark.parametrize("B,max_pages,N", [(1 << 16, 1 << 15, 1), (1 << 10, 1 << 20, 1 << 31),
                                           (1 << 20, 1 << 7, 1 << 13)])
def test_read(B, max_pages, N):
    c, b = _structs(B, max_pages, 0)
    assert _refused(S.lib().spade_cache_read(ctypes.byref(c), ctypes.byref(b), N, FAKE, 0x2000, None),
                    b"batch too large")


def test_append():
    c, b = _structs(1, 1 << 22, 1 << 28, H=4096)
    st = 4096 * 128
    assert _refused(S.lib().spade_cache_append(ctypes.byref(c), ctypes.byref(b), FAKE, st, FAKE, st, None, 0,
                                               0, None, None, None), b"batch too large")


def test_attention():
    c, b = _structs(1, 1 << 22, 1 << 28, H=4096)
    assert _refused(S.lib().spade_cache_attn(ctypes.byref(c), ctypes.byref(b), FAKE, 4096, None, None, 0, 1,
                                             0.1, 0x2000, None, FAKE, 1 << 50, None), b"batch too large")


def test_selection():
    c, b = _structs(1 << 20, 8, 1, H=4096)
    assert _refused(S.lib().spade_cache_select(ctypes.byref(c), ctypes.byref(b), FAKE, 4096, 4, 0, 1, 1, FAKE,
                                               FAKE, FAKE, 1 << 50, None), b"batch too large")
