"""CachePath on a stream that is not torch's current one: the tensors that a call makes for its
results belong to the call's stream, so work that is still queued elsewhere cannot reach
them."""
import pytest
import torch

from paper_2608_03335_amd.pipeline import CachePath

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _filled():
    p = CachePath(1, 4, 4, 64, n_pages=9, max_pages=8, max_tokens=200, page=32, device=DEV)
    gen = torch.Generator().manual_seed(1)
    x = [torch.randn(200, 4, 64, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(3)]
    p.plan([200])
    return p, x


def _busy():
    """Some 50 ms of work on the current stream."""
    a = torch.ones(8192, 8192, dtype=torch.bfloat16, device=DEV)
    b = torch.empty_like(a)
    for _ in range(50):
        torch.mm(a, a, out=b)


@pytest.mark.parametrize("handle", [False, True])
def test_read_on_another_stream(handle):
    p, x = _filled()
    p.run(*x)
    want = [t.clone() for t in p.read()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    _busy()
    got = p.read(stream=side.cuda_stream if handle else side)  # torch's own stream is still busy
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        assert torch.equal(g, w)


@pytest.mark.parametrize("handle", [False, True])
def test_run_on_another_stream(handle):
    p, x = _filled()
    want = p.run(*x).clone()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    _busy()
    old = torch.empty_like(want)
    old.fill_(float("nan"))   # queued behind the busy work; its memory is free for new tensors
    del old
    got = p.run(*x, stream=side.cuda_stream if handle else side)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_the_default_stream_by_its_handle():
    p, x = _filled()
    want = p.run(*x)
    got = p.run(*x, stream=torch.cuda.default_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(got, want)


def test_a_path_names_its_device():
    """Made on "cuda", a path stays on the device that was current then."""
    p, _ = _filled()
    assert p.device == p.k.device and p.device.index == torch.cuda.current_device()
