"""CachePath after a sequence was shortened or given up: what is read back, and which calls
wait for a plan."""
import pytest
import torch

from paper_2608_03335_amd.pipeline import CachePath

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _filled(fp4, lens=(100, 70)):
    p = CachePath(2, 2, 2, 64, n_pages=9, max_pages=4, max_tokens=200, page=32, fp4=fp4, device=DEV)
    gen = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(sum(lens), 2, 64, generator=gen).to(torch.bfloat16).to(DEV) for _ in range(3))
    p.plan(lens)
    p.run(q, k, v)
    return p, (q, k, v)


@pytest.mark.parametrize("fp4", [False, True])
def test_read_gives_zeros_behind_a_shortened_sequence(fp4):
    p, _ = _filled(fp4)
    before = [x.clone() for x in p.read(100)]
    p.rewind(0, 45)
    p.rewind(1, 64)
    for N in (None, 100):
        for got, old in zip(p.read(N), before):
            assert got.shape[2] == (64 if N is None else N)
            for b, L in enumerate((45, 64)):
                assert torch.equal(got[b, :, :L], old[b, :, :L])
                assert bool((got[b, :, L:] == 0).all()), (N, b)


@pytest.mark.parametrize("fp4", [False, True])
def test_read_gives_nothing_of_a_released_sequence(fp4):
    p, (q, k, v) = _filled(fp4)
    before = [x.clone() for x in p.read(100)]
    p.release(0)
    for got, old in zip(p.read(100), before):
        assert not bool(got[0].any()) and torch.equal(got[1], old[1])
    p.plan([0, 58])  # sequence 1 takes the pages that sequence 0 gave back
    p.run(q[:58], k[:58], v[:58])
    p.rewind(1, 70)
    for got, old in zip(p.read(100), before):
        assert not bool(got[0].any())
        assert torch.equal(got[1, :, :70], old[1, :, :70]) and not bool(got[1, :, 70:].any())


def test_run_waits_for_a_plan_of_the_new_lengths():
    p, (q, k, v) = _filled(False)
    for change in (lambda: p.rewind(0, 99), lambda: p.release(1)):
        change()
        with pytest.raises(ValueError, match="plan"):
            p.run(q, k, v)
        p.plan([1, 2])
        assert p.run(q[:3], k[:3], v[:3]).shape == (3, 2, 64)
