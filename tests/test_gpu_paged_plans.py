"""Plans of more than 512 sequences, several a thread, whose lengths are read again
once pages have gone back: with no new tokens, with slots that the plan's own launch
writes and with a launch for them, and refused."""
import numpy as np
import pytest
import torch

from tests.test_gpu_paged import Book

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("S", [513, 1024, 2048, 2049, 5000])
def test_decode_steps(S):
    """A token or two a sequence, or none, while some end, drop rows or come."""
    rng = np.random.default_rng(S)
    b = Book(S, 1, 1, 1, 64, 3 * S, 16, 6)
    for step in range(12):
        n_new = step % 3
        old = np.array(b.p.len)
        lens = np.minimum(old + rng.integers(0, n_new + 1, S), 96)
        some = rng.random(S)
        lens = np.where(some < 0.1, 0, lens)
        lens = np.where(some > 0.9, (old * rng.random(S)).astype(int), lens)
        b.plan(lens.tolist(), n_new)
        if step % 4 == 1:       # prompts
            lens = np.where(lens == 0, rng.integers(0, 40, S), lens)
            b.plan(lens.tolist(), 40)
    b.plan([0] * S)
    assert sorted(b.p.stack) == list(range(3 * S))


@pytest.mark.parametrize("S", [513, 1025, 2048])
@pytest.mark.parametrize("n_new", [1, 2, 8])
def test_refused(S, n_new):
    """Nothing changes, wherever in the batch the reason is."""
    b = Book(S, 1, 1, 1, 64, S + 1, 16, 2)
    b.plan([15] * S, 15)
    full = [15] * S
    for s in (0, 1, S // 2, S - 1):
        for n in (-1, 33, 15 + n_new + 1, 2**31 - 1):
            lens = [15 + (i % 5 == 0) for i in range(S)]
            lens[s] = n
            b.plan(lens, n_new)
        lens = list(full)
        lens[s] = 0             # three pages are asked for, two are free
        lens[(s + 7) % S] = lens[(s + 8) % S] = lens[(s + 9) % S] = 17
        if n_new > 1:
            b.plan(lens, n_new)
    assert b.p.len == full and b.p.stack == [S]
    b.plan([15 + (i % 5 == 0) for i in range(S)], n_new)
    b.plan(full)
