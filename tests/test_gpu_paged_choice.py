"""The choice of pages where more pages than a CTA has threads fall into one of the
256 parts of the scores' range, so that the budget's end is found digit by digit:
equal pages beside others, and pages that stretch the range.  Every launch form:
a cluster a unit (few units, tables of up to 2,048 pages), two launches with 256
threads a unit, and with 1,024 (few units of longer tables)."""
import numpy as np
import pytest
import torch

from oracle import paged
from paper_2608_15797_gb300 import kvr
from tests.test_gpu_paged import Book, dev, rnd

pytestmark = pytest.mark.gpu

P, D = 16, 64


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


def book(pages, many, dtype):
    """One unit of so many pages; with `many`, 24 units, six of them long: 152 SMs
    have no room for as many clusters of eight."""
    S, L = (4, 6) if many else (1, 1)
    return Book(S, L, 1, 2, D, pages + 1 + 2 * (S - 1), P, pages + 1, dtype,
                "f32")


def fill(b, k, pages):
    """Rows k [n][d] in the first sequence of every layer, five in the others."""
    c = b.c
    n = pages * P + 3
    x = rnd(7, (c.S, c.L, n, 1, D), b.dtype)
    x[0, :, :pages * P, 0] = k
    b.grow([n] + [5] * (c.S - 1), k=x)


FORMS = [(False, 390), (True, 390), (False, 2500)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("many,pages", FORMS)
def test_equal_pages_beside_others(dtype, many, pages):
    """300 of 390 pages alike, or 1,500 of 2,500, whose score is in the middle of
    the others': the budget ends among them, just before and just behind them."""
    alike = 300 if pages == 390 else 1500
    rng = np.random.default_rng(pages)
    k = rnd(11, (pages * P, D), dtype).reshape(pages, P, D)
    one = rnd(12, (P, D), dtype)
    at = rng.permutation(pages)[:alike]
    k[at] = one
    b = book(pages, many, dtype)
    fill(b, k.reshape(-1, D), pages)
    q = b.queries()
    lo, hi = k.min(1).astype(np.float64), k.max(1).astype(np.float64)
    x = q[0, 0].astype(np.float64)
    score = (np.maximum(x, 0) @ hi.T + np.minimum(x, 0) @ lo.T).max(0)
    above = int((score > score[at[0]]).sum())
    assert ((score == score[at[0]]).sum() >= alike) and above > 0
    for budget in (above, above + 1, above + alike // 2, above + alike,
                   above + alike + 1):
        b.check_pages(budget, 1, q)
    b.c.sync_status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("many,pages", [(False, 1500), (True, 700),
                                        (False, 3000)])
@pytest.mark.parametrize("far", [100.0, 8192.0])
def test_pages_that_stretch_the_range(dtype, many, pages, far):
    """Ordinary pages, all different, beside one of far greater and one of far
    lower score: all but those two lie in one part, and the greater `far`, the more
    of them lie within the rounding of the greatest score."""
    k = rnd(21, (pages * P, D), dtype).reshape(pages, P, D)
    k[pages // 3] = far
    k[pages // 2] = -far
    b = book(pages, many, dtype)
    fill(b, k.reshape(-1, D), pages)
    q = np.abs(b.queries())
    for budget in (1, 2, 100, pages // 2, pages - 2, pages - 1):
        b.check_pages(budget, 1, q)
    b.c.sync_status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("many,pages", [(False, 38), (True, 38), (False, 2100)])
def test_a_nan_ranks_above_infinity(dtype, many, pages):
    """One page of each kind beside ordinary ones, each budget's choice for itself:
    NaN, then +inf, then numbers, and -inf behind all of them."""
    k = rnd(31, (pages * P, D), dtype).reshape(pages, P, D)
    k[20, 3, 7] = np.nan
    k[9, 1, 8] = np.inf
    k[11, :, 9] = -np.inf       # both bounds
    b = book(pages, many, dtype)
    fill(b, k.reshape(-1, D), pages)
    c = b.c
    q = np.abs(b.queries()) + 1
    for budget in (1, 2, 3, pages - 1):
        got = torch.full((c.S, c.L, 1, budget + 1), -7, dtype=torch.int32,
                         device="cuda")
        c.attend_pages(dev(q, dtype), budget, 1, pages=got)
        want = paged.choose(q[0, 0], b.k[0][0, 0], P, budget, 1)
        first = got[0, 0, 0].tolist()
        assert first == want
        assert 20 in first and (budget == 1) == (9 not in first)
        assert 11 not in first
        for s in range(1, c.S):
            assert got[s, :, 0, 0].eq(0).all() and got[s, :, 0, 1:].eq(-1).all()
    with pytest.raises(kvr.KvrError, match="non-finite"):
        c.sync_status()
