"""The oracle of the paged cache against brute force on small inputs."""
import numpy as np
import pytest

from oracle import paged


def test_plan_takes_and_gives_back():
    p = paged.Plan(3, 6, 16, 4)
    slots, bad = p.plan([17, 0, 16], 17)
    assert bad is None and p.table == [[0, 1], [], [2]]
    assert slots[0].tolist() == list(range(17))
    assert slots[1].tolist() == [-1] * 17
    assert slots[2, :16].tolist() == list(range(32, 48)) and slots[2, 16] == -1
    before = (list(p.stack), p.table_array())
    slots, _ = p.plan([33, 1, 17], 17)
    assert p.table == [[0, 1, 3], [4], [2, 5]] and not p.stack
    assert slots[0, :16].tolist() == list(range(17, 32)) + [48]
    p.plan([17, 0, 16])
    assert p.stack == before[0]
    np.testing.assert_array_equal(p.table_array(), before[1])
    # what goes back is there to be taken in the same call
    p.plan([17, 40, 3], 40)
    assert p.table == [[0, 1], [3, 4, 5], [2]]
    p.plan([17, 0, 3])
    p.plan([0, 64, 3], 64)
    assert p.table[1] == [0, 1, 3, 4]


def test_plan_refuses_as_a_whole():
    p = paged.Plan(2, 4, 16, 3)
    for lens, n_new, why in (([49, 0], 99, "length"), ([-1, 0], 9, "length"),
                             ([5, 0], 4, "length"), ([48, 48], 48, "capacity")):
        slots, bad = p.plan(lens, n_new)
        assert bad == why and (slots == -1).all()
        assert p.len == [0, 0] and len(p.stack) == 4


def test_a_score_bounds_its_rows():
    rng = np.random.default_rng(0)
    for _ in range(50):
        k, q = rng.standard_normal((16, 8)), rng.standard_normal((3, 8))
        s = paged.score(q, *paged.bounds(k))
        assert s >= (q @ k.T).max() - 1e-12
    k = np.repeat(k[:1], 16, 0)   # where the rows are one, it is their logit
    assert paged.score(q, *paged.bounds(k)) == pytest.approx((q @ k[0]).max())


def test_choice():
    q = np.array([[1.0, -1.0]])
    k = np.zeros((16 * 6 + 3, 2))
    k[16 * 4 + 2] = (3, 0)
    k[16 * 1] = (0, -2)
    assert paged.choose(q, k, 16, 1, 1) == [4, 6]
    assert paged.choose(q, k, 16, 2, 2) == [1, 4, 5, 6]
    assert paged.choose(q, k, 16, 3, 1) == [0, 1, 4, 6]      # ties: the lower
    assert paged.choose(q, k, 16, 0, 2) == [5, 6]
    assert paged.choose(q, k, 16, 6, 1) == list(range(7))
    k[16 * 3 + 5, 1] = np.nan
    assert paged.choose(q, k, 16, 1, 1) == [3, 6]
    assert paged.rows_of([1, 6], len(k), 16).tolist() == [*range(16, 32),
                                                          96, 97, 98]


def test_attention():
    rng = np.random.default_rng(1)
    q, k, v = (rng.standard_normal(s) for s in ((2, 4), (5, 4), (5, 4)))
    out, mag, top = paged.attend(q, k, v)
    for g in range(2):
        x = np.array([np.dot(q[g], r) / 2.0 for r in k])
        w = np.exp(x) / np.exp(x).sum()
        np.testing.assert_allclose(out[g], sum(a * r for a, r in zip(w, v)))
        assert top[g] == pytest.approx(max(np.abs(q[g] * r).sum() / 2 for r in k))
    assert (mag >= np.abs(out) - 1e-15).all()
    assert (paged.attend(q, k[:0], v[:0])[0] == 0).all()
