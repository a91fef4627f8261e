"""The oracle of the 4-bit cache and of draft verification against what their
definitions imply."""
import numpy as np
import pytest
import torch

from oracle import kv4


@pytest.mark.parametrize("d", [64, 128])
def test_rounding_error_is_half_a_step(d):
    """|value - x| <= s/2, and where s or m were rounded towards the group's
    inside, what that cuts off: 15 half-ulps of s and one of m."""
    x = np.random.default_rng(0).standard_normal((50, d)).astype(np.float32)
    _, m, s = kv4.quantise(x)
    err = np.abs(kv4.values(x) - x).reshape(50, -1, 64).max(-1)
    slack = 15 * s * 2.0**-8 + np.abs(m) * 2.0**-8
    assert (err <= s / 2 + slack).all()


def test_bf16_matches_torch():
    x = np.random.default_rng(1).standard_normal(4096).astype(np.float32)
    x[:4] = [0.0, -0.0, 3e38, 1.00390625]
    np.testing.assert_array_equal(
        kv4.bf16(x), torch.from_numpy(x).bfloat16().float().numpy())


def test_two_level_groups_are_exact():
    """A group of two bf16 values fifteen steps apart is held exactly."""
    x = np.where(np.arange(128) % 3 == 0, -1.5, 6.0).astype(np.float32)
    np.testing.assert_array_equal(kv4.values(x[None])[0], x)


def test_constant_and_non_finite_groups():
    x = np.zeros((3, 128), np.float32)
    x[0] = 0.75
    x[1, 5] = np.inf
    x[2, 70] = np.nan
    y = kv4.values(x)
    assert (y[0] == 0.75).all()
    assert np.isnan(y[1, :64]).all() and (y[1, 64:] == 0).all()
    assert (y[2, :64] == 0).all() and np.isnan(y[2, 64:]).all()


def test_attend_matches_torch_and_conserves_scores():
    g = np.random.default_rng(2)
    q, k, v = (g.standard_normal(s) for s in ((3, 4, 64), (20, 64), (20, 64)))
    out, score, _ = kv4.attend(q, k, v)
    mask = torch.ones(3, 20, dtype=torch.bool).tril(17)
    ref = torch.nn.functional.scaled_dot_product_attention(
        torch.from_numpy(q).transpose(0, 1), torch.from_numpy(k)[None],
        torch.from_numpy(v)[None], attn_mask=mask).transpose(0, 1)
    np.testing.assert_allclose(out, ref.numpy(), atol=1e-12)
    assert abs(score.sum() - 3) < 1e-12


def test_evict_ties_and_windows():
    s = np.array([1, 3, 3, 2, 3, 0, 0], np.float32)
    assert kv4.evict(s, 2, 1).tolist() == [1, 2, 6]
    assert kv4.evict(s, 0, 2).tolist() == [5, 6]
    assert kv4.evict(s, 9, 2).tolist() == list(range(7))
    s[3] = np.nan
    assert kv4.evict(s, 1, 0).tolist() == [3]


def test_verified_tokens_follow_the_target():
    """What is emitted first, accepted draft or its replacement, is
    distributed as the target: frequencies within five standard deviations."""
    g = np.random.default_rng(3)
    target, draft = g.standard_normal((2, 6)), g.standard_normal((1, 6))
    p = np.exp(target[0]) / np.exp(target[0]).sum()
    q = np.exp(draft[0]) / np.exp(draft[0]).sum()
    n, hits = 20000, np.zeros(6)
    for _ in range(n):
        x = g.choice(6, p=q)
        a, nxt = kv4.verify(target, draft, [x], g.random(1),
                            g.exponential(size=6))
        hits[x if a else nxt] += 1
    assert (np.abs(hits - n * p) <= 5 * np.sqrt(n * p * (1 - p))).all()


def test_verify_edges():
    t = np.zeros((3, 4))
    one = np.ones(4)
    # equal distributions: always accepted, then the race's winner
    assert kv4.verify(t, t[:2], [1, 2], [0.9, 0.9],
                      np.array([2, 1, 3, 1.0])) == (2, 1)
    # a draft that the target excludes: its replacement is the target's
    x = t.copy()
    x[0, 1] = -np.inf
    assert kv4.verify(x, t[:2], [1, 2], [0.0, 0.0], one) == (0, 0)
    for bad in (np.nan, np.inf):
        x = t.copy()
        x[1, 0] = bad
        assert kv4.verify(x, t[:2], [0, 0], [0, 0], one) == (1, -1)
    assert kv4.verify(t, t[:2], [0, 4], [0, 0], one) == (1, -1)
