"""Verification at low temperatures (kvr_verify_drafts) against 64 bits.  A
logit enters as its distance to the row's greatest, which fp32 holds to 2^-24 of
itself; an exponent of up to 100, beyond which nothing is left of a probability,
is so off by 1e-5, and a probability by as much of itself, its normaliser's share
included 2e-5; twice that is allowed.  A decision has to be the one of 64 bits
unless it is that near to a tie, and the next token one whose weight may be the
greatest."""
import numpy as np
import pytest
import torch

from oracle import kv4
from tests.test_gpu_verify import call, make

pytestmark = pytest.mark.gpu

REL = 4e-5


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


def cold(temperature):
    return float(np.float32(temperature))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("temperature", [1e-1, 1e-2, 1e-3, 1e-4, 1e-5])
def test_decisions(dtype, temperature):
    """Drafts drawn from the draft at this temperature."""
    S, T, V = 60, 4, 1000
    temperature = cold(temperature)
    x = list(make(21, S, T, V, dtype, sigma=4.0, noise=0.1))
    target, draft, _, u, race = x
    d = draft.double().numpy() / temperature
    noise = np.random.default_rng(5).exponential(size=d.shape)
    x[2] = np.argmax(d - np.log(noise), -1).astype(np.int32)
    a, tok = call(x, temperature=temperature)
    told = 0
    for s in range(S):
        for t in range(T + 1):
            p = kv4._softmax(target[s, t].float().numpy(), temperature)
            if t == T:
                assert a[s] == T
                w, tol = p, REL * p
                break
            q = kv4._softmax(draft[s, t].float().numpy(), temperature)
            i = x[2][s, t]
            gap = p[i] - u[s, t] * q[i]
            if abs(gap) > REL * (p[i] + q[i]):
                assert (a[s] > t) == (gap > 0), (s, t, a[s])
                told += 1
            if a[s] == t:
                w, tol = np.maximum(p - q, 0), REL * (p + q)
                if w.max() <= tol.max():  # nothing may be left of it
                    w, tol = p, 2 * p
                break
        n = tok[s, a[s]]
        r = race[s].astype(np.float64)
        assert (w[n] + tol[n]) / r[n] >= ((w - tol) / r).max(), (s, n)
    assert told > S


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("temperature", [1e-2, 1e-3, 1e-4, 1e-5])
def test_one_token_of_probability_one_is_accepted(dtype, temperature):
    """Target and draft agree on one token, each with a maximum of its own: both
    give it all of the probability, and no uniform number below 1 rejects it."""
    S, T, V = 64, 3, 500
    x = list(make(22, S, T, V, dtype))
    top = 5 + 20 * np.random.default_rng(0).random((S, T, 2))
    token = np.random.default_rng(1).integers(0, V, (S, T))
    for s in range(S):
        for t in range(T):
            for i in range(2):
                row = x[i][s, t]
                row.clamp_(max=4.0)
                row[token[s, t]] = float(top[s, t, i])
    x[2] = token.astype(np.int32)
    x[3][:] = np.float32(1) - np.float32(2.0**-24)
    a, _ = call(x, temperature=cold(temperature))
    assert (a == T).all()
