"""Attention over the 4-bit cache where the references that probabilities are
held against rise along the context.  Bounds as in test_gpu_kv4."""
import numpy as np
import pytest
import torch

from oracle import kv4
from tests.test_gpu_kv4 import Pair, rnd

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("small", [0.0, 2.0**-50])
@pytest.mark.parametrize("G,T", [(7, 5), (8, 8), (2, 13), (1, 1)])
def test_rows_that_weigh_nothing_keep_their_probability(G, T, small):
    """A context that begins with rows whose values are zeros, or tiny, and goes
    on with rows of values up to 100 and logits about 3.4 higher: the first rows
    give nothing to the output, but have their share of the probability."""
    n, first = 500, 140  # four tiles of 128, which one CTA takes
    u = rnd(1, (128,))
    a = np.zeros(n, np.float32)
    a[first:] = np.linspace(0.05, 0.3, n - first)
    k = kv4.bf16(a[:, None] * u + 0.01 * rnd(5, (n, 128)))
    v = rnd(2, (n, 128)) * 32
    v[:first] *= small
    p = Pair(1, 1, 1, G, 128, n)
    p.append(k[None, None, :, None], kv4.bf16(v)[None, None, :, None])
    q = kv4.bf16(np.broadcast_to(u, (1, 1, T, G, 128)) *
                 np.linspace(0.9, 1, T * G, dtype=np.float32).reshape(
                     1, 1, T, G, 1))
    p.check_attend(q, scores=True)
    p.c.sync_status()
