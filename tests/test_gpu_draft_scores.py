"""What drafted tokens leave in the 4-bit cache's scores: the accepted ones
their weights, the rejected ones nothing.  A token's weights, over the rows that
it sees and the mean of its heads, add up to 1, so a cache whose tokens have
all attended holds scores that add up to its rows."""
import numpy as np
import pytest
import torch

from tests.test_gpu_kv4 import LOGIT, Pair, dev, rnd

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scores_count_emitted_tokens_alone(monkeypatch, dtype):
    """Drafts from few rows, so that many are rejected, sequences that finish
    at different times."""
    from examples import draft_and_verify as ex
    made = []

    def caches(*a):
        made.append(whole(*a))
        return made[-1]
    whole = ex.caches
    monkeypatch.setattr(ex, "caches", caches)
    m = ex.Decoder(d=128 if dtype == "bf16" else 64, dtype=dtype, seed=3)
    g = torch.Generator().manual_seed(5)
    prompts = [torch.randint(m.V, (n,), generator=g).tolist()
               for n in (150, 1, 77)]
    out, share = ex.generate(m, prompts, 20, 4, 16, 4, 1.0)
    assert 0 < share < 1
    full = made[0][0]
    score = full.scores_view().double().cpu().numpy()
    for s, n in enumerate(full.lengths()[:, 0]):
        assert n == len(prompts[s]) + len(out[s]) - 1
        total = score[s, :, :, :n].sum(-1)
        np.testing.assert_allclose(total, n, rtol=LOGIT)


@pytest.mark.parametrize("G,T", [(7, 3), (7, 6), (2, 4)])
def test_rejected_drafts_leave_no_weight(G, T):
    """Attended to without scores, truncated, and the rest again with scores:
    bit for bit the scores of a cache that never saw the rejected ones."""
    keep = [T, 1, 0]
    q = dev(rnd(3, (3, 1, T, 2 * G, 128)))
    k, v = (dev(rnd(i, (3, 1, T, 2, 128))) for i in (10, 11))
    got = []
    for drafts in (False, True):
        p = Pair(3, 1, 2, G, 128, 400)
        for s in range(3):
            p.load(s, 300 - 90 * s, 20 + s)
        n = p.c.lengths()[:, 0]
        if drafts:
            p.c.append(k, v)
            p.c.attend(q)
            p.c.truncate(n + keep)
        else:
            p.c.append(k, v, counts=keep)
        p.c.attend(q, counts=keep, scores=True)
        got.append([p.c.scores_view()[s, :, :, :int(n[s]) + keep[s]].clone()
                    for s in range(3)])
    assert all(map(torch.equal, *got))
    assert all(float(x.sum()) > 0 for x in got[0][:2])
