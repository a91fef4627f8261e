"""Verification of drafted tokens (kvr_verify_drafts) against rejection sampling
in 64 bits: whole numbers, compared for equality.  In fp32 a decision or a race
may go the other way where 64 bits leave it within about 1e-6 of a tie, which
one in some 1e5 of these seeded draws would be."""
import numpy as np
import pytest
import torch

from oracle import kv4
from paper_2608_15797_gb300 import kvr

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


def make(seed, S, T, V, dtype="bf16", sigma=2.0, noise=0.7, top=0):
    g = np.random.default_rng(seed)
    target = sigma * g.standard_normal((S, T + 1, V))
    draft = target[:, :T] + noise * g.standard_normal((S, T, V))
    if top:
        for x in (target, draft):
            cut = np.sort(x, -1)[..., -top:-top + 1 or None]
            x[x < cut] = -np.inf
    target, draft = (torch.from_numpy(x).to(DT[dtype]) for x in (target, draft))
    d = draft.float().numpy()
    tokens = np.argmax(d - np.log(g.exponential(size=d.shape)), -1) if T else \
        np.zeros((S, 0))
    return (target, draft, tokens.astype(np.int32),
            g.random((S, T)).astype(np.float32),
            np.maximum(g.exponential(size=(S, V)), 1e-6).astype(np.float32))


def reference(x, s, n, temperature):
    target, draft, tokens, u, race = x
    return kv4.verify(target[s, :n + 1].float().numpy(),
                      draft[s, :n].float().numpy(), tokens[s, :n], u[s, :n],
                      race[s], temperature)


def call(x, counts=None, temperature=1.0, **kw):
    target, draft, tokens, u, race = (
        t.cuda() if isinstance(t, torch.Tensor) else torch.from_numpy(t).cuda()
        for t in x)
    if counts is not None:
        counts = torch.tensor(counts, dtype=torch.int32, device="cuda")
    a, tok = kvr.verify_drafts(target, draft, tokens, u, race, n_draft=counts,
                               temperature=temperature, **kw)
    return a.cpu().numpy(), tok.cpu().numpy()


def check(x, counts=None, temperature=1.0, **kw):
    S, T = x[2].shape
    a, tok = call(x, counts, temperature, **kw)
    seen = set()
    for s in range(S):
        n = T if counts is None else min(max(counts[s], 0), T)
        ra, nxt = reference(x, s, n, temperature)
        assert a[s] == ra, (s, a[s], ra)
        want = list(x[2][s, :ra]) + [nxt] + [-1] * (T - ra)
        assert tok[s].tolist() == want, s
        seen.add(ra)
    return seen


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("S,T,V", [(1, 1, 5), (3, 3, 1000), (17, 4, 257),
                                   (2, 8, 32000), (5, 2, 50001), (70, 5, 33),
                                   (2, 64, 64), (300, 1, 1)])
def test_against_64_bits(dtype, S, T, V):
    check(make(S + T + V, S, T, V, dtype))


def test_every_number_of_acceptances_occurs():
    assert check(make(1, 60, 4, 500)) == {0, 1, 2, 3, 4}


def test_full_vocabulary_and_temperature():
    x = make(2, 3, 4, 152064)
    check(x)
    check(x, temperature=0.7)
    check(make(3, 2, 2, 151936, "f32"), temperature=1.3)


@pytest.mark.parametrize("top", [1, 20])
def test_filtered_logits(top):
    """Logits cut to the top few, -inf elsewhere."""
    check(make(4, 30, 3, 2000, top=top))


def test_ragged_counts():
    x = make(5, 6, 4, 300)
    check(x, counts=[0, 1, 2, 3, 4, 9])
    check(x, counts=[-3, 4, 0, 0, 1, 2])


def test_no_drafts():
    """T = 0: the next token alone."""
    check(make(6, 9, 0, 400))


def test_equal_distributions_accept_all():
    x = list(make(7, 20, 4, 777))
    x[1] = x[0][:, :4].clone()
    x[3][:] = np.float32(1) - np.float32(2.0**-24)
    assert check(x) == {4}


def test_disjoint_distributions_reject_all():
    x = list(make(8, 10, 2, 100))
    x[0][:, :, :50] = -np.inf
    x[1][:, :, 50:] = -np.inf
    x[2][:] = np.random.default_rng(0).integers(0, 50, x[2].shape)
    assert check(x) == {0}


def test_race_ties_go_to_the_lowest():
    V = 5000
    logits = torch.zeros(4, 1, V)
    logits[1, 0, :4000] = -np.inf
    logits[2, 0, 4999] = 3.0
    logits[3, 0, 1::2] = 1.0
    x = (logits, torch.zeros(4, 0, V), np.zeros((4, 0), np.int32),
         np.zeros((4, 0), np.float32), np.ones((4, V), np.float32))
    _, tok = call(x)
    assert tok[:, 0].tolist() == [0, 4000, 4999, 1]


def test_rows_without_a_softmax_end_a_sequence():
    for dtype in ("bf16", "f32"):
        x = list(make(9, 8, 3, 600, dtype))
        x[3][:] = 0  # every draft would be accepted
        x[0][0, 0, 17] = np.nan
        x[0][1, 1, 599] = np.inf
        x[0][2, 2, :] = -np.inf
        x[1][3, 1, 300] = np.nan
        x[1][4, 2, :] = -np.inf
        x[0][5, 3, 0] = np.nan        # the row after the last draft
        x[2][6, 1] = 600              # no such token
        x[2][7, 0] = -1
        check(x)
        a, tok = call(x)
        assert a.tolist() == [0, 1, 2, 1, 2, 3, 1, 0]
        assert all(tok[s, a[s]] == -1 for s in range(8))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strided_and_unaligned_rows(dtype):
    """Rows cut out of a wider, oddly placed buffer."""
    V, S, T = 1003, 4, 3
    x = make(10, S, T, V, dtype)
    wide = []
    for t, pad, off in ((x[0], 5, 1), (x[1], 2, 3)):
        n = t.shape[1]
        buf = torch.full((S * n * (V + pad) + off,), float("nan"),
                         dtype=t.dtype, device="cuda")[off:]
        view = buf.view(S, n, V + pad)[..., :V]
        view.copy_(t)
        wide.append(view)
    a, tok = call(x)
    dev = [torch.from_numpy(t).cuda() for t in x[2:]]
    b, tok2 = kvr.verify_drafts(*wide, *dev)
    np.testing.assert_array_equal(a, b.cpu().numpy())
    np.testing.assert_array_equal(tok, tok2.cpu().numpy())
    check(x)


def test_emitted_tokens_follow_the_target():
    """First emitted tokens of many sequences with the same logits: the
    target's frequencies within five standard deviations."""
    S, V = 40000, 8
    g = np.random.default_rng(11)
    t1, d1 = g.standard_normal((2, V)), g.standard_normal((1, V))
    p = np.exp(t1[0]) / np.exp(t1[0]).sum()
    q = np.exp(d1[0]) / np.exp(d1[0]).sum()
    x = (torch.from_numpy(np.broadcast_to(t1, (S, 2, V)).copy()).float(),
         torch.from_numpy(np.broadcast_to(d1, (S, 1, V)).copy()).float(),
         g.choice(V, (S, 1), p=q).astype(np.int32),
         g.random((S, 1)).astype(np.float32),
         np.maximum(g.exponential(size=(S, V)), 1e-9).astype(np.float32))
    _, tok = call(x)
    hits = np.bincount(tok[:, 0], minlength=V)
    assert (np.abs(hits - S * p) <= 5 * np.sqrt(S * p * (1 - p))).all()


def test_a_workspace_holds_nothing_between_calls():
    x = make(12, 5, 3, 4000)
    ws = kvr.verify_workspace(5, 3, 4000)
    ws.fill_(255)
    first = call(x, workspace=ws)
    for _ in range(3):
        call(make(13, 5, 3, 4000), workspace=ws)
        again = call(x, workspace=ws)
        np.testing.assert_array_equal(first[0], again[0])
        np.testing.assert_array_equal(first[1], again[1])


def test_refusals():
    x = make(14, 2, 2, 50)
    t, d, tok, u, race = (torch.as_tensor(v).cuda() for v in x)
    with pytest.raises(ValueError):
        kvr.verify_drafts(t, d[:, :1], tok, u, race)
    with pytest.raises(ValueError):
        kvr.verify_drafts(t, d.float(), tok, u, race)
    with pytest.raises(ValueError):
        kvr.verify_drafts(t, d, tok.long(), u, race)
    with pytest.raises(ValueError):
        kvr.verify_drafts(t, d, tok, u, race[:, :40])
    with pytest.raises(ValueError):
        kvr.verify_drafts(t[..., ::2], d[..., ::2], tok, u, race)
    with pytest.raises(kvr.KvrError, match="KVR_EINVAL"):
        kvr.verify_drafts(t, d, tok, u, race, temperature=-1.0)
    with pytest.raises(kvr.KvrError, match="KVR_ENOMEM"):
        kvr.verify_drafts(t, d, tok, u, race, workspace=torch.empty(
            16, dtype=torch.uint8, device="cuda"))
