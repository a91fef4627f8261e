"""The 4-bit full-context cache (kvr_kv4_*) against its definition: what it
stores, attention over it with accumulated weights, and its cut into an evicted
cache.  Storing and cutting are compared for equality.  Attention is compared
with 64 bits on the stored values within bounds of its arithmetic:
  - an output rounds to its type (2^-8 of it for bf16's 8 significant bits);
  - a probability is rounded to 16 bits once where the outputs are bf16
    (2^-11 of the probability-weighted mean of |v|), and is fp32 otherwise;
  - a logit of magnitude up to 30 carries about 2^-19 of fp32 rounding, which
    moves a probability by 2e-6 of itself; ten times that is allowed."""
import numpy as np
import pytest
import torch

from oracle import kv4
from paper_2608_15797_gb300 import kvr

pytestmark = pytest.mark.gpu

LOGIT = 2e-5


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


def rnd(seed, shape, dtype="bf16", heavy=False):
    """Seeded values: float32 that dtype represents."""
    x = np.random.default_rng(seed).standard_normal(shape).astype(np.float32)
    if heavy:
        hot = np.random.default_rng(seed + 1).random(shape[:-1]) < 0.05
        x[hot] *= 3
    return kv4.bf16(x) if dtype == "bf16" else x


def dev(x, dtype="bf16"):
    return torch.from_numpy(np.ascontiguousarray(x)).to(
        kvr.TORCH_DTYPES[dtype]).cuda()


def rounded(x, dtype):
    return kv4.bf16(x) if dtype == "bf16" else np.asarray(x, np.float32)


class Pair:
    """A cache and the rows it was given, per sequence: [L][H][n][d]."""

    def __init__(self, S, L, H, G, d, cap, dtype="bf16", out_dtype="bf16",
                 **kw):
        self.c = kvr.Kv4Cache(S, L, H, G, d, cap, dtype=dtype,
                              out_dtype=out_dtype, **kw)
        self.dtype, self.out_dtype = dtype, out_dtype
        none = np.zeros((L, H, 0, d), np.float32)
        self.k, self.v = [none] * S, [none] * S

    def load(self, s, n, seed):
        c = self.c
        k = rnd(seed, (c.L, c.H, n, c.d), self.dtype, heavy=True)
        v = rnd(seed + 7, (c.L, c.H, n, c.d), self.dtype)
        c.load(s, dev(k, self.dtype), dev(v, self.dtype))
        self.k[s], self.v[s] = k, v

    def append(self, k, v, counts=None):
        """k, v [S][L][n][H][d]"""
        c = self.c
        c.append(dev(k, self.dtype), dev(v, self.dtype), counts=counts)
        for s in range(c.S):
            n = k.shape[2] if counts is None else counts[s]
            for mine, x in ((self.k, k), (self.v, v)):
                mine[s] = np.concatenate(
                    (mine[s], x[s, :, :n].transpose(0, 2, 1, 3)), 2)

    def check_attend(self, q, counts=None, scores=False, **kw):
        """q [S][L][T][H*G][d]"""
        c = self.c
        before = c.scores_view().cpu().numpy().astype(np.float64)
        out = c.attend(dev(q, self.dtype), counts=counts, scores=scores, **kw)
        torch.cuda.synchronize()
        out = out.float().cpu().numpy()
        after = c.scores_view().cpu().numpy()
        T = q.shape[2]
        half = self.out_dtype == "bf16" and self.dtype == "bf16"
        rel = 2.0**-8 if self.out_dtype == "bf16" else 2.0**-24
        for s in range(c.S):
            m = T if counts is None else counts[s]
            assert (out[s, :, m:] == 0).all()
            for l in range(c.L):
                for h in range(c.H):
                    kk = kv4.values(self.k[s][l, h])
                    vv = kv4.values(self.v[s][l, h])
                    ref, sc, mag = kv4.attend(
                        q[s, l, :m, h * c.G:(h + 1) * c.G], kk, vv)
                    got = out[s, l, :m, h * c.G:(h + 1) * c.G]
                    tol = rel * np.abs(ref) + mag * (
                        LOGIT + (2.0**-11 if half else 0)) + 1e-30
                    assert (np.abs(got - ref) <= tol).all(), (
                        s, l, h, np.max(np.abs(got - ref) / tol))
                    n = len(sc)
                    want = before[s, l, h, :n] + (sc if scores else 0)
                    assert (np.abs(after[s, l, h, :n] - want)
                            <= LOGIT * want + 1e-9).all()
                    np.testing.assert_array_equal(after[s, l, h, n:],
                                                  before[s, l, h, n:])
        return out


# ---- what is stored -----------------------------------------------------------

@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128),
                                     ("f32", 64)])
def test_load_append_read(dtype, d):
    """Prompts, ragged appends across block ends, and reading back: bit for
    bit what the definition says."""
    S, L, H, cap = 3, 2, 3, 200
    p = Pair(S, L, H, 2, d, cap, dtype, dtype)
    for s, n in enumerate((0, 31, 97)):
        p.load(s, n, 10 * s + d)
    for i, (n, counts) in enumerate([(1, None), (5, [5, 0, 3]),
                                     (70, [1, 70, 69]), (2, None)]):
        k = rnd(100 + i, (S, L, n, H, d), dtype, heavy=True)
        v = rnd(200 + i, (S, L, n, H, d), dtype)
        p.append(k, v, counts)
    lens = [x.shape[2] for x in p.k]
    np.testing.assert_array_equal(p.c.lengths(), np.repeat(lens, L).reshape(
        S, L))
    most = max(lens)
    k, v = p.c.read_newest(most, counts=lens)
    for got, mine in ((k, p.k), (v, p.v)):
        got = got.float().cpu().numpy()
        for s in range(S):
            np.testing.assert_array_equal(
                got[s, :, :, :lens[s]], rounded(kv4.values(mine[s]), dtype))
            assert (got[s, :, :, lens[s]:] == 0).all()
    k, _ = p.c.read_newest(3)
    np.testing.assert_array_equal(
        k[2].float().cpu().numpy(),
        rounded(kv4.values(p.k[2][:, :, -3:]), dtype))
    p.c.sync_status()


def test_codes_at_ties_and_extremes():
    """Values half-way between codes, constant groups, huge ranges, tiny
    ranges, zeros of either sign and non-finite values."""
    d = 128
    rows = np.zeros((12, d), np.float32)
    rows[0] = np.tile(np.arange(64) / 2.0, 2)[:d] % 15.5   # s = 1: half codes
    rows[0, ::64] = 15.0
    rows[1] = 3.0
    rows[2, ::2], rows[2, 1::2] = 3e38, -3e38
    rows[3] = 1e-38 * (np.arange(d) % 16)
    rows[4, ::2] = -0.0
    rows[5, 3] = np.nan
    rows[6, 100] = -np.inf
    rows[7] = 1e4 + np.arange(d) % 7
    rows[8] = -(np.arange(d) % 16)
    rows[9] = 1e-45 * (np.arange(d) % 5)
    rows[10] = 2.0**-130 * np.random.default_rng(0).random(d)
    rows[11] = np.random.default_rng(1).standard_cauchy(d) * 1e3
    p = Pair(1, 1, 1, 1, d, 40, "f32", "f32")
    x = rows[None, None, :, None]
    p.append(x, -x)
    k, v = (t.cpu().numpy()[0, 0, 0] for t in p.c.read_newest(12))
    np.testing.assert_array_equal(k, kv4.values(rows))
    np.testing.assert_array_equal(v, kv4.values(-rows))


def test_many_sequences_in_spans():
    """More sequences than one launch takes."""
    S = 300
    p = Pair(S, 1, 1, 2, 64, 8, "f32", "f32")
    counts = [s % 4 for s in range(S)]
    p.append(rnd(1, (S, 1, 3, 1, 64), "f32"), rnd(2, (S, 1, 3, 1, 64), "f32"),
             counts)
    p.append(rnd(3, (S, 1, 2, 1, 64), "f32"), rnd(4, (S, 1, 2, 1, 64), "f32"))
    k, _ = p.c.read_newest(2)
    for s in (0, 255, 256, 299):
        np.testing.assert_array_equal(k[s, 0].cpu().numpy(),
                                      kv4.values(p.k[s][0, :, -2:]))
    p.check_attend(rnd(5, (S, 1, 2, 2, 64), "f32"), scores=True)


# ---- attention ----------------------------------------------------------------

CASES = [
    # dtype, out, d, H, G, lens, tokens, counts
    ("bf16", "bf16", 128, 2, 7, [1, 31, 32, 33, 200], 1, None),
    ("bf16", "bf16", 128, 1, 8, [63, 64, 65, 129], 1, None),
    ("bf16", "f32", 128, 2, 3, [40, 150], 1, None),
    ("bf16", "bf16", 64, 2, 5, [5, 77], 1, None),
    ("f32", "f32", 64, 2, 2, [129, 2], 1, None),
    ("f32", "f32", 128, 1, 7, [100], 1, None),
    ("f32", "bf16", 64, 1, 1, [33], 1, None),
    ("bf16", "bf16", 128, 2, 7, [40, 5, 190], 5, [5, 2, 4]),
    ("bf16", "bf16", 128, 1, 8, [70, 300], 2, None),
    ("bf16", "bf16", 128, 1, 6, [64, 65], 3, None),
    ("bf16", "bf16", 128, 1, 1, [96], 17, None),
    ("bf16", "bf16", 128, 1, 7, [130, 40], 32, [32, 31]),
    ("f32", "f32", 128, 1, 5, [90], 9, None),
    ("f32", "f32", 64, 1, 8, [150, 20], 20, [20, 19]),
    ("bf16", "f32", 64, 1, 7, [75], 40, None),
    ("bf16", "bf16", 128, 1, 7, [20, 33], 20, [20, 1]),
]


@pytest.mark.parametrize("scores", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attend(case, scores):
    dtype, out, d, H, G, lens, T, counts = CASES[case]
    S, L = len(lens), 2
    p = Pair(S, L, H, G, d, max(lens), dtype, out)
    for s, n in enumerate(lens):
        p.load(s, n, 1000 * case + 10 * s)
    q = rnd(case + 5, (S, L, T, H * G, d), dtype)
    p.check_attend(q, counts, scores)
    if scores:  # they accumulate
        p.check_attend(rnd(case + 6, q.shape, dtype), counts, True)
    p.c.sync_status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attend_of_sequences_that_hold_little(dtype):
    """Empty sequences, sequences without a token in the call, and tokens that
    lie before a sequence's first row."""
    lens, counts = [0, 0, 3, 50, 1], [0, 2, 4, 0, 1]
    p = Pair(5, 1, 2, 3, 128, 64, dtype, dtype)
    for s, n in enumerate(lens):
        p.load(s, n, 5 + s)
    q = rnd(1, (5, 1, 4, 6, 128), dtype)
    for scores in (False, True):
        out = p.c.attend(dev(q, dtype), counts=counts, scores=scores)
        got = out.float().cpu().numpy()
        assert (got[[0, 1, 3]] == 0).all() and (got[2, :, 0] == 0).all()
        ref, _, _ = kv4.attend(q[4, 0, :1, :3], kv4.values(p.k[4][0, 0]),
                               kv4.values(p.v[4][0, 0]))
        np.testing.assert_allclose(got[4, 0, :1, :3], ref, atol=2e-2)
        ref, _, _ = kv4.attend(q[2, 0, :4, 3:], kv4.values(p.k[2][0, 1]),
                               kv4.values(p.v[2][0, 1]))
        np.testing.assert_allclose(got[2, 0, :, 3:], ref, atol=2e-2)
    p.c.sync_status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 4, 30])
def test_long_and_ragged(dtype, T):
    lens = [2500, 64, 700]
    p = Pair(3, 1, 2, 7, 128, 2500, dtype, dtype)
    for s, n in enumerate(lens):
        p.load(s, n, 50 + s)
    p.check_attend(rnd(9, (3, 1, T, 14, 128), dtype), scores=True)


@pytest.mark.parametrize("T", [1, 3, 12])
def test_non_finite_rows_stay_with_those_who_see_them(T):
    """A non-finite key or value reaches the tokens that see its row, and no
    other: not earlier tokens of the call, and nobody once it was dropped."""
    p = Pair(2, 1, 1, 2, 128, 100)
    for s in range(2):
        p.load(s, 40 + s, 3 + s)
    lens = p.c.lengths()[:, 0]
    bad = rnd(1, (2, 1, T + 5, 1, 128))
    bad[..., 3], bad[..., 100] = np.inf, np.nan
    p.c.append(dev(bad), dev(bad))
    p.c.truncate(lens)
    q = rnd(2, (2, 1, T, 2, 128))
    p.check_attend(q, scores=True)
    k, v = (rnd(i, (2, 1, T, 1, 128)) for i in (4, 5))
    k[0, 0, T - 1, 0, 5] = np.inf
    v[1, 0, T - 1, 0, 70] = np.nan
    kd, vd = k.copy(), v.copy()
    kd[0, 0, T - 1] = vd[1, 0, T - 1] = 1.0
    p.append(kd, vd)
    p.c.truncate(lens)
    p.c.append(dev(k), dev(v))
    ref = p.c.attend(dev(q)).float().cpu().numpy()
    assert np.isnan(ref[0, 0, T - 1]).all()
    assert np.isnan(ref[1, 0, T - 1, :, 64:]).all()
    assert np.isfinite(ref[1, 0, T - 1, :, :64]).all()
    for s in range(2):
        n = lens[s]
        for t in range(T - 1):
            want, _, _ = kv4.attend(
                q[s, 0, t:t + 1], kv4.values(p.k[s][0, 0, :n + t + 1]),
                kv4.values(p.v[s][0, 0, :n + t + 1]))
            np.testing.assert_allclose(ref[s, 0, t], want[0], atol=2e-2)
    with pytest.raises(kvr.KvrError):
        p.c.sync_status()
    p.c.sync_status()


def test_scales_far_apart():
    """Keys and values whose scales span many powers of two, and one far
    outlier: the largest values decide what is small."""
    p = Pair(1, 1, 1, 4, 128, 300, "bf16", "f32")
    k, v = rnd(1, (1, 1, 300, 1, 128)), rnd(2, (1, 1, 300, 1, 128))
    f = 2.0 ** np.random.default_rng(3).integers(-30, 30, 300)
    v = kv4.bf16(v * f[None, None, :, None, None])
    p.append(k, v)
    p.check_attend(rnd(4, (1, 1, 1, 4, 128)))
    p.check_attend(kv4.bf16(rnd(5, (1, 1, 3, 4, 128)) * 2.0**-40), scores=True)


def test_peaked_logits():
    """Logits of magnitude 60: one row takes nearly all."""
    p = Pair(1, 1, 1, 8, 128, 500)
    p.load(0, 500, 8)
    q = rnd(6, (1, 1, 1, 8, 128))
    q[0, 0, 0] = kv4.bf16(p.k[0][0, 0, 100:500:50] * 5)
    out = p.c.attend(dev(q)).float().cpu().numpy()
    ref, _, mag = kv4.attend(q[0, 0], kv4.values(p.k[0][0, 0]),
                             kv4.values(p.v[0][0, 0]))
    assert (np.abs(out[0, 0] - ref) <= 2.0**-8 * np.abs(ref) +
            mag * (2.0**-11 + 1e-3)).all()


def test_rejected_drafts_leave_no_trace():
    """Append, attend, drop and append again: bit for bit as if the dropped
    rows had never been."""
    q = dev(rnd(3, (2, 1, 4, 14, 128)))
    outs = []
    for drafts in (False, True):
        p = Pair(2, 1, 2, 7, 128, 120)
        for s in range(2):
            p.load(s, 61 + s, 20 + s)
        if drafts:
            n = p.c.lengths()[:, 0]
            x = dev(rnd(8, (2, 1, 9, 2, 128)) * 30)
            p.c.append(x, x)
            p.c.attend(dev(rnd(9, (2, 1, 9, 14, 128))))
            p.c.truncate(n)
        x, y = (dev(rnd(i, (2, 1, 4, 2, 128))) for i in (10, 11))
        p.c.append(x, y, counts=[4, 2])
        outs.append(p.c.attend(q, counts=[4, 2], scores=True))
        outs.append(p.c.scores_view()[:, :, :, :65].clone())
    assert torch.equal(outs[0], outs[2])
    n = p.c.lengths()[:, 0]
    for s in range(2):
        assert torch.equal(outs[1][s, :, :, :n[s]], outs[3][s, :, :, :n[s]])


def test_layer_ranges_and_streams():
    """Layer by layer on another stream: the whole call's results."""
    L = 3
    p = Pair(2, L, 2, 7, 128, 300)
    for s in range(2):
        p.load(s, 250 - 90 * s, 30 + s)
    k, v = (rnd(i, (2, L, 2, 2, 128)) for i in (1, 2))
    q = dev(rnd(3, (2, L, 2, 14, 128)))
    p.append(k, v)
    whole = p.c.attend(q)
    p.c.truncate(p.c.lengths()[:, 0] - 2)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    kd, vd = dev(k), dev(v)
    st.wait_stream(torch.cuda.current_stream())
    parts = [torch.empty_like(q[:, :1]) for _ in range(L)]
    st.wait_stream(torch.cuda.current_stream())
    for l in range(L):
        one = [x[:, l:l + 1].contiguous() for x in (kd, vd, q)]
        st.wait_stream(torch.cuda.current_stream())
        p.c.append(one[0], one[1], layers=(l, l + 1), stream=st)
        p.c.attend(one[2], out=parts[l], layers=(l, l + 1), stream=st)
        if l < L - 1:
            with pytest.raises(kvr.KvrError, match="KVR_ESTATE"):
                p.c.attend(q)
        st.synchronize()
    assert torch.equal(whole, torch.cat(parts, 1))


def test_repeated_calls_agree_bit_for_bit():
    p = Pair(2, 2, 2, 7, 128, 3000)
    for s in range(2):
        p.load(s, 3000 - 1111 * s, 40 + s)
    ws = p.c.attend_workspace(3)
    ws.fill_(255)
    q = dev(rnd(3, (2, 2, 3, 14, 128)))
    first = p.c.attend(q, workspace=ws)
    for _ in range(5):
        assert torch.equal(first, p.c.attend(q, workspace=ws))


# ---- the cut into an evicted cache ---------------------------------------------

@pytest.mark.parametrize("dst", ["bf16", "f32"])
@pytest.mark.parametrize("d,budget,window", [(128, 16, 8), (64, 30, 0),
                                             (128, 0, 12), (128, 300, 4)])
def test_evict(dst, d, budget, window):
    lens = [0, 1, 20, 24, 25, 290]
    S, L, H = len(lens), 2, 2
    p = Pair(S, L, H, 2, d, 300)
    for s, n in enumerate(lens):
        p.load(s, n, 60 + s)
    g = np.random.default_rng(budget)
    # few different scores, so that many tie at the cut
    score = g.integers(0, 6, (S, L, H, 300)).astype(np.float32) / 4
    score[4, 0, 0, 3] = np.nan
    score[5, 1, 1, ::2] = -0.0
    score[5, 1, 1, 1::2] = 0.0
    p.c.scores_view().copy_(torch.from_numpy(score))
    c = kvr.Cache(S, L, H, 2, d, max(1, min(290, budget + window)),
                  kv_dtype=dst)
    p.c.evict_into(c, budget, window)
    p.c.sync_status()
    c.sync_status()
    for s, n in enumerate(lens):
        e = c.export(s)
        keep = min(n, budget + window)
        assert (e["len"] == keep).all() and (e["next_pos"] == n).all()
        assert (c.lengths()[s] == keep).all()
        for l in range(L):
            for h in range(H):
                pos = kv4.evict(score[s, l, h, :n], budget, window)
                np.testing.assert_array_equal(e["pos"][l, h, :keep], pos)
                np.testing.assert_array_equal(e["score"][l, h, :keep],
                                              score[s, l, h, pos])
                for name, mine in (("K", p.k), ("V", p.v)):
                    np.testing.assert_array_equal(
                        e[name][l, h, :keep],
                        rounded(kv4.values(mine[s][l, h, pos]), dst))


@pytest.mark.parametrize("n", [1000, 5000, 20000])
def test_evict_long(n):
    """Scores as attention leaves them, and a cache of many rows."""
    p = Pair(1, 1, 2, 2, 128, n)
    p.load(0, n, 70)
    score = np.exp(2 * np.random.default_rng(n).standard_normal(
        (1, 1, 2, n))).astype(np.float32) / n
    score[..., 10:500] = score[..., 9:10]
    p.c.scores_view().copy_(torch.from_numpy(score))
    c = kvr.Cache(1, 1, 2, 2, 128, 640)
    for budget, window in ((64, 8), (512, 128), (3, 1)):
        p.c.evict_into(c, budget, window)
        e = c.export(0)
        for h in range(2):
            pos = kv4.evict(score[0, 0, h], budget, window)
            np.testing.assert_array_equal(e["pos"][0, h, :len(pos)], pos)
            np.testing.assert_array_equal(
                e["V"][0, h, :len(pos)],
                kv4.bf16(kv4.values(p.v[0][0, h, pos])))


def test_decoding_goes_on_from_the_cut():
    """The evicted cache decodes as one that was given the same state."""
    p = Pair(2, 2, 2, 7, 128, 400)
    for s in range(2):
        p.load(s, 400 - 50 * s, 80 + s)
    p.c.attend(dev(rnd(1, (2, 2, 16, 14, 128))), scores=True)
    a, b = (kvr.Cache(2, 2, 2, 7, 128, 30) for _ in range(2))
    p.c.evict_into(a, 20, 8)
    for s in range(2):
        b.import_state(s, a.export(s))
    for t in range(4):
        x = [dev(rnd(90 + 3 * t + i, (2, 2, m, 128))) for i, m in
             enumerate((14, 2, 2))]
        assert torch.equal(a.step(*x, 20, 8), b.step(*x, 20, 8))
    a.sync_status()


def test_capacity_and_state_refusals():
    c = kvr.Kv4Cache(2, 2, 1, 2, 128, 40)
    x = torch.zeros(2, 2, 41, 1, 128, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(kvr.KvrError, match="KVR_ECAPACITY"):
        c.append(x, x)
    with pytest.raises(kvr.KvrError, match="KVR_ECAPACITY"):
        c.load(0, *[torch.zeros(2, 1, 41, 128, dtype=torch.bfloat16,
                                device="cuda")] * 2)
    c.append(x[:, :, :40].contiguous(), x[:, :, :40].contiguous(), [40, 7])
    with pytest.raises(kvr.KvrError, match="KVR_ECAPACITY"):
        c.append(x[:, :, :1].contiguous(), x[:, :, :1].contiguous())
    with pytest.raises(kvr.KvrError, match="KVR_EINVAL"):
        c.truncate([41, 7])
    with pytest.raises(kvr.KvrError, match="KVR_EINVAL"):
        c.read_newest(8)
    q = torch.zeros(2, 2, 1, 2, 128, dtype=torch.bfloat16, device="cuda")
    for bad in ([2, 0], [-1, 0]):
        with pytest.raises(kvr.KvrError, match="KVR_EINVAL"):
            c.attend(q, counts=bad)
    with pytest.raises(kvr.KvrError, match="KVR_EINVAL"):
        c.attend(q, layers=(1, 3))
    with pytest.raises(kvr.KvrError, match="KVR_ENOMEM"):
        c.attend(q, workspace=torch.empty(8, dtype=torch.uint8,
                                          device="cuda"))
    odd = torch.zeros(q.numel() + 1, dtype=torch.bfloat16, device="cuda")[1:]
    with pytest.raises(kvr.KvrError, match="16-byte"):
        c.attend(odd.view(q.shape))
    for bad in (q.float(), q[:, :, :, :1]):
        with pytest.raises(ValueError):
            c.attend(bad.contiguous())
    small = kvr.Cache(2, 2, 1, 2, 128, 10)
    with pytest.raises(kvr.KvrError, match="KVR_ECAPACITY"):
        c.evict_into(small, 10, 1)
    with pytest.raises(kvr.KvrError, match="KVR_EINVAL"):
        c.evict_into(kvr.Cache(2, 2, 2, 2, 128, 20), 10, 1)
    with pytest.raises(kvr.KvrError, match="KVR_EINVAL"):
        c.evict_into(small, 0, 0)
    np.testing.assert_array_equal(c.lengths(), [[40, 40], [7, 7]])
