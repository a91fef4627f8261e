"""The paged full-context cache (kvr_paged_*) against its definition.  Plans,
stored rows, bounds and chosen pages are compared for equality.  Attention is
compared with 64 bits within bounds of its arithmetic:
  - an output rounds to its type: 2^-8 of it in bf16, 2^-24 in fp32;
  - a logit is D products summed in fp32.  Plain sums: 40 additions or fewer in a
    chain, 2^-24 each of the sum of magnitudes.  Tensor-core sums (bf16): D / 16
    products of 16, whose 17 terms are cut at 2^-23 of the greatest: 2^-16 of the
    sum of magnitudes covers d = 128.  A logit that is off by x moves a
    probability by 2 x of itself;
  - an exponential is within 2^-22, its argument (below 2^6 for these inputs)
    within 2^-19: together below 2^-18 of a probability;
  - a probability may be held as two bf16 numbers: 2^-16 of it;
  - sums over rows are fp32: 2^-23 for each of n / 16 additions and 64 more."""
import numpy as np
import pytest
import torch

from oracle import kv4, paged
from paper_2608_15797_gb300 import kvr

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("needs a CUDA device")
    torch.cuda.set_device(0)


def rnd(seed, shape, dtype="bf16", heavy=False):
    x = np.random.default_rng(seed).standard_normal(shape).astype(np.float32)
    if heavy:
        x[np.random.default_rng(seed + 1).random(shape[:-1]) < 0.05] *= 3
    return kv4.bf16(x) if dtype == "bf16" else x


def dev(x, dtype="bf16"):
    return torch.from_numpy(np.ascontiguousarray(x)).to(
        kvr.TORCH_DTYPES[dtype]).cuda()


def bits(x):
    """bf16 values as whole numbers: rows that nothing wrote may hold NaN."""
    return x.view(torch.int16)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Book:
    """A cache, the oracle's plan of it and the rows it was given, per sequence
    [L][H][n][d]."""

    def __init__(self, S, L, H, G, d, n_pages, page=16, table=None,
                 dtype="bf16", out_dtype=None, **kw):
        out_dtype = out_dtype or dtype
        self.c = kvr.PagedCache(S, L, H, G, d, n_pages, page, table, dtype,
                                out_dtype, **kw)
        self.p = paged.Plan(S, n_pages, page, table or n_pages)
        self.dtype, self.out_dtype = dtype, out_dtype
        none = np.zeros((L, H, 0, d), np.float32)
        self.k, self.v = [none] * S, [none] * S
        self.seed = 0

    def plan(self, lens, n_new=0):
        slots = self.c.plan(i32(lens), n_new)
        want, bad = self.p.plan(lens, n_new)
        if n_new:
            np.testing.assert_array_equal(slots.cpu().numpy(), want)
        table, ln, free = (x.cpu().numpy() for x in self.c.tables_view())
        np.testing.assert_array_equal(table, self.p.table_array())
        assert ln.tolist() == self.p.len and free[0] == len(self.p.stack)
        if bad:
            with pytest.raises(kvr.KvrError, match=bad):
                self.c.sync_status()
        else:
            for s, n in enumerate(lens):
                self.k[s], self.v[s] = (x[s][:, :, :n] for x in (self.k, self.v))
        return slots

    def grow(self, counts, n_new=None, layers=None, k=None, v=None):
        """Plan and append counts[s] new tokens of random rows."""
        c, n_new = self.c, n_new or max(counts)
        old = list(self.p.len)
        slots = self.plan([a + b for a, b in zip(old, counts)], n_new)
        self.seed += 10
        shape = (c.S, c.L, n_new, c.H, c.d)
        k = rnd(self.seed, shape, self.dtype, True) if k is None else k
        v = rnd(self.seed + 2, shape, self.dtype) if v is None else v
        for lb, le in layers or [(0, c.L)]:
            c.append(dev(k[:, lb:le], self.dtype), dev(v[:, lb:le], self.dtype),
                     slots, layers=(lb, le))
        for s, n in enumerate(counts):
            for mine, x in ((self.k, k), (self.v, v)):
                mine[s] = np.concatenate(
                    (mine[s], x[s, :, :n].transpose(0, 2, 1, 3)), 2)
        return slots

    def check_rows(self):
        """Every row is where the tables say, every full page has its bounds."""
        c, P = self.c, self.p.P
        k, v = (x.float().cpu().numpy() for x in c.rows_view())
        b = c.bounds_view().float().cpu().numpy()
        for s, t in enumerate(self.p.table):
            n = self.p.len[s]
            if not n:
                continue
            for pool, rows in ((k, self.k[s]), (v, self.v[s])):
                got = np.concatenate([pool[:, p] for p in t], 2)[:, :, :n]
                np.testing.assert_array_equal(got, rows)
            for i in range(n // P):
                part = self.k[s][:, :, i * P:(i + 1) * P]
                np.testing.assert_array_equal(b[:, t[i], :, 0], part.min(2))
                np.testing.assert_array_equal(b[:, t[i], :, 1], part.max(2))

    def check_out(self, q, out, pages=None, scale=None):
        """q and out [S][L][H*G][d]; pages [S][L][H][.]: those that were read."""
        c = self.c
        rel = 2.0**-8 if self.out_dtype == "bf16" else 2.0**-24
        logit = 2.0**-16 if self.dtype == "bf16" else 40 * 2.0**-24
        worst = 0.0
        for s in range(c.S):
            n = self.p.len[s]
            if n == 0:
                assert (out[s] == 0).all()
                continue
            for l in range(c.L):
                for h in range(c.H):
                    kk, vv = self.k[s][l, h], self.v[s][l, h]
                    if pages is not None:
                        at = pages[s, l, h]
                        at = paged.rows_of(at[at >= 0], n, self.p.P)
                        kk, vv = kk[at], vv[at]
                    g = slice(h * c.G, (h + 1) * c.G)
                    ref, mag, top = paged.attend(q[s, l, g], kk, vv, scale)
                    some = 2 * logit * top[:, None] + 2.0**-18 + 2.0**-16 \
                        + (len(kk) / 16 + 64) * 2.0**-23
                    tol = rel * np.abs(ref) + mag * some + 1e-30
                    r = np.abs(out[s, l, g] - ref) / tol
                    worst = max(worst, r.max())
                    assert (r <= 1).all(), (s, l, h, r.max())
        return worst

    def queries(self):
        c = self.c
        self.seed += 10
        return rnd(self.seed, (c.S, c.L, c.H * c.G, c.d), self.dtype)

    def check_attend(self, scale=None, **kw):
        q = self.queries()
        out = self.c.attend(dev(q, self.dtype), **kw).float().cpu().numpy()
        self.check_out(q, out, scale=scale)
        return out

    def check_pages(self, budget, window, q=None):
        c = self.c
        q = self.queries() if q is None else q
        got = torch.full((c.S, c.L, c.H, budget + window), -7,
                         dtype=torch.int32, device="cuda")
        out = c.attend_pages(dev(q, self.dtype), budget, window, pages=got)
        got, out = got.cpu().numpy(), out.float().cpu().numpy()
        for s in range(c.S):
            for l in range(c.L):
                for h in range(c.H):
                    want = paged.choose(q[s, l, h * c.G:(h + 1) * c.G],
                                        self.k[s][l, h], self.p.P, budget,
                                        window)
                    want += [-1] * (budget + window - len(want))
                    assert got[s, l, h].tolist() == want, (s, l, h)
        self.check_out(q, out, got)
        return out


# ---- plans ------------------------------------------------------------------

@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_plans_at_random(page):
    """Sequences grow, shrink, end and come, also several at once."""
    rng = np.random.default_rng(page)
    b = Book(7, 1, 1, 1, 64, 40, page, 20)
    most = 20 * page
    for step in range(60):
        kind = rng.integers(4)
        old = np.array(b.p.len)
        if kind == 0:
            lens = np.minimum(old + rng.integers(0, 3, 7), most)
        elif kind == 1:
            lens = np.where(rng.random(7) < 0.3, 0, old)
        elif kind == 2:
            lens = (old * rng.random(7)).astype(int)
        else:
            lens = rng.integers(0, most // 2, 7)
        n_new = max(int((lens - old).max()), 0)
        b.plan(lens.tolist(), n_new + int(rng.integers(0, 3)))
    b.plan([0] * 7)
    assert sorted(b.p.stack) == list(range(40))


@pytest.mark.parametrize("S", [1, 31, 33, 255, 256, 257, 511, 513, 1024, 2500,
                               9000])
def test_plans_of_many_sequences(S):
    rng = np.random.default_rng(S)
    b = Book(S, 1, 1, 1, 64, 3 * S + 1, 16, 6)
    for _ in range(4):
        lens = rng.integers(0, 6 * 16 + 1, S)
        while -(-lens // 16).sum() > 3 * S + 1:
            lens[rng.integers(S)] = 0
        b.plan(lens.tolist(), 96)


def test_a_long_sequence():
    """One sequence of more pages than the plan has threads, and many slots."""
    b = Book(2, 1, 1, 1, 64, 5000, 16, 5000)
    b.plan([16 * 2900 + 5, 3], 16 * 2900 + 5)
    b.plan([16 * 2900 + 21, 0], 16)
    b.plan([7, 16 * 4000], 16 * 4000)


def test_refused_plans_change_nothing():
    b = Book(3, 1, 2, 2, 64, 8, 16, 5)
    b.grow([40, 3, 0])
    rows = bits(b.c.rows_view()[0]).clone()
    for lens, n_new in (([81, 3, 0], 99),       # longer than a table
                        ([40, -1, 0], 9), ([40, 3, -2**31], 9),
                        ([44, 3, 1], 3),        # grows by more than n_new
                        ([41, 3, 0], 0),
                        ([80, 17, 17], 80),     # the pool ends
                        ([2**31 - 1, 3, 0], 9),
                        ([81, 3, 0], 6000),     # slots by a launch of their own
                        ([80, 17, 17], 6000)):
        b.plan(lens, n_new)
    assert torch.equal(rows, bits(b.c.rows_view()[0]))
    b.plan([80, 16, 17], 80)                    # all eight
    assert not b.p.stack


# ---- append -----------------------------------------------------------------

@pytest.mark.parametrize("dtype,d,page", [
    ("bf16", 128, 16), ("bf16", 128, 64), ("bf16", 64, 32), ("f32", 128, 128),
    ("f32", 64, 16)])
def test_append(dtype, d, page):
    """Prompts, single tokens across page ends, ragged batches, idle places,
    rows dropped from the end and written again; layers in one call and in
    several."""
    b = Book(4, 3, 2, 2, d, 4 * 7, page, 7, dtype)
    b.grow([page * 2 + 5, 1, 0, page])
    b.check_rows()
    for i in range(4):
        b.grow([1, 1, 0, 1], layers=[(0, 1), (1, 3)] if i % 2 else None)
    b.grow([page - 9, page - 5, 3, 2 * page + 1], n_new=2 * page + 7)
    b.check_rows()
    # rejected drafts: back into the middle of a full page, and on
    b.plan([page + 3, 2, 3, page - 1])
    b.grow([2 * page, page - 2, 0, 1])
    b.check_rows()
    b.c.sync_status()


def test_append_any_rows_of_a_plan():
    """Sequences in another order, one by one, one not at all."""
    b = Book(3, 2, 2, 1, 128, 12, 16, 4)
    slots = b.plan([20, 33, 16], 33)
    shape = (3, 2, 33, 2, 128)
    k, v = rnd(1, shape), rnd(2, shape)
    before = bits(b.c.rows_view()[0])[:, b.p.table[2]].clone()
    order = torch.tensor([1, 0], device="cuda")
    b.c.append(dev(k)[order].contiguous(), dev(v)[order].contiguous(),
               slots[order].contiguous())
    assert torch.equal(before, bits(b.c.rows_view()[0])[:, b.p.table[2]])
    b.c.append(dev(k)[2:], dev(v)[2:], slots[2:])
    for s, n in enumerate((20, 33, 16)):
        b.k[s], b.v[s] = (x[s, :, :n].transpose(0, 2, 1, 3) for x in (k, v))
    b.check_rows()


def test_a_prompt_in_parts():
    """Columns of a plan's slots, one part after the other."""
    b = Book(2, 2, 2, 1, 64, 20, 32, 10)
    slots = b.plan([150, 77], 150)
    shape = (2, 2, 150, 2, 64)
    k, v = rnd(1, shape, heavy=True), rnd(2, shape)
    for a, e in ((0, 40), (40, 41), (41, 96), (96, 150)):
        b.c.append(dev(k[:, :, a:e]), dev(v[:, :, a:e]),
                   slots[:, a:e].contiguous())
    for s, n in enumerate((150, 77)):
        b.k[s], b.v[s] = (x[s, :, :n].transpose(0, 2, 1, 3) for x in (k, v))
    b.check_rows()
    b.check_pages(1, 1)
    b.c.sync_status()


def test_bounds_of_extreme_keys():
    """Infinities, NaN and the types' ends are in the bounds of their page."""
    for dtype in ("bf16", "f32"):
        big = float(torch.finfo(kvr.TORCH_DTYPES[dtype]).max)
        b = Book(1, 1, 1, 1, 64, 3, 16, 3, dtype)
        k = rnd(3, (1, 1, 40, 1, 64), dtype)
        k[0, 0, 3, 0, 5], k[0, 0, 4, 0, 6] = np.inf, -np.inf
        k[0, 0, 20, 0, 7], k[0, 0, 30, 0, 8] = np.nan, big
        k[0, 0, 31, 0, 9], k[0, 0, 35, 0, 0] = -big, np.nan
        b.grow([40], k=k)
        b.check_rows()


def test_slots_outside_the_pool_are_not_written():
    """What a plan would not give: the call says so and writes none of it."""
    b = Book(1, 1, 2, 1, 128, 4, 16, 4)
    b.grow([40])
    before = bits(b.c.rows_view()[0]).clone()
    x = dev(rnd(5, (1, 1, 3, 2, 128)))
    for slots in ([64, 65, 66], [62, 63, 64], [2**31 - 1, 5, 6], [33, 35, 36],
                  [31, 33, 34]):
        b.c.append(x, x, i32([slots]))
        with pytest.raises(kvr.KvrError, match="length"):
            b.c.sync_status()
    b.c.append(x, x, i32([[-1, 5, 6]]))     # a row ends at its first -1
    b.c.sync_status()
    same = (before == bits(b.c.rows_view()[0])).all(-1).cpu().numpy()[0]
    # of [62, 63, 64] and [31, 33, 34] the part in one page may be written
    wrong = list(zip(*np.nonzero(~same.all(1))))
    assert set(wrong) <= {(3, 14), (3, 15), (1, 15)}


# ---- attention --------------------------------------------------------------

@pytest.mark.parametrize("dtype,out_dtype,d,G,page", [
    ("bf16", "bf16", 128, 7, 16), ("bf16", "f32", 128, 8, 64),
    ("bf16", "bf16", 64, 5, 32), ("bf16", "f32", 64, 1, 128),
    ("f32", "f32", 128, 8, 16), ("f32", "bf16", 128, 3, 128),
    ("f32", "f32", 64, 2, 64), ("f32", "f32", 64, 7, 32)])
@pytest.mark.parametrize("lens", [
    [1], [15, 16, 17], [0, 129, 0, 64, 1], [300, 0, 2000, 31]])
def test_attend(dtype, out_dtype, d, G, page, lens):
    most = max(lens)
    pages = sum(-(-n // page) for n in lens)
    b = Book(len(lens), 2, 2, G, d, pages, page, -(-most // page), dtype,
             out_dtype)
    b.grow([n // 2 for n in lens], n_new=most)
    b.grow([n - n // 2 for n in lens], n_new=most)
    b.check_attend()
    b.c.sync_status()


@pytest.mark.parametrize("dtype,d,G", [("bf16", 128, 7), ("bf16", 64, 8),
                                       ("f32", 128, 5), ("f32", 64, 1)])
@pytest.mark.parametrize("lens", [[1], [16], [17], [1023], [1025, 0], [5000]])
def test_attend_few_units(dtype, d, G, lens):
    """A layer a call: few units, from one row to some thousand."""
    most = max(lens)
    b = Book(len(lens), 2, 2, G, d, sum(-(-n // 16) for n in lens), 16,
             -(-most // 16), dtype, "f32")
    b.grow(lens)
    q = b.queries()
    out = torch.cat([b.c.attend(dev(q[:, l:l + 1], dtype), layers=(l, l + 1))
                     for l in range(2)], 1)
    b.check_out(q, out.cpu().numpy())
    b.c.sync_status()


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64),
                                     ("f32", 128), ("f32", 64)])
def test_one_long_unit(dtype, d):
    """Shared by many CTAs: lengths around the ends of their spans."""
    n = 40000
    b = Book(1, 1, 1, 3, d, n // 16, 16, n // 16, dtype, "f32")
    b.grow([n])
    for m in (n, n - 1, 3 * 16 * 4 * 100 + 1, 3 * 16 * 4 * 100, 12289):
        b.plan([m])
        b.check_attend()
    b.c.sync_status()


def test_several_waves():
    """More CTAs than run at once; some units are looked at."""
    n, P = 8000, 64
    b = Book(8, 4, 4, 7, 128, 8 * 125, P, 125, out_dtype="f32")
    b.grow([n, 1, 0, n - 1, n // 2, n, 77, n])
    q = b.queries()
    out = b.c.attend(dev(q)).cpu().numpy()
    b.c.sync_status()
    for s in range(8):
        for l, h in ((0, 0), (1, 2), (3, 3)):
            g = slice(7 * h, 7 * h + 7)
            ref, mag, top = paged.attend(q[s, l, g], b.k[s][l, h], b.v[s][l, h])
            some = 2 * 2.0**-16 * top[:, None] + 2.0**-18 + 2.0**-16 \
                + (n / 16 + 64) * 2.0**-23 if len(b.k[s][l, h]) else 0
            assert (np.abs(out[s, l, g] - ref)
                    <= 2.0**-24 * np.abs(ref) + mag * some + 1e-30).all()


@pytest.mark.parametrize("scale", [0.3, 1e-3])
def test_softmax_scale(scale):
    b = Book(2, 1, 2, 4, 128, 8, 64, 4, "bf16", "f32", softmax_scale=scale)
    b.grow([100, 5])
    b.check_attend(scale=scale)


def test_many_short_sequences():
    """More units than warps, several of them in one warp's span."""
    rng = np.random.default_rng(8)
    lens = rng.integers(0, 60, 150).tolist()
    b = Book(150, 3, 8, 8, 128, 150 * 4, 16, 4, out_dtype="f32")
    b.grow(lens)
    b.check_attend()


def test_equal_calls_give_equal_bits():
    """Also through other pages."""
    lens = [1500, 3, 700]
    out = []
    for first in (0, 1):
        b = Book(3, 2, 2, 7, 128, 80, 32, 50, out_dtype="f32")
        if first:      # the pool is handed round before
            b.plan([1000, 50, 500], 1000)
            b.plan([0, 900, 70], 900)
            b.plan([0, 0, 0])
        b.seed = 0
        b.grow(lens)
        b.seed = 99
        q = dev(b.queries())
        x = b.c.attend(q)
        for _ in range(5):
            assert torch.equal(x, b.c.attend(q))
        p = b.c.attend_pages(q, 3, 1)
        for _ in range(5):
            assert torch.equal(p, b.c.attend_pages(q, 3, 1))
        out.append((x, p))
    assert torch.equal(out[0][0], out[1][0])
    assert torch.equal(out[0][1], out[1][1])


def test_nothing_behind_a_sequence_is_read():
    """The rest of the last page holds NaN, other sequences' pages infinities,
    workspace and outputs are full of NaN."""
    b = Book(2, 1, 2, 7, 128, 6, 64, 3)
    b.grow([70, 64])
    other = np.full((2, 1, 40, 2, 128), np.nan, np.float32)
    slots = b.c.plan(i32([110, 64]), 40)
    b.c.append(dev(other), dev(other), slots)
    b.c.plan(i32([70, 64]))
    c = b.c
    for scale in (1, 2):
        ws = c.attend_pages_workspace(1, 1)
        ws.fill_(255)
        q = b.queries()
        out = torch.full((2, 1, 14, 128), float("nan"), dtype=torch.bfloat16,
                         device="cuda")
        c.attend(dev(q), out=out, workspace=ws)
        b.check_out(q, out.float().cpu().numpy())
        ws.fill_(255)
        out.fill_(float("nan"))
        c.attend_pages(dev(q), 1, 1, out=out, workspace=ws)
        b.check_out(q, out.float().cpu().numpy())
    c.sync_status()


def test_extreme_values():
    """Logits far apart and equal; keys that give -inf everywhere but in one row;
    an infinite one sets the error word."""
    for dtype in ("bf16", "f32"):
        b = Book(1, 1, 1, 2, 64, 5, 16, 5, dtype, "f32")
        k = np.zeros((1, 1, 70, 1, 64), np.float32)
        b.grow([70], k=k)
        b.check_attend()            # all rows alike
        k[0, 0, 33] = 64.0
        b = Book(1, 1, 1, 2, 64, 5, 16, 5, dtype, "f32")
        b.grow([70], k=k)
        q = np.full((1, 1, 2, 64), 8.0, np.float32)
        q[0, 0, 1] = -8.0
        out = b.c.attend(dev(q, dtype)).cpu().numpy()
        np.testing.assert_allclose(out[0, 0, 0], b.v[0][0, 0, 33], rtol=1e-6)
        rest = np.delete(b.v[0][0, 0], 33, 0).astype(np.float64).mean(0)
        np.testing.assert_allclose(out[0, 0, 1], rest, atol=1e-4)
        b.c.sync_status()
        k[0, 0, 12, 0, 0] = -np.inf  # 8 x -inf: a row without weight
        b = Book(1, 1, 1, 1, 64, 5, 16, 5, dtype, "f32")
        b.grow([70], k=k)
        q = np.full((1, 1, 1, 64), 8.0, np.float32)
        out = b.c.attend(dev(q, dtype)).cpu().numpy()
        np.testing.assert_allclose(out[0, 0, 0], b.v[0][0, 0, 33], rtol=1e-6)
        b.c.sync_status()
        out = b.c.attend(dev(-q, dtype)).cpu().numpy()
        assert np.isnan(out).all()
        with pytest.raises(kvr.KvrError, match="non-finite"):
            b.c.sync_status()


# ---- attention over chosen pages --------------------------------------------

@pytest.mark.parametrize("dtype,d,G,page", [
    ("bf16", 128, 7, 16), ("bf16", 64, 8, 32), ("f32", 128, 4, 16),
    ("f32", 64, 1, 64)])
@pytest.mark.parametrize("budget,window", [(0, 1), (1, 1), (5, 2), (40, 3),
                                           (1000, 1)])
def test_attend_pages(dtype, d, G, page, budget, window):
    lens = [page * 50 + 3, 0, page * 6, 1, page * 43]
    b = Book(5, 1, 2, G, d, 103, page, 60, dtype, "f32")
    b.grow(lens)
    b.check_pages(budget, window)
    b.c.sync_status()


@pytest.mark.parametrize("dtype,d,page", [("bf16", 128, 16), ("bf16", 64, 32),
                                          ("f32", 128, 16), ("f32", 64, 16)])
def test_attend_pages_of_many_units(dtype, d, page):
    """Scores and choice in launches of their own: all layers of a batch."""
    lens = [page * 40 + 1, 0, page * 33, page * 9 + 5, page * 40, page * 12]
    b = Book(6, 4, 2, 3, d, 136, page, 41, dtype, "f32")
    b.grow(lens)
    for budget, window in ((1, 1), (7, 3), (30, 1), (0, 2)):
        b.check_pages(budget, window)
    b.c.sync_status()


def test_many_pages_of_fp32():
    b = Book(1, 1, 1, 2, 64, 2200, 16, 2200, "f32")
    k = rnd(3, (1, 1, 16 * 2190, 1, 64), "f32")
    k[0, 0, 16 * 2000:] = k[0, 0, :16 * 190]
    b.grow([16 * 2190], k=k)
    for budget in (1, 60, 900):
        b.check_pages(budget, 2)


def test_equal_scores_keep_the_lower_page():
    """Every page alike, and pages alike in groups."""
    for dtype in ("bf16", "f32"):
        b = Book(1, 1, 1, 3, 128, 400, 16, 400, dtype, "f32")
        k = np.repeat(rnd(3, (1, 1, 1, 1, 128), dtype), 16 * 390, 2)
        b.grow([16 * 390], k=k)
        b.check_pages(7, 2)
        b = Book(1, 1, 1, 3, 128, 400, 16, 400, dtype, "f32")
        k = rnd(3, (1, 1, 16 * 13, 1, 128), dtype)
        b.grow([16 * 390], k=np.tile(k, (1, 1, 30, 1, 1)))
        for budget in (1, 30, 45, 61):
            b.check_pages(budget, 1)


@pytest.mark.parametrize("pages", [8190, 8193, 9000])
def test_more_pages_than_are_held_on_chip(pages):
    """Ordinary scores, and ties across the whole sequence."""
    b = Book(1, 1, 1, 2, 64, pages, 16, pages)
    k = rnd(3, (1, 1, 16 * pages, 1, 64))
    k[0, 0, 16 * (pages - 300):] = k[0, 0, :16 * 300]
    b.grow([16 * pages], k=k)
    for budget in (1, 100, 4000):
        b.check_pages(budget, 5)


def test_scores_that_round_alike():
    """Scores that differ by less than fp32 can tell: the choice is that of 64
    bits."""
    for dtype in ("bf16", "f32"):
        n = 120
        k = np.zeros((1, 1, 16 * n, 1, 128), np.float32)
        rng = np.random.default_rng(4)
        big = kv4.bf16(rng.standard_normal(64).astype(np.float32))
        k[..., :64] = big
        tiny = rng.permutation(n).astype(np.float32) * 2.0**-24
        k[0, 0, :, 0, 100] = np.repeat(kv4.bf16(tiny), 16)
        q = np.zeros((1, 1, 2, 128), np.float32)
        q[..., :64] = kv4.bf16(rng.standard_normal((2, 64)).astype(np.float32))
        q[..., 100] = 1.0
        b = Book(1, 1, 1, 2, 128, n, 16, n, dtype, "f32")
        b.grow([16 * n], k=k)
        b.check_pages(20, 1, q)
        b.check_pages(59, 1, q)


def test_nan_and_infinite_scores():
    """A NaN ranks above every number, whatever else is there."""
    for dtype in ("bf16", "f32"):
        b = Book(1, 1, 1, 2, 64, 40, 16, 40, dtype, "f32")
        k = rnd(3, (1, 1, 16 * 38, 1, 64), dtype)
        k[0, 0, 16 * 20 + 3, 0, 7] = np.nan
        k[0, 0, 16 * 9 + 1, 0, 8] = np.inf
        k[0, 0, 16 * 11 + 1, 0, 8] = -np.inf
        b.grow([16 * 38], k=k)
        q = np.abs(rnd(9, (1, 1, 2, 64), dtype)) + 1
        got = torch.empty((1, 1, 1, 4), dtype=torch.int32, device="cuda")
        for budget in (1, 2, 3):
            b.c.attend_pages(dev(q, dtype), budget, 1, pages=got[..., :budget + 1]
                             .contiguous())
        b.c.attend_pages(dev(q, dtype), 3, 1, pages=got)
        want = paged.choose(q[0, 0], b.k[0][0, 0], 16, 3, 1)
        assert got.flatten().tolist() == want
        assert 20 in want and 9 in want
        with pytest.raises(kvr.KvrError, match="non-finite"):
            b.c.sync_status()


# ---- how calls go together --------------------------------------------------

def test_a_captured_step_replays_as_sequences_grow():
    """plan, append and both attentions of every layer in one graph: lengths,
    tables and rows are the device's own."""
    S, L = 3, 2
    b = Book(S, L, 2, 7, 128, 40, 16, 20, out_dtype="f32")
    b.grow([30, 0, 77])
    c = b.c
    lens = i32([0] * S)
    k, v = (torch.zeros((S, L, 1, 2, 128), dtype=torch.bfloat16, device="cuda")
            for _ in range(2))
    q = torch.zeros((S, L, 14, 128), dtype=torch.bfloat16, device="cuda")
    slots = torch.zeros((S, 1), dtype=torch.int32, device="cuda")
    out, some = (torch.zeros((S, L, 14, 128), device="cuda") for _ in range(2))
    ws = c.attend_pages_workspace(3, 1)

    def step():
        c.plan(lens, 1, slots=slots)
        for l in range(L):
            part = [x[:, l:l + 1].contiguous() for x in (k, v, q)]
            c.append(part[0], part[1], slots, layers=(l, l + 1))
            out[:, l:l + 1] = c.attend(part[2], layers=(l, l + 1), workspace=ws)
            some[:, l:l + 1] = c.attend_pages(part[2], 3, 1, layers=(l, l + 1),
                                              workspace=ws)

    lens.copy_(i32(b.p.len))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()      # nothing grows
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(40):
        want = [n + 1 for n in b.p.len]
        if i == 10:
            want[2] = 0          # a sequence ends
        if i == 20:
            want[0] -= 8         # rejected
        x = [rnd(1000 + 10 * i + j, t.shape) for j, t in enumerate((k, v, q))]
        for t, y in zip((k, v, q), x):
            t.copy_(dev(y))
        lens.copy_(i32(want))
        old = list(b.p.len)
        graph.replay()
        b.p.plan(want, 1)
        for s in range(S):
            keep = min(old[s], want[s])
            for mine, y in ((b.k, x[0]), (b.v, x[1])):
                mine[s] = mine[s][:, :, :keep]
                if want[s] > keep:
                    mine[s] = np.concatenate(
                        (mine[s], y[s].transpose(0, 2, 1, 3)), 2)
        b.check_out(x[2], out.cpu().numpy())
        table, ln, free = c.tables_view()
        assert ln.tolist() == want
        np.testing.assert_array_equal(table.cpu().numpy(), b.p.table_array())
        chosen = np.full((S, L, 2, 4), -1)
        for s in range(S):
            for l in range(L):
                for h in range(2):
                    w = paged.choose(x[2][s, l, 7 * h:7 * h + 7], b.k[s][l, h],
                                     16, 3, 1)
                    chosen[s, l, h, :len(w)] = w
        b.check_out(x[2], some.cpu().numpy(), chosen)
    b.check_rows()
    c.sync_status()


def test_a_call_of_every_layer_equals_calls_by_layer():
    """Within rounding: the spans of warps differ."""
    b = Book(2, 3, 2, 5, 128, 40, 32, 20, out_dtype="f32")
    b.grow([500, 333])
    q = b.queries()
    whole = b.c.attend(dev(q))
    parts = torch.cat([b.c.attend(dev(q[:, l:l + 1]), layers=(l, l + 1))
                       for l in range(3)], 1)
    b.check_out(q, whole.cpu().numpy())
    b.check_out(q, parts.cpu().numpy())


def test_two_caches_and_two_streams():
    """Each on its own stream, with workspaces of the streams' own."""
    books, streams = [], [torch.cuda.Stream() for _ in range(2)]
    for i in range(2):
        b = Book(2, 2, 2, 7, 128, 60, 16, 40, out_dtype="f32")
        b.seed = 1000 * i
        b.grow([600, 77 + i])
        books.append((b, b.queries()))
    torch.cuda.synchronize()
    qs = [dev(q) for _, q in books]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            outs[i].append(books[i][0].c.attend(qs[i], stream=s))
            outs[i].append(books[i][0].c.attend_pages(qs[i], 60, 1, stream=s))
    torch.cuda.synchronize()
    for i, (b, q) in enumerate(books):
        for x in outs[i]:
            b.check_out(q, x.cpu().numpy())


def test_refusals():
    b = Book(2, 2, 2, 7, 128, 8, 16, 4)
    b.grow([5, 0])
    q = dev(b.queries())
    c = b.c
    for call in (lambda: c.attend(q[:, :1].contiguous(), layers=(1, 1)),
                 lambda: c.attend(q, layers=(1, 3)),
                 lambda: c.attend_pages(q, -1, 2), lambda: c.attend_pages(q, 1, 0),
                 lambda: c.attend_pages(q, 1 << 24, 1),
                 lambda: c.attend_pages_workspace(1, 0),
                 lambda: c.attend_workspace((0, 5))):
        with pytest.raises((kvr.KvrError, ValueError)):
            call()
    ws = c.attend_workspace()
    with pytest.raises(kvr.KvrError, match="KVR_ENOMEM"):
        c.attend(q, workspace=ws[:-16])
    with pytest.raises(kvr.KvrError, match="KVR_ENOMEM"):
        c.attend_pages(q, 1, 1, workspace=ws)
    with pytest.raises(kvr.KvrError, match="aligned"):
        c.attend(q, workspace=torch.empty(ws.numel() + 8, dtype=torch.uint8,
                                          device="cuda")[8:])
    odd = torch.empty(q.numel() + 4, dtype=q.dtype, device="cuda")[4:]
    with pytest.raises(kvr.KvrError, match="aligned"):
        c.attend(odd.view(q.shape))
    n = c.launch_count()
    c.attend(q)
    assert c.launch_count() == n + 1
    c.sync_status()


# ---- sizes that pass 32 bits, and long ones ---------------------------------

def test_offsets_past_32_bits():
    """Rows in pages whose place in the pool passes 2^32 bytes and 2^31
    elements, keys and values alike."""
    S, L, H, G, d, P, n_pages = 2, 2, 8, 2, 128, 64, 20000
    c = kvr.PagedCache(S, L, H, G, d, n_pages, P, n_pages - 50)
    first = n_pages - 60
    c.plan(i32([first * P, 0]), first * P)
    n = 300
    slots = c.plan(i32([first * P, n]), n)
    c.plan(i32([0, n]))
    assert int(c.tables_view()[0][1, 0]) == first
    assert 2 * ((n_pages * L - 60) * H * P * d) > 2**32
    k, v = (rnd(i, (1, L, n, H, d), heavy=True) for i in (1, 2))
    c.append(dev(k), dev(v), slots[1:])
    q = rnd(3, (S, L, H * G, d))
    pages = torch.empty((S, L, H, 3), dtype=torch.int32, device="cuda")
    out = c.attend(dev(q)).float().cpu().numpy()
    some = c.attend_pages(dev(q), 2, 1, pages=pages).float().cpu().numpy()
    pages = pages.cpu().numpy()
    assert (out[0] == 0).all() and (some[0] == 0).all()
    for l in range(L):
        for h in range(H):
            g = slice(G * h, G * h + G)
            kk, vv = k[0, l, :, h], v[0, l, :, h]
            want = paged.choose(q[1, l, g], kk, P, 2, 1)
            assert pages[1, l, h].tolist() == want
            for got, rows in ((out, np.arange(n)),
                              (some, paged.rows_of(want, n, P))):
                ref, mag, top = paged.attend(q[1, l, g], kk[rows], vv[rows])
                tol = 2.0**-8 * np.abs(ref) + mag * (
                    2 * 2.0**-16 * top[:, None] + 2.0**-15) + 1e-30
                assert (np.abs(got[1, l, g] - ref) <= tol).all()
    c.sync_status()


def test_a_very_long_sequence():
    """Four million rows of one unit: all of them, and 65 of 262,145 pages.  A
    warp of 608 sums 432 tiles one after the other, and as many parts are joined:
    2^-13 covers what their sums round by."""
    n, d, P = (1 << 22) + 5, 64, 16
    pages = -(-n // P)
    g = torch.Generator(device="cuda").manual_seed(5)
    k, v = (torch.randn((1, 1, n, 1, d), generator=g, device="cuda",
                        dtype=torch.bfloat16) for _ in range(2))
    c = kvr.PagedCache(1, 1, 1, 2, d, pages, P, pages, out_dtype="f32")
    c.append(k, v, c.plan(i32([n]), n))
    q = dev(rnd(6, (1, 1, 2, d)))
    qd = q[0, 0].double()

    def check(out, kk, vv):
        x = qd @ kk.double().T / 8.0
        p = torch.softmax(x, -1)
        ref, mag = p @ vv.double(), p @ vv.double().abs()
        top = (qd.abs() @ kk.double().abs().T).amax(-1, keepdim=True) / 8.0
        tol = mag * (2 * 2.0**-16 * top + 2.0**-13 + 2.0**-15)
        assert ((out[0, 0].double() - ref).abs() <= tol).all()

    check(c.attend(q), k[0, 0, :, 0], v[0, 0, :, 0])
    got = torch.empty((1, 1, 1, 65), dtype=torch.int32, device="cuda")
    out = c.attend_pages(q, 64, 1, pages=got)
    full = k[0, 0, :(n // P) * P, 0].view(-1, P, d)
    lo, hi = full.amin(1).double(), full.amax(1).double()
    score = (qd.clamp(min=0) @ hi.T + qd.clamp(max=0) @ lo.T).amax(0)
    order = torch.sort(score, descending=True, stable=True).indices[:64]
    want = torch.cat((order.sort().values,
                      torch.tensor([pages - 1], device="cuda")))
    assert torch.equal(got.flatten().long(), want)
    rows = (want[:, None] * P + torch.arange(P, device="cuda")).flatten()
    rows = rows[rows < n]
    check(out, k[0, 0, rows, 0], v[0, 0, rows, 0])
    c.sync_status()
