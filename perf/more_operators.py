"""The operators around a paged full-context cache, as they are timed, with their
plain forms.

A server whose sequences come and go keeps the full context in pages of a pool
that all of them share.  Four operators carry a decode step over it:

  plan     from the lengths that the sequences are to have: pages taken and
           given back, the tables of pages, and the slots of the new tokens
  append   the new tokens' keys and values go to their slots; a page that is
           full gets the least and the greatest key of every channel
  attend   attention of one new token a sequence over all of its pages
  sparse   attention of one new token over some of them: the newest, and those
           whose least and greatest keys promise the greatest logits

Free pages are a stack, page 0 on top at first.  The i-th page that a call takes,
in order of sequence and page, is the i-th from the top; of those it gives back
(before it takes any) the first comes to lie on top.

A page's score for a query is the greatest, over the query heads that share its
KV head, of sum_c max(q_c, 0) hi_c + min(q_c, 0) lo_c: no logit of its rows is
above it.  Equal scores keep the lower page.
"""
from __future__ import annotations

import math

import torch

own = False

# layers, KV heads, query heads per KV head, head dim, element type
GEOMETRY = {
    "tiny": (1, 2, 2, 64, "f32"),
    "1p5b": (28, 2, 6, 128, "bf16"),
    "7b": (28, 4, 7, 128, "bf16"),
    "72b": (80, 8, 8, 128, "bf16"),
}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
HEAVY_FRAC, HEAVY_SCALE = 0.05, 3.0
TOPIC_ROWS, TOPIC_SCALE = 64, 0.7
MOST_ROWS = 16 * 16384 * 56     # cached rows (token, layer, head) of a case
MOST_SPARSE = 131072 * 112      # the same where most of them are not read
MOST_READ = 131072 * 28         # rows that a sparse case reads
MOST_NEW = 2 * 8191 * 56        # appended rows of a case
MOST_SLOTS = 256 * 8191         # slots of a plan


def listed():
    return [
        # Rejected drafts leave, the next five tokens of a whole batch get
        # their slots: once a decode step, latency.
        dict(name="plan_64seq_5tok", kind="plan", n_seq=64, tokens=5, page=64,
             shortest=512, longest=16384, empty=False),
        # A queue of prompts is admitted at once to an empty pool.
        dict(name="plan_256seq_prompts", kind="plan", n_seq=256, tokens=8191,
             page=16, shortest=100, longest=8191, empty=True),
        # One decoded token of a single user's sequence: latency.
        dict(name="append_7b_1seq_1tok", kind="append", geometry="7b",
             n_seq=1, tokens=1, page=16, shortest=4099, longest=4099),
        # One decoded token of a whole batch; some of them fill their page.
        dict(name="append_7b_64seq_1tok", kind="append", geometry="7b",
             n_seq=64, tokens=1, page=64, shortest=63, longest=1023),
        # Two prompts of odd length.
        dict(name="append_1p5b_2seq_8191", kind="append", geometry="1p5b",
             n_seq=2, tokens=8191, page=64, shortest=0, longest=0),
        # The smallest attention: one layer, fp32, head dim 64.
        dict(name="attend_tiny_f32", kind="attend", geometry="tiny", n_seq=1,
             page=16, shortest=129, longest=129, idle=False, by_layer=False),
        # One user's token as a model decodes it, a call a layer.
        dict(name="attend_7b_1seq_by_layer", kind="attend", geometry="7b",
             n_seq=1, page=16, shortest=4099, longest=4099, idle=False,
             by_layer=True),
        # The full-context helper's step at its longest context.
        dict(name="attend_1p5b_16seq_16k", kind="attend", geometry="1p5b",
             n_seq=16, page=64, shortest=16384, longest=16384, idle=False,
             by_layer=False),
        # A batch of very different contexts, one place of it free.
        dict(name="attend_7b_28seq_ragged", kind="attend", geometry="7b",
             n_seq=28, page=32, shortest=512, longest=16384, idle=True,
             by_layer=False),
        # A long document of one user, a call a layer: 32 of 513 pages.
        dict(name="sparse_7b_1seq_by_layer", kind="sparse", geometry="7b",
             n_seq=1, page=64, shortest=32771, longest=32771, budget=28,
             window=4, idle=False, by_layer=True),
        # Several of them in one call.
        dict(name="sparse_7b_6seq_16k_32k", kind="sparse", geometry="7b",
             n_seq=6, page=64, shortest=16384, longest=30000, budget=56,
             window=8, idle=False, by_layer=False),
        # The longest context, small pages: 4,096 of them to choose from.
        dict(name="sparse_7b_1seq_131k", kind="sparse", geometry="7b",
             n_seq=1, page=32, shortest=131072, longest=131072, budget=120,
             window=8, idle=False, by_layer=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithm."""
    kind = rng.choice(["plan", "append", "attend", "attend", "sparse",
                       "sparse"])
    page = rng.choice([16, 32, 64, 128])
    if kind == "plan":
        empty = rng.random() < 0.4
        n_seq = _log_int(rng, 1, 256)
        tokens = _log_int(rng, 1, min(8191, MOST_SLOTS // n_seq)) if empty \
            else rng.randint(1, 8)
        most = tokens if empty else 16384
        lo, hi = sorted(_log_int(rng, 1, most) for _ in range(2))
        return dict(kind=kind, n_seq=n_seq, tokens=tokens, page=page,
                    shortest=lo, longest=hi, empty=empty)
    geometry = rng.choice(["7b", "7b", "1p5b", "72b", "tiny"])
    layers, heads = GEOMETRY[geometry][:2]
    units = layers * heads
    if kind == "append":
        tokens = rng.choice([1, _log_int(rng, 1, 8191)])
        tokens = min(tokens, MOST_NEW // units)
        n_seq = min(_log_int(rng, 1, 64), max(1, MOST_NEW // (units * tokens)))
        most = min(1024, MOST_ROWS // (2 * units * n_seq))
        lo, hi = sorted(_log_int(rng, 1, most) for _ in range(2))
        return dict(kind=kind, geometry=geometry, n_seq=n_seq, tokens=tokens,
                    page=page, shortest=lo if n_seq > 1 else hi, longest=hi)
    sparse = kind == "sparse"
    most = (MOST_SPARSE if sparse else MOST_ROWS) // units
    lo, hi = sorted(_log_int(rng, 30, min(131072 if sparse else 16384, most))
                    for _ in range(2))
    n_seq = max(1, min(_log_int(rng, 1, 64), most // hi))
    more = {}
    if sparse:
        read = max(2, MOST_READ // (units * n_seq * page))
        keep = _log_int(rng, 2, min(read, 256))
        window = rng.randint(1, max(1, min(16, keep // 2)))
        more = dict(budget=keep - window, window=window)
    return dict(kind=kind, geometry=geometry, n_seq=n_seq, page=page,
                shortest=lo if n_seq > 1 else hi, longest=hi, **more,
                idle=n_seq > 2 and rng.random() < 0.5, by_layer=n_seq == 1)


# ---- inputs -----------------------------------------------------------------

def _gen(seed, *tags):
    g = torch.Generator(device="cuda")
    mixed = int(seed)
    for t in tags:
        mixed = (mixed * 1000003 + t + 1) % (1 << 40)
    g.manual_seed(mixed * 7919 + 17)
    return g


def _normal(g, shape, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _lengths(case):
    """Cached rows of each sequence: shortest to longest in equal ratios; one in
    the middle is idle where the case says so."""
    n, lo, hi = case["n_seq"], case["shortest"], case["longest"]
    lens = [hi] * n if n == 1 or lo == hi else \
        [int(round(lo * (hi / lo) ** (s / (n - 1)))) for s in range(n)]
    if case.get("idle"):
        lens[n // 2] = 0
    return lens


def _targets(case, seed):
    """Of a plan: the lengths before the new tokens, and with them.  Sequences
    come in any order, and end anywhere in their last page."""
    n = torch.tensor(_lengths(case))
    g = torch.Generator()
    g.manual_seed(int(seed) * 31 + 5)
    n = n[torch.randperm(len(n), generator=g)]
    inside = (n - 1) % case["page"] + 1
    n -= (torch.rand(len(n), generator=g) * inside).long()
    if case["empty"]:
        return [0] * len(n), n.tolist()
    more = torch.randint(0, case["tokens"] + 1, n.shape, generator=g)
    return n.tolist(), (n + more).tolist()


def _rows(case, seed, s, n):
    """Sequence s's n keys and values, [L][n][H][d]; 5% of the keys scaled by 3.
    Where pages are chosen, groups of keys share a direction, as the passages of
    a document do: that is what makes one page better than another."""
    L, H, _, d, dtype = GEOMETRY[case["geometry"]]
    g = _gen(seed, 1, s)
    dt = DTYPES[dtype]
    k = _normal(g, (L, n, H, d), dt)
    heavy = torch.rand((L, n, H), generator=g, device="cuda") < HEAVY_FRAC
    k *= torch.where(heavy, HEAVY_SCALE, 1.0).to(dt)[..., None]
    if case["kind"] == "sparse":
        many = -(-n // TOPIC_ROWS)
        t = TOPIC_SCALE * _normal(g, (L, many, H, d), dt)
        k += t.repeat_interleave(TOPIC_ROWS, dim=1)[:, :n]
    return k, _normal(g, (L, n, H, d), dt)


def _new_rows(case, seed):
    L, H, _, d, dtype = GEOMETRY[case["geometry"]]
    g = _gen(seed, 2)
    shape = (case["n_seq"], L, case["tokens"], H, d)
    return tuple(_normal(g, shape, DTYPES[dtype]) for _ in range(2))


def _queries(case, seed):
    L, H, G, d, dtype = GEOMETRY[case["geometry"]]
    return _normal(_gen(seed, 3), (case["n_seq"], L, H * G, d), DTYPES[dtype])


# ---- the plain forms --------------------------------------------------------

class _Pool:
    """A plain paged cache: tables, a stack of free pages, rows and bounds."""

    def __init__(self, S, n_pages, page, table_pages, geometry=None):
        z = dict(device="cuda")
        self.P = page
        self.table = torch.full((S, table_pages), -1, dtype=torch.int32, **z)
        self.lens = torch.zeros(S, dtype=torch.int32, **z)
        self.stack = torch.arange(n_pages - 1, -1, -1, dtype=torch.int32, **z)
        self.free = torch.full((1,), n_pages, dtype=torch.int32, **z)
        if geometry is not None:
            L, H, _, d, dtype = GEOMETRY[geometry]
            z["dtype"] = DTYPES[dtype]
            self.k = torch.zeros((L, n_pages, H, page, d), **z)
            self.v = torch.zeros((L, n_pages, H, page, d), **z)
            self.bounds = torch.zeros((L, n_pages, H, 2, d), **z)

    def plan(self, want, n_new=0):
        """Lengths become `want`; slots [S][n_new] of the tokens that come."""
        P, table = self.P, self.table
        have = (self.lens.long() + P - 1) // P
        need = (want.long() + P - 1) // P
        at = torch.arange(table.shape[1], device="cuda")
        gone = (at >= need[:, None]) & (at < have[:, None])
        come = (at >= have[:, None]) & (at < need[:, None])
        back = table[gone]              # in order of sequence and page
        top = int(self.free) + back.numel()
        self.stack[top - back.numel():top] = back.flip(0)
        table[gone] = -1
        taken = int(come.sum())
        table[come] = self.stack[top - taken:top].flip(0)
        self.free.fill_(top - taken)
        old = self.lens.long()
        self.lens.copy_(want)
        if not n_new:
            return None
        pos = old[:, None] + torch.arange(n_new, device="cuda")
        new = pos < want[:, None]
        pos = torch.where(new, pos, 0)
        slot = table.long().gather(1, pos // P) * P + pos % P
        return torch.where(new, slot, -1).to(torch.int32)

    def append(self, k, v, slots):
        """k, v [N][L][T][H][d], slots [N][T] (-1: no token)."""
        P = self.P
        n, t = torch.nonzero(slots >= 0, as_tuple=True)
        slot = slots[n, t].long()
        page, row = slot // P, slot % P
        full = page[row == P - 1]
        for l in range(k.shape[1]):
            self.k[l][page, :, row] = k[n, l, t]
            self.v[l][page, :, row] = v[n, l, t]
            rows = self.k[l][full]      # [full pages][H][P][d]
            self.bounds[l][full] = torch.stack((rows.amin(2), rows.amax(2)), 2)


def _plain_softmax(q, k, v, sees):
    """Attention of q [S][H][G][d] over k, v [S][H][n][d] where sees [S][n] or
    [S][H][n], in 32 bits."""
    if sees.dim() == 2:
        sees = sees[:, None]
    x = torch.matmul(q.float(), k.float().transpose(-1, -2))
    x = (x / math.sqrt(q.shape[-1])).masked_fill(~sees[:, :, None], -math.inf)
    p = torch.exp(x - x.amax(-1, keepdim=True).clamp(min=-1e30))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    return torch.matmul(p, v.float()).to(q.dtype)


def _plain_attend(pool, q):
    S, L, HG, d = q.shape
    H, P = pool.k.shape[2], pool.P
    most = (int(pool.lens.max()) + P - 1) // P
    pages = pool.table[:, :most].long().clamp(min=0)
    sees = torch.arange(most * P, device="cuda") < pool.lens[:, None]
    out = torch.empty_like(q)
    for l in range(L):
        k, v = (x[l][pages].transpose(1, 2).reshape(S, H, most * P, d)
                for x in (pool.k, pool.v))
        qs = q[:, l].view(S, H, HG // H, d)
        out[:, l] = _plain_softmax(qs, k, v, sees).reshape(S, HG, d)
    return out


def _plain_select(pool, l, q, budget, window):
    """Pages [S][H][budget + window], ascending, then -1, for q [S][H][G][d]."""
    S, H = q.shape[:2]
    P = pool.P
    have = (pool.lens.long() + P - 1) // P
    most = int(have.max())
    pages = pool.table[:, :most].long().clamp(min=0)
    b = pool.bounds[l][pages].double().permute(0, 2, 1, 3, 4)  # [S][H][.][2][d]
    qd = q.double()
    x = torch.matmul(qd.clamp(min=0), b[..., 1, :].transpose(-1, -2)) \
        + torch.matmul(qd.clamp(max=0), b[..., 0, :].transpose(-1, -2))
    x = x.amax(2)                                              # [S][H][.]
    got = torch.full((S, H, budget + window), -1, device="cuda")
    for s, n in enumerate(have.tolist()):
        old = max(n - window, 0)
        best = torch.sort(x[s, :, :old], dim=-1, descending=True,
                          stable=True).indices[:, :budget]
        new = torch.arange(old, n, device="cuda").expand(H, n - old)
        kept = torch.cat((best, new), -1).sort(dim=-1).values
        got[s, :, :kept.shape[1]] = kept
    return got


def _plain_sparse(pool, q, budget, window):
    S, L, HG, d = q.shape
    H, P = pool.k.shape[2], pool.P
    heads = torch.arange(H, device="cuda")[:, None]
    out = torch.empty_like(q)
    chosen = torch.empty((S, L, H, budget + window), dtype=torch.int32,
                         device="cuda")
    for l in range(L):
        qs = q[:, l].view(S, H, HG // H, d)
        kept = _plain_select(pool, l, qs, budget, window)
        chosen[:, l] = kept
        # a page's place in the pool, per sequence and head
        at = pool.table.long()[:, None].expand(S, H, -1).gather(
            2, kept.clamp(min=0)).clamp(min=0)
        k, v = (x[l][at, heads].reshape(S, H, -1, d) for x in (pool.k, pool.v))
        row = kept[..., None] * P + torch.arange(P, device="cuda")
        sees = (kept[..., None] >= 0) & (row < pool.lens[:, None, None, None])
        out[:, l] = _plain_softmax(qs, k, v, sees.reshape(S, H, -1)).reshape(
            S, HG, d)
    return out, chosen


# ---- a state, and one pass --------------------------------------------------

def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _pages_of(lens, page):
    return [-(-n // page) for n in lens]


def _fill(cache, case, seed, lens):
    """The sequences' rows, as a server comes by them: prompts in two parts, so
    that the pages of one sequence do not lie side by side."""
    half = [n // 2 for n in lens]
    parts = []
    for a, b in (([0] * len(lens), half), (half, lens)):
        most = max(y - x for x, y in zip(a, b))
        parts.append(cache.plan(_i32(b), most) if most else None)
    for s, n in enumerate(lens):
        if not n:
            continue
        slots = torch.cat([p[s:s + 1, :m] for p, m in
                           zip(parts, (half[s], n - half[s])) if m], 1)
        k, v = _rows(case, seed, s, n)
        cache.append(k[None], v[None], slots.contiguous())


def prepare(case, seed):
    kind, page, S = case["kind"], case["page"], case["n_seq"]
    st = {"kind": kind, "own": own}
    if own:
        from paper_2608_15797_gb300 import kvr
    if kind == "plan":
        base, want = _targets(case, seed)
        most = max(_lengths(case)) + (0 if case["empty"] else case["tokens"])
        pages, table = sum(_pages_of(want, page)) + 64, -(-most // page)
        # a plan does not touch rows: the smallest cache that has these tables
        if own:
            cache = kvr.PagedCache(S, 1, 1, 1, 64, pages, page_rows=page,
                                   table_pages=table)
        else:
            cache = _Pool(S, pages, page, table)
        half = [n // 2 for n in base]
        most = max(max(half), max(b - h for b, h in zip(base, half)), 1)
        for n in (half, base):
            cache.plan(_i32(n), most)
        st.update(cache=cache, base=_i32(base), want=_i32(want),
                  tokens=case["tokens"])
        if own:
            st["slots"] = torch.empty((S, case["tokens"]), dtype=torch.int32,
                                      device="cuda")
        return st
    L, H, G, d, dtype = GEOMETRY[case["geometry"]]
    lens = _lengths(case)
    new = case["tokens"] if kind == "append" else 0
    many = _pages_of([n + new for n in lens], page)
    if own:
        desc = (S, L, H, G, d, sum(many))
        more = dict(page_rows=page, table_pages=max(many), dtype=dtype,
                    out_dtype=dtype)
        room = torch.zeros(kvr.PagedCache.required_bytes(*desc, **more),
                           dtype=torch.uint8, device="cuda")
        cache = kvr.PagedCache(*desc, **more, buf=room)
    else:
        cache = _Pool(S, sum(many), page, max(many), case["geometry"])
    _fill(cache, case, seed, lens)
    st["cache"] = cache
    if kind == "append":
        st["new"] = _new_rows(case, seed)
        st["slots"] = cache.plan(_i32([n + new for n in lens]), new)
        return st
    st["q"], st["by_layer"] = _queries(case, seed), case["by_layer"]
    if kind == "sparse":
        st.update(budget=case["budget"], window=case["window"])
    if own:
        keep = case.get("budget", 0) + case.get("window", 0)
        layers = (0, 1) if case["by_layer"] else None
        st["workspace"] = cache.attend_workspace(layers) if kind == "attend" \
            else cache.attend_pages_workspace(case["budget"], case["window"],
                                              layers)
        st["out"] = torch.empty((S, L, H * G, d), dtype=DTYPES[dtype],
                                device="cuda")
        st["pages"] = torch.empty((S, L, H, keep), dtype=torch.int32,
                                  device="cuda")
        if case["by_layer"]:   # (one sequence: a layer's part is dense)
            st["q"] = [st["q"][:, l:l + 1].contiguous() for l in range(L)]
    return st


def _own_attend(st, q, out, pages, layers):
    cache = st["cache"]
    if st["kind"] == "attend":
        cache.attend(q, out=out, layers=layers, workspace=st["workspace"])
    else:
        cache.attend_pages(q, st["budget"], st["window"], out=out, pages=pages,
                           layers=layers, workspace=st["workspace"])


def run(st):
    kind, cache = st["kind"], st["cache"]
    if kind == "plan":
        cache.plan(st["base"])
        if st["own"]:
            slots = cache.plan(st["want"], st["tokens"], slots=st["slots"])
            table, lens, free = cache.tables_view()
            return {"slots": slots, "table": table, "lens": lens, "free": free}
        slots = cache.plan(st["want"], st["tokens"])
        return {"slots": slots, "table": cache.table, "lens": cache.lens,
                "free": cache.free}
    if kind == "append":
        cache.append(*st["new"], st["slots"])
        if st["own"]:
            (k, v), bounds = cache.rows_view(), cache.bounds_view()
            return {"k": k, "v": v, "bounds": bounds}
        return {"k": cache.k, "v": cache.v, "bounds": cache.bounds}
    if not st["own"]:
        if kind == "attend":
            return {"out": _plain_attend(cache, st["q"])}
        out, pages = _plain_sparse(cache, st["q"], st["budget"], st["window"])
        return {"out": out, "pages": pages}
    if st["by_layer"]:
        for l, q in enumerate(st["q"]):
            _own_attend(st, q, st["out"][:, l:l + 1], st["pages"][:, l:l + 1],
                        (l, l + 1))
    else:
        _own_attend(st, st["q"], st["out"], st["pages"], None)
    return {"out": st["out"]} if kind == "attend" else \
        {"out": st["out"], "pages": st["pages"]}


def work(case):
    kind, page = case["kind"], case["page"]
    if kind == "plan":
        S = case["n_seq"]
        lens = _lengths(case)
        new = sum(_pages_of(lens, page)) if case["empty"] else S
        # lengths read and written twice; pages taken and given back: stack
        # and table
        return {"bytes": 4 * S * case["tokens"] + 16 * S + 16 * new,
                "flops": S * case["tokens"] * 4}
    L, H, G, d, dtype = GEOMETRY[case["geometry"]]
    es = 2 if dtype == "bf16" else 4
    if kind == "append":
        rows = case["n_seq"] * case["tokens"] * L * H
        full = sum((n + case["tokens"]) // page - n // page
                   for n in _lengths(case)) * L * H
        return {"bytes": rows * 4 * d * es + full * 2 * d * es
                + 4 * case["n_seq"] * case["tokens"],
                "flops": full * page * 2 * d}
    lens = _lengths(case)
    ends = case["n_seq"] * L * H * G * d * 2 * es    # q and the outputs
    if kind == "attend":
        rows = sum(lens) * L * H
        return {"bytes": rows * 2 * d * es + ends, "flops": rows * G * 4 * d}
    B, W = case["budget"], case["window"]
    rows = scored = 0
    for n in lens:
        have = -(-n // page)
        kept = min(have, B + W)
        rows += n - (have - kept) * page
        scored += max(have - W, 0) if have > kept else 0
    rows, scored = rows * L * H, scored * L * H
    return {"bytes": rows * 2 * d * es + scored * 2 * d * es + ends
            + 4 * case["n_seq"] * L * H * (B + W),
            "flops": rows * G * 4 * d + scored * G * 4 * d}


# ---- the definitions in 64 bits ---------------------------------------------

def _exact_pool(case, seed):
    """The pool after an append: rows and bounds, page by page."""
    L, H, _, d, _ = GEOMETRY[case["geometry"]]
    P, S, new = case["page"], case["n_seq"], case["tokens"]
    lens = _lengths(case)
    total = sum(_pages_of([n + new for n in lens], P))
    k, v = (torch.zeros((L, total, H, P, d), dtype=torch.float64, device="cuda")
            for _ in range(2))
    bounds = torch.zeros((L, total, H, 2, d), dtype=torch.float64,
                         device="cuda")
    # pages go to the halves of all sequences, then to their ends, then to the
    # new tokens, from page 0 on
    owner, page = [[] for _ in range(S)], 0
    for upto in ([n // 2 for n in lens], lens, [n + new for n in lens]):
        for s in range(S):
            while len(owner[s]) * P < upto[s]:
                owner[s].append(page)
                page += 1
    kn, vn = _new_rows(case, seed)
    for s in range(S):
        ko, vo = _rows(case, seed, s, lens[s])
        n = lens[s] + new
        for pool, old, fresh in ((k, ko, kn), (v, vo, vn)):
            rows = torch.cat((old, fresh[s]), 1).double()       # [L][n][H][d]
            for i, p in enumerate(owner[s]):
                part = rows[:, i * P:min((i + 1) * P, n)].transpose(1, 2)
                pool[:, p, :, :part.shape[2]] = part
                if pool is k and part.shape[2] == P:
                    bounds[:, p, :, 0] = part.min(2).values
                    bounds[:, p, :, 1] = part.max(2).values
    return {"k": k, "v": v, "bounds": bounds}


def _exact_attention(q, k, v):
    """q [H][G][d] over k, v [H][n][d], 64 bits."""
    x = torch.einsum("hgd,hnd->hgn", q, k) / math.sqrt(q.shape[-1])
    return torch.einsum("hgn,hnd->hgd", torch.softmax(x, -1), v)


def _exact_attends(case, seed):
    L, H, G, d, _ = GEOMETRY[case["geometry"]]
    S, P = case["n_seq"], case["page"]
    sparse = case["kind"] == "sparse"
    q = _queries(case, seed).double().view(S, L, H, G, d)
    out = torch.zeros_like(q)
    if sparse:
        B, W = case["budget"], case["window"]
        pages = torch.full((S, L, H, B + W), -1, dtype=torch.int32,
                           device="cuda")
    for s, n in enumerate(_lengths(case)):
        if not n:
            continue
        k, v = _rows(case, seed, s, n)
        have = -(-n // P)
        for l in range(L):
            kl, vl = k[l].transpose(0, 1), v[l].transpose(0, 1)    # [H][n][d]
            if not sparse:
                out[s, l] = _exact_attention(q[s, l], kl.double(), vl.double())
                continue
            kept = torch.arange(have, device="cuda").expand(H, have)
            old = max(have - W, 0)
            if have > B + W:
                block = kl[:, :old * P].reshape(H, old, P, d)
                lo = block.min(2).values.double()
                hi = block.max(2).values.double()
                # a channel gives at most q hi or q lo, whichever is greater
                bound = torch.stack([
                    torch.maximum(q[s, l, :, g, None] * hi,
                                  q[s, l, :, g, None] * lo).sum(-1)
                    for g in range(G)]).max(0).values           # [H][old]
                order = torch.argsort(-bound, dim=-1, stable=True)[:, :B]
                kept = torch.cat((order, kept[:, old:]), -1).sort(-1).values
            pages[s, l, :, :kept.shape[1]] = kept
            row = (kept[..., None] * P
                   + torch.arange(P, device="cuda")).reshape(H, -1)
            inside = row < n    # the newest page ends where the sequence does
            row = row[inside].view(H, -1)[..., None].expand(-1, -1, d)
            out[s, l] = _exact_attention(q[s, l], kl.gather(1, row).double(),
                                         vl.gather(1, row).double())
    out = out.view(S, L, H * G, d)
    return {"out": out, "pages": pages} if sparse else {"out": out}


def exact(case, seed):
    if case["kind"] == "plan":
        return None      # whole numbers alone
    if case["kind"] == "append":
        return _exact_pool(case, seed)
    return _exact_attends(case, seed)
