"""The operators around a full-context cache held in 4 bits, as they are timed,
with their plain forms.

A program that decodes with an evicted cache can draft with it: the drafter
decodes a few tokens from its budget of rows, and one pass over the full
context, held in 4 bits, says which of them the model itself would have
emitted.  Four operators carry that:

  append  quantise new tokens' keys and values into the 4-bit cache
  attend  causal attention of a sequence's newest tokens over it; optionally
          each cached row's accumulated attention weight
  evict   the rows of highest accumulated weight, and the newest ones, as the
          drafter's evicted cache
  verify  drafted tokens accepted or rejected against the target's
          probabilities, and the token that follows them

The 4-bit format: 64 channels of one token and head share a scale s and a
minimum m, both bfloat16.  With lo and hi their least and greatest value,
m = bf16(lo), s = bf16(hi * (1/15) - lo * (1/15)), and the code of x is
(x - m) / s rounded to the nearest even whole number within 0..15 (0 where s
is 0); it stands for m + s * code.
"""
from __future__ import annotations

import math

import torch

own = False

GROUP = 64
# layers, KV heads, query heads per KV head, head dim, element type
GEOMETRY = {
    "tiny": (1, 2, 2, 64, "f32"),
    "1p5b": (28, 2, 6, 128, "bf16"),
    "7b": (28, 4, 7, 128, "bf16"),
    "72b": (80, 8, 8, 128, "bf16"),
}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
VOCAB = 152064
HEAVY_FRAC, HEAVY_SCALE = 0.05, 3.0
MOST_ROWS = 16 * 16384 * 56   # cached rows (token, layer, head) of a case
MOST_NEW = 2 * 8191 * 56      # appended rows of a case
MOST_PAIRS = 2 * 8191 * 112 * 32 * 7   # pairs of a query head and a row


def listed():
    return [
        # One decoded token of a single user's sequence enters the cache:
        # latency.
        dict(name="append_7b_1seq_1tok", kind="append", geometry="7b",
             n_seq=1, tokens=1, shortest=4099, longest=4099),
        # Four drafted tokens and the one before them, of a whole batch.
        dict(name="append_7b_64seq_5tok", kind="append", geometry="7b",
             n_seq=64, tokens=5, shortest=64, longest=1024),
        # Two prompts of odd length are stored.
        dict(name="append_1p5b_2seq_8191", kind="append", geometry="1p5b",
             n_seq=2, tokens=8191, shortest=0, longest=0),
        # The smallest attention: one layer, fp32, head dim 64.
        dict(name="attend_tiny_f32", kind="attend", geometry="tiny", n_seq=1,
             tokens=1, shortest=129, longest=129, scores=False, ragged=False,
             by_layer=False),
        # One user's token as a model decodes it, a call a layer.
        dict(name="attend_7b_1seq_by_layer", kind="attend", geometry="7b",
             n_seq=1, tokens=1, shortest=4099, longest=4099, scores=False,
             ragged=False, by_layer=True),
        # The full-context helper's step at its longest context.
        dict(name="attend_1p5b_16seq_16k", kind="attend", geometry="1p5b",
             n_seq=16, tokens=1, shortest=16384, longest=16384, scores=False,
             ragged=False, by_layer=False),
        # Four drafted tokens of each sequence verified at once, contexts of
        # very different lengths.
        dict(name="attend_7b_16seq_5tok", kind="attend", geometry="7b",
             n_seq=16, tokens=5, shortest=512, longest=16384, scores=False,
             ragged=False, by_layer=False),
        # The last 32 tokens of two prompts say which rows are worth keeping.
        dict(name="attend_7b_2seq_32tok_scores", kind="attend", geometry="7b",
             n_seq=2, tokens=32, shortest=8191, longest=8191, scores=True,
             ragged=False, by_layer=False),
        # A short prompt is cut to the smallest budget: latency.
        dict(name="evict_7b_1seq_2k_b64", kind="evict", geometry="7b",
             n_seq=1, budget=64, window=8, shortest=2048, longest=2048),
        # Long prompts of different lengths are cut to the paper's own budget
        # and window.
        dict(name="evict_7b_4seq_16k_b512", kind="evict", geometry="7b",
             n_seq=4, budget=512, window=128, shortest=4000, longest=16384),
        # A single user's three drafted tokens, fp32 logits.
        dict(name="verify_1x3_32000_f32", kind="verify", n_seq=1, tokens=3,
             vocab=32000, dtype="f32", temperature=1.0, top=0, ragged=False),
        # Four drafted tokens of a whole batch, full vocabulary.
        dict(name="verify_64x4_152064_bf16", kind="verify", n_seq=64,
             tokens=4, vocab=VOCAB, dtype="bf16", temperature=1.0, top=0,
             ragged=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges, sizes spread over their logarithm."""
    kind = rng.choice(["append", "attend", "attend", "evict", "verify"])
    if kind == "verify":
        tokens = rng.randint(1, 8)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = 64 * 9 // max(9, 2 * tokens + 1) // (1 if dtype == "bf16" else 2)
        return dict(kind=kind, n_seq=_log_int(rng, 1, most), tokens=tokens,
                    vocab=rng.choice([VOCAB, 151936, 50001, 32000]),
                    dtype=dtype,
                    temperature=rng.choice([1.0, 0.7]),
                    top=rng.choice([0, 0, 20]), ragged=rng.random() < 0.4)
    geometry = rng.choice(["7b", "7b", "1p5b", "72b", "tiny"])
    layers, heads, group = GEOMETRY[geometry][:3]
    if kind == "append":
        tokens = _log_int(rng, 1, 8191)
        most = max(1, MOST_NEW // (layers * heads * tokens))
        if most < 2:
            tokens = min(tokens, MOST_NEW // (layers * heads))
        lo, hi = sorted(_log_int(rng, 1, 1024) for _ in range(2))
        n_seq = min(_log_int(rng, 1, 64), most)
        return dict(kind=kind, geometry=geometry, n_seq=n_seq, tokens=tokens,
                    shortest=lo, longest=hi if n_seq > 1 else lo)
    if kind == "evict":
        n_seq = rng.randint(1, 4) if layers * heads < 300 else 1
        most = 16384 if layers * heads < 300 else 6400
        lo, hi = sorted(_log_int(rng, 700, most) for _ in range(2))
        return dict(kind=kind, geometry=geometry, n_seq=n_seq,
                    budget=rng.choice([64, 128, 256, 512]),
                    window=rng.choice([8, 32, 128]),
                    shortest=lo if n_seq > 1 else hi, longest=hi)
    tokens = rng.choice([1, 1, 2, 3, 5, 8, 17, 32])
    most = min(MOST_ROWS, MOST_PAIRS // (tokens * group)) // (layers * heads)
    lo, hi = sorted(_log_int(rng, 100, min(16384, most)) for _ in range(2))
    n_seq = max(1, min(_log_int(rng, 1, 16), most // hi))
    return dict(kind=kind, geometry=geometry, n_seq=n_seq, tokens=tokens,
                shortest=lo if n_seq > 1 else hi, longest=hi,
                scores=rng.random() < 0.3,
                ragged=tokens > 1 and rng.random() < 0.4,
                by_layer=tokens == 1 and n_seq == 1)


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


def _keys(g, shape, dtype):
    """N(0, 1) keys [..., d], 5% of the rows scaled by 3."""
    k = _normal(g, shape, dtype)
    heavy = torch.rand(shape[:-1], generator=g, device="cuda") < HEAVY_FRAC
    return torch.where(heavy[..., None], k * HEAVY_SCALE, k)


def _lengths(case):
    """Cached rows of each sequence: shortest to longest in equal ratios."""
    n, lo, hi = case["n_seq"], case["shortest"], case["longest"]
    if n == 1 or lo == hi:
        return [hi] * n
    return [int(round(lo * (hi / lo) ** (s / (n - 1)))) for s in range(n)]


def _counts(case, seed):
    """Tokens of each sequence in a ragged batch: 1 to `tokens`, or all."""
    n, most = case["n_seq"], case["tokens"]
    if not case.get("ragged"):
        return [most] * n
    g = torch.Generator()
    g.manual_seed(int(seed) * 31 + 5)
    return torch.randint(1, most + 1, (n,), generator=g).tolist()


def _rows(case, seed, s, n):
    """Sequence s's n cached keys and values, [L][H][n][d]."""
    L, H, _, d, dtype = GEOMETRY[case["geometry"]]
    g = _gen(seed, 1, s)
    dt = DTYPES[dtype]
    return _keys(g, (L, H, n, d), dt), _normal(g, (L, H, n, d), dt)


def _new_rows(case, seed):
    L, H, _, d, dtype = GEOMETRY[case["geometry"]]
    g = _gen(seed, 2)
    shape = (case["n_seq"], L, case["tokens"], H, d)
    return _keys(g, shape, DTYPES[dtype]), _normal(g, shape, DTYPES[dtype])


def _queries(case, seed):
    L, H, G, d, dtype = GEOMETRY[case["geometry"]]
    return _normal(_gen(seed, 3), (case["n_seq"], L, case["tokens"], H * G, d),
                   DTYPES[dtype])


def _weights(case, seed, s, n):
    """Accumulated attention weights of sequence s's rows, [L][H][n]: a few
    rows hold most of it."""
    L, H = GEOMETRY[case["geometry"]][:2]
    return torch.exp(2.0 * torch.randn((L, H, n), generator=_gen(seed, 4, s),
                                       device="cuda")) / n


def _drafts(case, seed):
    """Target and draft logits, drafted tokens (drawn from the draft), and the
    random numbers: one uniform a draft, one exponential a vocabulary entry."""
    g = _gen(seed, 5)
    S, T, V = case["n_seq"], case["tokens"], case["vocab"]
    dt = DTYPES[case["dtype"]]
    sharp = 2.0 + 2.0 * torch.rand((S, T + 1, 1), generator=g, device="cuda")
    target = sharp * torch.randn((S, T + 1, V), generator=g, device="cuda")
    draft = target[:, :T] + 0.7 * torch.randn((S, T, V), generator=g,
                                              device="cuda")
    if case["top"]:
        cut = torch.topk(target, case["top"], dim=-1).values[..., -1:]
        target = target.masked_fill(target < cut, -math.inf)
        cut = torch.topk(draft, case["top"], dim=-1).values[..., -1:]
        draft = draft.masked_fill(draft < cut, -math.inf)
    target, draft = target.to(dt), draft.to(dt)
    race = torch.empty((S, T, V), device="cuda").exponential_(generator=g)
    tokens = torch.argmax(draft.float() / case["temperature"]
                          - torch.log(race), dim=-1).to(torch.int32)
    u = torch.rand((S, T), generator=g, device="cuda")
    race = torch.empty((S, V), device="cuda").exponential_(generator=g)
    return target, draft, tokens, u, race.clamp_(min=1e-30)


# ---- the plain forms --------------------------------------------------------

def _quantise(x):
    """[..., d] to packed codes uint8 [..., d / 2] (even channel low), minima
    and scales bf16 [..., d / 64]."""
    x = x.float().unflatten(-1, (-1, GROUP))
    lo, hi = x.amin(-1), x.amax(-1)
    fifteenth = torch.tensor(1.0 / 15.0, dtype=torch.float32, device=x.device)
    m = lo.to(torch.bfloat16)
    s = (hi * fifteenth - lo * fifteenth).to(torch.bfloat16)
    sf = s.float()[..., None]
    c = torch.round((x - m.float()[..., None]) / sf).clamp(0, 15)
    c = torch.where(sf > 0, c, torch.zeros_like(c)).to(torch.uint8).flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), m, s


def _values(packed, m, s):
    """What packed codes stand for, in 32 bits: [..., d]."""
    c = torch.stack((packed & 15, packed >> 4), dim=-1).flatten(-2)
    c = c.float().unflatten(-1, (-1, GROUP))
    return (c * s.float()[..., None] + m.float()[..., None]).flatten(-2)


class _Packed:
    """A plain 4-bit cache: [S][L][H][cap] rows of codes, minima, scales."""

    def __init__(self, S, L, H, d, cap):
        lead = (S, L, H, cap)
        z = dict(device="cuda")
        self.codes = [torch.zeros((*lead, d // 2), dtype=torch.uint8, **z)
                      for _ in range(2)]
        self.m = [torch.zeros((*lead, d // GROUP), dtype=torch.bfloat16, **z)
                  for _ in range(2)]
        self.s = [torch.zeros((*lead, d // GROUP), dtype=torch.bfloat16, **z)
                  for _ in range(2)]
        self.score = torch.zeros(lead, **z)

    def load(self, s, k, v):
        n = k.shape[2]
        for i, x in enumerate((k, v)):
            p, m, sc = _quantise(x)
            self.codes[i][s, :, :, :n] = p
            self.m[i][s, :, :, :n] = m
            self.s[i][s, :, :, :n] = sc


def _plain_append(st):
    cache, at = st["cache"], st["at"]      # at: [S][T] row of each new token
    S, T = at.shape
    L, H = cache.score.shape[1:3]
    where = (torch.arange(S, device="cuda")[:, None, None, None],
             torch.arange(L, device="cuda")[None, :, None, None],
             torch.arange(H, device="cuda")[None, None, :, None],
             at[:, None, None, :])
    got = []
    for i, x in enumerate(st["new"]):      # keys, then values
        p, m, s = _quantise(x.transpose(2, 3))
        cache.codes[i][where] = p
        cache.m[i][where] = m
        cache.s[i][where] = s
        got.append(_values(cache.codes[i][where], cache.m[i][where],
                           cache.s[i][where]).to(x.dtype))
    cache.score[where] = 0.0
    return {"k": got[0], "v": got[1]}


def _plain_attend(st):
    cache, q = st["cache"], st["q"]
    S, L, T, _, d = q.shape
    H, G = st["heads"], q.shape[3] // st["heads"]
    n = cache.score.shape[3]
    qf = q.float().view(S, L, T, H, G, d).permute(0, 1, 3, 2, 4, 5)
    k = _values(cache.codes[0], cache.m[0], cache.s[0])
    logits = torch.matmul(qf.reshape(S, L, H, T * G, d), k.transpose(-1, -2))
    del k
    logits = logits.view(S, L, H, T, G, n) / math.sqrt(d)
    # query t of sequence s sees rows 0 .. last[s][t]; -1: none
    sees = torch.arange(n, device="cuda") <= st["last"][..., None]
    sees = sees[:, None, None, :, None, :]
    logits = logits.masked_fill(~sees, -math.inf)
    top = logits.amax(-1, keepdim=True).clamp(min=-1e30)
    p = torch.exp(logits - top)
    del logits
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    v = _values(cache.codes[1], cache.m[1], cache.s[1])
    out = torch.matmul(p.view(S, L, H, T * G, n), v).view(S, L, H, T, G, d)
    out = out.permute(0, 1, 3, 2, 4, 5).reshape(S, L, T, H * G, d).to(q.dtype)
    if not st["scores"]:
        return {"out": out}
    cache.score += p.mean(4).sum(3)
    return {"out": out, "score": cache.score}


def _plain_evict(st):
    cache, n, B, W = st["cache"], st["lens"], st["budget"], st["window"]
    most = cache.score.shape[3]
    row = torch.arange(most, device="cuda")
    old = (row < n[:, None] - W)[:, None, None]
    best = torch.where(old, cache.score, torch.full_like(cache.score, -1.0))
    best = torch.sort(best, dim=-1, descending=True, stable=True).indices
    newest = (n[:, None] - W + torch.arange(W, device="cuda"))[:, None, None]
    newest = newest.expand(*best.shape[:3], W)
    kept = torch.cat((torch.sort(best[..., :B], dim=-1).values, newest), -1)
    got = {"pos": kept.to(torch.int32), "score": cache.score.gather(3, kept)}
    for i, name in enumerate("kv"):
        rows = [x.gather(3, kept[..., None].expand(*kept.shape, x.shape[4]))
                for x in (cache.codes[i], cache.m[i], cache.s[i])]
        got[name] = _values(*rows).to(st["dtype"])
    return got


def _softmax(logits, temperature):
    x = logits.float() / temperature
    e = torch.exp(x - x.amax(-1, keepdim=True))
    return e / e.sum(-1, keepdim=True)


def _plain_verify(st):
    p = _softmax(st["target"], st["temperature"])
    q = _softmax(st["draft"], st["temperature"])
    S, T, V = q.shape
    x = st["tokens"].long()[..., None]
    ok = st["u"] * q.gather(2, x)[..., 0] < p[:, :T].gather(2, x)[..., 0]
    step = torch.arange(T, device="cuda")
    if st["counts"] is not None:
        ok = ok & (step < st["counts"][:, None])
    taken = torch.cumprod(ok.int(), dim=1).sum(1)
    every = torch.full_like(taken, T) if st["counts"] is None \
        else st["counts"].long()
    one = torch.arange(S, device="cuda")
    last = p[one, taken]
    rest = (last - q[one, taken.clamp(max=T - 1)]).clamp(min=0)
    plain = (taken == every)[:, None] | (rest.amax(-1, keepdim=True) <= 0)
    w = torch.where(plain, last, rest) / st["race"]
    index = torch.arange(V, device="cuda")
    nxt = torch.where(w == w.amax(-1, keepdim=True), index, V).amin(-1)
    at = torch.arange(T + 1, device="cuda")
    drafted = torch.cat((st["tokens"], st["tokens"][:, :1]), 1)
    tokens = torch.where(at < taken[:, None], drafted,
                         torch.where(at == taken[:, None], nxt[:, None], -1))
    return {"accepted": taken.to(torch.int32), "tokens": tokens.to(torch.int32)}


# ---- a state, and one pass --------------------------------------------------

def prepare(case, seed):
    kind = case["kind"]
    st = {"kind": kind, "own": own}
    if kind == "verify":
        names = ("target", "draft", "tokens", "u", "race")
        st.update(zip(names, _drafts(case, seed)))
        st["temperature"] = case["temperature"]
        st["counts"] = torch.tensor(_counts(case, seed), dtype=torch.int32,
                                    device="cuda") if case["ragged"] else None
        if own:
            from paper_2608_15797_gb300 import kvr
            st["kvr"] = kvr
            st["workspace"] = kvr.verify_workspace(
                case["n_seq"], case["tokens"], case["vocab"])
        return st
    L, H, G, d, dtype = GEOMETRY[case["geometry"]]
    S, lens = case["n_seq"], _lengths(case)
    new = case["tokens"] if kind == "append" else 0
    cap = max(lens) + new
    if own:
        from paper_2608_15797_gb300 import kvr
        st["kvr"] = kvr
        cache = kvr.Kv4Cache(S, L, H, G, d, cap, dtype=dtype, out_dtype=dtype)
    else:
        cache = _Packed(S, L, H, d, cap)
    for s in range(S):
        if lens[s]:
            cache.load(s, *_rows(case, seed, s, lens[s]))
    st.update(cache=cache, heads=H, dtype=DTYPES[dtype])
    if kind == "append":
        st["new"] = _new_rows(case, seed)
        st["lens"] = lens
        if not own:
            st["at"] = torch.tensor(lens, device="cuda")[:, None] \
                + torch.arange(new, device="cuda")
    elif kind == "attend":
        st["q"] = _queries(case, seed)
        st["scores"] = case["scores"]
        counts = _counts(case, seed)
        st["counts"] = counts if case["ragged"] else None
        st["by_layer"] = case["by_layer"]
        if own:
            st["workspace"] = cache.attend_workspace(case["tokens"])
            if case["by_layer"]:
                st["q"] = [st["q"][:, l:l + 1].contiguous() for l in range(L)]
                st["out"] = torch.empty((L, S, 1, case["tokens"], H * G, d),
                                        dtype=DTYPES[dtype], device="cuda")
        else:
            last = [[n - c + t if t < c else -1
                     for t in range(case["tokens"])]
                    for n, c in zip(lens, counts)]
            st["last"] = torch.tensor(last, device="cuda")
    else:
        st.update(budget=case["budget"], window=case["window"])
        score = cache.scores_view() if own else cache.score
        for s in range(S):
            score[s, :, :, :lens[s]] = _weights(case, seed, s, lens[s])
        if own:
            keep = case["budget"] + case["window"]
            st["kept"] = kvr.Cache(S, L, H, G, d, keep + 1, kv_dtype=dtype,
                                   out_dtype=dtype)
        else:
            st["lens"] = torch.tensor(lens, device="cuda")
    return st


def run(st):
    kind = st["kind"]
    if not st["own"]:
        return {"append": _plain_append, "attend": _plain_attend,
                "evict": _plain_evict, "verify": _plain_verify}[kind](st)
    if kind == "verify":
        accepted, tokens = st["kvr"].verify_drafts(
            st["target"], st["draft"], st["tokens"], st["u"], st["race"],
            n_draft=st["counts"], temperature=st["temperature"],
            workspace=st["workspace"])
        return {"accepted": accepted, "tokens": tokens}
    cache = st["cache"]
    if kind == "append":
        cache.append(*st["new"])
        k, v = cache.read_newest(st["new"][0].shape[2])
        cache.truncate(st["lens"])  # the drafts were rejected
        return {"k": k, "v": v}
    if kind == "attend":
        if st["by_layer"]:
            for l, q in enumerate(st["q"]):
                cache.attend(q, out=st["out"][l], layers=(l, l + 1),
                             counts=st["counts"], scores=st["scores"],
                             workspace=st["workspace"])
            out = st["out"][:, :, 0].transpose(0, 1)
        else:
            out = cache.attend(st["q"], counts=st["counts"],
                               scores=st["scores"], workspace=st["workspace"])
        return {"out": out, "score": cache.scores_view()} if st["scores"] \
            else {"out": out}
    B, W, kept = st["budget"], st["window"], st["kept"]
    cache.evict_into(kept, B, W)
    k, v = kept.rows_view()
    score, pos, _ = kept.scores_view()
    return {"pos": pos[..., :B + W], "score": score[..., :B + W],
            "k": k[..., :B + W, :], "v": v[..., :B + W, :]}


def work(case):
    kind = case["kind"]
    if kind == "verify":
        S, T, V = case["n_seq"], case["tokens"], case["vocab"]
        es = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": S * ((2 * T + 1) * V * es + 4 * V + 12 * T + 8),
                "flops": S * V * ((2 * T + 1) * 4 + 3)}
    L, H, G, d, dtype = GEOMETRY[case["geometry"]]
    es = 2 if dtype == "bf16" else 4
    row = d + 8 * (d // GROUP)         # key and value: codes, scales, minima
    if kind == "append":
        rows = case["n_seq"] * L * H * case["tokens"]
        return {"bytes": rows * (2 * d * es * 2 + 2 * row + 4),
                "flops": rows * 2 * d * 6}
    lens = _lengths(case)
    rows = sum(lens) * L * H
    if kind == "attend":
        T = case["tokens"]
        return {"bytes": rows * (row + (8 if case["scores"] else 0))
                + case["n_seq"] * L * T * H * G * d * 2 * es,
                "flops": rows * T * G * 4 * d}
    keep = case["n_seq"] * L * H * (case["budget"] + case["window"])
    return {"bytes": rows * 4 + keep * (row + 2 * d * es + 8),
            "flops": rows + keep * 4 * d}


# ---- the definitions in 64 bits ---------------------------------------------

def _stands_for(x):
    """The values, in 64 bits, that the cache holds for x [..., d]."""
    y = x.double().reshape(*x.shape[:-1], x.shape[-1] // GROUP, GROUP)
    lo = y.min(dim=-1, keepdim=True).values
    hi = y.max(dim=-1, keepdim=True).values
    m = lo.to(torch.bfloat16).double()
    s = ((hi - lo) / 15.0).to(torch.bfloat16).double()
    code = torch.where(s > 0, (y - m) / s, torch.zeros_like(y)).round()
    return (m + s * code.clamp(0, 15)).reshape(x.shape)


def _exact_attend(case, seed):
    L, H, G, d, dtype = GEOMETRY[case["geometry"]]
    q = _queries(case, seed)
    lens, counts = _lengths(case), _counts(case, seed)
    T = case["tokens"]
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    score = torch.zeros((len(lens), L, H, max(lens)), dtype=torch.float64,
                        device="cuda")
    for s, n in enumerate(lens):
        k, v = _rows(case, seed, s, n)
        for l in range(L):
            kd, vd = _stands_for(k[l]), _stands_for(v[l])
            for t in range(counts[s]):
                end = n - counts[s] + t + 1
                qd = q[s, l, t].double().view(H, G, d)
                x = (qd @ kd[:, :end].transpose(1, 2)) / math.sqrt(d)
                p = torch.softmax(x, dim=-1)
                out[s, l, t] = (p @ vd[:, :end]).view(H * G, d)
                score[s, l, :, :end] += p.mean(1)
    return {"out": out, "score": score} if case["scores"] else {"out": out}


def _exact_evict(case, seed):
    L, H, _, d, _ = GEOMETRY[case["geometry"]]
    B, W = case["budget"], case["window"]
    got = {"pos": [], "score": [], "k": [], "v": []}
    for s, n in enumerate(_lengths(case)):
        k, v = _rows(case, seed, s, n)
        w = _weights(case, seed, s, n)
        # weight first, then the lower position: whole numbers of 64 bits
        # (a positive float's bits are in the order of its value)
        key = (w.view(torch.int32).long() << 24) \
            - torch.arange(n, device="cuda")
        old = torch.topk(key[..., :n - W], B, dim=-1).indices
        new = torch.arange(n - W, n, device="cuda").expand(L, H, W)
        pos = torch.cat((old, new), dim=-1).sort(dim=-1).values
        got["pos"].append(pos.to(torch.int32))
        got["score"].append(torch.take_along_dim(w, pos, dim=-1).double())
        for name, x in (("k", k), ("v", v)):
            x = torch.take_along_dim(x, pos[..., None], dim=2)
            got[name].append(_stands_for(x))
    return {name: torch.stack(x) for name, x in got.items()}


def _exact_verify(case, seed):
    target, draft, tokens, u, race = _drafts(case, seed)
    counts = _counts(case, seed)
    S, T = tokens.shape
    accepted = torch.zeros(S, dtype=torch.int32, device="cuda")
    emitted = torch.full((S, T + 1), -1, dtype=torch.int32, device="cuda")
    for s in range(S):
        t = 0
        rest = None
        while t < counts[s]:
            p = torch.softmax(target[s, t].double() / case["temperature"], -1)
            q = torch.softmax(draft[s, t].double() / case["temperature"], -1)
            x = int(tokens[s, t])
            if not bool(u[s, t].double() * q[x] < p[x]):
                rest = torch.relu(p - q)
                rest = rest if bool((rest > 0).any()) else p
                break
            emitted[s, t] = x
            t += 1
        if rest is None:
            rest = torch.softmax(target[s, t].double() / case["temperature"],
                                 -1)
        accepted[s] = t
        emitted[s, t] = int(torch.argmax(rest / race[s].double()))
    return {"accepted": accepted, "tokens": emitted}


def exact(case, seed):
    kind = case["kind"]
    if kind == "append":
        k, v = (_stands_for(x).transpose(2, 3) for x in _new_rows(case, seed))
        return {"k": k, "v": v}
    if kind == "attend":
        return _exact_attend(case, seed)
    return _exact_evict(case, seed) if kind == "evict" \
        else _exact_verify(case, seed)
