"""Drafting from an evicted cache, verified over the full context in 4 bits.

    python -m examples.draft_and_verify [--seqs 4] [--new 64] [--draft 4] ...

A small random decoder (its projections are plain matrix products) generates
for several prompts at once.  The full context is a Kv4Cache; the drafter
decodes from an evicted Cache of budget + window rows a KV head.  A round:

1. the drafter proposes `draft` tokens, a Cache.step a layer and token;
2. the pending token and the drafts enter the full cache (append) and attend
   over it at once (attend, which leaves the rows' scores alone: some of these
   tokens may never have been);
3. verify_drafts accepts a prefix of the drafts and draws the next token, so
   that what is emitted is distributed as the model's own samples;
4. truncate drops the rejected rows, the tokens that stay attend once more and
   accumulate the rows' scores, and evict_into cuts the drafter's cache from the
   full one by them.
"""
from __future__ import annotations

import argparse
import math

import torch

from paper_2608_15797_gb300 import kvr


class Decoder:
    """Random weights: L layers of attention alone, tied to nothing."""

    def __init__(self, layers=2, heads=2, group=4, d=64, vocab=1000, width=256,
                 dtype="f32", seed=0):
        self.L, self.H, self.G, self.d, self.V = layers, heads, group, d, vocab
        self.dtype = dtype
        g = torch.Generator("cuda").manual_seed(seed)

        def w(*shape, gain=1.0):
            x = torch.randn(shape, generator=g, device="cuda")
            return x * (gain / math.sqrt(shape[0]))

        hd = heads * d
        self.embed = w(vocab, width, gain=math.sqrt(vocab))
        self.wq = [w(width, group * hd) for _ in range(layers)]
        self.wk = [w(width, hd) for _ in range(layers)]
        self.wv = [w(width, hd) for _ in range(layers)]
        self.wo = [w(group * hd, width) for _ in range(layers)]
        self.head = w(width, vocab, gain=3.0)

    def forward(self, tokens, attend):
        """tokens [S][n] -> logits [S][n][V]; attend(layer, q, k, v) with
        q [S][1][n][H*G][d] and k, v [S][1][n][H][d]."""
        S, n = tokens.shape
        h = self.embed[tokens.long().clamp(min=0)]
        to = kvr.TORCH_DTYPES[self.dtype]
        for l in range(self.L):
            x = torch.nn.functional.rms_norm(h, h.shape[-1:])
            q = (x @ self.wq[l]).view(S, 1, n, self.H * self.G, self.d)
            k = (x @ self.wk[l]).view(S, 1, n, self.H, self.d)
            v = (x @ self.wv[l]).view(S, 1, n, self.H, self.d)
            o = attend(l, *(t.to(to).contiguous() for t in (q, k, v)))
            h = h + o.float().view(S, n, -1) @ self.wo[l]
        return torch.nn.functional.rms_norm(h, h.shape[-1:]) @ self.head

    def full(self, cache, tokens, counts=None, scores=True, queries=None):
        """Append the tokens to a Kv4Cache and run them over it.  queries: a
        list that gets each layer's."""
        def attend(l, q, k, v):
            if queries is not None:
                queries.append(q)
            cache.append(k, v, counts=counts, layers=(l, l + 1))
            return cache.attend(q, counts=counts, layers=(l, l + 1),
                                scores=scores)
        return self.forward(tokens, attend)

    def weigh(self, cache, queries, counts):
        """Accumulate the scores that the newest counts[s] tokens give the rows,
        which are the first ones of their call."""
        for l, q in enumerate(queries):
            cache.attend(q, counts=counts, layers=(l, l + 1), scores=True)

    def draft(self, cache, tokens, budget, window):
        """One token a sequence over an evicted Cache -> logits [S][V]."""
        def attend(l, q, k, v):
            o = cache.step(q[:, :, 0], k[:, :, 0], v[:, :, 0], budget, window,
                           layers=(l, l + 1))
            return o.unsqueeze(2)
        return self.forward(tokens[:, None], attend)[:, 0]


def caches(m, n_seq, capacity, budget, window):
    full = kvr.Kv4Cache(n_seq, m.L, m.H, m.G, m.d, capacity, dtype=m.dtype,
                        out_dtype=m.dtype)
    small = kvr.Cache(n_seq, m.L, m.H, m.G, m.d, budget + window + 1,
                      kv_dtype=m.dtype, out_dtype=m.dtype)
    return full, small


def padded(rows):
    n = max(len(r) for r in rows)
    return torch.tensor([r + [0] * (n - len(r)) for r in rows], device="cuda")


def prefill(m, full, prompts):
    """All but the last token of each prompt; that one is pending."""
    counts = [len(p) - 1 for p in prompts]
    if max(counts) > 0:
        m.full(full, padded([p[:-1] for p in prompts]), counts)
    return torch.tensor([p[-1] for p in prompts], device="cuda")


def check_sizes(new, draft, budget, window, temperature):
    if new < 1:
        raise ValueError(f"new must be 1 or more, not {new}")
    if not 1 <= draft <= 64:
        raise ValueError(f"draft must be 1 to 64, not {draft}")
    if budget < 0 or window < 0 or budget + window < 1:
        raise ValueError(f"budget {budget} and window {window} keep no row")
    if not temperature > 0:
        raise ValueError(f"temperature must be above 0, not {temperature}")


def generate(m, prompts, new, draft=4, budget=64, window=16, temperature=1.0,
             seed=1):
    """At least `new` tokens a prompt.  Returns them, and the share of drafted
    tokens that were accepted."""
    check_sizes(new, draft, budget, window, temperature)
    S = len(prompts)
    if not S or not all(prompts):
        raise ValueError("every prompt needs a token")
    g = torch.Generator("cuda").manual_seed(seed)
    most = max(len(p) for p in prompts) + new + 2 * draft + 2
    full, small = caches(m, S, most, budget, window)
    pending = prefill(m, full, prompts)
    out = [[] for _ in prompts]
    drafted = kept = 0
    while min(len(o) for o in out) < new:
        full.evict_into(small, budget, window)
        x, tokens, logits = pending, [], []
        for _ in range(draft):
            y = m.draft(small, x, budget, window)
            race = torch.empty_like(y).exponential_(generator=g)
            x = (torch.softmax(y / temperature, -1) / race).argmax(-1)
            logits.append(y)
            tokens.append(x)
        tokens = torch.stack(tokens, 1).int()
        before = full.lengths()[:, 0]
        queries = []
        target = m.full(full, torch.cat((pending[:, None].int(), tokens), 1),
                        scores=False, queries=queries)
        u = torch.rand((S, draft), generator=g, device="cuda")
        race = torch.empty((S, m.V), device="cuda").exponential_(generator=g)
        accepted, emitted = kvr.verify_drafts(
            target.contiguous(), torch.stack(logits, 1), tokens, u, race,
            temperature=temperature)
        accepted, emitted = accepted.tolist(), emitted.tolist()
        # Sequences that have enough stay where they are.
        done = [len(o) >= new for o in out]
        kept_rows = [0 if d else 1 + a for d, a in zip(done, accepted)]
        full.truncate([int(n) + k for n, k in zip(before, kept_rows)])
        m.weigh(full, queries, kept_rows)
        nxt = pending.tolist()
        for s in range(S):
            if not done[s]:
                out[s] += emitted[s][:accepted[s] + 1]
                nxt[s] = emitted[s][accepted[s]]
                drafted += draft
                kept += accepted[s]
        pending = torch.tensor(nxt, device="cuda")
    full.sync_status()
    small.sync_status()
    return out, kept / drafted


def greedy(m, prompts, new):
    """The full cache alone, one token at a time, the likeliest each time."""
    full, _ = caches(m, len(prompts), max(map(len, prompts)) + new, 1, 0)
    x, out = prefill(m, full, prompts), []
    for _ in range(new):
        x = m.full(full, x[:, None], scores=False)[:, 0].argmax(-1)
        out.append(x)
    return torch.stack(out, 1).tolist()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--seqs", type=int, default=4)
    ap.add_argument("--prompt", type=int, default=300)
    ap.add_argument("--new", type=int, default=64)
    ap.add_argument("--draft", type=int, default=4)
    ap.add_argument("--budget", type=int, default=64)
    ap.add_argument("--window", type=int, default=16)
    ap.add_argument("--temperature", type=float, default=1.0)
    ap.add_argument("--dtype", choices=("f32", "bf16"), default="bf16")
    a = ap.parse_args(argv)
    try:
        check_sizes(a.new, a.draft, a.budget, a.window, a.temperature)
    except ValueError as e:
        ap.error(str(e))
    if a.seqs < 1:
        ap.error(f"seqs must be 1 or more, not {a.seqs}")
    m = Decoder(d=128 if a.dtype == "bf16" else 64, dtype=a.dtype)
    g = torch.Generator().manual_seed(3)
    prompts = [torch.randint(m.V, (max(1, a.prompt - 37 * s),),
                             generator=g).tolist() for s in range(a.seqs)]
    out, share = generate(m, prompts, a.new, a.draft, a.budget, a.window,
                          a.temperature)
    for s, o in enumerate(out):
        print(f"sequence {s}: {len(prompts[s])} + {len(o)} tokens, "
              f"first {o[:8]}")
    print(f"accepted {share:.0%} of the drafted tokens")


if __name__ == "__main__":
    main()
