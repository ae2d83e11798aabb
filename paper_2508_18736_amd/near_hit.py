"""From a lookup to answers: what is done with a hit, a near hit and a miss.

A query whose closest centroid passes the retrieval threshold is answered with the stored answer.  One that only passes a lower one is
a near hit: the stored answer is probably right for the most part, so its tokens are a draft that the target model verifies several
at a time.  All others are answered token by token.  The target model's keys and values are kept in pages (``PagedKV``): a
prompt is written and attended to as one chunk, then each step writes a sequence's last token and its draft, attends to the pages, and
``verify`` says how many of them stand and which token follows.

Several stored answers may be close.  They agree for a while and then part: a tree of drafted tokens, which the model reads at once (``tree``, ``attend``
with it), ``verify_tree`` says which path of it stands, and ``keep`` moves that path behind the context.  A cache that must not grow keeps so many
positions of a sequence: what attention weighs is added up (``weigh``), and the lightest go (``evict``).

    python -m paper_2508_18736_amd.near_hit [--storage bf16|fp8] [--drafts 4] [--tokens 48] [--branches 1] [--keep 0]

runs it with a small model of random weights, on synthetic prompts and stored answers.
"""

import argparse
from typing import List, Optional, Sequence, Tuple

import torch

from . import siso


class Target:
    """A causal transformer of random weights: what surrounds attention is torch's, in single precision."""

    def __init__(self, layers: int = 2, heads: int = 8, kv_heads: int = 2, head_dim: int = 64, vocab: int = 2048, seed: int = 0,
                 device: str = "cuda:0"):
        g = torch.Generator().manual_seed(seed)
        width = heads * head_dim
        rand = lambda *shape: (torch.randn(shape, generator=g) * shape[0] ** -0.5).to(device)  # noqa: E731
        self.heads, self.kv_heads, self.head_dim, self.vocab, self.device = heads, kv_heads, head_dim, vocab, device
        self.embed = torch.randn(vocab, width, generator=g).to(device)
        self.layers = [(rand(width, width + 2 * kv_heads * head_dim), rand(width, width), rand(width, 2 * width), rand(2 * width, width))
                       for _ in range(layers)]
        self.frequency = (10000.0 ** (-torch.arange(0, width, 2) / width)).to(device)

    @staticmethod
    def _norm(x: torch.Tensor) -> torch.Tensor:
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    def logits(self, kv: siso.PagedKV, batch: siso.KvBatch, tokens: torch.Tensor, positions: torch.Tensor, tree: Optional[siso.KvTree] = None,
               noted: Optional[list] = None) -> torch.Tensor:
        """[rows, vocab] of the batch's rows (of trees: ``tree``), whose keys and values go into the cache.  ``noted``: each layer's queries
        and the logarithms of their rows' sums are put there."""
        angle = positions[:, None] * self.frequency
        x = self.embed[tokens.long()] + torch.cat((angle.sin(), angle.cos()), 1)
        n = self.heads * self.head_dim
        for layer, (w_qkv, w_out, w_up, w_down) in enumerate(self.layers):
            qkv = (self._norm(x) @ w_qkv).to(torch.bfloat16)
            q, k, v = qkv.split((n, self.kv_heads * self.head_dim, self.kv_heads * self.head_dim), 1)
            heads = lambda t: t.unflatten(1, (-1, self.head_dim))  # noqa: E731  (strides as they are)
            kv.write(batch, heads(k), heads(v), layer=layer)
            how = {} if tree is None else {"tree": tree}
            if noted is None:
                out = kv.attend(batch, heads(q), layer=layer, **how)
            else:
                out, lse = kv.attend(batch, heads(q), layer=layer, with_lse=True, **how)
                noted.append((heads(q), lse))
            x = x + out.flatten(1).float() @ w_out
            x = x + torch.nn.functional.silu(self._norm(x) @ w_up) @ w_down
        return self._norm(x) @ self.embed.t()


def _ends(counts: Sequence[int], device) -> torch.Tensor:
    return torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], dtype=torch.int32, device=device)


def _branches(answers: Sequence[Sequence[int]], done: int, most: int, deepest: int) -> Tuple[List[int], List[int], List[int]]:
    """The answers' tokens from ``done`` on as a tree of at most ``most`` rows behind row 0: ``(tokens, parents, depths)``.  What answers have in common
    they share; token by token, the first answer first."""
    tokens: List[int] = []
    parents: List[int] = []
    depths: List[int] = []
    at: List[Optional[int]] = [0] * len(answers)
    known = {}
    for depth in range(deepest):
        for i, a in enumerate(answers):
            if at[i] is None:
                continue
            place = (at[i], a[done + depth]) if done + depth < len(a) else None
            if place is not None and place not in known and len(tokens) < most:
                tokens.append(place[1])
                parents.append(place[0])
                depths.append(depth + 1)
                known[place] = len(tokens)
            at[i] = known.get(place)
    return tokens, parents, depths


def serve(target: Target, prompts: Sequence[Sequence[int]], drafts: Sequence[Optional[Sequence]], tokens: int, most: int = 4,
          dtype: int = siso.BF16, page_tokens: int = 16, temperature: float = 0.0, seed: int = 0, keep: int = 0, recent: Optional[int] = None,
          early: int = 1) -> Tuple[List[List[int]], int]:
    """``tokens`` tokens behind each prompt, and the number of the model's steps.  ``drafts[b]``: the stored answer of sequence b, a list of
    several, or None; at most ``most`` of their tokens are verified at a time.  Temperature 0: greedy.  ``keep`` > 0: behind each step a sequence keeps
    so many positions of its cache: the newest ``recent`` (None: half), those before position ``early``, and those that attention has weighed most."""
    n, dev = len(prompts), target.device
    if most < 0:
        raise ValueError(f"most: {most} drafted tokens at a time")
    recent = keep // 2 if recent is None else recent
    if keep < 0 or recent < 0 or early < 0 or (keep > 0 and recent + early > keep):
        raise ValueError(f"keep: {keep} positions, {recent} recent and {early} early ones among them")
    several = any(d and isinstance(d[0], (list, tuple)) for d in drafts)
    if several and most >= siso.TREE:
        raise ValueError(f"most: trees of at most {siso.TREE - 1} drafted tokens")
    if n == 0 or tokens <= 0:
        return [[] for _ in prompts], 0
    if not all(len(p) for p in prompts):
        raise ValueError("prompts: every one has a token at least")
    # (with a bound a sequence has so many positions, or its prompt's, and a step's rows)
    need = [-(-(max(len(p), keep) + 1 + most if 0 < keep < len(p) + tokens else len(p) + tokens + most) // page_tokens) for p in prompts]
    kv = siso.PagedKV(target.kv_heads, target.head_dim, sum(need), page_tokens=page_tokens, layers=len(target.layers), dtype=dtype, device=dev)
    weights = kv.weights() if keep else None
    pages = torch.zeros(n, max(need), dtype=torch.int32)
    for b, at in enumerate(_ends(need, "cpu").tolist()[:-1]):
        pages[b, :need[b]] = torch.arange(at, at + need[b], dtype=torch.int32)
    pages = pages.to(dev)
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)  # noqa: E731
    g = torch.Generator(device=dev).manual_seed(seed)
    answers: List[List[int]] = [[] for _ in prompts]
    held = [0] * n  # positions of the cache whose keys and values stand
    stand = [0] * n  # tokens that they are of, the evicted ones too
    rows = [list(p) for p in prompts]
    guess = [([], [], []) for _ in prompts]  # the drafted ones at the end of a sequence's rows: tokens, the rows that they continue, how deep
    steps = 0
    while any(rows):
        flat = ints([t for r in rows for t in r])
        deep = [(list(range(len(r))) if not d[0] else [0, *d[2]]) for r, d in zip(rows, guess)]
        positions = torch.tensor([stand[b] + i for b, r in enumerate(deep) for i in r], device=dev)
        counts = [len(r) for r in rows]
        length = ints([h + c for h, c in zip(held, counts)])
        batch = kv.batch(_ends(counts, dev), length, pages, rows=sum(counts), max_new=max(counts), max_length=max(h + c for h, c in zip(held, counts)))
        drafted = any(d[0] for d in guess)
        tree = kv.tree(batch, ints([p for r, d in zip(rows, guess) if r for p in (-1, *d[1])])) if several and drafted else None
        noted: Optional[list] = [] if keep else None
        logits = target.logits(kv, batch, flat, positions, tree, noted)
        # what is judged: of every sequence the last token that stands, and the draft behind it
        judged = [1 + len(d[0]) if r else 0 for r, d in zip(rows, guess)]
        ends = _ends(counts, "cpu").tolist()
        pick = torch.tensor([i for b in range(n) for i in range(ends[b + 1] - judged[b], ends[b + 1])], device=dev)
        judge = kv.batch(_ends(judged, dev), rows=sum(judged), max_new=max(judged))
        p = torch.softmax(logits[pick] / temperature, 1) if temperature > 0 else logits[pick]
        path = None
        if tree is not None:  # (all rows are judged: a prompt has no draft)
            u = torch.rand(sum(judged), generator=g, device=dev) if temperature > 0 else None
            accepted, path, out = kv.verify_tree(judge, tree, flat, p, u)
            kv.keep(batch, path)
            path = path.tolist()
        elif temperature > 0:
            u = torch.rand(sum(judged) + n, generator=g, device=dev)
            accepted, out = kv.verify(judge, flat[pick], p, u_accept=u[:sum(judged)], u_sample=u[sum(judged):])
        else:
            accepted, out = kv.verify(judge, flat[pick], p)
        accepted, out = accepted.tolist(), out.tolist()
        at = 0
        standing: List[List[int]] = [[] for _ in prompts]  # rows of the batch whose tokens stand now
        for b in range(n):
            if judged[b]:
                answers[b] += out[at:at + accepted[b] + 1]
                new = counts[b] - len(guess[b][0]) + accepted[b]  # (the rest of the draft is written over)
                standing[b] = [ends[b] + i for i in (range(new) if path is None else path[at:at + new])]
                held[b] += new
                stand[b] += new
                done = len(answers[b])
                left = tokens - done
                d = drafts[b] or []
                if left <= 0 or not d:
                    guess[b] = ([], [], [])
                elif isinstance(d[0], (list, tuple)):
                    guess[b] = _branches(d, done, most, min(most, left - 1))
                else:
                    line = list(d[done:done + min(most, left - 1)])
                    guess[b] = (line, list(range(len(line))), list(range(1, len(line) + 1)))
                rows[b] = [answers[b][-1], *guess[b][0]] if left > 0 else []
            at += judged[b]
        if keep:
            some = torch.tensor([r for s in standing for r in s], device=dev)
            now = kv.batch(_ends([len(s) for s in standing], dev), ints(held), pages, rows=len(some), max_new=max(map(len, standing)), max_length=max(held))
            for layer, (q, lse) in enumerate(noted):
                kv.weigh(now, q[some], lse[some], weights, layer=layer, newest=ints([s - 1 for s in stand]))
            if max(held) > keep:
                kv.evict(now, weights, keep, recent=recent, early=early)
                held = [min(h, keep) for h in held]
        steps += 1
    return answers, steps


def answer(cache: siso.SisoCache, stored: Sequence[Sequence[int]], target: Target, queries: torch.Tensor, prompts: Sequence[Sequence[int]],
           theta: float, theta_near: float, tokens: int, branches: int = 1, **how):
    """Answers of all queries: ``(answers, kinds, steps)``, a kind each of "hit", "near", "miss"; ``stored[i]``: the answer of centroid i.
    ``branches``: the drafts of a near hit are the stored answers of so many of the closest centroids, as far as they pass ``theta_near``."""
    idx, _, flags = cache.lookup_multi(queries, [theta_near, theta], count_index=1)
    idx, flags = idx.tolist(), flags.tolist()
    kinds = ["hit" if f[1] else "near" if f[0] else "miss" for f in flags]
    ask = [b for b, kind in enumerate(kinds) if kind != "hit"]
    drafts = {b: stored[idx[b]] for b in ask if kinds[b] == "near"}
    if branches > 1 and drafts:
        closest, similarity = (x.tolist() for x in cache.lookup_topk(queries, k=branches))
        drafts = {b: [stored[idx[b]], *(stored[i] for i, s in zip(closest[b], similarity[b]) if i not in (-1, idx[b]) and s > theta_near)] for b in drafts}
    got, steps = serve(target, [prompts[b] for b in ask], [drafts.get(b) for b in ask], tokens, **how)
    answers = [list(stored[i])[:tokens] if kind == "hit" else [] for i, kind in zip(idx, kinds)]  # (no stored answer behind a miss: the cache may be empty)
    for b, a in zip(ask, got):
        answers[b] = a
    return answers, kinds, steps


def example(target: Target, tokens: int, dim: int = 768, seed: int = 3):
    """Synthetic queries at three distances of a small cache's centroids, prompts, and stored answers: what the model itself
    answers, with every sixth token another one."""
    g = torch.Generator().manual_seed(seed)
    centroids = torch.nn.functional.normalize(torch.randn(12, dim, generator=g), dim=1)
    noise = torch.nn.functional.normalize(torch.randn(12, dim, generator=g), dim=1)
    near = torch.tensor([0.95, 0.85, 0.4])[torch.arange(12) % 3]
    queries = torch.nn.functional.normalize(near[:, None] * centroids + (1 - near[:, None].square()).sqrt() * noise, dim=1)
    prompts = [torch.randint(0, target.vocab, (int(torch.randint(5, 200, (1,), generator=g)),), generator=g).tolist() for _ in range(12)]
    plain, _ = serve(target, prompts, [None] * 12, tokens)
    stored = [[(t + 1) % target.vocab if i % 6 == 5 else t for i, t in enumerate(a)] for a in plain]
    cache = siso.SisoCache(dim, 12, siso.BF16)
    cache.load(centroids.to(target.device, torch.bfloat16))
    return cache, stored, queries.to(target.device, torch.bfloat16), prompts


def main() -> None:
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--storage", choices=["bf16", "fp8"], default="bf16")
    ap.add_argument("--drafts", type=int, default=4, help="drafted tokens that are verified at a time")
    ap.add_argument("--tokens", type=int, default=48)
    ap.add_argument("--temperature", type=float, default=0.0)
    ap.add_argument("--branches", type=int, default=1, help="stored answers that are drafts of one near hit, at most")
    ap.add_argument("--keep", type=int, default=0, help="positions of its cache that a sequence keeps (0: all)")
    args = ap.parse_args()
    target = Target()
    cache, stored, queries, prompts = example(target, args.tokens)
    how = dict(most=args.drafts, dtype=siso.FP8 if args.storage == "fp8" else siso.BF16, temperature=args.temperature)
    if args.keep:
        how["keep"] = args.keep
    answers, kinds, steps = answer(cache, stored, target, queries, prompts, 0.9, 0.7, args.tokens, **({"branches": args.branches} if args.branches > 1 else {}), **how)
    for b, kind in enumerate(kinds):
        same = sum(x == y for x, y in zip(answers[b], stored[b]))
        print(f"query {b}: {kind:4s} prompt of {len(prompts[b])} tokens, {same} of {len(answers[b])} tokens as in the stored answer")
    near = [b for b, kind in enumerate(kinds) if kind == "near"]
    _, alone = serve(target, [prompts[b] for b in near], [stored[b] for b in near], args.tokens, **how)
    print(f"{len(kinds)} queries, {kinds.count('hit')} hits, {kinds.count('near')} near hits; {steps} steps for all that missed, "
          f"{alone} for the near hits, {args.tokens} without drafts")


if __name__ == "__main__":
    main()
