"""From a lookup to answers: what is done with a hit, a near hit and a miss.

A query whose closest centroid passes the retrieval threshold is answered with the stored answer.  One that only passes a lower one is
a near hit: the stored answer is probably right for the most part, so its tokens are a draft that the target model verifies several
at a time.  All others are answered token by token.  The target model's keys and values are kept in pages (``PagedKV``): a
prompt is written and attended to as one chunk, then each step writes a sequence's last token and its draft, attends to the pages, and
``verify`` says how many of them stand and which token follows.

    python -m paper_2508_18736_amd.near_hit [--storage bf16|fp8] [--drafts 4] [--tokens 48]

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

    def logits(self, kv: siso.PagedKV, batch: siso.KvBatch, tokens: torch.Tensor, positions: torch.Tensor) -> torch.Tensor:
        """[rows, vocab] of the batch's rows, whose keys and values go into the cache."""
        angle = positions[:, None] * self.frequency
        x = self.embed[tokens.long()] + torch.cat((angle.sin(), angle.cos()), 1)
        n = self.heads * self.head_dim
        for layer, (w_qkv, w_out, w_up, w_down) in enumerate(self.layers):
            qkv = (self._norm(x) @ w_qkv).to(torch.bfloat16)
            q, k, v = qkv.split((n, self.kv_heads * self.head_dim, self.kv_heads * self.head_dim), 1)
            heads = lambda t: t.unflatten(1, (-1, self.head_dim))  # noqa: E731  (strides as they are)
            kv.write(batch, heads(k), heads(v), layer=layer)
            x = x + kv.attend(batch, heads(q), layer=layer).flatten(1).float() @ w_out
            x = x + torch.nn.functional.silu(self._norm(x) @ w_up) @ w_down
        return self._norm(x) @ self.embed.t()


def _ends(counts: Sequence[int], device) -> torch.Tensor:
    return torch.tensor([0, *torch.tensor(counts).cumsum(0).tolist()], dtype=torch.int32, device=device)


def serve(target: Target, prompts: Sequence[Sequence[int]], drafts: Sequence[Optional[Sequence[int]]], tokens: int, most: int = 4,
          dtype: int = siso.BF16, page_tokens: int = 16, temperature: float = 0.0, seed: int = 0) -> Tuple[List[List[int]], int]:
    """``tokens`` tokens behind each prompt, and the number of the model's steps.  ``drafts[b]``: the stored answer of sequence b or
    None; at most ``most`` of its tokens are verified at a time.  Temperature 0: greedy."""
    n, dev = len(prompts), target.device
    if most < 0:
        raise ValueError(f"most: {most} drafted tokens at a time")
    if n == 0 or tokens <= 0:
        return [[] for _ in prompts], 0
    if not all(len(p) for p in prompts):
        raise ValueError("prompts: every one has a token at least")
    need = [-(-(len(p) + tokens + most) // page_tokens) for p in prompts]
    kv = siso.PagedKV(target.kv_heads, target.head_dim, sum(need), page_tokens=page_tokens, layers=len(target.layers), dtype=dtype, device=dev)
    pages = torch.zeros(n, max(need), dtype=torch.int32)
    for b, at in enumerate(_ends(need, "cpu").tolist()[:-1]):
        pages[b, :need[b]] = torch.arange(at, at + need[b], dtype=torch.int32)
    pages = pages.to(dev)
    g = torch.Generator(device=dev).manual_seed(seed)
    answers: List[List[int]] = [[] for _ in prompts]
    held = [0] * n  # tokens whose keys and values are in the cache and stand
    rows = [list(p) for p in prompts]
    guess = [[] for _ in prompts]  # the drafted ones at the end of a sequence's rows
    steps = 0
    while any(rows):
        flat = torch.tensor([t for r in rows for t in r], dtype=torch.int32, device=dev)
        positions = torch.tensor([held[b] + i for b, r in enumerate(rows) for i in range(len(r))], device=dev)
        counts = [len(r) for r in rows]
        length = torch.tensor([h + c for h, c in zip(held, counts)], dtype=torch.int32, device=dev)
        batch = kv.batch(_ends(counts, dev), length, pages, rows=sum(counts), max_new=max(counts), max_length=max(h + c for h, c in zip(held, counts)))
        logits = target.logits(kv, batch, flat, positions)
        # what is judged: of every sequence the last token that stands, and the draft behind it
        judged = [1 + len(d) if r else 0 for r, d in zip(rows, guess)]
        ends = _ends(counts, "cpu").tolist()
        pick = torch.tensor([i for b in range(n) for i in range(ends[b + 1] - judged[b], ends[b + 1])], device=dev)
        judge = kv.batch(_ends(judged, dev), rows=sum(judged), max_new=max(judged))
        if temperature > 0:
            p = torch.softmax(logits[pick] / temperature, 1)
            u = torch.rand(sum(judged) + n, generator=g, device=dev)
            accepted, out = kv.verify(judge, flat[pick], p, u_accept=u[:sum(judged)], u_sample=u[sum(judged):])
        else:
            accepted, out = kv.verify(judge, flat[pick], logits[pick])
        accepted, out = accepted.tolist(), out.tolist()
        at = 0
        for b in range(n):
            if judged[b]:
                answers[b] += out[at:at + accepted[b] + 1]
                held[b] += counts[b] - len(guess[b]) + accepted[b]  # (the rest of the draft is written over)
                done = len(answers[b])
                left = tokens - done
                guess[b] = list((drafts[b] or [])[done:done + min(most, left - 1)]) if left > 0 else []
                rows[b] = [answers[b][-1], *guess[b]] if left > 0 else []
            at += judged[b]
        steps += 1
    return answers, steps


def answer(cache: siso.SisoCache, stored: Sequence[Sequence[int]], target: Target, queries: torch.Tensor, prompts: Sequence[Sequence[int]],
           theta: float, theta_near: float, tokens: int, **how):
    """Answers of all queries: ``(answers, kinds, steps)``, a kind each of "hit", "near", "miss"; ``stored[i]``: the answer of centroid i."""
    idx, _, flags = cache.lookup_multi(queries, [theta_near, theta], count_index=1)
    idx, flags = idx.tolist(), flags.tolist()
    kinds = ["hit" if f[1] else "near" if f[0] else "miss" for f in flags]
    ask = [b for b, kind in enumerate(kinds) if kind != "hit"]
    got, steps = serve(target, [prompts[b] for b in ask], [stored[idx[b]] if kinds[b] == "near" else None for b in ask], tokens, **how)
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
    args = ap.parse_args()
    target = Target()
    cache, stored, queries, prompts = example(target, args.tokens)
    how = dict(most=args.drafts, dtype=siso.FP8 if args.storage == "fp8" else siso.BF16, temperature=args.temperature)
    answers, kinds, steps = answer(cache, stored, target, queries, prompts, 0.9, 0.7, args.tokens, **how)
    for b, kind in enumerate(kinds):
        same = sum(x == y for x, y in zip(answers[b], stored[b]))
        print(f"query {b}: {kind:4s} prompt of {len(prompts[b])} tokens, {same} of {len(answers[b])} tokens as in the stored answer")
    near = [b for b, kind in enumerate(kinds) if kind == "near"]
    _, alone = serve(target, [prompts[b] for b in near], [stored[b] for b in near], args.tokens, **how)
    print(f"{len(kinds)} queries, {kinds.count('hit')} hits, {kinds.count('near')} near hits; {steps} steps for all that missed, "
          f"{alone} for the near hits, {args.tokens} without drafts")


if __name__ == "__main__":
    main()
