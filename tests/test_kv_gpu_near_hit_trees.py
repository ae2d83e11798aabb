"""From a lookup to answers with several stored answers as drafts and a bound on the cache: every attention and every verification against their
definitions in 64 bits."""

import pytest
import torch

import kv_oracle
import kv_tree_oracle as oracle

pytestmark = pytest.mark.gpu


def checks(monkeypatch, seen):
    from paper_2508_18736_amd import siso
    attend, verify_tree, keep, evict = siso.PagedKV.attend, siso.PagedKV.verify_tree, siso.PagedKV.keep, siso.PagedKV.evict

    def checked_attend(self, batch, q, layer=0, tree=None, with_lse=False, **kw):
        out, lse = attend(self, batch, q, layer=layer, tree=tree, with_lse=True, **kw)
        if tree is not None:
            first, length, parent = batch.first.tolist(), batch.length.tolist(), tree.parent.tolist()
            ends = torch.tensor([0, *torch.tensor(length).cumsum(0).tolist()], dtype=torch.int32, device=q.device)
            k, v = (x.double().cpu() for x in self.read(self.batch(ends, batch.length, batch.pages), layer=layer, dtype=torch.float32))
            for b, l in enumerate(length):
                r, at = slice(first[b], first[b + 1]), int(ends[b])
                if first[b + 1] > first[b]:
                    want = oracle.attend(q[r].cpu(), k[at:at + l], v[at:at + l], oracle.seen_by(oracle.ancestors(parent[r]), l), float(torch.tensor(64 ** -0.5)))
                    kv_oracle.check_attend(out[r], lse[r], want, 64, f"sequence {b}")
            seen["attend"] += 1
        return (out, lse) if with_lse else out

    def checked_verify(self, batch, tree, tokens, target, u=None):
        got = verify_tree(self, batch, tree, tokens, target, u)
        first, parent, tok = batch.first.tolist(), tree.parent.tolist(), tokens.tolist()
        accepted, rows, out = (x.tolist() for x in got)
        for b in range(batch.n):
            r = slice(first[b], first[b + 1])
            want = oracle.verify(parent[r], tok[r], target[r].double().cpu().numpy(), None if u is None else u[r].cpu().numpy())
            assert (accepted[b], rows[r], out[r]) == want
            seen["accepted"] += max(want[0], 0)
            seen["jumps"] += any(x > j for j, x in enumerate(rows[r]))
        seen["verify"] += 1
        return got

    def checked_keep(self, batch, rows, layer=None):
        before = [self.read(batch, layer=i) for i in range(self.layers)]
        keep(self, batch, rows, layer)
        path, first = rows.tolist(), batch.first.tolist()
        for i in range(self.layers):
            for x, y in zip(self.read(batch, layer=i), before[i]):
                for b in range(batch.n):
                    for j, r in enumerate(path[first[b]:first[b + 1]]):
                        if r >= 0:
                            assert torch.equal(x[first[b] + j], y[first[b] + r])

    def counted_evict(self, batch, weights, bound, **kw):
        seen["evict"] += 1
        seen["longest"] = max(seen["longest"], int(batch.length.max()))
        evict(self, batch, weights, bound, **kw)

    for name, f in (("attend", checked_attend), ("verify_tree", checked_verify), ("keep", checked_keep), ("evict", counted_evict)):
        monkeypatch.setattr(siso.PagedKV, name, f)


@pytest.mark.parametrize("storage", ["bf16", "fp8"])
@pytest.mark.parametrize("temperature", [0.0, 1.0])
@pytest.mark.parametrize("keep", [0, 40])
def test_answers(monkeypatch, storage, temperature, keep):
    from paper_2508_18736_amd import near_hit, siso

    print(f"case: near hits with trees {storage} {temperature} keep={keep}", flush=True)
    tokens, target = 14, near_hit.Target(layers=2, heads=4, kv_heads=2, head_dim=64, vocab=301)
    cache, stored, queries, prompts = near_hit.example(target, tokens)
    # the stored answers of a near hit: the model's with every sixth token another one, two that part from it early, and one of their own
    drafts = [[[t if i != 3 else (t + 7) % 301 for i, t in enumerate(stored[b])], stored[b], stored[b][:2] + [5, 6, 7], [11, 12]] if b % 3 == 1 else None for b in range(12)]
    seen = {"attend": 0, "verify": 0, "accepted": 0, "jumps": 0, "evict": 0, "longest": 0}
    checks(monkeypatch, seen)
    ask = [b for b in range(12) if b % 3]
    got, steps = near_hit.serve(target, [prompts[b] for b in ask], [drafts[b] for b in ask], tokens, most=9, dtype=siso.FP8 if storage == "fp8" else siso.BF16,
                                temperature=temperature, keep=keep)
    assert all(len(a) == tokens and all(0 <= t < 301 for t in a) for a in got)
    assert steps == tokens and 0 < seen["verify"] < steps and seen["attend"] == 2 * seen["verify"]
    assert (seen["evict"] > 0) == (keep > 0)
    if keep == 0 and temperature == 0.0 and storage == "bf16":
        assert seen["accepted"] > 0 and seen["jumps"] > 0
        _, near_steps = near_hit.serve(target, [prompts[1]], [drafts[1]], tokens, most=9)
        assert near_steps < tokens


@pytest.mark.parametrize("most", [0, 4])
def test_a_bound_with_single_drafts_and_with_none(monkeypatch, most):
    """A bound that no sequence reaches changes nothing; one that they all reach holds."""
    from paper_2508_18736_amd import near_hit

    tokens, target = 20, near_hit.Target(layers=1, heads=4, kv_heads=2, head_dim=64, vocab=301)
    prompts = [list(range(3, 40)), [5], list(range(100, 110))]
    plain, steps = near_hit.serve(target, prompts, [None, [7] * 20, None], tokens, most=most)
    bounded, bounded_steps = near_hit.serve(target, prompts, [None, [7] * 20, None], tokens, most=most, keep=1000)
    assert bounded == plain and bounded_steps == steps
    seen = {"attend": 0, "verify": 0, "accepted": 0, "jumps": 0, "evict": 0, "longest": 0}
    checks(monkeypatch, seen)
    short, _ = near_hit.serve(target, prompts, [None, [7] * 20, None], tokens, most=most, keep=12, recent=4, early=2)
    assert all(len(a) == tokens for a in short) and seen["evict"] > 0 and seen["longest"] == 37


def test_several_of_the_closest_stored_answers(monkeypatch):
    """branches: the stored answers of the centroids that pass the lower threshold are one near hit's drafts, the closest first."""
    from paper_2508_18736_amd import near_hit, siso

    asked = []
    monkeypatch.setattr(near_hit, "serve", lambda target, prompts, drafts, tokens, **how: (asked.append(drafts) or [[1] * tokens for _ in prompts], 1))
    g = torch.Generator().manual_seed(2)
    base = torch.nn.functional.normalize(torch.randn(1, 64, generator=g), dim=1)
    near = lambda c: c * base + (1 - c * c) ** 0.5 * torch.nn.functional.normalize(torch.randn(1, 64, generator=g) - 0 * base, dim=1)  # noqa: E731
    rows = torch.cat([near(0.9), torch.randn(1, 64, generator=g), near(0.97), near(0.93)])
    rows = torch.nn.functional.normalize(rows, dim=1).cuda().bfloat16()
    cache = siso.SisoCache(64, 4, siso.BF16)
    cache.load(rows)
    query = base.cuda().bfloat16()
    similarity = (query.double() @ rows.double().t() / query.double().norm() / rows.double().norm(dim=1))[0].cpu()
    order = [i for i in similarity.argsort(descending=True).tolist() if similarity[i] > 0.6]
    assert len(order) >= 2
    stored = [[10], [20], [30], [40]]
    near_hit.answer(cache, stored, None, query, [[1]], 0.999, 0.6, 2, branches=3)
    assert asked == [[[stored[i] for i in order[:3]]]]
