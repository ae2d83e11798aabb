"""From a lookup to answers: every attention and every verification of the loop against their definitions in 64 bits."""

import pytest
import torch

import kv_oracle

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("storage", ["bf16", "fp8"])
@pytest.mark.parametrize("temperature", [0.0, 1.0])
def test_answers(monkeypatch, storage, temperature):
    from paper_2508_18736_amd import near_hit, siso

    print(f"case: near hit {storage} {temperature}", flush=True)
    tokens, target = 14, near_hit.Target(layers=2, heads=4, kv_heads=2, head_dim=64, vocab=301)
    cache, stored, queries, prompts = near_hit.example(target, tokens)
    seen = {"attend": 0, "verify": 0, "accepted": 0, "drafted": 0}
    attend, verify = siso.PagedKV.attend, siso.PagedKV.verify

    def checked_attend(self, batch, q, layer=0, **kw):
        out, lse = attend(self, batch, q, layer=layer, with_lse=True, **kw)
        first, length = batch.first.tolist(), batch.length.tolist()
        ends = torch.tensor([0, *torch.tensor(length).cumsum(0).tolist()], dtype=torch.int32, device=q.device)
        everything = self.batch(ends, batch.length, batch.pages)
        k, v = self.read(everything, layer=layer, dtype=torch.float32)  # (code times scale, rounded to 24 bits: 2^-24 of a score, in the bar's four)
        k, v = k.double().cpu(), v.double().cpu()
        for b, l in enumerate(length):
            m, at = first[b + 1] - first[b], int(ends[b])
            keep = min(m, 6)  # (of a prompt the last rows)
            r = slice(first[b + 1] - keep, first[b + 1])
            want = kv_oracle.attend(q[r], k[at:at + l], v[at:at + l], l, keep, float(torch.tensor(64 ** -0.5)))
            kv_oracle.check_attend(out[r], lse[r], want, 64, f"sequence {b}")
        seen["attend"] += 1
        return out

    def checked_verify(self, batch, toks, target_rows, draft=None, u_accept=None, u_sample=None):
        accepted, out = verify(self, batch, toks, target_rows, draft, u_accept, u_sample)
        rows = batch.first.diff().tolist()
        wide = lambda t: None if t is None else t.double().cpu().numpy()  # noqa: E731
        want = kv_oracle.verify(toks.tolist(), rows, wide(target_rows), None, wide(u_accept), wide(u_sample))
        assert accepted.tolist() == want[0]
        assert out.tolist() == want[1]
        seen["verify"] += 1
        seen["accepted"] += sum(max(a, 0) for a in want[0])
        seen["drafted"] += sum(max(m - 1, 0) for m in rows)
        return accepted, out

    monkeypatch.setattr(siso.PagedKV, "attend", checked_attend)
    monkeypatch.setattr(siso.PagedKV, "verify", checked_verify)
    answers, kinds, steps = near_hit.answer(cache, stored, target, queries, prompts, 0.9, 0.7, tokens, most=4,
                                            dtype=siso.FP8 if storage == "fp8" else siso.BF16, temperature=temperature)
    assert kinds == ["hit", "near", "miss"] * 4
    assert all(len(a) == tokens and all(0 <= t < 301 for t in a) for a in answers)
    assert all(answers[b] == stored[b] for b in range(0, 12, 3))
    assert steps == tokens and seen["verify"] == steps and seen["attend"] == 2 * steps  # (the misses take a step for each token)
    assert seen["drafted"] > 0
    if temperature == 0.0 and storage == "bf16":
        assert seen["accepted"] > 0
        _, near_steps = near_hit.serve(target, [prompts[1]], [stored[1]], tokens)
        assert near_steps < tokens


def test_nothing_to_answer():
    from paper_2508_18736_amd import near_hit
    assert near_hit.serve(near_hit.Target(layers=1, heads=2, vocab=50), [], [], 5) == ([], 0)
