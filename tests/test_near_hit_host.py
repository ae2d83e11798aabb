"""What near_hit does before and around the model's steps, without a GPU."""

import pytest
import torch

from test_kv_abi import siso  # noqa: F401


class Lookup:
    """Answers of a lookup that are given."""

    def __init__(self, idx, flags):
        self.idx, self.flags = torch.tensor(idx), torch.tensor(flags)

    def lookup_multi(self, queries, thetas, count_index):
        return self.idx, None, self.flags


def test_an_empty_cache_has_no_stored_answers(siso, monkeypatch):  # noqa: F811
    from paper_2508_18736_amd import near_hit

    asked = []
    monkeypatch.setattr(near_hit, "serve", lambda target, prompts, drafts, tokens, **how: (asked.append((prompts, drafts)) or [[7] * tokens for _ in prompts], 3))
    got = near_hit.answer(Lookup([-1, -1], [[0, 0], [0, 0]]), [], None, None, [[1], [2, 3]], 0.9, 0.7, 4)
    assert got == ([[7] * 4, [7] * 4], ["miss", "miss"], 3)
    assert asked == [([[1], [2, 3]], [None, None])]
    # and beside others
    got = near_hit.answer(Lookup([0, -1, 0], [[1, 1], [0, 0], [1, 0]]), [[5, 6, 8, 9, 9]], None, None, [[1], [2, 3], [4]], 0.9, 0.7, 4)
    assert got == ([[5, 6, 8, 9], [7] * 4, [7] * 4], ["hit", "miss", "near"], 3)
    assert asked[1] == ([[2, 3], [4]], [None, [5, 6, 8, 9, 9]])


@pytest.mark.parametrize("tokens", [0, -1])
def test_no_tokens_are_no_steps(siso, tokens):  # noqa: F811
    from paper_2508_18736_amd import near_hit

    target = near_hit.Target(layers=1, heads=2, vocab=50, device="cpu")
    assert near_hit.serve(target, [[1, 2], [3]], [None, [4]], tokens) == ([[], []], 0)


def test_a_prompt_without_tokens_is_refused(siso):  # noqa: F811
    from paper_2508_18736_amd import near_hit

    target = near_hit.Target(layers=1, heads=2, vocab=50, device="cpu")
    with pytest.raises(ValueError):
        near_hit.serve(target, [[1, 2], []], [None, None], 3)


def test_the_command_serves_all_its_calls_alike(siso, monkeypatch, capsys):  # noqa: F811
    """The steps that are printed side by side are steps of one storage and one temperature."""
    import sys

    from paper_2508_18736_amd import near_hit

    calls = []

    def serve(target, prompts, drafts, tokens, **how):
        calls.append(how)
        return [[1] * tokens for _ in prompts], 2

    monkeypatch.setattr(near_hit, "serve", serve)
    monkeypatch.setattr(near_hit, "Target", lambda: None)
    monkeypatch.setattr(near_hit, "example", lambda target, tokens: (Lookup([0, 0], [[1, 0], [0, 0]]), [[1] * 5] * 2, None, [[1], [2]]))
    monkeypatch.setattr(sys, "argv", ["near_hit", "--storage", "fp8", "--temperature", "0.5", "--drafts", "3", "--tokens", "5"])
    near_hit.main()
    assert calls == [dict(most=3, dtype=siso.FP8, temperature=0.5)] * 2
    assert "1 near hits; 2 steps" in capsys.readouterr().out


def test_fewer_drafts_than_none_are_refused(siso):  # noqa: F811
    from paper_2508_18736_amd import near_hit

    target = near_hit.Target(layers=1, heads=2, vocab=50, device="cpu")
    with pytest.raises(ValueError):
        near_hit.serve(target, [[1, 2]], [[3, 4]], 3, most=-1)
