"""What the binding hands to siso_kv_evict for the pages that what is kept goes to, on the CPU: the call is looked at, not made."""

import pytest
import torch

from test_kv_abi import siso  # noqa: F401


@pytest.mark.parametrize("n,width", [(1, 0), (3, 0), (2, 5)])
def test_other_pages_are_never_taken_for_none(siso, monkeypatch, n, width):  # noqa: F811
    """A tensor without elements has no address, and no address means in place: pages of a sequence that are none at all are not the batch's own."""
    calls = []

    class Library:
        def siso_kv_evict(self, *args):
            calls.append(args)
            return 0

    monkeypatch.setattr(siso, "_lib", Library())
    kv = siso.PagedKV.__new__(siso.PagedKV)
    kv.kv_heads, kv.head_dim, kv.pages, kv.page_tokens, kv.layers = 2, 64, 5, 16, 2
    kv.device, kv._index, kv._h, kv._stream, kv._raw_stream = torch.device("cpu"), -1, None, None, 0
    kv._elsewhere = lambda: False
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32)  # noqa: E731
    batch = siso.KvBatch(i32(n + 1), i32(n), i32(n, 2), 0, 0, 0)
    kv.evict(batch, kv.weights(), 10, to=i32(n, width))
    kv.evict(batch, kv.weights(), 10)
    assert calls[0][8] and calls[0][9] == width
    assert calls[1][8] is None and calls[1][9] == 0
