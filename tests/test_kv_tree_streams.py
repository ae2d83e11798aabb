"""What the tree's and the eviction's calls on another stream than torch's tell torch's allocator, with tensors on the CPU and no handle."""

import pytest
import torch

from test_kv_abi import siso  # noqa: F401
from test_kv_streams import Noted


@pytest.mark.parametrize("call", ["tree", "attend", "verify_tree", "keep", "weigh", "evict"])
def test_what_a_call_reads_and_writes_is_noted(siso, monkeypatch, call):  # noqa: F811
    kv = siso.PagedKV.__new__(siso.PagedKV)
    kv.layers, kv.pages, kv.kv_heads, kv.page_tokens, kv.head_dim = 1, 4, 2, 16, 64
    kv.device, kv._index, kv._stream, kv._h = torch.device("cpu"), -1, None, None
    monkeypatch.setattr(siso.PagedKV, "_elsewhere", lambda self: True)
    monkeypatch.setattr(torch.Tensor, "record_stream", Noted.record_stream)  # (of what the call makes)
    make = lambda *shape, dtype=torch.int32: torch.zeros(shape, dtype=dtype).as_subclass(Noted)  # noqa: E731
    batch = siso.KvBatch(make(2), make(1), make(1, 1), 3, 0, 0)
    tree = siso.KvTree(make(3), make(3, 8), make(3))
    weights = siso.KvWeights(make(1, 4, 2, 16, dtype=torch.float32), make(1, 4, 2, 16))
    q, lse = make(3, 64, 4, dtype=torch.bfloat16).transpose(1, 2), make(3, 4, dtype=torch.float32)  # (without unit stride: copied)
    a, b, c, d = make(3), make(3, 50, dtype=torch.float32), make(3, dtype=torch.float32), make(1, 2)
    fresh, newest, accepted, rows, tokens = make(1), make(1), make(1), make(3), make(3)
    calls = {
        "tree": (lambda: kv.tree(batch, a), [a, batch.first]),
        "attend": (lambda: kv.attend(batch, q, lse=lse, tree=tree), [q, lse, tree.mask, *batch.tensors]),
        "verify_tree": (lambda: kv.verify_tree(batch, tree, a, b, c, out_accepted=accepted, out_rows=rows, out_tokens=tokens),
                        [tree.parent, a, b, c, accepted, rows, tokens, batch.first]),
        "keep": (lambda: kv.keep(batch, a), [a, *batch.tensors]),
        "weigh": (lambda: kv.weigh(batch, q, lse, weights, fresh=fresh, newest=newest), [q, lse, fresh, newest, weights.mass, weights.born, *batch.tensors]),
        "evict": (lambda: kv.evict(batch, weights, 10, to=d), [d, weights.mass, weights.born, *batch.tensors]),
    }
    go, used = calls[call]
    Noted.noted = []
    with pytest.raises(siso.SisoError):  # (there is no handle)
        go()
    assert {t.data_ptr() for t in used} <= {at for at, _ in Noted.noted}
