"""What the paged cache's calls on another stream than torch's tell torch's allocator, with tensors on the CPU and no handle."""

import pytest
import torch

from test_kv_abi import siso  # noqa: F401


class Noted(torch.Tensor):
    noted = []

    def record_stream(self, stream):
        Noted.noted.append((self.data_ptr(), stream))


@pytest.mark.parametrize("call", ["write", "attend"])
def test_what_is_copied_is_kept_until_it_is_read(siso, monkeypatch, call):  # noqa: F811
    """Rows without unit stride are copied on the handle's stream, which reads the caller's own memory then."""
    kv = siso.PagedKV.__new__(siso.PagedKV)
    kv.kv_heads, kv.head_dim, kv.device, kv._index, kv._stream, kv._h = 2, 64, torch.device("cpu"), -1, None, None
    monkeypatch.setattr(siso.PagedKV, "_elsewhere", lambda self: True)
    make = lambda *shape, dtype: torch.zeros(shape, dtype=dtype).as_subclass(Noted)  # noqa: E731
    batch = siso.KvBatch(make(2, dtype=torch.int32), make(1, dtype=torch.int32), make(1, 1, dtype=torch.int32), 3, 0, 0)
    rows = [make(3, 64, 2, dtype=torch.bfloat16).transpose(1, 2) for _ in range(2)]
    Noted.noted = []
    with pytest.raises(siso.SisoError):  # (there is no handle)
        kv.write(batch, *rows) if call == "write" else kv.attend(batch, rows[0])
    noted = {at for at, _ in Noted.noted}
    assert {t.data_ptr() for t in batch.tensors} <= noted
    assert {t.data_ptr() for t in (rows if call == "write" else rows[:1])} <= noted
