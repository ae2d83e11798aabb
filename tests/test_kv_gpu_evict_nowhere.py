"""Eviction to other pages where a sequence has none of them."""

import pytest
import torch

from gpu_util import DEV
from test_gpu_kv import siso  # noqa: F401
from test_kv_gpu_evict import Full

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("length", [[300, 20, 0], [40000]])
def test_no_other_pages_leave_all_as_it_was(siso, dtype, length):  # noqa: F811
    print(f"case: evict to nowhere {dtype} {length}", flush=True)
    s = Full(siso, dtype, 64, 2, 16, length, seed=3, layers=2)
    before = [x for i in range(2) for x in s.kv.read(s.all, layer=i)]
    s.kv.evict(s.all, s.weights, 50, recent=9, early=2, to=torch.zeros(len(length), 0, dtype=torch.int32, device=DEV))
    after = [x for i in range(2) for x in s.kv.read(s.all, layer=i)]
    assert all(torch.equal(x, y) for x, y in zip(after, before))
    assert torch.equal(s.weights.mass.cpu(), s.mass) and torch.equal(s.weights.born.cpu(), s.born)
    assert s.kv.bad_pages() == 0
