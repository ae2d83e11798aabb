"""Page numbers that are none, where eviction meets them (siso_kv_evict)."""

import pytest
import torch

from gpu_util import DEV
from test_gpu_kv import ends, siso  # noqa: F401
from test_kv_gpu_evict import Full

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("born", [True, False])
@pytest.mark.parametrize("length", [[300, 200], [20000, 60], [40000], [100] * 300])
def test_pages_that_are_none_are_counted_though_nothing_of_them_is_kept(siso, length, born):  # noqa: F811
    """Their slots are the first to go, so nothing of them moves; each is counted once at least, and for each layer.  A page beyond the length is
    not met, nor is any of a sequence that keeps all it has."""
    print(f"case: evict, pages that are none {length[:3]} born={born}", flush=True)
    s = Full(siso, "fp8", 64, 2, 16, length, seed=8, layers=2)
    weights = s.weights if born else s.kv.weights(s.weights.mass)
    table = torch.cat([s.pages, torch.full((len(length), 1), -1, dtype=torch.int32, device=DEV)], 1)
    kept = s.kv.batch(ends([0] * len(length)), s.length_dev, table)
    s.kv.evict(kept, weights, 50, recent=9)
    assert s.kv.bad_pages() == 0
    s.weights.mass.copy_(s.mass)
    for b, l in enumerate(length):
        table[b, 4], table[b, l // 16 - 1] = -1, s.pool  # (beyond the slots that stay)
    batch = s.kv.batch(ends([0] * len(length)), s.length_dev, table)
    s.kv.evict(batch, weights, max(length))
    assert s.kv.bad_pages() == 0
    before = 0
    for layer, layers in ((1, 1), (None, 2)):
        s.kv.evict(batch, weights, 50, recent=9, layer=layer)
        after = s.kv.bad_pages()
        assert after - before >= 2 * layers * sum(l > 60 for l in length)
        before = after
