"""Which entries of the page table the attention of wide trees looks up, where sequences have fewer positions than rows."""

import pytest

from test_gpu_kv import ends, siso  # noqa: F401
from test_kv_gpu_tree_chunks import Heavy

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,heads", [(128, 4), (256, 8), (64, 4)])
@pytest.mark.parametrize("window", [0, 50])
def test_rows_below_position_zero_look_up_nothing(siso, dtype, d, heads, window):  # noqa: F811
    """Tiles whose rows all stand below position 0, behind and ahead of other sequences.  All that the table holds beyond a sequence's own pages is
    no page, the last entry of every row among it, which lies ahead of the next row's first: none of it is met."""
    print(f"case: tiles without positions {dtype} d={d} window={window}", flush=True)
    new, length = [256, 200, 32, 256, 250], [100, 1500, 10, 1, 250]
    s = Heavy(siso, dtype, d, 1, 16, new, length, seed=d)
    s.write()
    for b, l in enumerate(length):
        s.pages[b, -(-l // 16):] = -1
    s.batch = s.kv.batch(ends(new), s.length_dev, s.pages, max_new=256)
    s.check_tree(s.queries(heads), window=window, label=f"{dtype} d={d}")
    assert s.kv.bad_pages() == 0


def test_more_sequences_than_a_wave_plans_for(siso):  # noqa: F811
    new, length = [256, 40] * 35, [100, 41] * 35
    s = Heavy(siso, "bf16", 64, 1, 16, new, length, seed=5)
    s.write()
    for b, l in enumerate(length):
        s.pages[b, -(-l // 16):] = -1
    s.batch = s.kv.batch(ends(new), s.length_dev, s.pages, max_new=256)
    s.check_tree(s.queries(4), label="many")
    assert s.kv.bad_pages() == 0
