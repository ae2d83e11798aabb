"""Attention under windows as large as a number can be."""

import pytest
import torch

from gpu_util import DEV
from test_gpu_kv import Setup, ends, ints, siso  # noqa: F401
from test_gpu_kv_heavy import Wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,kind", [(64, Setup), (128, Setup), (64, Wide), (128, Wide), (256, Setup)])
@pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 2 ** 20, 2 ** 23, 208, 207])
def test_windows_of_any_size_and_rows_without_a_position(siso, dtype, d, kind, window):  # noqa: F811
    """More rows than tokens: the first ones have no position.  The others of their tile see everything."""
    print(f"case: wide window {dtype} d={d} {kind.__name__} {window}", flush=True)
    s = kind(siso, dtype, d, 1, 16, [1, 1], [207, 40], seed=150)  # (tables of 208 positions)
    s.write()
    rows = [219, 41]  # (207 and 40 tokens)
    q = torch.randn(sum(rows), 1, d, generator=torch.Generator().manual_seed(1)).bfloat16()
    batch = s.kv.batch(ends(rows), s.length_dev, s.pages)
    out, lse = s.kv.attend(batch, q.to(DEV), window=window, with_lse=True)
    without = [torch.arange(0, 12), torch.arange(219, 220)]
    for at in without:
        assert (out[at] == 0).all() and torch.isneginf(lse[at]).all()
    have = torch.cat([torch.arange(12, 219), torch.arange(220, 260)])
    s.new = [207, 40]
    s.check(q[have], got=(out[have], lse[have]), label=f"window {window}")
