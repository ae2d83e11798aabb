"""First rows that decrease, which no batch may have: what such a call returns is not said, the calls behind it are as ever."""

import pytest
import torch

from gpu_util import DEV
from test_gpu_kv import Setup, ends, ints, siso  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("times", [1, 40])  # (40: the plan has a launch of its own)
@pytest.mark.parametrize("d", [64, 128])
def test_calls_behind_rows_that_two_sequences_claim(siso, dtype, d, times):  # noqa: F811
    """The device meets more tiles than the host counted workgroups for; sequences of many positions, which would be cut."""
    print(f"case: decreasing first rows {dtype} d={d} {times}", flush=True)
    s = Setup(siso, dtype, d, 1, 64, [1, 3, 40], [3500, 900, 2000], seed=140)
    s.write()
    q = s.queries(2)
    want = s.kv.attend(s.batch, q.to(DEV), with_lse=True)
    s.check(q, got=want, label="before")
    first = [0] + [1000, 0] * times + [1000]
    n = len(first) - 1
    table = s.pages[0].expand(n, -1).contiguous()
    x = torch.randn(1000, 1, d, device=DEV).bfloat16()
    for bound in (1, 0):
        s.kv.attend(s.kv.batch(ints(first), ints([3500] * n), table, rows=1000, max_length=bound), x)
        for _ in range(2):
            got = s.kv.attend(s.batch, q.to(DEV), with_lse=True)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
            s.check(q, got=got, label="behind")
    assert s.kv.bad_pages() == 0
