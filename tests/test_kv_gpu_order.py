"""Batches that no caller may give: first rows that decrease (what such a call returns is not said, the calls behind it are as ever) and
tables wider than kernels count."""

import ctypes as C

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


@pytest.mark.parametrize("page", [16, 1024])
def test_tables_of_more_positions_than_kernels_count(siso, page):  # noqa: F811
    """The widest table is taken (none of it beyond the length is read), one page more is refused by every call that takes one."""
    kv = siso.PagedKV(1, 64, 2, page_tokens=page)
    widest = (2 ** 31 - 2 ** 25) // page
    first, length, pages = ints([0, 2]), ints([2]), ints([[1]])
    x = torch.randn(2, 1, 64, device=DEV).bfloat16()
    for width, rc in ((widest, siso.OK), (widest + 1, siso.EINVAL), ((2 ** 31 - 1) // page, siso.EINVAL)):
        batch = siso._KvBatchStruct(n=1, rows=2, first=first.data_ptr(), length=length.data_ptr(), pages=pages.data_ptr(), width=width, max_new=0, max_length=0)
        out = [torch.zeros_like(x) for _ in range(3)]
        assert siso._lib.siso_kv_write(kv._h, 0, C.byref(batch), x.data_ptr(), 64, 64, x.data_ptr(), 64, 64) == rc
        assert siso._lib.siso_kv_read(kv._h, 0, C.byref(batch), siso.BF16, out[0].data_ptr(), out[1].data_ptr()) == rc
        assert siso._lib.siso_kv_attend(kv._h, 0, C.byref(batch), x.data_ptr(), 64, 64, 1, 0.125, 0, out[2].data_ptr(), None) == rc
        if rc == siso.OK:
            assert torch.equal(out[0], x) and torch.equal(out[1], x) and torch.equal(out[2][0], x[0])
        else:
            assert b"pages" in siso._lib.siso_kv_last_error(kv._h)
    assert kv.bad_pages() == 0
