"""siso_kv_weigh with a page table without columns, on the CPU: there are no positions, and nothing is asked of the GPU."""

import pytest

from test_kv_abi import siso  # noqa: F401
from test_kv_tree_abi import A, at, batch  # noqa: F401


@pytest.mark.parametrize("n,rows,max_new", [(1, 3, 0), (1, 300, 0), (2, 600, 300), (70, 70, 1), (70, 7000, 0)])
def test_a_table_without_columns(siso, at, n, rows, max_new):  # noqa: F811
    b = batch(siso, n=n, rows=rows, max_new=max_new, width=0)
    assert siso._lib.siso_kv_weigh(at[0], 0, b, A, 256, 64, 4, 1.0, 0, A, None, None, 1.0, A, A) == siso.OK
    assert siso._lib.siso_kv_weigh(at[0], 0, b, A, 256, 64, 4, 1.0, 5, A, None, None, 0.5, A, None) == siso.OK
    # what is refused is refused
    assert siso._lib.siso_kv_weigh(at[0], 0, b, A, 256, 64, 4, 1.0, 0, None, None, None, 1.0, A, A) == siso.EINVAL
