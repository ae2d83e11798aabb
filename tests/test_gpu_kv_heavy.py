"""Attention of long chunks over the paged cache in the kernel for heavy work.  Which kernel takes a call goes by how long sequences can
be, not by how long they are: a table with room for millions of positions sends small cases there.  Work that is heavy by itself,
under a window, is checked at some of its rows and heads."""

import math

import pytest
import torch

import kv_oracle
import test_gpu_kv_batch as batches
import test_gpu_kv_chunk as chunks
from gpu_util import DEV
from test_gpu_kv import Setup, ends, siso  # noqa: F401

pytestmark = pytest.mark.gpu


class Wide(Setup):
    def __init__(self, *args, **kwargs):
        super().__init__(*args, **kwargs)
        wide = torch.zeros(len(self.new), (1 << 23) // self.page, dtype=torch.int32, device=DEV)
        wide[:, :self.pages.shape[1]] = self.pages
        self.pages = wide
        self.all = self.kv.batch(ends(self.length), self.length_dev, self.pages)
        self.batch = self.kv.batch(ends(self.new), self.length_dev, self.pages, max_new=max(self.new))


@pytest.fixture
def wide(monkeypatch):
    monkeypatch.setattr(chunks, "Setup", Wide)
    monkeypatch.setattr(batches, "Setup", Wide)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("case", range(len(chunks.CASES)))
def test_chunks(siso, wide, dtype, case):  # noqa: F811
    chunks.test_chunks(siso, dtype, case, 0)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,new,length", [(64, [150], [2500]), (128, [140], [3001]), (128, [150, 2, 131], [1700, 900, 140])])
def test_chunks_over_a_long_axis(siso, wide, dtype, d, new, length):  # noqa: F811
    chunks.test_chunks_over_a_long_axis(siso, dtype, d, new, length)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_does_not_touch_it(siso, wide, dtype, what):  # noqa: F811
    chunks.test_what_a_row_does_not_see_does_not_touch_it(siso, dtype, what)


def test_infinite_values_reach_the_rows_that_see_them(siso, wide):  # noqa: F811
    chunks.test_infinite_values_reach_the_rows_that_see_them(siso)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_large_and_small_scores(siso, wide, dtype):  # noqa: F811
    chunks.test_large_and_small_scores(siso, dtype)


def test_pages_that_are_none_and_rows_without_a_position(siso, wide):  # noqa: F811
    chunks.test_pages_that_are_none_and_rows_without_a_position(siso)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_queries_in_any_order_of_memory_and_the_same_bits_twice(siso, wide, dtype):  # noqa: F811
    chunks.test_queries_in_any_order_of_memory_and_the_same_bits_twice(siso, dtype)


def test_recorded_in_a_graph(siso, wide):  # noqa: F811
    chunks.test_recorded_in_a_graph(siso)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_many_sequences_and_chunks_among_them(siso, wide, dtype):  # noqa: F811
    batches.test_many_sequences_and_chunks_among_them(siso, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,rows", [(64, 140), (128, 300), (192, 130)])
@pytest.mark.parametrize("grow", [40.0, 400.0])
def test_a_maximum_that_grows_beyond_any_power(siso, wide, dtype, d, rows, grow):  # noqa: F811
    batches.test_a_maximum_that_grows_beyond_any_power(siso, dtype, d, rows, grow)


def test_values_whose_sums_leave_the_range(siso, wide):  # noqa: F811
    batches.test_values_whose_sums_leave_the_range(siso)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,window", [(64, 1), (64, 90), (128, 70), (128, 700)])
def test_windows(siso, dtype, d, window):  # noqa: F811
    """Two sequences of 1,300 or, under the smallest window, 4,100 rows of 96 or 128 heads (as many rows each: the smaller bound)."""
    m = 4100 if window == 1 else 1300
    heads, kv_heads, new, length = (128 if window < 100 else 96), 32, [m, m], [m + 233, m + 100]
    print(f"case: heavy window {dtype} d={d} {window}", flush=True)
    s = Setup(siso, dtype, d, kv_heads, 32, new, length, seed=95)
    if window < 700:  # values behind the window that are not finite
        s.k[:100], s.v[:100] = math.nan, math.inf
    s.write()
    q = s.queries(heads)
    s.batch = s.kv.batch(ends(new), s.length_dev, s.pages, max_new=max(new))
    out, lse = s.kv.attend(s.batch, q.to(DEV), window=window, with_lse=True)
    hk, hv = kv_oracle.held(s.k, dtype), kv_oracle.held(s.v, dtype)
    g, first = torch.Generator().manual_seed(1), 0
    for b, (m, l) in enumerate(zip(new, length)):
        for i in {*torch.randint(0, max(m, 1), (24,), generator=g).tolist(), 0, max(m - 1, 0)} if m else ():
            pos = l - m + i
            if b == 0 and pos - window < 100:  # (sees some of them)
                continue
            for h in torch.randint(0, heads, (3,), generator=g).tolist():
                at, kh = s.starts[b], h // (heads // kv_heads)
                want = kv_oracle.attend(q[first + i:first + i + 1, h:h + 1], hk[at:at + pos + 1, kh:kh + 1], hv[at:at + pos + 1, kh:kh + 1], pos + 1, 1,
                                        float(torch.tensor(d ** -0.5)), window)
                kv_oracle.check_attend(out[first + i:first + i + 1, h:h + 1], lse[first + i:first + i + 1, h:h + 1], want, d, f"row {i} of {b}, head {h}")
        first += m
    assert s.kv.bad_pages() == 0
