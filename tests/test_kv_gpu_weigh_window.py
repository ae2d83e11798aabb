"""Attention weights under a window (siso_kv_weigh): what is ahead of it, and rows that are cut into stretches."""

import random

import pytest
import torch

import kv_oracle
import kv_tree_oracle as oracle
from gpu_util import DEV
from test_gpu_kv import ends, ints, siso  # noqa: F401
from test_kv_gpu_weigh import Weighed

pytestmark = pytest.mark.gpu

# (new, length, heads of two kv heads, window): few rows of work, many, both, more sequences than a wave takes in, rows below position 0
CASES = [([1, 7, 0], [900, 300, 40], 4, 33), ([100, 300], [2000, 900], 8, 70), ([3, 200, 1], [1500, 700, 64], 4, 100), ([1, 90, 2] * 30, [333, 400, 90] * 30, 4, 47),
         ([20, 80], [10, 700], 6, 5), ([300], [301], 4, 1000)]


def ahead(s, window, page=16):
    """Of every sequence the first page with a position that one of its rows sees."""
    return [max(0, l - m - window + 1) // page for m, l in zip(s.new, s.length)]


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_pages_ahead_of_a_window_may_be_given_up(siso, dtype, case):  # noqa: F811
    """Without decay what no row sees keeps its weight: its pages are not met, whatever the table has for them."""
    new, length, heads, window = CASES[case]
    print(f"case: weigh, pages given up {dtype} {new[:4]} {length[:4]} window={window}", flush=True)
    s = Weighed(siso, dtype, 64, 2, 16, new, length, seed=case)
    s.write()
    q = s.queries(heads)
    pages = s.pages.clone()
    for b, first in enumerate(ahead(s, window)):
        pages[b, :first] = -1
        pages[b, -(-length[b] // 16):] = -1
    batch = s.kv.batch(ends(new), s.length_dev, pages, max_new=max(new))
    lse = s.kv.attend(batch, q.to(DEV), window=window, with_lse=True)[1]
    assert s.kv.bad_pages() == 0
    s.start()
    s.kv.weigh(batch, q.to(DEV), lse, s.weights, window=window)
    s.check_weigh(q, lse, window, label="given up")
    assert s.kv.bad_pages() == 0
    # a position that is noted anew is none of these
    fresh = [max(0, l - m - window + 1) // 16 * 16 for m, l in zip(new, length)]
    s.start()
    s.kv.weigh(batch, q.to(DEV), lse, s.weights, window=window, fresh=ints(fresh))
    s.check_weigh(q, lse, window, fresh=fresh, label="given up, fresh")
    assert s.kv.bad_pages() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("rows", [2, 150])
def test_pages_given_up_and_taken_by_another(siso, dtype, rows):  # noqa: F811
    """The page of a position ahead of the window is another sequence's by now: that one's weights are its own."""
    print(f"case: weigh, pages taken by another {dtype} {rows}", flush=True)
    window = 40
    s = Weighed(siso, dtype, 64, 2, 16, [rows] * 6, [1000, 200, 1000, 230, 900, 180], seed=rows)
    s.write()
    q = s.queries(4)
    for at in (0, 2, 4):  # (the pages of sequence at + 1 were sequence at's first)
        own = -(-s.length[at + 1] // 16)
        s.pages[at, :own] = s.pages[at + 1, :own]
    lse = s.kv.attend(s.batch, q.to(DEV), window=window, with_lse=True)[1]
    table = s.pages.cpu()
    assert all(ahead(s, window)[at] >= -(-s.length[at + 1] // 16) for at in (0, 2, 4))
    s.start()
    s.kv.weigh(s.batch, q.to(DEV), lse, s.weights, window=window)
    got = s.weights.mass.cpu()
    at = 0
    for b, (m, l) in enumerate(zip(s.new, s.length)):  # where each sequence's own pages are
        begin = ahead(s, window)[b] * 16 if b % 2 == 0 else 0
        r = slice(s.starts[b], s.starts[b] + l)
        sums, tol = oracle.weigh(q[at:at + m], kv_oracle.held(s.k, dtype)[r], lse[at:at + m].cpu(), l, window, float(torch.tensor(s.d ** -0.5)))
        j = torch.arange(begin, l)
        pg, slot = table[b, j // 16].long(), j % 16
        had = torch.where(j[:, None] < l - m, s.mass[0, pg, :, slot].double(), torch.zeros((), dtype=torch.float64)).t()
        want = had + sums[:, begin:]
        err = (got[0, pg, :, slot].double().t() - want).abs()
        assert (err <= tol[:, begin:] + 2.0 ** -23 * want).all(), f"sequence {b}"
        at += m


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("rows", [1, 40, 200])
def test_where_it_begins_without_decay(siso, dtype, rows):  # noqa: F811
    """`fresh` at, ahead of and behind what the rows see, anywhere in a page; and none."""
    print(f"case: weigh, fresh and a window {dtype} {rows}", flush=True)
    rng = random.Random(rows)
    new, length = [rows, 1, rows], [700, 333, rows]
    s = Weighed(siso, dtype, 128, 2, 16, new, length, seed=rows)
    s.write()
    q = s.queries(4)
    for window in (1, 20, 300, 5000):
        lse = s.lse_of(q, window=window)
        for fresh in (None, [0, 0, 0], [700, 333, rows], [5, 100, -4], [2000, -2, 1], [rng.randrange(0, l + 1) for l in length]):
            s.start()
            s.kv.weigh(s.batch, q.to(DEV), lse, s.weights, window=window, fresh=None if fresh is None else ints(fresh))
            s.check_weigh(q, lse, window, fresh=fresh, label=f"window {window} fresh {fresh}")
    assert s.kv.bad_pages() == 0
