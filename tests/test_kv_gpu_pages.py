"""Attention over tables with page numbers that are none: nothing of the page that stands in for them reaches a row, and those ahead
of a window are not met."""

import math

import pytest
import torch

from gpu_util import DEV
from test_gpu_kv import Setup, ints, siso  # noqa: F401
from test_gpu_kv_heavy import Wide

pytestmark = pytest.mark.gpu


def without_the_first_page(s):
    """The cache's first page is in no table: whatever a test writes there belongs to nobody."""
    used = set(s.pages.flatten().tolist())
    spare = next(p for p in range(1, s.pool) if p not in used)
    at = torch.zeros_like(s.pages, dtype=torch.bool)
    for b, l in enumerate(s.length):
        at[b, :-(-l // s.page)] = True
    s.pages[at & (s.pages == 0)] = spare


# positions behind 0 in whole stages that all rows see; one piece, and cut into some
@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,rows,length,none", [(64, 140, 250, 1), (64, 150, 2500, 70), (128, 260, 500, 3), (128, 260, 3001, 130), (192, 130, 900, 5)])
@pytest.mark.parametrize("there", [25.0, math.inf])
@pytest.mark.parametrize("grows", [False, True])
def test_scores_of_no_page_do_not_weigh(siso, dtype, d, rows, length, none, there, grows):  # noqa: F811
    """Scores that a row sees lie far below zero, those of the first page far above, or at infinity; later ones may pass the first
    by more than single precision's powers."""
    print(f"case: scores of no page {dtype} d={d} {rows} of {length} {there} {grows}", flush=True)
    s = Wide(siso, dtype, d, 1, 16, [rows], [length], seed=120)
    without_the_first_page(s)
    s.k -= 25
    if grows:
        s.k[length - rows - 20] += 15
    s.write()
    first = s.kv.batch(ints([0, 16]), ints([16]), ints([[0]]))
    x = torch.full((16, 1, d), there, dtype=torch.bfloat16, device=DEV)
    s.kv.write(first, x, x)
    s.pages[0, none] = -1
    q = (1 + 0.1 * s.queries(1).float()).bfloat16()
    s.check(q, hidden={0: range(16 * none, 16 * none + 16)}, label="no page")
    assert s.kv.bad_pages() > 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,page,new,length", [(64, 16, [1, 4], [900, 333]), (64, 32, [150], [700]), (128, 16, [3, 1, 2], [2100, 60, 515]),
                                               (128, 64, [270, 140], [1000, 300]), (192, 16, [1, 130], [777, 400]), (256, 16, [2], [450])])
@pytest.mark.parametrize("window", [1, 17, 45, 100, 250])
@pytest.mark.parametrize("kind", [Setup, Wide])
def test_pages_given_up_ahead_of_a_window(siso, dtype, d, page, new, length, window, kind):  # noqa: F811
    """Whoever keeps a window gives up the pages that no row sees any more: they are not met, and the bits are the same."""
    print(f"case: pages given up {dtype} d={d} {page} {new} {length} {window} {kind.__name__}", flush=True)
    s = kind(siso, dtype, d, 1, page, new, length, seed=121)
    s.k[:2], s.v[:2] = math.nan, math.inf  # (of the first sequence, ahead of all windows)
    s.write()
    q = s.queries(2)
    want = s.kv.attend(s.batch, q.to(DEV), window=window, with_lse=True)
    for b, (m, l) in enumerate(zip(new, length)):
        s.pages[b, :max(0, l - m - window + 1) // page] = -1
    got = s.kv.attend(s.batch, q.to(DEV), window=window, with_lse=True)
    assert s.kv.bad_pages() == 0
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    s.check(q, window=window, got=got, label="pages given up")
