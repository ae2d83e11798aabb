"""Attention of long chunks over tables with page numbers that are none: nothing of the page that stands in for them reaches a row."""

import math

import pytest
import torch

from gpu_util import DEV
from test_gpu_kv import ends, ints, siso  # noqa: F401
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
