"""Trees of drafted tokens over the paged cache (siso_kv_tree, siso_kv_attend_tree) against their definition in 64 bits."""

import math
import random

import pytest
import torch

import kv_oracle
import kv_tree_oracle as oracle
from gpu_util import DEV
from test_gpu_kv import Setup, ends, ints, siso  # noqa: F401

pytestmark = pytest.mark.gpu


def random_tree(m, branch, seed):
    rng = random.Random(seed)
    return [-1] + [i - 1 if rng.randrange(100) >= branch else rng.randrange(-1, i) for i in range(1, m)] if m else []


class Trees(Setup):
    def __init__(self, siso, dtype, d, kv_heads, page, new, length, branch=40, seed=0, **more):  # noqa: F811
        super().__init__(siso, dtype, d, kv_heads, page, new, length, seed=seed, **more)
        self.parents = [random_tree(m, branch, seed + b) for b, m in enumerate(new)]
        self.tree = self.kv.tree(self.batch, ints([p for t in self.parents for p in t]))

    def check_tree(self, q, lists=None, scale=None, window=0, hidden=None, label="", got=None):
        scale = self.d ** -0.5 if scale is None else scale
        out, lse = got if got is not None else self.kv.attend(self.batch, q.to(DEV), scale=scale, window=window, with_lse=True, tree=self.tree)
        torch.cuda.synchronize()
        lists = [oracle.ancestors(p) for p in self.parents] if lists is None else lists
        hk, hv = kv_oracle.held(self.k, self.dtype), kv_oracle.held(self.v, self.dtype)
        at = 0
        for b, (m, l) in enumerate(zip(self.new, self.length)):
            s = self.starts[b]
            seen = oracle.seen_by(lists[b], l, window, (hidden or {}).get(b, ()))
            want = oracle.attend(q[at:at + m], hk[s:s + l], hv[s:s + l], seen, float(torch.tensor(scale)))
            kv_oracle.check_attend(out[at:at + m], lse[at:at + m], want, self.d, f"{label} sequence {b} ({m} of {l})")
            at += m


@pytest.mark.parametrize("sizes", [[1], [256], [0, 1, 2, 31, 32, 33, 64, 65, 200, 256, 0], [1] * 100])
@pytest.mark.parametrize("branch", [0, 40, 100])
def test_masks_and_depths(siso, sizes, branch):  # noqa: F811
    print(f"case: masks {sizes[:12]} {branch}", flush=True)
    kv = siso.PagedKV(1, 64, 1)
    batch = kv.batch(ends(sizes), rows=sum(sizes), max_new=max(sizes))
    parents = [random_tree(m, branch, 7 * b + branch) for b, m in enumerate(sizes)]
    tree = kv.tree(batch, ints([p for t in parents for p in t]))
    lists = [x for p in parents for x in oracle.ancestors(p)]
    assert torch.equal(tree.mask.cpu(), oracle.words(lists))
    assert tree.depth.tolist() == [len(x) - 1 for x in lists]


def test_parents_that_are_none(siso):  # noqa: F811
    """A row that names itself, a later row or a number that is no row continues the context."""
    kv = siso.PagedKV(1, 64, 1)
    parents = [0, 0, 2, 9, -7, 1 << 30, 3, -(1 << 31)]
    tree = kv.tree(kv.batch(ints([0, 8])), ints(parents))
    lists = oracle.ancestors(parents)
    assert torch.equal(tree.mask.cpu(), oracle.words(lists)) and tree.depth.tolist() == [len(x) - 1 for x in lists]


# (heads of kv_heads, dimension, page): of the last four more than 128 rows of work go to the kernel for heavy work
@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,page,kv_heads,heads", [(64, 16, 2, 4), (128, 64, 2, 8), (72, 16, 3, 3), (8, 32, 1, 5), (192, 32, 2, 8), (256, 16, 1, 4), (136, 128, 1, 8), (200, 16, 2, 2)])
def test_rows_see_the_context_and_their_ancestors(siso, dtype, d, page, kv_heads, heads):  # noqa: F811
    print(f"case: tree {dtype} d={d} page={page} heads={heads}/{kv_heads}", flush=True)
    new, length = [1, 7, 33, 64, 0, 200], [1, 300, 33, 65, 40, 777]
    s = Trees(siso, dtype, d, kv_heads, page, new, length, seed=d)
    s.write()
    s.check_tree(s.queries(heads), label=f"{dtype} d={d}")
    assert s.kv.bad_pages() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128, 192])
@pytest.mark.parametrize("window", [1, 2, 5, 40, 100000])
def test_windows_count_depth_not_rows(siso, dtype, d, window):  # noqa: F811
    print(f"case: tree window {window} {dtype} d={d}", flush=True)
    s = Trees(siso, dtype, d, 2, 16, [9, 100, 60], [9, 400, 61], branch=20, seed=window % 97)
    s.write()
    s.check_tree(s.queries(4), window=window, label=f"window {window}")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,new,length", [(128, [256, 250], [20000, 9001]), (64, [256] * 3, [30000, 7, 15000])])
def test_wide_trees_behind_long_contexts(siso, dtype, d, new, length):  # noqa: F811
    """So much work that the kernel for chunks takes it, positions cut into pieces."""
    print(f"case: wide trees {dtype} d={d}", flush=True)
    length = [max(l, m) for l, m in zip(length, new)]
    s = Trees(siso, dtype, d, 1, 64, new, length, branch=60, seed=5)
    s.write()
    s.check_tree(s.queries(8), label="wide")
    s.check_tree(s.queries(8), window=700, label="wide, window")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 192])
def test_any_mask(siso, dtype, d):  # noqa: F811
    """Masks that are no trees, bits of later rows, and rows that see nothing."""
    print(f"case: any mask {dtype} d={d}", flush=True)
    new, length = [100, 70, 3], [100, 300, 3]
    s = Trees(siso, dtype, d, 1, 16, new, length, seed=3)
    s.write()
    rng = random.Random(4)
    lists = [[sorted(rng.sample(range(256), rng.randrange(0, 40))) if rng.random() < 0.8 else [] for _ in range(m)] for m in new]
    lists[2] = [[], [2], []]
    s.tree = siso.KvTree(s.tree.parent, oracle.words([x for t in lists for x in t]).to(DEV), s.tree.depth)
    s.check_tree(s.queries(2), lists=lists, label="any mask")
    s.check_tree(s.queries(2), lists=lists, window=3, label="any mask, window")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 192])
def test_what_a_row_does_not_see_does_not_touch_it(siso, dtype, d):  # noqa: F811
    """Infinities and NaN in keys and values of other branches and ahead of a window."""
    print(f"case: not seen {dtype} d={d}", flush=True)
    new, length = [90, 12], [300, 12]
    s = Trees(siso, dtype, d, 1, 16, new, length, branch=0, seed=11)
    s.parents = [[-1] + [0 if i in (1, 40) else i - 1 for i in range(1, 90)], [-1, 0, 1, 0, 3, 4, 4, 4, 7, 7, 7, 7]]
    s.tree = s.kv.tree(s.batch, ints([p for t in s.parents for p in t]))
    for at in (210 + 39, 300 + 6, 300 + 8):  # the end of the first branch, leaves
        s.k[at], s.v[at] = math.nan, math.inf
    s.k[3], s.v[3], s.v[4, 0, 5] = math.inf, math.nan, -math.inf  # ahead of the window
    s.write()
    out, lse = s.kv.attend(s.batch, s.queries(2).to(DEV), window=150, with_lse=True, tree=s.tree)
    touched = [39, 90 + 6, 90 + 8]
    fine = [i for i in range(102) if i not in touched]
    assert torch.isfinite(out[fine].float()).all() and torch.isfinite(lse[fine]).all()
    assert not torch.isfinite(out[touched].float()).any()
    at = 0
    hk, hv = kv_oracle.held(s.k, dtype), kv_oracle.held(s.v, dtype)
    for b, (m, l) in enumerate(zip(new, length)):
        seen = oracle.seen_by([oracle.ancestors(s.parents[b])[i] if at + i in fine else [] for i in range(m)], l, 150)
        rows = [i for i in range(m) if at + i in fine]
        want = oracle.attend(s.queries(2)[at:at + m], hk[s.starts[b]:s.starts[b] + l], hv[s.starts[b]:s.starts[b] + l], seen, float(torch.tensor(d ** -0.5)))
        kv_oracle.check_attend(out[at:at + m][rows], lse[at:at + m][rows], [x[rows] for x in want], d, f"sequence {b}")
        at += m


@pytest.mark.parametrize("d", [128, 192])
def test_pages_that_are_none(siso, d):  # noqa: F811
    print(f"case: tree, pages that are none d={d}", flush=True)
    s = Trees(siso, "bf16", d, 2, 16, [70, 5], [200, 60], seed=6)
    s.write()
    pages = s.pages.clone()
    pages[0, 2], pages[0, 10], pages[1, 3] = -1, s.pool, 1 << 30
    s.batch = s.kv.batch(ends(s.new), s.length_dev, pages, max_new=70)
    s.check_tree(s.queries(4), hidden={0: [*range(32, 48), *range(160, 176)], 1: [*range(48, 60)]}, label="no page")
    assert s.kv.bad_pages() > 0


def test_more_rows_than_positions_and_a_chain_is_what_attend_computes(siso):  # noqa: F811
    s = Trees(siso, "bf16", 64, 2, 16, [40, 33, 8], [25, 90, 50], branch=0, seed=8)
    s.parents = [[-1, *range(m - 1)] for m in s.new]
    s.tree = s.kv.tree(s.batch, ints([p for t in s.parents for p in t]))
    s.write()
    q = s.queries(4)
    s.check_tree(q, label="more rows than positions")
    s.check(q, label="a chain", got=s.kv.attend(s.batch, q.to(DEV), with_lse=True, tree=s.tree))  # (the bar of siso_kv_attend)


def test_many_sequences_strides_and_scale(siso):  # noqa: F811
    """More sequences than a wave plans for; queries within a wider tensor; a scale below zero."""
    print("case: many trees", flush=True)
    rng = random.Random(2)
    new = [rng.randrange(0, 6) for _ in range(90)]
    length = [m + rng.randrange(0, 60) for m in new]
    s = Trees(siso, "fp8", 64, 2, 16, new, length, seed=9)
    s.write()
    q = s.queries(4)
    wide = torch.zeros(sum(new), 4, 3, 65, dtype=torch.bfloat16, device=DEV)
    wide[:, :, 1, :64] = q.to(DEV)
    got = s.kv.attend(s.batch, wide[:, :, 1, :64], scale=-0.3, with_lse=True, tree=s.tree)
    s.check_tree(q, scale=-0.3, got=got, label="many")


def test_sequences_with_more_rows_than_a_tree_has_are_left_out(siso):  # noqa: F811
    s = Setup(siso, "bf16", 64, 1, 16, [3, 257, 2], [50, 300, 20], seed=10)
    s.write()
    batch = s.kv.batch(ends(s.new), s.length_dev, s.pages, max_new=256)  # (which is not so)
    q = s.queries(2).to(DEV)
    parents = [random_tree(m, 40, b) for b, m in enumerate(s.new)]
    out, lse = torch.full_like(q, 7.0), torch.full((262, 2), 5.0, device=DEV)
    tree = s.kv.tree(batch, ints([p for t in parents for p in t]))
    s.kv.attend(batch, q, out=out, lse=lse, tree=tree)
    accepted, rows, tokens = (torch.full((k,), -9, dtype=torch.int32, device=DEV) for k in (3, 262, 262))
    s.kv.verify_tree(batch, tree, ints([0] * 262), torch.zeros(262, 10, device=DEV), out_accepted=accepted, out_rows=rows, out_tokens=tokens)
    torch.cuda.synchronize()
    assert (out[3:260] == 7).all() and (lse[3:260] == 5).all() and accepted[1] == -9 and (rows[3:260] == -9).all() and (tokens[3:260] == -9).all()
    assert accepted[0] >= 0 and accepted[2] >= 0 and rows[0] == 0 and rows[260] == 0
    hk, hv = kv_oracle.held(s.k, "bf16"), kv_oracle.held(s.v, "bf16")
    for b, at in ((0, 0), (2, 260)):
        m, l, start = s.new[b], s.length[b], s.starts[b]
        want = oracle.attend(q[at:at + m].cpu(), hk[start:start + l], hv[start:start + l], oracle.seen_by(oracle.ancestors(parents[b]), l), 0.125)
        kv_oracle.check_attend(out[at:at + m], lse[at:at + m], want, 64, f"sequence {b}")


@pytest.mark.parametrize("d", [128, 192])
def test_replayed_with_another_tree(siso, d):  # noqa: F811
    print(f"case: tree in a graph d={d}", flush=True)
    s = Trees(siso, "fp8", d, 2, 16, [40, 5], [300, 70], seed=12)
    s.write()
    q, parent = s.queries(8).to(DEV), s.tree.parent.clone()
    stream = torch.cuda.Stream()
    s.kv.set_stream(stream)
    with torch.cuda.stream(stream):
        s.kv.attend(s.batch, q, with_lse=True, tree=s.kv.tree(s.batch, parent))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            tree = s.kv.tree(s.batch, parent)
            got = s.kv.attend(s.batch, q, with_lse=True, tree=tree)
        for turn in range(4):
            s.parents = [random_tree(m, 50, 100 + turn) for m in s.new]
            parent.copy_(ints([p for t in s.parents for p in t]))
            graph.replay()
            torch.cuda.synchronize()
            s.check_tree(s.queries(8), got=got, label=f"replay {turn}")
            want = s.kv.attend(s.batch, q, with_lse=True, tree=s.kv.tree(s.batch, parent))
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got, want))
