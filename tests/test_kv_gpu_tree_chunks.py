"""Trees of many rows by the kernel for heavy work, which a table of many pages asks for (without max_length the calls count with all of it), against the definition."""

import math
import random

import pytest
import torch

import kv_oracle
import kv_tree_oracle as oracle
from gpu_util import DEV
from test_gpu_kv import ends, ints, siso  # noqa: F401
from test_kv_gpu_tree import Trees

pytestmark = pytest.mark.gpu


class Heavy(Trees):
    """Behind the sequences' own pages the table has others, of 2^22 positions."""

    def __init__(self, *args, **how):
        super().__init__(*args, **how)
        extra = torch.zeros(len(self.new), (1 << 22) // self.page - self.pages.shape[1], dtype=torch.int32, device=DEV)
        self.pages = torch.cat([self.pages, extra], 1)
        self.batch = self.kv.batch(ends(self.new), self.length_dev, self.pages, max_new=max(self.new))
        self.all = self.kv.batch(ends(self.length), self.length_dev, self.pages)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,page,kv_heads,heads", [(64, 16, 2, 8), (96, 64, 1, 8), (128, 16, 2, 8), (72, 32, 1, 5), (128, 128, 1, 128), (256, 16, 2, 4)])
def test_rows_see_the_context_and_their_ancestors(siso, dtype, d, page, kv_heads, heads):  # noqa: F811
    print(f"case: heavy trees {dtype} d={d} page={page} heads={heads}/{kv_heads}", flush=True)
    s = Heavy(siso, dtype, d, kv_heads, page, [1, 200, 0, 33, 64, 3, 100], [1, 777, 40, 33, 1065, 2000, 130], seed=d)
    s.write()
    s.check_tree(s.queries(heads), label=f"{dtype} d={d}")
    assert s.kv.bad_pages() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,kv_heads,heads,window", [(64, 1, 26, 7000), (128, 2, 32, 3000), (128, 2, 32, 100000)])
def test_windows(siso, dtype, d, kv_heads, heads, window):  # noqa: F811
    """(A window that is short makes the work light: these are heavy for their rows.)"""
    print(f"case: heavy trees, window {window} {dtype} d={d}", flush=True)
    long = min(window, 3000 if d == 128 else 7000)
    s = Heavy(siso, dtype, d, kv_heads, 16, [256, 5, 250, 240], [long + 200, 5, long + 700, 241], branch=20, seed=window % 97)
    s.write()
    s.check_tree(s.queries(heads), window=window, label=f"window {window}")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_any_mask(siso, dtype):  # noqa: F811
    print(f"case: heavy trees, any mask {dtype}", flush=True)
    new, length = [100, 70, 40], [100, 900, 40]
    s = Heavy(siso, dtype, 128, 1, 16, new, length, seed=3)
    s.write()
    rng = random.Random(4)
    lists = [[sorted(rng.sample(range(256), rng.randrange(0, 40))) if rng.random() < 0.8 else [] for _ in range(m)] for m in new]
    lists[2] = [[] for _ in range(40)]  # (all of it is rows: nothing is seen)
    s.tree = siso.KvTree(s.tree.parent, oracle.words([x for t in lists for x in t]).to(DEV), s.tree.depth)
    s.check_tree(s.queries(4), lists=lists, label="any mask")
    s.check_tree(s.queries(4), lists=lists, window=3, label="any mask, window")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_what_is_not_seen_and_large_scores(siso, dtype):  # noqa: F811
    """Infinities and NaN in other branches and ahead of a window, and maxima that grow far beyond the first ones."""
    print(f"case: heavy trees, not seen {dtype}", flush=True)
    new, length = [130, 70], [1500, 700]
    s = Heavy(siso, dtype, 128, 1, 16, new, length, branch=0, seed=11)
    s.parents = [[-1] + [0 if i in (1, 65) else i - 1 for i in range(1, 130)], [-1, *range(69)]]
    s.tree = s.kv.tree(s.batch, ints([p for t in s.parents for p in t]))
    q = s.queries(4)
    s.k[900] = (q[120, 0].float() * 6).bfloat16()  # a score far above those before it
    at = 1370 + 64  # the end of the first branch
    s.k[at], s.v[at] = math.nan, math.inf
    s.k[3], s.v[3], s.v[4, 0, 5] = math.inf, math.nan, -math.inf  # ahead of the window
    s.write()
    out, lse = s.kv.attend(s.batch, q.to(DEV), window=1200, with_lse=True, tree=s.tree)
    fine = [i for i in range(200) if i != 64]
    assert torch.isfinite(out[fine].float()).all() and torch.isfinite(lse[fine]).all() and not torch.isfinite(out[64].float()).any()
    hk, hv = kv_oracle.held(s.k, dtype), kv_oracle.held(s.v, dtype)
    first = 0
    for b, (m, l) in enumerate(zip(new, length)):
        rows = [i for i in range(m) if first + i != 64]
        lists = [oracle.ancestors(s.parents[b])[i] if i in rows else [] for i in range(m)]
        seen = oracle.seen_by(lists, l, 1200)
        if b == 0:
            seen[64] = False
        want = oracle.attend(q[first:first + m], hk[s.starts[b]:s.starts[b] + l], hv[s.starts[b]:s.starts[b] + l], seen, float(torch.tensor(128 ** -0.5)))
        kv_oracle.check_attend(out[first:first + m][rows], lse[first:first + m][rows], [x[rows] for x in want], 128, f"sequence {b}")
        first += m


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_pages_that_are_none(siso, dtype):  # noqa: F811
    print(f"case: heavy trees, pages that are none {dtype}", flush=True)
    s = Heavy(siso, dtype, 128, 2, 16, [170, 65], [900, 400], seed=6)
    s.write()
    pages = s.pages.clone()
    pages[0, 2], pages[0, 50], pages[1, 3] = -1, s.pool, 1 << 30
    s.batch = s.kv.batch(ends(s.new), s.length_dev, pages, max_new=170)
    s.check_tree(s.queries(8), hidden={0: [*range(32, 48), *range(800, 816)], 1: [*range(48, 64)]}, label="no page")
    assert s.kv.bad_pages() > 0


@pytest.mark.parametrize("n", [64, 65, 90])
def test_many_sequences(siso, n):  # noqa: F811
    """As many as a wave plans for, and more."""
    print(f"case: heavy trees, {n} sequences", flush=True)
    rng = random.Random(n)
    new = [rng.choice([0, 3, 20, 60, 90]) for _ in range(n)]
    new[5] = 256
    length = [m + rng.randrange(0, 400) for m in new]
    s = Heavy(siso, "bf16", 64, 1, 16, new, length, seed=n)
    s.write()
    s.check_tree(s.queries(6), label="many")


def test_replayed_with_other_lengths(siso):  # noqa: F811
    """Pieces go by the lengths that the device finds: replays with others, each twice the same as the eager call."""
    print("case: heavy trees in a graph", flush=True)
    s = Heavy(siso, "bf16", 128, 2, 16, [70, 130], [3000, 2000], seed=12)
    s.write()
    q, length = s.queries(8).to(DEV), s.length_dev.clone()
    stream = torch.cuda.Stream()
    s.kv.set_stream(stream)
    batch = s.kv.batch(ends(s.new), length, s.pages, rows=200, max_new=130)
    with torch.cuda.stream(stream):
        s.kv.attend(batch, q, with_lse=True, tree=s.tree)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = s.kv.attend(batch, q, with_lse=True, tree=s.tree)
        for lengths in ([3000, 2000], [70, 130], [2999, 131], [1, 1500]):
            length.copy_(ints(lengths))
            for _ in range(2):
                graph.replay()
                out, lse = got[0].clone(), got[1].clone()
                eager = s.kv.attend(batch, q, with_lse=True, tree=s.tree)
                torch.cuda.synchronize()
                assert torch.equal(out, eager[0]) and torch.equal(lse, eager[1])
            at, hk, hv = 0, kv_oracle.held(s.k, "bf16"), kv_oracle.held(s.v, "bf16")
            for b, (m, l) in enumerate(zip(s.new, lengths)):
                r = slice(s.starts[b], s.starts[b] + l)
                want = oracle.attend(q[at:at + m].cpu(), hk[r], hv[r], oracle.seen_by(oracle.ancestors(s.parents[b]), l), float(torch.tensor(128 ** -0.5)))
                kv_oracle.check_attend(out[at:at + m], lse[at:at + m], want, 128, f"{lengths} sequence {b}")
                at += m


def test_sequences_without_positions(siso):  # noqa: F811
    """Rows of sequences without tokens, or with fewer tokens than rows, among others: zeros and minus infinity where nothing is seen."""
    print("case: heavy trees, no positions", flush=True)
    s = Heavy(siso, "bf16", 128, 1, 16, [200, 100, 0, 256, 90], [0, 1500, 0, 100, 90], seed=21)
    s.write()
    s.check_tree(s.queries(4), label="no positions")
    s.check_tree(s.queries(4), window=1000000, label="no positions, window")


def test_a_sequence_of_too_many_rows_among_many_tiles(siso):  # noqa: F811
    """It is left out; the others, whose tiles are more than are ever cut or fewer, are whole."""
    print("case: heavy trees, too many rows", flush=True)
    new, length = [256] * 3 + [3000], [300, 1700, 256, 3000]
    s = Heavy(siso, "bf16", 136, 8, 16, new[:3] + [2], length, seed=22)
    s.write()
    q = torch.cat([s.queries(64)[:768], torch.zeros(3000, 64, 136, dtype=torch.bfloat16)])
    batch = s.kv.batch(ends(new), s.length_dev, s.pages, max_new=256)
    parent = torch.cat([s.tree.parent[:768], torch.zeros(3000, dtype=torch.int32, device=DEV)])
    out, lse = s.kv.attend(batch, q.to(DEV), with_lse=True, tree=s.kv.tree(batch, parent))
    hk, hv = kv_oracle.held(s.k, "bf16"), kv_oracle.held(s.v, "bf16")
    for b in range(3):
        at, r = 256 * b, slice(s.starts[b], s.starts[b] + length[b])
        rows = [0, 1, 31, 100, 128, 200, 255]
        lists = [x if i in rows else [] for i, x in enumerate(oracle.ancestors(s.parents[b]))]
        seen = oracle.seen_by(lists, length[b])
        seen[[i for i in range(256) if i not in rows]] = False
        want = oracle.attend(q[at:at + 256], hk[r], hv[r], seen, float(torch.tensor(136 ** -0.5)))
        kv_oracle.check_attend(out[at:at + 256][rows], lse[at:at + 256][rows], [x[rows] for x in want], 136, f"sequence {b}")
