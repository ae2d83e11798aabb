"""Which path of a tree stands, and where its keys and values go (siso_kv_verify_tree, siso_kv_keep), against their definition."""

import math
import random

import numpy as np
import pytest
import torch

import kv_oracle
import kv_tree_oracle as oracle
from gpu_util import DEV
from test_gpu_kv import Setup, ends, ints, siso  # noqa: F401
from test_kv_gpu_tree import random_tree

pytestmark = pytest.mark.gpu


def make(sizes, vocab, kind, greedy, seed, branch=40, right=0.7):
    """Trees whose rows' tokens mostly are what their parents' targets name, so that walks go deep."""
    g = torch.Generator().manual_seed(seed)
    rng = random.Random(seed)
    total = sum(sizes)
    logits = torch.randn(total, vocab, generator=g) * 2
    target = (logits if greedy else torch.softmax(logits * 3, 1)).to(kind)
    u = None if greedy else torch.rand(total, generator=g)
    parents, tokens, at = [], [], 0
    for b, m in enumerate(sizes):
        tree = random_tree(m, branch, seed + b)
        exact = target[at:at + m].double().numpy()
        say = [oracle.verify([-1], [0], exact[i:i + 1], None if greedy else u[at + i:at + i + 1].numpy())[2][0] for i in range(m)]
        tokens += [say[p] if p >= 0 and rng.random() < right else rng.randrange(vocab) for p in tree]
        parents.append(tree)
        at += m
    return parents, tokens, target, u


def check(siso, sizes, parents, tokens, target, u, got=None):  # noqa: F811
    if got is None:
        kv = siso.PagedKV(1, 64, 1)
        batch = kv.batch(ends(sizes), rows=sum(sizes), max_new=max(sizes))
        tree = kv.tree(batch, ints([p for t in parents for p in t]))
        got = kv.verify_tree(batch, tree, ints(tokens), target.to(DEV), None if u is None else u.to(DEV))
    torch.cuda.synchronize()
    accepted, rows, out = (x.tolist() for x in got)
    at, deep = 0, 0
    for b, m in enumerate(sizes):
        want = oracle.verify(parents[b], tokens[at:at + m], target[at:at + m].double().cpu().numpy(), None if u is None else u[at:at + m].numpy())
        assert (accepted[b], rows[at:at + m], out[at:at + m]) == want, f"sequence {b}"
        deep = max(deep, want[0])
        at += m
    return deep


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("greedy", [True, False])
@pytest.mark.parametrize("sizes,vocab", [([1], 1), ([5, 0, 1], 7), ([256], 513), ([30, 64, 65, 200, 2], 8191), ([40, 3, 17], 8193), ([25] * 3, 32000), ([9, 33], 128001)])
def test_walks(siso, kind, greedy, sizes, vocab):  # noqa: F811
    print(f"case: walk {kind} {'greedy' if greedy else 'drawn'} {sizes} {vocab}", flush=True)
    for branch in (10, 60):
        parents, tokens, target, u = make(sizes, vocab, kind, greedy, 31 * vocab + branch, branch)
        check(siso, sizes, parents, tokens, target, u)
    parents, tokens, target, u = make(sizes, vocab, kind, greedy, 17 * vocab, branch=0, right=1.0)  # chains that stand as a whole
    assert check(siso, sizes, parents, tokens, target, u) == max(sizes) - 1


def test_many_sequences(siso):  # noqa: F811
    rng = random.Random(3)
    sizes = [rng.randrange(0, 20) for _ in range(700)]
    for greedy in (True, False):
        check(siso, sizes, *make(sizes, 300, torch.float32, greedy, 5))


@pytest.mark.parametrize("greedy", [True, False])
def test_special_values(siso, greedy):  # noqa: F811
    """Equal entries, rows of NaN and without weight, weights below zero, u at its ends, children with one token, tokens that are none."""
    vocab, m = 5000, 12
    target = torch.rand(m, vocab, generator=torch.Generator().manual_seed(1))
    target[0] = 0
    target[0, 100] = target[0, 4000] = 1.0
    target[1] = math.nan
    target[2] = 0.0 if not greedy else -math.inf
    target[3, ::2] = math.nan
    target[4] = -1.0
    target[4, 4999] = 2.0
    target[5] = 0
    target[5, 0] = 1e-30
    target[6, 7] = -3.0
    u = torch.tensor([0.0, 0.5, 0.5, 0.9, 0.99999994, 0.99999994, 0.0, 0.3, 0.6, 0.7, 0.1, 0.2])
    named = [oracle.verify([-1], [0], target[i:i + 1].double().numpy(), None if greedy else u[i:i + 1].numpy())[2][0] for i in range(m)]
    # from the root to each row in turn, by two children of the same token: the first counts
    for end in range(1, m):
        parents = [[-1, 0, 0, 1]]
        rows = torch.stack([target[0], target[end], target[(end + 1) % m], target[(end + 2) % m]])
        uu = torch.stack([u[0], u[end], u[(end + 1) % m], u[(end + 2) % m]])
        tokens = [0, named[0], named[0], named[end]]
        check(siso, [4], parents, tokens, rows, None if greedy else uu)
    check(siso, [4], [[-1, 0, 0, 0]], [0, -1, vocab, 1 << 30], target[:4], None if greedy else u[:4])
    check(siso, [3], [[-1, 0, -1]], [0, named[0], named[1]], target[[0, 1, 2]], None if greedy else u[:3])


def test_drawn_tokens_are_the_targets(siso):  # noqa: F811
    """Over many random numbers, the first token's frequencies are the target's probabilities, whatever the tree offers."""
    n, vocab = 20000, 6
    g = torch.Generator().manual_seed(4)
    p = torch.tensor([0.4, 0.25, 0.2, 0.1, 0.05, 0.0])
    target = p.expand(3 * n, vocab).contiguous()
    kv = siso.PagedKV(1, 64, 1)
    batch = kv.batch(ints(list(range(0, 3 * n + 1, 3))), rows=3 * n, max_new=3)
    tree = kv.tree(batch, ints([-1, 0, 0] * n))
    accepted, _, out = kv.verify_tree(batch, tree, ints([0, 3, 0] * n), target.to(DEV), torch.rand(3 * n, generator=g).to(DEV))
    first = out.view(n, 3)[:, 0].cpu()
    share = torch.bincount(first.long(), minlength=vocab).double() / n
    assert ((share - p.double()).abs() <= 5 * (p.double() * (1 - p.double()) / n).sqrt() + 1e-12).all()  # (five standard deviations)
    assert torch.equal(accepted.cpu() > 0, (first == 0) | (first == 3))


def test_rows_within_wider_ones_and_a_graph(siso):  # noqa: F811
    sizes, vocab = [20, 7], 3001
    kv = siso.PagedKV(1, 64, 1)
    stream = torch.cuda.Stream()
    kv.set_stream(stream)
    batch = kv.batch(ends(sizes), rows=27, max_new=20)
    wide, tokens_dev, u_dev, parent = torch.zeros(27, vocab + 5, device=DEV), ints([0] * 27), torch.zeros(27, device=DEV), ints([-1] * 27)
    with torch.cuda.stream(stream):
        step = lambda: kv.verify_tree(batch, kv.tree(batch, parent), tokens_dev, wide[:, 3:3 + vocab], u_dev)  # noqa: E731
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = step()
        for turn in range(3):
            parents, tokens, target, u = make(sizes, vocab, torch.float32, False, 50 + turn)
            wide[:, 3:3 + vocab] = target.to(DEV)
            tokens_dev.copy_(ints(tokens))
            u_dev.copy_(u.to(DEV))
            parent.copy_(ints([p for t in parents for p in t]))
            graph.replay()
            check(siso, sizes, parents, tokens, target, u, got=got)


# ------------------------------------------------------------------ what stands moves
@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,page,kv_heads", [(8, 16, 1), (64, 64, 3), (72, 16, 2), (128, 32, 8), (192, 128, 1), (256, 16, 2)])
@pytest.mark.parametrize("layer", [None, 1])
def test_a_path_moves_behind_the_context(siso, dtype, d, page, kv_heads, layer):  # noqa: F811
    print(f"case: keep {dtype} d={d} page={page} kv_heads={kv_heads} layer={layer}", flush=True)
    rng = random.Random(d)
    new, length = [1, 9, 0, 40, 150, 256], [5, 9, 30, 77, 201, 300]
    s = Setup(siso, dtype, d, kv_heads, page, new, length, seed=d, layers=3)
    shift = lambda x, by: torch.roll(x, by, 0)  # noqa: E731  (layers hold unlike tokens)
    for lay in range(3):
        s.kv.write(s.all, shift(s.k, lay).to(DEV), shift(s.v, lay).to(DEV), layer=lay)
    paths = [[0], [0, 1, 2, 5, 8], [], sorted(rng.sample(range(40), 17)), list(range(100)) + [120, 149], [0] + sorted(rng.sample(range(1, 256), 99))]
    flat = [x for p, m in zip(paths, new) for x in p + [-1] * (m - len(p))]
    s.kv.keep(s.batch, ints(flat), layer=layer)
    want = torch.arange(sum(length))
    for b, p in enumerate(paths):
        base = s.starts[b] + length[b] - new[b]
        for j, r in enumerate(p):
            want[base + j] = base + r
    for lay in range(3):
        at = want if layer in (None, lay) else torch.arange(sum(length))
        got = s.kv.read(s.all, layer=lay, dtype=torch.float32)
        for x, y in zip(got, (s.k, s.v)):
            assert torch.equal(x.cpu(), kv_oracle.held(shift(y, lay), dtype).float()[at]), f"layer {lay}"
    assert s.kv.bad_pages() == 0


def test_paths_that_are_none_and_pages_that_are_none(siso):  # noqa: F811
    """What does not increase, or lies ahead of its place or beyond the rows, ends a path; pages that are none give zeros and take nothing."""
    s = Setup(siso, "bf16", 64, 2, 16, [6, 6, 6, 6, 40], [60, 40, 3, 30, 60], seed=3)
    s.write()
    flat = [0, 2, 1, 5, -1, -1, 3, 4, 6, 5, -1, -1, 0, 4, 5, -1, -1, -1, 1, 0, 3, 4, 5, 5] + [0, 17, 18, 39] + [-1] * 36
    pages = s.pages.clone()
    pages[4, 2] = s.pool  # positions 32 to 47
    batch = s.kv.batch(ends(s.new), s.length_dev, pages, max_new=40)
    s.kv.keep(batch, ints(flat))
    moved = [(0, 55, 56), (1, 34, 37), (1, 35, 38), (2, 0, None), (3, 24, 25)]
    moved = [x for x in moved if x[2] is not None]
    want_k, want_v = kv_oracle.held(s.k, "bf16").float(), kv_oracle.held(s.v, "bf16").float()
    new_k, new_v = want_k.clone(), want_v.clone()
    for b, to, of in moved:
        new_k[s.starts[b] + to], new_v[s.starts[b] + to] = want_k[s.starts[b] + of], want_v[s.starts[b] + of]
    # sequence 4 begins at position 20: rows 17, 18 (37, 38: no page) give zeros at 21, 22, row 39 (59) goes to 23
    for to, of in ((21, None), (22, None), (23, 59)):
        for x, y in ((new_k, want_k), (new_v, want_v)):
            x[s.starts[4] + to] = 0 if of is None else y[s.starts[4] + of]
    got = s.kv.read(s.all, dtype=torch.float32)
    # sequence 2 has 3 positions for 6 rows: its rows 4 and 5 stand at 1 and 2, rows 1 and 2 nowhere
    assert torch.equal(got[0].cpu(), new_k) and torch.equal(got[1].cpu(), new_v)
    assert s.kv.bad_pages() > 0


def test_a_path_in_a_graph(siso):  # noqa: F811
    """Written, kept and read back by one graph, replayed with other paths."""
    new, length = [30, 5], [90, 20]
    s = Setup(siso, "fp8", 128, 2, 16, new, length, seed=5, layers=2)
    stream = torch.cuda.Stream()
    s.kv.set_stream(stream)
    k, v, path = s.k.to(DEV), s.v.to(DEV), ints([-1] * 35)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        def step():
            for layer in range(2):
                s.kv.write(s.all, k, v, layer=layer)
            s.kv.keep(s.batch, path)
            return [s.kv.read(s.all, layer=layer, dtype=torch.float32) for layer in range(2)]
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = step()
        rng = random.Random(1)
        for turn in range(4):
            paths = [[0] + sorted(rng.sample(range(1, 30), rng.randrange(0, 20))), [0, 2, 4][:1 + turn % 3]]
            path.copy_(ints([x for p, m in zip(paths, new) for x in p + [-1] * (m - len(p))]))
            graph.replay()
            torch.cuda.synchronize()
            want = torch.arange(110)
            for b, p in enumerate(paths):
                base = s.starts[b] + length[b] - new[b]
                for j, r in enumerate(p):
                    want[base + j] = base + r
            for layer in range(2):
                for x, y in zip(got[layer], (s.k, s.v)):
                    assert torch.equal(x.cpu(), kv_oracle.held(y, "fp8").float()[want])
            eager = step()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for a, b in zip(eager, got) for x, y in zip(a, b))
