"""Trees and eviction as their callers may call them: on another stream, by graphs that share a workspace, behind 4 GiB, with hints that are too small."""

import math
import random

import pytest
import torch

import kv_oracle
import kv_tree_oracle as oracle
from gpu_util import DEV
from test_gpu_kv import ends, ints, siso  # noqa: F401
from test_kv_gpu_evict import Full
from test_kv_gpu_tree import Trees, random_tree
from test_kv_gpu_weigh import Weighed

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [3, 90])
def test_a_stream_that_is_not_torchs(siso, rows):  # noqa: F811
    """All calls on the handle's stream, one behind the other, while torch's own stream allocates and frees: as on one stream."""
    print(f"case: a stream of its own, {rows} rows", flush=True)

    def go(kv_of, side):
        s = kv_of()
        s.write()
        q, vocab = s.queries(4).to(DEV), 501
        target = torch.randn(sum(s.new), vocab, generator=torch.Generator().manual_seed(4)).to(DEV)
        tokens = ints([i % vocab for i in range(sum(s.new))])
        parent = ints([p for t in s.parents for p in t])
        weights = s.kv.weights()
        torch.cuda.synchronize()
        if side:
            s.kv.set_stream(side)
        tree = s.kv.tree(s.batch, parent)
        out, lse = s.kv.attend(s.batch, q.transpose(0, 2).contiguous().transpose(0, 2) if not side else q, tree=tree, with_lse=True)
        accepted, path, named = s.kv.verify_tree(s.batch, tree, tokens, target)
        s.kv.keep(s.batch, path)
        s.kv.weigh(s.batch, q, lse, weights, fresh=ints([0] * len(s.new)))
        s.kv.evict(s.batch, weights, 50, recent=10, early=2)
        back = s.kv.read(s.kv.batch(ends([50, 50]), ints([50, 50]), s.pages))
        got = [out, lse, accepted, path, named, weights.mass, weights.born, *back]
        junk = [torch.full((rows + 1, 4, 64), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(4)]
        if side:
            torch.cuda.current_stream().wait_stream(side)
        copies = [x.clone() for x in got]
        torch.cuda.synchronize()
        del junk
        return copies

    make = lambda: Trees(siso, "fp8", 64, 2, 16, [rows, 2], [400, 90], seed=31)  # noqa: E731
    want = go(make, None)
    for _ in range(3):
        for x, y in zip(go(make, torch.cuda.Stream()), want):
            assert torch.equal(x, y)


def test_graphs_that_share_a_workspace(siso):  # noqa: F811
    """Two graphs of one handle, replayed in turn with eager calls between them: weights of many rows (parts that are joined), drafts, eviction."""
    print("case: two graphs, one handle", flush=True)
    s = Weighed(siso, "bf16", 128, 2, 16, [300, 1], [900, 500], seed=12)
    stream = torch.cuda.Stream()
    s.kv.set_stream(stream)
    k, v, q = s.k.to(DEV), s.v.to(DEV), s.queries(8).to(DEV)
    sizes, vocab = [20, 1, 7], 9001
    walks = s.kv.batch(ends(sizes), rows=28, max_new=20)
    parent, tokens = ints([p for b, m in enumerate(sizes) for p in random_tree(m, 40, b)]), ints([i % 5 for i in range(28)])
    target = torch.zeros(28, vocab, device=DEV)
    target[torch.arange(28), torch.arange(28) % 5] = 1.0
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        def weigh(w):
            s.kv.write(s.all, k, v)
            s.kv.weigh(s.batch, q, s.kv.attend(s.batch, q, with_lse=True)[1], w, fresh=zero)
            s.kv.evict(s.batch, w, 200, recent=20)
            return s.kv.read(kept)
        zero, kept = ints([0, 0]), s.kv.batch(ends([200, 200]), ints([200, 200]), s.pages)
        walk = lambda: s.kv.verify_tree(walks, s.kv.tree(walks, parent), tokens, target)  # noqa: E731
        a, b = s.kv.weights(), s.kv.weights()
        want, want_walk = [x.clone() for x in weigh(a)], [x.clone() for x in walk()]
        want += [a.mass.clone(), a.born.clone()]
        torch.cuda.synchronize()
        graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
        with torch.cuda.graph(graphs[0], stream=stream):
            got = weigh(b)
        with torch.cuda.graph(graphs[1], stream=stream):
            got_walk = walk()
        for turn in range(4):
            graphs[turn & 1].replay()
            if turn == 2:
                walk()
            graphs[~turn & 1].replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip([*got, b.mass, b.born], want)), f"turn {turn}"
            assert all(torch.equal(x, y) for x, y in zip(got_walk, want_walk)), f"turn {turn}"


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_offsets_beyond_32_bits(siso, dtype):  # noqa: F811
    """Pages whose bytes lie beyond 4 GiB of either pool: a tree's attention, its path, its weights (few rows and many) and eviction, there and back."""
    print(f"case: large offsets {dtype}", flush=True)
    pages = 40000 if dtype == "bf16" else 80000  # of 64 tokens, 8 heads, 128 elements: 5.2 GB of keys
    kv = siso.PagedKV(8, 128, pages, page_tokens=64, dtype=siso.FP8 if dtype == "fp8" else siso.BF16)
    g = torch.Generator().manual_seed(16)
    k, v = (torch.randn(150, 8, 128, generator=g).bfloat16() for _ in range(2))
    hk, hv = kv_oracle.held(k, dtype), kv_oracle.held(v, dtype)
    table = ints([[pages - 1, 5, pages - 2]])
    kv.write(kv.batch(ints([0, 150]), ints([150]), table), k.to(DEV), v.to(DEV))
    scale = float(torch.tensor(128 ** -0.5))
    weights = kv.weights()
    for m in (4, 40, 100):
        q = torch.randn(m, 8, 128, generator=g).bfloat16()
        parents = random_tree(m, 40, m)
        batch = kv.batch(ints([0, m]), ints([150]), table)
        out, lse = kv.attend(batch, q.to(DEV), with_lse=True, tree=kv.tree(batch, ints(parents)))
        want = oracle.attend(q, hk, hv, oracle.seen_by(oracle.ancestors(parents), 150), scale)
        kv_oracle.check_attend(out, lse, want, 128, f"large offsets, {m} rows")
        lse = kv.attend(batch, q.to(DEV), with_lse=True)[1]
        kv.weigh(batch, q.to(DEV), lse, weights, fresh=ints([0]))
        sums, tol = oracle.weigh(q, hk, lse.cpu(), 150, 0, scale)
        mass = torch.cat([weights.mass[0, p].cpu() for p in table[0].tolist()], 1)[:, :150].double()
        assert ((mass - sums).abs() <= tol).all(), f"{m} rows"
    path = [0, 30, 99] + [-1] * 97
    kv.keep(kv.batch(ints([0, 100]), ints([150]), table), ints(path))
    order = torch.tensor([*range(51), 80, 149, *range(53, 150)])
    back = kv.read(kv.batch(ints([0, 150]), ints([150]), table), dtype=torch.float32)
    k32, v32 = hk[order].float(), hv[order].float()  # (code * scale, rounded once)
    assert torch.equal(back[0].cpu(), k32) and torch.equal(back[1].cpu(), v32)
    to = ints([[9, pages - 3]])
    mass = [float(x) for x in torch.cat([weights.mass[0, p].cpu() for p in table[0].tolist()], 1)[3, :150]]
    of = oracle.evict(mass, [*range(150)], 100, 10, 2)
    kv.evict(kv.batch(ints([0, 0]), ints([150]), table), weights, 100, recent=10, early=2, to=to)
    got = kv.read(kv.batch(ints([0, 100]), ints([100]), to), dtype=torch.float32)
    assert torch.equal(got[0][:, 3].cpu(), k32[of, 3]) and torch.equal(got[1][:, 3].cpu(), v32[of, 3])
    assert kv.bad_pages() == 0


def test_hints_that_are_too_small(siso):  # noqa: F811
    """max_length weighs on speed alone, for a tree's attention and for eviction, too."""
    print("case: small hints", flush=True)
    for rows in (3, 150):
        s = Trees(siso, "bf16", 128, 2, 16, [rows, 1], [1500, 700], seed=40)
        s.write()
        s.batch = s.kv.batch(ends(s.new), s.length_dev, s.pages, max_new=rows, max_length=20)
        s.check_tree(s.queries(4), label="a small max_length")
    for length in ([700, 90], [9000, 3000], [20000, 10]):
        s = Full(siso, "fp8", 64, 1, 64, length, seed=41)
        s.all = s.kv.batch(ends(length), s.length_dev, s.pages, max_length=20)
        s.check(60, 9, 2, label="a small max_length")


def test_many_sequences_of_many_rows(siso):  # noqa: F811
    """More than 64 sequences, of few rows and of many in one batch, and more blocks of positions than are joined at once."""
    print("case: many sequences weigh", flush=True)
    rng = random.Random(3)
    new = [rng.choice([0, 1, 2, 40, 70, 130]) for _ in range(100)]
    length = [m + rng.randrange(0, 150) for m in new]
    s = Weighed(siso, "bf16", 64, 2, 16, new, length, seed=13)
    s.write()
    q = s.queries(4)
    lse = s.lse_of(q)
    s.start()
    s.kv.weigh(s.batch, q.to(DEV), lse, s.weights, decay=0.5)
    s.check_weigh(q, lse, decay=0.5, label="many rows")


@pytest.mark.parametrize("rows", [1, 50])
def test_without_decay_it_does_not_matter_what_was_there(siso, rows):  # noqa: F811
    s = Weighed(siso, "fp8", 64, 2, 16, [rows], [300], seed=14)
    s.write()
    q = s.queries(8)
    lse = s.lse_of(q)
    s.start()
    s.mass.zero_()
    s.weights.mass.fill_(math.nan)
    s.kv.weigh(s.batch, q.to(DEV), lse, s.weights, decay=0.0)
    pages = s.pages.cpu()[0].long()
    got = torch.stack([s.weights.mass.cpu()[0, pages[j // 16], :, j % 16] for j in range(300)], 1).double()
    sums, tol = oracle.weigh(q, kv_oracle.held(s.k, "fp8"), lse.cpu(), 300, 0, float(torch.tensor(s.d ** -0.5)))
    assert ((got - sums).abs() <= tol).all()


@pytest.mark.parametrize("rows", [1, 3, 50])
@pytest.mark.parametrize("apart", [0, 1])
def test_keys_that_are_infinite_where_they_weigh_nothing(siso, rows, apart):  # noqa: F811
    """A score of minus infinity is a weight of zero, whatever a tile of rows is filled up with."""
    s = Weighed(siso, "bf16", 64, 1, 16, [rows], [300], seed=15)
    q = s.queries(4).abs()
    s.k[10, 0, 5] = -math.inf
    s.write()
    wide = torch.zeros(rows, 4, 64 + apart, dtype=torch.bfloat16, device=DEV)
    wide[:, :, :64] = q.to(DEV)
    lse = s.lse_of(q)
    assert torch.isfinite(lse).all()
    s.start()
    s.kv.weigh(s.batch, wide[:, :, :64], lse, s.weights, fresh=ints([0]))
    mass = s.weights.mass.cpu()[0, s.pages.cpu()[0, 0].long(), 0]
    assert mass[10] == 0 and (mass[:10] > 0).all()


def test_thousands_of_sequences(siso):  # noqa: F811
    """More sequences than a workgroup plans for at a time: trees, their paths, weights and eviction."""
    print("case: thousands of sequences", flush=True)
    rng = random.Random(8)
    n = 1500
    new = [rng.randrange(0, 4) for _ in range(n)]
    length = [m + rng.randrange(0, 20) for m in new]
    s = Trees(siso, "bf16", 8, 1, 16, new, length, seed=17)
    s.write()
    q = s.queries(2)
    s.check_tree(q, label="thousands")
    first, tokens = s.batch.first.tolist(), [rng.randrange(5) for _ in range(sum(new))]
    target = torch.rand(sum(new), 5, generator=torch.Generator().manual_seed(5))
    for u in (None, torch.rand(sum(new), generator=torch.Generator().manual_seed(6))):
        accepted, path, out = (x.tolist() for x in s.kv.verify_tree(s.batch, s.tree, ints(tokens), target.to(DEV), None if u is None else u.to(DEV)))
        for b in range(n):
            r = slice(first[b], first[b + 1])
            assert (accepted[b], path[r], out[r]) == oracle.verify(s.parents[b], tokens[r], target[r].double().numpy(), None if u is None else u[r].numpy())
    w = Weighed(siso, "bf16", 8, 1, 16, new, length, seed=17)
    w.write()
    w.start()
    lse = w.lse_of(q)
    w.kv.weigh(w.batch, q.to(DEV), lse, w.weights)
    w.check_weigh(q, lse, label="thousands")
    Full(siso, "fp8", 8, 1, 16, length, seed=18).check(9, 3, 1, label="thousands")
