"""Eviction from the paged cache (siso_kv_evict) against its definition."""

import math
import random

import pytest
import torch

import kv_oracle
import kv_tree_oracle as oracle
from gpu_util import DEV
from test_gpu_kv import Setup, ends, ints, siso  # noqa: F401

pytestmark = pytest.mark.gpu


class Full(Setup):
    """All tokens written in every layer, masses and ages of every kind; `apart`: pages for what is kept."""

    def __init__(self, siso, dtype, d, kv_heads, page, length, seed=0, layers=1, apart=0, kind="spread"):  # noqa: F811
        extra = sum(-(-min(l, apart) // page) for l in length) if apart else 0
        super().__init__(siso, dtype, d, kv_heads, page, [0] * len(length), length, seed=seed, layers=layers, spare=2 + extra)
        g = torch.Generator().manual_seed(seed + 1)
        for layer in range(layers):
            self.kv.write(self.all, torch.roll(self.k, layer, 0).to(DEV), torch.roll(self.v, layer, 0).to(DEV), layer=layer)
        shape = (layers, self.pool, kv_heads, page)
        if kind == "spread":
            self.mass = torch.exp(3 * torch.randn(shape, generator=g))
        elif kind == "ties":
            self.mass = torch.randint(0, 3, shape, generator=g).float()
        elif kind == "same":
            self.mass = torch.full(shape, 0.25)
        else:  # odd values
            values = torch.tensor([math.nan, math.inf, -math.inf, -0.0, 0.0, 1e-40, -2.0, 3.4e38, 1.0, -1e-45])
            self.mass = values[torch.randint(0, len(values), shape, generator=g)]
        self.born = torch.randint(0, 4 * max(max(length), 1), shape, generator=g, dtype=torch.int32)
        self.weights = self.kv.weights(self.mass.to(DEV), self.born.to(DEV))
        self.to = None
        if apart:
            used = set(self.pages.cpu()[b, j].item() for b, l in enumerate(length) for j in range(-(-l // page)))
            free = [p for p in range(self.pool) if p not in used]
            need = [-(-min(l, apart) // page) for l in length]
            self.to = torch.zeros(len(length), max(max(need), 1), dtype=torch.int32)
            for b, c in enumerate(need):
                self.to[b, :c] = torch.tensor([free.pop() for _ in range(c)], dtype=torch.int32)

    def check(self, keep, recent, early, layer=None, born=True, label=""):
        before = [[x.cpu() for x in self.kv.read(self.all, layer=i, dtype=torch.float32)] for i in range(self.kv.layers)]
        weights = self.weights if born else self.kv.weights(self.weights.mass)
        self.kv.evict(self.all, weights, keep, recent, early, layer=layer, to=None if self.to is None else self.to.to(DEV))
        torch.cuda.synchronize()
        mass, age = self.mass.clone(), self.born.clone()
        stay = [min(l, keep) for l in self.length]
        table = self.pages if self.to is None else self.to.to(DEV)
        after_batch = self.kv.batch(ends(stay), ints(stay), table)
        pages, to = self.pages.cpu(), table.cpu()
        for i in range(self.kv.layers):
            if layer not in (None, i):
                continue
            got = [x.cpu() for x in self.kv.read(after_batch, layer=i, dtype=torch.float32)]
            at = 0
            for b, l in enumerate(self.length):
                j = torch.arange(l)
                pg, slot = pages[b, j // self.page].long(), j % self.page
                jj = j[:stay[b]]
                tpg, tslot = to[b, jj // self.page].long(), jj % self.page
                for h in range(self.kv.kv_heads):
                    w, a = self.mass[i, pg, h, slot], self.born[i, pg, h, slot]
                    of = torch.tensor(oracle.evict(w.tolist(), a.tolist() if born else None, keep, recent, early), dtype=torch.long)
                    for x, y in zip(got, before[i]):
                        assert torch.equal(x[at:at + stay[b], h].nan_to_num(), y[self.starts[b] + of, h].nan_to_num()), f"{label} layer {i} sequence {b} head {h}"
                    mass[i, tpg, h, tslot] = w[of]
                    age[i, tpg, h, tslot] = a[of]
                at += stay[b]
        assert torch.equal(self.weights.mass.cpu().nan_to_num(nan=7.0), mass.nan_to_num(nan=7.0)), f"{label}: mass"
        if born:
            assert torch.equal(self.weights.born.cpu(), age), f"{label}: born"
        if self.to is not None:  # what was there stays
            for i in range(self.kv.layers):
                assert all(torch.equal(x.cpu(), y) for x, y in zip(self.kv.read(self.all, layer=i, dtype=torch.float32), before[i]))


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,page,kv_heads", [(8, 16, 1), (64, 64, 3), (72, 16, 2), (128, 32, 4), (192, 128, 1), (256, 16, 2)])
@pytest.mark.parametrize("apart", [False, True])
def test_the_heaviest_stay(siso, dtype, d, page, kv_heads, apart):  # noqa: F811
    print(f"case: evict {dtype} d={d} page={page} kv_heads={kv_heads} apart={apart}", flush=True)
    length = [0, 1, 99, 100, 101, 164, 500, 250]
    s = Full(siso, dtype, d, kv_heads, page, length, seed=d, apart=100 if apart else 0)
    s.check(100, 20, 4, label=f"{dtype} d={d}")
    assert s.kv.bad_pages() == 0


@pytest.mark.parametrize("kind", ["spread", "ties", "same", "odd"])
@pytest.mark.parametrize("keep,recent,early", [(1, 0, 0), (1, 1, 0), (64, 64, 0), (100, 0, 100), (333, 40, 7), (1200, 0, 0), (2999, 1, 1), (3000, 10, 10)])
def test_orders_and_ties(siso, kind, keep, recent, early):  # noqa: F811
    print(f"case: evict {kind} {keep} {recent} {early}", flush=True)
    s = Full(siso, "bf16", 64, 2, 64, [3000, 1100, 65], seed=keep, kind=kind)
    s.check(keep, recent, early, label=kind)


@pytest.mark.parametrize("born", [True, False])
def test_layers_and_slots_as_ages(siso, born):  # noqa: F811
    for layer in (None, 1):
        s = Full(siso, "fp8", 64, 2, 16, [200, 77, 30], seed=4, layers=3)
        s.check(64, 16, 4, layer=layer, born=born, label=f"layer {layer}")


@pytest.mark.parametrize("kind,apart", [("spread", 0), ("ties", 700)])
def test_long_contexts(siso, kind, apart):  # noqa: F811
    """More positions than a workgroup holds the numbers of."""
    print(f"case: evict long {kind}", flush=True)
    s = Full(siso, "fp8", 64, 1, 128, [70001, 300, 45000], seed=6, kind=kind, apart=apart)
    s.check(700 if apart else 40001, 100, 3, label="long")


def test_many_sequences_more_than_fit_the_workspace(siso):  # noqa: F811
    """keep is so large that the workspace holds a part of the units at a time."""
    rng = random.Random(1)
    length = [rng.randrange(0, 40) for _ in range(40)]
    s = Full(siso, "bf16", 64, 2, 16, length, seed=2, layers=2)
    s.check(1 << 21, 5, 2, label="large keep")
    s = Full(siso, "bf16", 64, 2, 16, [rng.randrange(0, 60) for _ in range(300)], seed=3)
    s.check(20, 5, 2, label="many")


def test_pages_that_are_none(siso):  # noqa: F811
    """Slots of such pages count as nothing: they are the first to go; what is kept of them is zeros, and nothing is written there."""
    s = Full(siso, "bf16", 64, 1, 16, [64, 48], seed=5)
    pages = s.pages.clone()
    pages[0, 3], pages[1, 0] = -1, s.pool
    batch = s.kv.batch(ends([0, 0]), s.length_dev, pages)
    before = [x.cpu() for x in s.kv.read(s.all, dtype=torch.float32)]
    s.kv.evict(batch, s.weights, 40, 0, 0)
    pg = s.pages.cpu()
    w = [s.mass[0, pg[b, torch.arange(l) // 16].long(), 0, torch.arange(l) % 16].tolist() for b, l in enumerate((64, 48))]
    w[0][48:], w[1][:16] = [math.nan] * 16, [math.nan] * 16
    got = [x.cpu() for x in s.kv.read(s.all, dtype=torch.float32)]
    for b, l in enumerate((64, 48)):
        of = oracle.evict(w[b], None, 40, 0, 0)
        for x, y in zip(got, before):
            for i in range(l):
                want = y[s.starts[b] + i] if i >= 40 or of[i] == i or (b == 1 and i < 16) else y[s.starts[b] + of[i]]
                assert torch.equal(x[s.starts[b] + i], want), f"sequence {b} slot {i}"
    assert s.kv.bad_pages() > 0


def test_too_few_pages_for_what_is_kept(siso):  # noqa: F811
    """Slots beyond the pages given are left out, and nothing else is touched."""
    s = Full(siso, "fp8", 64, 2, 16, [200, 100], seed=7, apart=100)
    to = s.to[:, :3].contiguous().to(DEV)
    s.kv.evict(s.all, s.weights, 100, 10, 2, to=to)
    got = s.kv.read(s.kv.batch(ints([0, 48, 96]), ints([48, 48]), to), dtype=torch.float32)
    hk, pg, j = kv_oracle.held(s.k, "fp8").float(), s.pages.cpu(), torch.arange(200)
    for h in range(2):
        of = torch.tensor(oracle.evict(*(x[0, pg[0, j // 16].long(), h, j % 16].tolist() for x in (s.mass, s.born)), 100, 10, 2))
        assert torch.equal(got[0].cpu()[:48, h], hk[of[:48], h])
        assert torch.equal(got[0].cpu()[48:, h], hk[200:248, h])


def test_an_answer_that_goes_on(siso):  # noqa: F811
    """Tokens are appended, attended to and weighed, and the cache is cut down every few steps: what it then holds, and how attention answers over it,
    against the same done on the host."""
    print("case: a long answer", flush=True)
    heads, kvh, d, page, keep, recent, early, steps = 4, 2, 64, 16, 48, 12, 2, 90
    g = torch.Generator().manual_seed(1)
    kv = siso.PagedKV(kvh, d, 12, page_tokens=page)
    weights = kv.weights()
    pages = ints([[3, 1, 7, 0, 9]])
    table = [3, 1, 7, 0, 9]
    k, v = (torch.randn(steps, kvh, d, generator=g).bfloat16() for _ in range(2))
    q = (torch.randn(steps, heads, d, generator=g) * 2).bfloat16()
    have = [[] for _ in range(kvh)]  # of every head the tokens that its slots hold
    length = 0
    for step in range(steps):
        length += 1
        batch = kv.batch(ints([0, 1]), ints([length]), pages, rows=1, max_new=1, max_length=length)
        kv.write(batch, k[step:step + 1].to(DEV), v[step:step + 1].to(DEV))
        out, lse = kv.attend(batch, q[step:step + 1].to(DEV), with_lse=True)
        for h in range(kvh):
            have[h].append(step)
        want = [torch.zeros(1, heads, d, dtype=torch.float64), torch.zeros(1, heads, d, dtype=torch.float64), torch.zeros(1, heads, dtype=torch.float64),
                torch.zeros(1, heads, dtype=torch.float64)]
        for h in range(kvh):
            part = kv_oracle.attend(q[step:step + 1, 2 * h:2 * h + 2], k[have[h], h:h + 1].double(), v[have[h], h:h + 1].double(), length, 1, float(torch.tensor(d ** -0.5)))
            for x, y in zip(want, part):
                x[:, 2 * h:2 * h + 2] = y
        kv_oracle.check_attend(out, lse, want, d, f"step {step}")
        kv.weigh(batch, q[step:step + 1].to(DEV), lse, weights, newest=ints([step]))
        born = [[weights.born.cpu()[0, table[i // page], h, i % page].item() for i in range(length)] for h in range(kvh)]
        assert born == have, f"step {step}"
        if length == keep + 7:
            mass = [[weights.mass.cpu()[0, table[i // page], h, i % page].item() for i in range(length)] for h in range(kvh)]
            kv.evict(batch, weights, keep, recent, early)
            for h in range(kvh):
                of = oracle.evict(mass[h], have[h], keep, recent, early)
                have[h] = [have[h][i] for i in of]
                assert set(range(step - recent + 1, step + 1)) <= set(have[h]) and {0, 1} <= set(have[h])
            length = keep
    assert have[0] != have[1]


def test_in_a_graph(siso):  # noqa: F811
    """Written and evicted by one graph, replayed with other masses."""
    s = Full(siso, "bf16", 64, 2, 16, [300, 64, 90], seed=8)
    stream = torch.cuda.Stream()
    s.kv.set_stream(stream)
    k, v = s.k.to(DEV), s.v.to(DEV)
    start, ages = s.weights.mass.clone(), s.weights.born.clone()
    stays = s.kv.batch(ints([0, 64, 128, 192]), ints([64, 64, 64]), s.pages)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        def step():
            s.weights.mass.copy_(start)
            s.weights.born.copy_(ages)
            s.kv.write(s.all, k, v)
            s.kv.evict(s.all, s.weights, 64, 16, 4)
            return [*s.kv.read(stays), s.weights.mass.clone(), s.weights.born.clone()]
        step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            got = step()
        for turn in range(4):
            start.copy_(torch.rand_like(start))
            graph.replay()
            torch.cuda.synchronize()
            s.kv.write(s.all, k, v)
            torch.cuda.synchronize()
            replayed = [x.clone() for x in got]
            eager = step()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(replayed, eager)), f"replay {turn}"


@pytest.mark.parametrize("length", [4090, 5119, 5121, 5600, 6144, 6145, 8191, 16384, 16385, 32768, 32769])
def test_lengths_where_the_room_in_shared_memory_changes(siso, length):  # noqa: F811
    print(f"case: evict {length}", flush=True)
    s = Full(siso, "fp8", 8, 1, 128, [length, 3], seed=length % 100, kind="ties" if length % 2 else "spread")
    s.all = s.kv.batch(ends(s.length), s.length_dev, s.pages, max_length=length)
    s.check(length // 3, 100, 4, label=str(length))
