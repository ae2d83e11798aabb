"""Attention weights of cached positions, added up (siso_kv_weigh), against their definition in 64 bits."""

import math

import pytest
import torch

import kv_oracle
import kv_tree_oracle as oracle
from gpu_util import DEV
from test_gpu_kv import Setup, ends, ints, siso  # noqa: F401

pytestmark = pytest.mark.gpu


class Weighed(Setup):
    def start(self, layers=1, seed=0):
        g = torch.Generator().manual_seed(seed)
        shape = (layers, self.pool, self.kv.kv_heads, self.page)
        self.mass, self.born = torch.rand(shape, generator=g), torch.randint(0, 1000, shape, generator=g, dtype=torch.int32)
        self.weights = self.kv.weights(self.mass.to(DEV), self.born.to(DEV))

    def check_weigh(self, q, lse, window=0, decay=1.0, fresh=None, newest=None, scale=None, layer=0, got=None, label=""):
        scale = self.d ** -0.5 if scale is None else scale
        want, tol, born = self.mass.double().clone(), torch.zeros(self.mass.shape, dtype=torch.float64), self.born.clone()
        hk = kv_oracle.held(self.k, self.dtype)
        pages, at = self.pages.cpu(), 0
        for b, (m, l) in enumerate(zip(self.new, self.length)):
            if m > 0 and l > 0:
                s = self.starts[b]
                sums, off = oracle.weigh(q[at:at + m], hk[s:s + l], lse[at:at + m].cpu(), l, window, float(torch.tensor(scale)))
                j = torch.arange(l)
                pg, slot = pages[b, j // self.page].long(), j % self.page
                begin = l - m if fresh is None else fresh[b]
                had = torch.where(j < begin, want[layer, pg, :, slot].t() * decay, torch.zeros((), dtype=torch.float64))
                want[layer, pg, :, slot] = (had + sums).t()
                tol[layer, pg, :, slot] = (off + 2.0 ** -23 * (had + sums)).t()
                new = j >= begin
                born[layer, pg[new], :, slot[new]] = ((l - 1 if newest is None else newest[b]) - (l - 1 - j[new]))[:, None].int().expand(-1, born.shape[2])
            at += m
        mass, got_born = (self.weights.mass, self.weights.born) if got is None else got
        torch.cuda.synchronize()
        err = (mass.double().cpu() - want).abs()
        assert torch.isfinite(mass).all() and (err <= tol).all(), f"{label}: {float((err - tol).max()):.3e} beyond the bar"
        assert torch.equal(got_born.cpu(), born), f"{label}: born"

    def lse_of(self, q, **how):
        return self.kv.attend(self.batch, q.to(DEV), with_lse=True, **how)[1]


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,page,kv_heads,heads", [(64, 16, 2, 4), (128, 64, 2, 8), (72, 16, 3, 3), (8, 32, 1, 5), (192, 32, 2, 2), (256, 16, 1, 4), (128, 16, 1, 128)])
def test_weights_are_added(siso, dtype, d, page, kv_heads, heads):  # noqa: F811
    print(f"case: weigh {dtype} d={d} page={page} heads={heads}/{kv_heads}", flush=True)
    s = Weighed(siso, dtype, d, kv_heads, page, [1, 7, 0, 33, 1, 150], [1, 300, 40, 33, 257, 400], seed=d)
    s.write()
    s.start()
    q = s.queries(heads)
    lse = s.lse_of(q)
    s.kv.weigh(s.batch, q.to(DEV), lse, s.weights)
    s.check_weigh(q, lse, label=f"{dtype} d={d}")
    assert s.kv.bad_pages() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("window", [1, 30, 200, 100000])
def test_windows_decay_and_where_it_begins(siso, dtype, window):  # noqa: F811
    print(f"case: weigh window {window} {dtype}", flush=True)
    new, length = [1, 100, 40], [90, 300, 41]
    s = Weighed(siso, dtype, 128, 2, 16, new, length, seed=window % 89)
    s.write()
    q = s.queries(4)
    lse = s.lse_of(q, window=window)
    for decay, fresh, newest in ((1.0, None, None), (0.0, None, [1000, 5, 70]), (0.75, [0, 250, 100], [89, 2000, 40]), (0.5, [90, 0, -3], None)):
        s.start()
        s.kv.weigh(s.batch, q.to(DEV), lse, s.weights, window=window, decay=decay, fresh=None if fresh is None else ints(fresh),
                   newest=None if newest is None else ints(newest))
        s.check_weigh(q, lse, window, decay, fresh, newest, label=f"decay {decay}")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,new,length,heads", [(128, [1500], [4000], 4), (64, [600, 1, 900], [900, 9000, 901], 6), (128, [1, 1], [70001, 300], 8), (256, [300], [2000], 2)])
def test_chunks_and_long_contexts(siso, dtype, d, new, length, heads):  # noqa: F811
    print(f"case: weigh chunk {dtype} d={d} {new} {length}", flush=True)
    s = Weighed(siso, dtype, d, 2, 64, new, length, seed=7)
    s.write()
    s.start()
    q = s.queries(heads)
    lse = s.lse_of(q)
    s.kv.weigh(s.batch, q.to(DEV), lse, s.weights)
    s.check_weigh(q, lse, label="chunk")


def test_a_row_spreads_one(siso):  # noqa: F811
    """What a row weighs adds up to one for each of its heads."""
    s = Weighed(siso, "bf16", 64, 2, 16, [50], [500], seed=3)
    s.write()
    weights = s.kv.weights()
    q = s.queries(8).to(DEV)
    s.kv.weigh(s.batch, q, s.kv.attend(s.batch, q, with_lse=True)[1], weights, fresh=ints([0]))
    total = weights.mass.double().sum((1, 3))[0]
    assert ((total - 50 * 4).abs() < 50 * 4 * 1e-5).all()
    assert weights.born.max() == 499


def test_strides_scale_layers_and_many_sequences(siso):  # noqa: F811
    import random
    rng = random.Random(5)
    new = [rng.randrange(0, 4) for _ in range(150)]
    length = [max(m, rng.randrange(0, 200)) for m in new]
    s = Weighed(siso, "fp8", 64, 2, 16, new, length, seed=9, layers=2)
    s.write(layer=1)
    q = s.queries(4)
    wide = torch.zeros(sum(new), 4, 3, 65, dtype=torch.bfloat16, device=DEV)
    wide[:, :, 1, :64] = q.to(DEV)
    lse = s.lse_of(q, scale=-0.3, layer=1)
    s.start(layers=2)
    s.kv.weigh(s.batch, wide[:, :, 1, :64], lse, s.weights, layer=1, scale=-0.3)
    s.check_weigh(q, lse, scale=-0.3, layer=1, label="many")
    # a length that the caller has too small weighs on speed alone
    s.start(layers=2)
    s.batch = s.kv.batch(ends(new), s.length_dev, s.pages, max_new=3, max_length=20)
    s.kv.weigh(s.batch, q.to(DEV), lse, s.weights, layer=1, scale=-0.3)
    s.check_weigh(q, lse, scale=-0.3, layer=1, label="a small max_length")


def test_rows_that_saw_nothing_and_values_that_are_not_finite(siso):  # noqa: F811
    """Rows with lse = -inf add nothing; NaN in a key is its own position's, and of positions that no row sees nobody's."""
    s = Weighed(siso, "bf16", 64, 2, 16, [4, 30], [100, 20], seed=4)
    s.write()
    q = s.queries(4)
    lse = s.lse_of(q)
    assert torch.isneginf(lse[4:14]).all()  # rows without a position
    lse[2] = -math.inf
    s.start()
    s.kv.weigh(s.batch, q.to(DEV), lse, s.weights)
    s.check_weigh(q, lse, label="rows that saw nothing")
    s.k[10, 0, 5], s.k[2] = math.nan, math.inf
    s.write()
    s.start()
    s.kv.weigh(s.batch, q.to(DEV), lse, s.weights, window=94)
    mass = s.weights.mass.cpu()[0, s.pages.cpu()[0, 0].long()]
    before = s.mass[0, s.pages.cpu()[0, 0].long()]
    assert torch.isnan(mass[0, 10]) and torch.isfinite(mass[1, 10]) and torch.isfinite(mass[0, 11])
    assert torch.equal(mass[:, 2], before[:, 2])  # (the first row stands at 96 and sees what is beyond 96 - 94)


def test_pages_that_are_none(siso):  # noqa: F811
    s = Weighed(siso, "fp8", 64, 2, 16, [3], [100], seed=6)
    s.write()
    pages = s.pages.clone()
    pages[0, 2], pages[0, 5] = -1, s.pool
    q = s.queries(4)
    batch = s.kv.batch(ends([3]), s.length_dev, pages, max_new=3)
    lse = s.kv.attend(batch, q.to(DEV), with_lse=True)[1]
    s.start()
    s.kv.weigh(batch, q.to(DEV), lse, s.weights)
    before = s.kv.bad_pages()
    held = [j for j in range(100) if j // 16 not in (2, 5)]
    sums, tol = oracle.weigh(q, kv_oracle.held(s.k, "fp8"), lse.cpu(), 100, 0, float(torch.tensor(s.d ** -0.5)))
    pg = s.pages.cpu()[0]
    for j in range(100):
        got, had = s.weights.mass.cpu()[0, pg[j // 16].long(), :, j % 16].double(), s.mass[0, pg[j // 16].long(), :, j % 16].double()
        want = had if j not in held else sums[:, j] + (had if j < 97 else 0)
        assert ((got - want).abs() <= tol[:, j] + 2.0 ** -22 * want.abs()).all(), f"position {j}"
    assert before > 0


@pytest.mark.parametrize("rows", [1, 70])
def test_in_a_graph(siso, rows):  # noqa: F811
    """Written, attended to and weighed by one graph, replayed: sums grow as eager calls make them grow."""
    s = Weighed(siso, "bf16", 128, 2, 16, [rows, 1], [200, 90], seed=8)
    stream = torch.cuda.Stream()
    s.kv.set_stream(stream)
    k, v, q = s.k.to(DEV), s.v.to(DEV), s.queries(8).to(DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        weights = s.kv.weights()
        def step(w):
            s.kv.write(s.all, k, v)
            s.kv.weigh(s.batch, q, s.kv.attend(s.batch, q, with_lse=True)[1], w)
        step(weights)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(weights)
        eager = s.kv.weights(weights.mass.clone(), weights.born.clone())
        for _ in range(4):
            q.copy_(torch.randn_like(q))
            graph.replay()
            step(eager)
            torch.cuda.synchronize()
            assert torch.equal(weights.mass, eager.mass) and torch.equal(weights.born, eager.born)
