"""The paged key/value cache (siso_kv.h) against its definition in 64 bits: writing, reading back, attention."""

import ctypes as C
import math

import pytest
import torch

import kv_oracle
from gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def siso():
    from paper_2508_18736_amd import siso as m
    return m


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def ends(x):
    return ints([sum(x[:i]) for i in range(len(x) + 1)])


class Setup:
    """A cache whose sequences' tokens are all written, in pages of a random order, and the same tokens on the host."""

    def __init__(self, siso, dtype, d, kv_heads, page, new, length, seed=0, layers=1, spare=2, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.new, self.length, self.page, self.d, self.dtype = new, length, page, d, dtype
        need = [-(-x // page) for x in length]
        self.pool = sum(need) + spare
        order = torch.randperm(self.pool, generator=g)
        width = max(max(need), 1)
        self.pages = torch.full((len(new), width), 0, dtype=torch.int32)
        at = 0
        for b, c in enumerate(need):
            self.pages[b, :c] = order[at:at + c].int()
            at += c
        self.pages = self.pages.to(DEV)
        total = sum(length)
        self.k = (torch.randn(total, kv_heads, d, generator=g) * spread).bfloat16()
        self.v = (torch.randn(total, kv_heads, d, generator=g) * torch.exp2(torch.randn(total, kv_heads, 1, generator=g))).bfloat16()
        self.kv = siso.PagedKV(kv_heads, d, self.pool, page_tokens=page, layers=layers, dtype=siso.FP8 if dtype == "fp8" else siso.BF16)
        self.length_dev = ints(length)
        self.all = self.kv.batch(ends(length), self.length_dev, self.pages)
        self.batch = self.kv.batch(ends(new), self.length_dev, self.pages, max_new=max(new))
        self.starts = [sum(length[:b]) for b in range(len(length) + 1)]

    def write(self, layer=0):
        self.kv.write(self.all, self.k.to(DEV), self.v.to(DEV), layer=layer)

    def queries(self, heads, seed=1):
        g = torch.Generator().manual_seed(seed)
        return torch.randn(sum(self.new), heads, self.d, generator=g).bfloat16()

    def check(self, q, scale=None, window=0, hidden=None, label="", got=None):
        scale = self.d ** -0.5 if scale is None else scale
        out, lse = got if got is not None else self.kv.attend(self.batch, q.to(DEV), scale=scale, window=window, with_lse=True)
        torch.cuda.synchronize()
        at = 0
        hk, hv = kv_oracle.held(self.k, self.dtype), kv_oracle.held(self.v, self.dtype)
        for b, (m, l) in enumerate(zip(self.new, self.length)):
            s = self.starts[b]
            want = kv_oracle.attend(q[at:at + m], hk[s:s + l], hv[s:s + l], l, m, float(torch.tensor(scale)), window, (hidden or {}).get(b, ()))
            kv_oracle.check_attend(out[at:at + m], lse[at:at + m], want, self.d, f"{label} sequence {b} ({m} of {l})")
            at += m


# ------------------------------------------------------------------ writing and reading back
@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,page,kv_heads", [(8, 16, 1), (64, 64, 3), (72, 16, 2), (128, 32, 8), (192, 128, 1), (256, 16, 2)])
def test_what_is_written_is_read_back(siso, dtype, d, page, kv_heads):
    print(f"case: write and read {dtype} d={d} page={page} kv_heads={kv_heads}", flush=True)
    s = Setup(siso, dtype, d, kv_heads, page, [1, 1, 1, 1], [1, 37, 16, 200], seed=d + page)
    s.k[5] = 0  # a vector without length
    s.v[7, 0] *= 1e30
    s.k[9, 0] *= 1e-30
    s.write()
    for out, exact in ((torch.float32, True), (torch.bfloat16, False)):
        k, v = s.kv.read(s.all, dtype=out)
        for got, x in ((k, s.k), (v, s.v)):
            want = kv_oracle.held(x, dtype).float().to(out)  # (code * scale in 32 bits: the exact product has at most 28, rounded once)
            assert torch.equal(got.cpu(), want)
    assert s.kv.bad_pages() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_tokens_are_appended_one_by_one_and_in_chunks(siso, dtype):
    """Sequences grow by chunks that begin and end anywhere in a block; what stands beside them stays."""
    print(f"case: appending {dtype}", flush=True)
    steps = [[1, 5, 0], [1, 1, 15], [3, 11, 1], [40, 16, 2], [1, 1, 33], [0, 17, 1]]
    final = [sum(x) for x in zip(*steps)]
    s = Setup(siso, dtype, 96, 2, 16, [1, 1, 1], final, seed=3)
    have = [0, 0, 0]
    for step in steps:
        rows = torch.cat([torch.arange(s.starts[b] + have[b], s.starts[b] + have[b] + step[b]) for b in range(3)])
        have = [h + x for h, x in zip(have, step)]
        batch = s.kv.batch(ends(step), ints(have), s.pages, max_new=max(step))
        s.kv.write(batch, s.k[rows].to(DEV), s.v[rows].to(DEV))
        back = s.kv.read(batch, dtype=torch.float32)
        assert torch.equal(back[0].cpu(), kv_oracle.held(s.k[rows], dtype).float())
    k, v = s.kv.read(s.all, dtype=torch.float32)
    assert torch.equal(k.cpu(), kv_oracle.held(s.k, dtype).float()) and torch.equal(v.cpu(), kv_oracle.held(s.v, dtype).float())


def test_vectors_that_are_not_finite(siso):
    s = Setup(siso, "fp8", 64, 2, 16, [1], [20], seed=4)
    s.k[3, 1, 5], s.v[4, 0, 0], s.v[6, 1, 63] = math.nan, math.inf, -math.inf
    s.write()
    k, v = s.kv.read(s.all, dtype=torch.float32)
    for got, x in ((k, s.k), (v, s.v)):
        want = kv_oracle.held(x, "fp8").float()
        assert torch.equal(torch.isnan(got.cpu()), torch.isnan(want)) and torch.equal(torch.nan_to_num(got.cpu()), torch.nan_to_num(want))
    s = Setup(siso, "bf16", 64, 2, 16, [1], [20], seed=4)
    s.k[3, 1, 5], s.v[4, 0, 0], s.v[6, 1, 63] = math.nan, math.inf, -math.inf
    s.write()
    k, v = s.kv.read(s.all)
    assert torch.equal(torch.nan_to_num(k.cpu()), torch.nan_to_num(s.k)) and torch.equal(torch.nan_to_num(v.cpu()), torch.nan_to_num(s.v))


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_rows_in_any_order_of_memory(siso, dtype):
    """Keys and values as slices of a fused projection, as a transposed view, and at addresses no vector load takes."""
    s = Setup(siso, dtype, 64, 3, 32, [1, 1], [50, 21], seed=5)
    total = sum(s.length)
    fused = torch.zeros(total, 5 * 3 * 64 + 1, dtype=torch.bfloat16, device=DEV)
    for off in (0, 64, 1):
        kk, vv = fused[:, off:off + 192].view(total, 3, 64), fused[:, off + 192:off + 384].view(total, 3, 64)
        kk.copy_(s.k), vv.copy_(s.v)
        s.kv.write(s.all, kk, vv)
        k, v = s.kv.read(s.all, dtype=torch.float32)
        assert torch.equal(k.cpu(), kv_oracle.held(s.k, dtype).float()) and torch.equal(v.cpu(), kv_oracle.held(s.v, dtype).float())
    s.kv.write(s.all, s.v.to(DEV).transpose(0, 1).contiguous().transpose(0, 1), s.k.to(DEV).transpose(1, 2).contiguous().transpose(1, 2))
    k, v = s.kv.read(s.all, dtype=torch.float32)
    assert torch.equal(v.cpu(), kv_oracle.held(s.k, dtype).float()) and torch.equal(k.cpu(), kv_oracle.held(s.v, dtype).float())


def test_layers_are_apart(siso):
    s = Setup(siso, "fp8", 64, 2, 16, [1, 1], [33, 10], seed=6, layers=3)
    s.write(layer=1)
    zero = s.kv.read(s.all, layer=0)
    assert (zero[0] == 0).all() and (s.kv.read(s.all, layer=2)[1] == 0).all()
    assert torch.equal(s.kv.read(s.all, layer=1, dtype=torch.float32)[0].cpu(), kv_oracle.held(s.k, "fp8").float())


def test_bad_pages_and_lengths_touch_nothing(siso):
    """Page numbers that are none are counted and left out; rows at positions below zero are no positions."""
    s = Setup(siso, "bf16", 64, 2, 16, [1, 1], [40, 40], seed=7)
    s.write()
    before = s.kv.read(s.all)
    pages = s.pages.clone()
    pages[0, 1], pages[1, 2] = -1, s.pool
    bad = s.kv.batch(ends([40, 40]), s.length_dev, pages)
    assert s.kv.bad_pages() == 0
    s.kv.write(bad, torch.ones(80, 2, 64, dtype=torch.bfloat16, device=DEV), s.v.to(DEV))
    assert s.kv.bad_pages() >= 2
    k, v = s.kv.read(bad)
    assert (k[16:32] == 0).all() and (k[40 + 32:] == 0).all() and (k[:16] == 1).all() and (k[32:40 + 32] == 1).all()
    now = s.kv.read(s.all)
    assert torch.equal(now[1], before[1])  # (the values were the same, the left out ones stand as before)
    # more rows than tokens: the first ones have no position
    short = s.kv.batch(ints([0, 30]), ints([10]), s.pages[:1].contiguous())
    s.kv.write(short, torch.full((30, 2, 64), 2.0, dtype=torch.bfloat16, device=DEV), torch.zeros(30, 2, 64, dtype=torch.bfloat16, device=DEV))
    k, _ = s.kv.read(short)
    assert (k[:20] == 0).all() and (k[20:] == 2).all()
    # lengths and first rows outside their ranges
    for first, length in (([0, 90, 80], [5, 40]), ([-5, 200, 80], [-3, 10 ** 9]), ([70, 10, 80], [40, 40])):
        odd = s.kv.batch(ints(first), ints(length), s.pages, rows=80)
        x = torch.zeros(80, 2, 64, dtype=torch.bfloat16, device=DEV)
        s.kv.write(odd, x, x)
        s.kv.read(odd)
        s.kv.attend(odd, x)
    torch.cuda.synchronize()


# ------------------------------------------------------------------ attention
CASES = [
    # d, page, heads, kv_heads, new, length
    (64, 16, 4, 4, [1, 1, 1], [1, 2, 17]),
    (64, 32, 2, 1, [1, 0, 5, 33, 17], [1, 7, 40, 33, 200]),
    (128, 16, 8, 2, [1, 1, 1, 1], [300, 31, 32, 33]),
    (128, 64, 4, 4, [64, 3], [64, 130]),
    (96, 16, 6, 3, [7, 1, 20], [100, 515, 21]),
    (8, 16, 1, 1, [3], [19]),
    (192, 16, 5, 1, [2, 9], [70, 9]),
    (256, 128, 4, 2, [1, 12], [257, 90]),
    (64, 16, 40, 1, [1, 2], [50, 3]),   # a group of 40: more rows than a tile for one token
    (128, 16, 12, 4, [100], [150]),     # a group of 3: tiles begin inside a token
]


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("window", [0, 1, 20])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(siso, dtype, case, window):
    d, page, heads, kv_heads, new, length = CASES[case]
    print(f"case: attention {dtype} window={window} {CASES[case]}", flush=True)
    s = Setup(siso, dtype, d, kv_heads, page, new, length, seed=case)
    s.write()
    s.check(s.queries(heads), window=window, label=f"{dtype} {CASES[case]}")
    assert s.kv.bad_pages() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("new,length", [([1], [5000]), ([1, 1, 1], [3, 4100, 900]), ([4, 2], [2049, 700]), ([40, 1], [3000, 1030])])
def test_attention_over_a_long_axis(siso, dtype, new, length):
    """Work is split over the positions; with and without a bound on the lengths, and with one that is too low."""
    print(f"case: long axis {dtype} {new} {length}", flush=True)
    s = Setup(siso, dtype, 64, 2, 64, new, length, seed=8, spread=2.0)
    s.write()
    q = s.queries(4)
    for bound in (0, max(length), 64):
        s.batch = s.kv.batch(ends(new), s.length_dev, s.pages, max_new=max(new), max_length=bound)
        s.check(q, label=f"bound {bound}")
    s.check(q, window=777, label="window")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_attention_of_large_scores(siso, dtype):
    """Scores of hundreds, of both signs: one key takes all; and a scale of zero and below."""
    s = Setup(siso, dtype, 64, 2, 16, [3, 1], [90, 40], seed=9, spread=20.0)
    s.write()
    q = (s.queries(4).float() * 20).bfloat16()
    for scale in (None, -0.125, 0.0, 1e-3):
        s.check(q, scale=scale, label=f"scale {scale}")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf, -3.3895e38])
def test_what_a_row_does_not_see_does_not_touch_it(siso, dtype, what):
    """Later tokens of the chunk, tokens ahead of the window, the rest of a page and pages that were used before hold anything."""
    s = Setup(siso, dtype, 64, 2, 32, [8, 20], [50, 61], seed=10)
    s.write()
    q = s.queries(4)
    bad = torch.full((s.pool * 32, 2, 64), what, dtype=torch.bfloat16, device=DEV)
    # every slot of every page holds it first
    everything = s.kv.batch(ints([0, s.pool * 32]), ints([s.pool * 32]), torch.arange(s.pool, dtype=torch.int32, device=DEV)[None].contiguous())
    s.kv.write(everything, bad, bad)
    s.write()
    s.check(q, label="unused slots")
    # the last token of each sequence holds it: only the last row sees that
    for b in range(2):
        s.k[s.starts[b + 1] - 1] = what
        s.v[s.starts[b + 1] - 1] = what
    s.write()
    out, lse = s.kv.attend(s.batch, q.to(DEV), with_lse=True)
    hk, hv = kv_oracle.held(s.k, dtype), kv_oracle.held(s.v, dtype)
    at = 0
    for b, (m, l) in enumerate(zip(s.new, s.length)):
        a = s.starts[b]
        want = kv_oracle.attend(q[at:at + m - 1], hk[a:a + l - 1], hv[a:a + l - 1], l - 1, m - 1, 0.125)
        kv_oracle.check_attend(out[at:at + m - 1], lse[at:at + m - 1], want, 64, "later tokens")
        if not math.isfinite(what):
            assert not torch.isfinite(out[at + m - 1].float()).any()
        at += m
    # the first token holds it, ahead of every row's window
    s = Setup(siso, dtype, 64, 2, 32, [8, 20], [50, 61], seed=10)
    for b in range(2):
        s.k[s.starts[b]:s.starts[b] + 10] = what
        s.v[s.starts[b]:s.starts[b] + 10] = what
    s.write()
    hk, hv = kv_oracle.held(s.k, dtype), kv_oracle.held(s.v, dtype)
    out, lse = s.kv.attend(s.batch, q.to(DEV), window=30, with_lse=True)
    at = 0
    for b, (m, l) in enumerate(zip(s.new, s.length)):
        a = s.starts[b]
        want = kv_oracle.attend(q[at:at + m], hk[a + 10:a + l], hv[a + 10:a + l], l - 10, m, 0.125, 30)
        kv_oracle.check_attend(out[at:at + m], lse[at:at + m], want, 64, "ahead of the window")
        at += m


def test_infinite_values_reach_the_rows_that_see_them(siso):
    """An infinity among the values of the chunk's middle token: rows from there on get it, rows before do not."""
    s = Setup(siso, "bf16", 64, 1, 16, [9], [40], seed=11)
    s.v[35, 0, 7], s.v[35, 0, 9] = math.inf, -math.inf
    s.write()
    q = s.queries(2)
    out = s.kv.attend(s.batch, q.to(DEV)).float().cpu()
    assert torch.isfinite(out[:4]).all()
    assert torch.isposinf(out[4:, :, 7]).all() and torch.isneginf(out[4:, :, 9]).all()
    others = [d for d in range(64) if d not in (7, 9)]
    hk, hv = kv_oracle.held(s.k, "bf16"), torch.nan_to_num(kv_oracle.held(s.v, "bf16"), posinf=0, neginf=0)
    want = kv_oracle.attend(q, hk, hv, 40, 9, 0.125)[0]
    assert ((out[:, :, others].double() - want[:, :, others]).abs() < 0.05).all()


def test_rows_that_see_nothing(siso):
    """Rows at positions below zero and rows whose only pages are none: zeros and -inf."""
    s = Setup(siso, "fp8", 64, 2, 16, [1, 1], [30, 16], seed=12)
    s.write()
    q = torch.randn(26, 4, 64, device=DEV).bfloat16()
    pages = s.pages.clone()
    pages[1, 0] = -7
    batch = s.kv.batch(ints([0, 20, 26]), ints([5, 16]), pages)
    out, lse = s.kv.attend(batch, q, with_lse=True)
    assert (out[:15] == 0).all() and torch.isneginf(lse[:15]).all() and torch.isfinite(lse[15:20]).all()
    assert (out[20:] == 0).all() and torch.isneginf(lse[20:]).all()
    assert s.kv.bad_pages() > 0
    # an empty sequence, an empty batch
    out, lse = s.kv.attend(s.kv.batch(ints([0, 3]), ints([0]), s.pages[:1].contiguous()), q[:3].contiguous(), with_lse=True)
    assert (out == 0).all() and torch.isneginf(lse).all()
    assert s.kv.attend(s.kv.batch(ints([0]), ints([]), s.pages[:0]), q[:0]).shape == (0, 4, 64)
    # a page that is none in the middle hides its tokens
    s = Setup(siso, "bf16", 64, 2, 16, [3], [70], seed=13)
    s.write()
    s.pages[0, 2] = 10 ** 6
    s.check(s.queries(4), hidden={0: range(32, 48)}, label="a page that is none")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_queries_in_any_order_of_memory(siso, dtype):
    s = Setup(siso, dtype, 64, 2, 16, [5, 1], [60, 40], seed=14)
    s.write()
    q = s.queries(4)
    want = s.kv.attend(s.batch, q.to(DEV))
    for off in (0, 1, 8):
        fused = torch.zeros(6, 4 * 64 + 9, dtype=torch.bfloat16, device=DEV)
        view = fused[:, off:off + 256].view(6, 4, 64)
        view.copy_(q)
        assert torch.equal(s.kv.attend(s.batch, view), want)
    assert torch.equal(s.kv.attend(s.batch, q.to(DEV).transpose(0, 1).contiguous().transpose(0, 1)), want)
    assert torch.equal(s.kv.attend(s.batch, q.to(DEV).transpose(1, 2).contiguous().transpose(1, 2)), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_a_sequence_does_not_depend_on_its_neighbours(siso, dtype):
    """A sequence alone and among others, with pages of another order: results within the bar of each other's rounding, and the
    same call twice: the same bits."""
    s = Setup(siso, dtype, 128, 2, 16, [2, 1, 30], [700, 300, 100], seed=15)
    s.write()
    q = s.queries(8)
    a = s.kv.attend(s.batch, q.to(DEV), with_lse=True)
    b = s.kv.attend(s.batch, q.to(DEV), with_lse=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    s.check(q, got=a, label="together")


def test_offsets_beyond_32_bits(siso):
    """Pages whose bytes lie beyond 4 GiB of either pool."""
    print("case: large offsets", flush=True)
    pages = 40000  # of 64 tokens, 8 heads, 128 elements: 5.2 GB of keys in 16 bits
    kv = siso.PagedKV(8, 128, pages, page_tokens=64)
    g = torch.Generator().manual_seed(16)
    k, v = (torch.randn(150, 8, 128, generator=g).bfloat16() for _ in range(2))
    table = ints([[pages - 1, 5, pages - 2]])
    batch = kv.batch(ints([0, 150]), ints([150]), table)
    kv.write(batch, k.to(DEV), v.to(DEV))
    back = kv.read(batch)
    assert torch.equal(back[0].cpu(), k) and torch.equal(back[1].cpu(), v)
    q = torch.randn(1, 8, 128, generator=g).bfloat16()
    out, lse = kv.attend(kv.batch(ints([0, 1]), ints([150]), table), q.to(DEV), with_lse=True)
    kv_oracle.check_attend(out, lse, kv_oracle.attend(q, k.double(), v.double(), 150, 1, 128 ** -0.5), 128, "large offsets")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_recorded_in_a_graph(siso, dtype):
    """Writing, reading and attending in a graph, replayed while lengths, pages and rows change between the replays."""
    print(f"case: graph {dtype}", flush=True)
    s = Setup(siso, dtype, 64, 2, 16, [1, 1], [900, 400], seed=17)
    s.write()
    stream = torch.cuda.Stream()
    s.kv.set_stream(stream)
    q, k, v = (torch.zeros(2, h, 64, dtype=torch.bfloat16, device=DEV) for h in (4, 2, 2))
    length = ints([880, 390])
    batch = s.kv.batch(ints([0, 1, 2]), length, s.pages, rows=2, max_new=1, max_length=900)
    out, lse = torch.empty(2, 4, 64, dtype=torch.bfloat16, device=DEV), torch.empty(2, 4, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        s.kv.write(batch, k, v)
        s.kv.attend(batch, q, out=out, lse=lse)
    for step in range(4):
        q.copy_(s.queries(4, seed=step)[:2]), length.copy_(ints([880 + step, 390 + step]))
        rows = [s.starts[0] + 879 + step, s.starts[1] + 389 + step]
        k.copy_(s.k[rows]), v.copy_(s.v[rows])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        eager = s.kv.attend(batch, q, with_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])
        hk, hv = kv_oracle.held(s.k, dtype), kv_oracle.held(s.v, dtype)
        for b, l in enumerate((880 + step, 390 + step)):
            a = s.starts[b]
            want = kv_oracle.attend(q[b:b + 1].cpu(), hk[a:a + l], hv[a:a + l], l, 1, 0.125)
            kv_oracle.check_attend(got[0][b:b + 1], got[1][b:b + 1], want, 64, f"replay {step}")


# ------------------------------------------------------------------ refusals
def test_refusals(siso):
    for bad in (dict(kv_heads=0), dict(head_dim=12), dict(head_dim=264), dict(head_dim=0), dict(page_tokens=8), dict(page_tokens=48),
                dict(page_tokens=2048), dict(pages=0), dict(layers=0), dict(dtype=siso.F32), dict(kv_heads=2000)):
        with pytest.raises(siso.SisoError):
            siso.PagedKV(**{**dict(kv_heads=2, head_dim=64, pages=4), **bad})
    kv = siso.PagedKV(2, 64, 4, page_tokens=16, layers=2)
    batch = kv.batch(ints([0, 2]), ints([2]), ints([[0]]))
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16, device=DEV)
    x = torch.zeros(2, 2, 64, dtype=torch.bfloat16, device=DEV)
    for call in (lambda: kv.attend(batch, q[:, :3]), lambda: kv.attend(batch, q, layer=2), lambda: kv.attend(batch, q, layer=-1),
                 lambda: kv.attend(batch, q, scale=math.inf), lambda: kv.attend(batch, q, scale=math.nan), lambda: kv.attend(batch, q, window=-1),
                 lambda: kv.write(batch, x, x, layer=2), lambda: kv.read(batch, layer=5),
                 lambda: kv.attend(batch, torch.zeros(2, 2 * 129, 64, dtype=torch.bfloat16, device=DEV)),
                 lambda: kv.attend(kv.batch(ints([0, 2])), q)):
        with pytest.raises(siso.SisoError) as e:
            call()
        assert e.value.code == siso.EINVAL and "siso_kv" in str(e.value)
    for call in (lambda: kv.attend(batch, q.float()), lambda: kv.attend(batch, q[:1]), lambda: kv.attend(batch, q.cpu()),
                 lambda: kv.write(batch, q, x), lambda: kv.read(batch, dtype=torch.float16), lambda: kv.attend(batch, q, out=q[:1]),
                 lambda: kv.batch(ints([0, 2]), ints([2])), lambda: kv.batch(ints([0, 2]), ints([2, 3]), ints([[0]])),
                 lambda: kv.batch(ints([0, 2]).long(), ints([2]), ints([[0]]))):
        with pytest.raises(ValueError):
            call()


def test_refusals_of_the_c_calls(siso):
    """Arguments that the binding does not let through."""
    lib = siso._lib
    kv = siso.PagedKV(2, 64, 4, page_tokens=16)
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16, device=DEV)
    first, length, pages = ints([0, 2]), ints([2]), ints([[0]])
    make = lambda **over: siso._KvBatchStruct(**{**dict(n=1, rows=2, first=first.data_ptr(), length=length.data_ptr(), pages=pages.data_ptr(),  # noqa: E731
                                                        width=1, max_new=0, max_length=0), **over})
    p = x.data_ptr()
    attend = lambda b, q=p, out=p, lse=None: lib.siso_kv_attend(kv._h, 0, C.byref(b), q, 128, 64, 2, 0.125, 0, out, lse)  # noqa: E731
    for over in (dict(n=-1), dict(n=70000), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(first=None), dict(length=None), dict(pages=None),
                 dict(width=-1), dict(width=1 << 40), dict(max_new=-1), dict(max_length=-1)):
        assert attend(make(**over)) == siso.EINVAL, over
        assert lib.siso_kv_last_error(kv._h)
    good = make()
    assert attend(good, q=None) == siso.EINVAL and attend(good, out=None) == siso.EINVAL and attend(good, out=p + 8) == siso.EINVAL
    assert attend(good, q=p + 1) == siso.EINVAL and attend(good, lse=p + 2) == siso.EINVAL
    assert lib.siso_kv_attend(kv._h, 0, None, p, 128, 64, 2, 0.125, 0, p, None) == siso.EINVAL
    assert lib.siso_kv_write(kv._h, 0, C.byref(good), None, 128, 64, p, 128, 64) == siso.EINVAL
    assert lib.siso_kv_write(kv._h, 0, C.byref(good), p, 128, 64, p + 1, 128, 64) == siso.EINVAL
    assert lib.siso_kv_read(kv._h, 0, C.byref(good), siso.FP8, p, p) == siso.EINVAL
    assert lib.siso_kv_read(kv._h, 0, C.byref(good), siso.BF16, p, p + 4) == siso.EINVAL
    assert attend(make(n=0, rows=0, first=None, length=None, pages=None)) == siso.OK and attend(make(rows=0)) == siso.OK
    for call in (lib.siso_kv_set_stream(None, None), lib.siso_kv_bad_pages(None),
                 lib.siso_kv_write(None, 0, C.byref(good), p, 0, 0, p, 0, 0), lib.siso_kv_read(None, 0, C.byref(good), 1, p, p),
                 lib.siso_kv_attend(None, 0, C.byref(good), p, 0, 0, 2, 1.0, 0, p, None)):
        assert call == siso.EINVAL
    lib.siso_kv_destroy(None)
