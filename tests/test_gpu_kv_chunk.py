"""Attention of long chunks over the paged cache (siso_kv_attend where a sequence has more than 128 rows of work, new
tokens times query heads of a kv head) against its definition in 64 bits: tiles that fill up and that do not, positions cut into
pieces, chunks beside single tokens."""

import math

import pytest
import torch

import kv_oracle
from gpu_util import DEV
from test_gpu_kv import Setup, ends, ints, siso  # noqa: F401

pytestmark = pytest.mark.gpu

CASES = [
    # d, page, heads, kv_heads, new, length
    (64, 16, 1, 1, [129], [129]),                    # one row more than the other kernel takes
    (64, 32, 4, 2, [100, 1, 65], [150, 40, 65]),     # beside single tokens
    (64, 64, 3, 1, [300], [300]),                    # groups of three: tiles begin inside a token
    (128, 16, 4, 1, [70, 33], [200, 33]),
    (128, 64, 8, 2, [257, 0, 128], [257, 9, 500]),
    (96, 16, 2, 2, [131], [180]),
    (192, 32, 2, 1, [140], [177]),
    (256, 16, 4, 2, [75], [90]),
    (8, 16, 2, 1, [90], [111]),
    (64, 16, 80, 1, [2, 3], [33, 3]),                # a group of 80
]


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("window", [0, 1, 50])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_chunks(siso, dtype, case, window):  # noqa: F811
    d, page, heads, kv_heads, new, length = CASES[case]
    print(f"case: chunk {dtype} window={window} {CASES[case]}", flush=True)
    s = Setup(siso, dtype, d, kv_heads, page, new, length, seed=50 + case)
    s.write()
    s.check(s.queries(heads), window=window, label=f"{dtype} {CASES[case]}")
    assert s.kv.bad_pages() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,new,length", [(64, [150], [2500]), (128, [140], [3001]), (256, [130], [1200]), (128, [150, 2, 131], [1700, 900, 140])])
def test_chunks_over_a_long_axis(siso, dtype, d, new, length):  # noqa: F811
    """Few tiles: their positions are cut into pieces, which are joined; with a bound on the new tokens and without."""
    print(f"case: pieces {dtype} d={d} {new} {length}", flush=True)
    s = Setup(siso, dtype, d, 1, 64, new, length, seed=70, spread=2.0)
    s.write()
    q = s.queries(1)
    s.check(q, label="pieces")
    s.check(q, window=600, label="pieces, window")
    s.batch = s.kv.batch(ends(new), s.length_dev, s.pages)
    s.check(q, label="no bound")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_what_a_row_does_not_see_does_not_touch_it(siso, dtype, what):  # noqa: F811
    s = Setup(siso, dtype, 64, 1, 32, [140], [200], seed=71)
    q = s.queries(2)
    bad = torch.full((s.pool * 32, 1, 64), what, dtype=torch.bfloat16, device=DEV)
    everything = s.kv.batch(ints([0, s.pool * 32]), ints([s.pool * 32]), torch.arange(s.pool, dtype=torch.int32, device=DEV)[None].contiguous())
    s.kv.write(everything, bad, bad)
    s.write()
    s.check(q, label="unused slots")
    # one later token: the rows before it as if it were not there, it and the rows behind it are touched
    s.k[150] = what
    s.v[150] = what
    s.write()
    out, lse = s.kv.attend(s.batch, q.to(DEV), with_lse=True)
    hk, hv = kv_oracle.held(s.k, dtype), kv_oracle.held(s.v, dtype)
    want = kv_oracle.attend(q[:90], hk[:150], hv[:150], 150, 90, 0.125)
    kv_oracle.check_attend(out[:90], lse[:90], want, 64, "before it")
    if dtype == "fp8" or math.isnan(what):
        assert torch.isnan(out[90:].float()).all()
    # tokens ahead of the window
    s = Setup(siso, dtype, 64, 1, 32, [140], [200], seed=72)
    s.k[:20], s.v[:20] = what, what
    s.write()
    hk, hv = kv_oracle.held(s.k, dtype), kv_oracle.held(s.v, dtype)
    out, lse = s.kv.attend(s.batch, q.to(DEV), window=40, with_lse=True)
    want = kv_oracle.attend(q, hk[20:], hv[20:], 180, 140, 0.125, 40)
    kv_oracle.check_attend(out, lse, want, 64, "ahead of the window")


def test_infinite_values_reach_the_rows_that_see_them(siso):  # noqa: F811
    s = Setup(siso, "bf16", 128, 1, 16, [200], [260], seed=73)
    s.v[160, 0, 7], s.v[160, 0, 9], s.v[170, 0, 100] = math.inf, -math.inf, math.inf
    s.write()
    out = s.kv.attend(s.batch, s.queries(1).to(DEV)).float().cpu()[:, 0]
    assert torch.isfinite(out[:100]).all()
    assert torch.isposinf(out[100:, 7]).all() and torch.isneginf(out[100:, 9]).all()
    assert torch.isfinite(out[:110, 100]).all() and torch.isposinf(out[110:, 100]).all()
    assert torch.isfinite(out[:, [d for d in range(128) if d not in (7, 9, 100)]]).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_large_and_small_scores(siso, dtype):  # noqa: F811
    s = Setup(siso, dtype, 64, 1, 16, [150], [400], seed=74, spread=10.0)
    s.k[300:] *= 4  # the maximum rises late
    s.write()
    q = (s.queries(1).float() * 8).bfloat16()
    for scale in (None, -0.125, 0.0, 1e-3):
        s.check(q, scale=scale, label=f"scale {scale}")


def test_pages_that_are_none_and_rows_without_a_position(siso):  # noqa: F811
    s = Setup(siso, "bf16", 64, 1, 16, [150], [200], seed=75)
    s.write()
    s.pages[0, 3], s.pages[0, 10] = -1, 1 << 30
    s.check(s.queries(1), hidden={0: [*range(48, 64), *range(160, 176)]}, label="no pages")
    assert s.kv.bad_pages() > 0
    q = torch.randn(300, 1, 64, device=DEV).bfloat16()
    out, lse = s.kv.attend(s.kv.batch(ints([0, 300]), ints([100]), s.pages), q, with_lse=True)
    assert (out[:200] == 0).all() and torch.isneginf(lse[:200]).all() and torch.isfinite(lse[200:]).all()
    out, lse = s.kv.attend(s.kv.batch(ints([0, 300]), ints([0]), s.pages), q, with_lse=True)
    assert (out == 0).all() and torch.isneginf(lse).all()


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_queries_in_any_order_of_memory_and_the_same_bits_twice(siso, dtype):  # noqa: F811
    s = Setup(siso, dtype, 64, 2, 16, [70, 90], [600, 90], seed=76)
    s.write()
    q = s.queries(4)
    want = s.kv.attend(s.batch, q.to(DEV), with_lse=True)
    for off in (0, 1, 8):
        fused = torch.zeros(160, 4 * 64 + 9, dtype=torch.bfloat16, device=DEV)
        view = fused[:, off:off + 256].view(160, 4, 64)
        view.copy_(q)
        got = s.kv.attend(s.batch, view, with_lse=True)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.equal(s.kv.attend(s.batch, q.to(DEV).transpose(0, 1).contiguous().transpose(0, 1)), want[0])


def test_recorded_in_a_graph(siso):  # noqa: F811
    print("case: chunk in a graph", flush=True)
    s = Setup(siso, "fp8", 64, 1, 16, [150, 1], [700, 500], seed=77)
    s.write()
    stream = torch.cuda.Stream()
    s.kv.set_stream(stream)
    q = torch.zeros(151, 2, 64, dtype=torch.bfloat16, device=DEV)
    out, lse = torch.empty(151, 2, 64, dtype=torch.bfloat16, device=DEV), torch.empty(151, 2, device=DEV)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        s.kv.attend(s.batch, q, out=out, lse=lse)
    for seed in range(4):
        q.copy_(s.queries(2, seed=seed))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        eager = s.kv.attend(s.batch, q, with_lse=True)
        torch.cuda.synchronize()
        assert torch.equal(got[0], eager[0]) and torch.equal(got[1], eager[1])
        s.check(q.cpu(), got=got, label=f"replay {seed}")
