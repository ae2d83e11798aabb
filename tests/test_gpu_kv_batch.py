"""The paged key/value cache with batches of many sequences, which attention plans in a launch of its own, with maxima that
grow late in a chunk, on a stream that is not torch's, and sizes that are refused."""

import ctypes as C
import random

import pytest
import torch

import kv_oracle
from gpu_util import DEV
from test_gpu_kv import Setup, ends, ints, siso  # noqa: F401

pytestmark = pytest.mark.gpu


def _spread(seed, n, new, length):
    rng = random.Random(seed)
    m = [rng.randint(0, new) for _ in range(n)]
    return m, [max(x, int(length ** rng.random())) for x in m]


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("n,d,page,kv_heads,heads,new,length", [
    (64, 64, 16, 1, 2, 2, 300),        # the most that needs no plan
    (65, 64, 16, 2, 2, 1, 200),        # one more
    (130, 128, 32, 1, 4, 3, 700),      # tiles that are cut into stretches, in every part of the plan
    (70, 256, 16, 1, 1, 40, 120),      # more than one tile of a sequence
    (4161, 8, 16, 1, 1, 1, 3),         # the plan has two levels: more than 64 parts of 64
])
def test_many_sequences(siso, dtype, n, d, page, kv_heads, heads, new, length):  # noqa: F811
    print(f"case: many sequences {dtype} {n} {d} {new} {length}", flush=True)
    m, l = _spread(n, n, new, length)
    m[0] = m[-1] = 0
    l[5], l[n - 2] = 1500 if n < 1000 else 40, 1800 if n < 1000 else 50
    s = Setup(siso, dtype, d, kv_heads, page, m, l, seed=90)
    s.write()
    back = s.kv.read(s.all, dtype=torch.float32)
    for got, x in zip(back, (s.k, s.v)):
        assert torch.equal(got.cpu(), kv_oracle.held(x, dtype).float())  # (code times scale in single precision)
    q = s.queries(heads)
    s.check(q, label="many")
    s.check(q, window=33, label="many, window")
    want = s.kv.attend(s.batch, q.to(DEV), with_lse=True)
    for hints in (dict(), dict(max_new=max(m), max_length=max(l)), dict(max_length=1)):  # (a bound on lengths that does not hold costs time only)
        got = s.kv.attend(s.kv.batch(ends(m), s.length_dev, s.pages, **hints), q.to(DEV), with_lse=True)
        if hints != dict(max_length=1):
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        s.check(q, got=got, label=f"hints {hints}")
    assert s.kv.bad_pages() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
def test_many_sequences_and_chunks_among_them(siso, dtype):  # noqa: F811
    print(f"case: chunks among many {dtype}", flush=True)
    m, l = _spread(7, 100, 2, 90)
    m[3], m[64], m[99] = 140, 70, 33
    l[3], l[64], l[99] = 300, 70, 400
    s = Setup(siso, dtype, 64, 1, 16, m, l, seed=91)
    s.write()
    s.check(s.queries(2), label="chunks among many")
    s.check(s.queries(2), window=40, label="chunks among many, window")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,rows", [(64, 140), (128, 300), (192, 130)])
@pytest.mark.parametrize("grow", [40.0, 400.0])
def test_a_maximum_that_grows_beyond_any_power(siso, dtype, d, rows, grow):  # noqa: F811
    """Rows whose later scores pass the first ones by far more than single precision's powers take in, and rows of the same tile
    that see none of them, or nothing else."""
    print(f"case: growing maximum {dtype} d={d} {rows} {grow}", flush=True)
    length = 700
    s = Setup(siso, dtype, d, 1, 32, [rows], [length], seed=92)
    q = s.queries(1)
    direction = q[rows // 2, 0].float()
    direction /= (direction * direction).sum().sqrt()
    for at, size in ((320, grow / 2), (length - rows + rows // 2 - 1, grow), (length - 2, -grow)):
        s.k[at] = (direction * size).bfloat16()
    s.write()
    s.check(q, scale=1.0, label=f"grows by {grow}")
    s.check(q, scale=1.0, window=64, label=f"grows by {grow}, window")


def test_values_whose_sums_leave_the_range(siso):  # noqa: F811
    """Large values under weights that would overflow against the first maximum, and do not against the last one."""
    s = Setup(siso, "bf16", 64, 1, 16, [150], [500], seed=93)
    q = s.queries(1)
    s.k[350] = (q[149, 0].float() * 2).bfloat16()
    s.v[350] = 1.0e38
    s.v[349] = -1.0e38
    s.write()
    s.check(q, scale=0.125, label="large values")


@pytest.mark.parametrize("rows", [1, 150])
def test_a_stream_that_is_not_torchs(siso, rows):  # noqa: F811
    """Calls work on the handle's stream; what they return is used behind it, while torch's own stream allocates and frees."""
    s = Setup(siso, "fp8", 64, 2, 16, [rows, 1], [400, 90], seed=94)
    s.write()
    q = s.queries(4).to(DEV)
    want = s.kv.attend(s.batch, q, with_lse=True)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    s.kv.set_stream(side)
    for _ in range(3):
        view = q.transpose(0, 2).contiguous().transpose(0, 2)  # (no unit stride: copied on the handle's stream)
        side.wait_stream(torch.cuda.current_stream())
        s.write()
        out, lse = s.kv.attend(s.batch, view, with_lse=True)
        back = s.kv.read(s.all)
        del view
        junk = [torch.full((rows + 1, 4, 64), float("nan"), dtype=torch.bfloat16, device=DEV) for _ in range(4)]
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]) and torch.equal(back[0].double().cpu(), kv_oracle.held(s.k, "fp8").bfloat16().double())
        del junk


def test_more_rows_of_work_than_launches_count(siso):  # noqa: F811
    kv = siso.PagedKV(1, 64, 4, page_tokens=16)
    first, length, pages = ints([0, 2]), ints([2]), ints([[0]])
    x = torch.zeros(2, 128, 64, dtype=torch.bfloat16, device=DEV)
    batch = siso._KvBatchStruct(n=1, rows=(1 << 23) + 1, first=first.data_ptr(), length=length.data_ptr(), pages=pages.data_ptr(), width=1, max_new=0,
                                max_length=0)
    rc = siso._lib.siso_kv_attend(kv._h, 0, C.byref(batch), x.data_ptr(), 128 * 64, 64, 128, 0.125, 0, x.data_ptr(), None)
    assert rc == siso.EINVAL and b"rows" in siso._lib.siso_kv_last_error(kv._h)
