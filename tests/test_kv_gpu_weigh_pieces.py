"""Attention weights where the pieces of work are many (siso_kv_weigh): more than there are workgroups or places for their sums, and rows cut under windows."""

import pytest
import torch

import kv_oracle
import kv_tree_oracle as oracle
from gpu_util import DEV
from test_gpu_kv import ends, ints, siso  # noqa: F401
from test_kv_gpu_weigh import Weighed

pytestmark = pytest.mark.gpu


def check_heads(s, q, lse, some, label):
    """Of the kv heads `some` (one query head each) all positions; sums alone (nothing was there), ages of all."""
    table, mass, born, at = s.pages.cpu(), s.weights.mass.cpu(), s.weights.born.cpu(), 0
    for b, (m, l) in enumerate(zip(s.new, s.length)):
        j = torch.arange(l)
        pg, slot = table[b, j // s.page].long(), j % s.page
        sums, tol = oracle.weigh(q[at:at + m][:, some], kv_oracle.held(s.k[s.starts[b]:s.starts[b] + l, some], s.dtype), lse[at:at + m][:, some].cpu(), l, 0,
                                 float(torch.tensor(s.d ** -0.5)))
        got = mass[0, pg, :, slot][:, some].double().t()
        assert ((got - sums).abs() <= tol + 2.0 ** -23 * sums).all(), f"{label}: sequence {b}"
        assert torch.equal(born[0, pg, :, slot], j[:, None].int().expand(-1, s.kv.kv_heads)), f"{label}: sequence {b}, born"
        at += m


@pytest.mark.parametrize("n", [70, 64])
def test_more_pieces_than_workgroups(siso, n):  # noqa: F811
    """1,024 kv heads: more blocks than a launch has workgroups, which take several one after the other."""
    print(f"case: weigh, {1024 * n} blocks and more", flush=True)
    new, length = [129 + b % 3 for b in range(n)], [131 + 60 * (b % 4) for b in range(n)]
    s = Weighed(siso, "fp8", 8, 1024, 16, new, length, seed=n)
    s.write()
    s.weights = s.kv.weights()
    q = s.queries(1024)
    lse = s.lse_of(q)
    s.kv.weigh(s.batch, q.to(DEV), lse, s.weights, fresh=ints([0] * n))
    check_heads(s, q, lse, [0, 1, 63, 500, 940, 1023], f"{n} sequences")


@pytest.mark.parametrize("many", [False, True])
def test_more_pieces_than_are_joined(siso, many):  # noqa: F811
    """Rows that the launch would cut, by a length that the caller has too small, into more pieces than there are places for sums: they are not cut."""
    print(f"case: weigh, more pieces than are joined, many={many}", flush=True)
    new, length = ([300], [8600]) if not many else ([257] * 66, [257] * 66)
    heads = 1000 if not many else 15
    if many:
        length = [257 + 256 * (b % 70) for b in range(66)]
    s = Weighed(siso, "bf16", 8, heads, 64, new, length, seed=6)
    s.write()
    s.weights = s.kv.weights()
    q = s.queries(heads)
    lse = s.lse_of(q)
    batch = s.kv.batch(ends(new), s.length_dev, s.pages, max_new=max(new), max_length=1)
    s.kv.weigh(batch, q.to(DEV), lse, s.weights, fresh=ints([0] * len(new)))
    check_heads(s, q, lse, [0, heads // 2, heads - 1], "not cut")


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("window", [1, 200, 3000])
@pytest.mark.parametrize("apart", [0, 1])
def test_windows_of_rows_that_are_cut(siso, dtype, window, apart):  # noqa: F811
    """Stretches of rows that see nothing of a block, some of it and all of it, whose sums are joined; queries aligned and not."""
    print(f"case: weigh, cut rows, window {window} {dtype} apart={apart}", flush=True)
    new, length = [1500, 700], [4000, 700]
    s = Weighed(siso, dtype, 64, 2, 16, new, length, seed=window % 83)
    s.write()
    q = s.queries(4)
    wide = torch.zeros(sum(new), 4, 64 + apart, dtype=torch.bfloat16, device=DEV)
    wide[:, :, :64] = q.to(DEV)
    lse = s.lse_of(q, window=window)
    for decay, fresh in ((1.0, None), (0.75, [0, 300]), (1.0, [1000, 0]), (0.5, None)):
        s.start()
        s.kv.weigh(s.batch, wide[:, :, :64], lse, s.weights, window=window, decay=decay, fresh=None if fresh is None else ints(fresh))
        s.check_weigh(q, lse, window, decay, fresh, label=f"window {window} decay {decay} fresh {fresh}")
    assert s.kv.bad_pages() == 0
