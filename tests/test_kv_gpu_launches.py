"""Attention of so many sequences and heads that one launch does not take them."""

import pytest
import torch

from gpu_util import DEV
from test_gpu_kv import ints, siso  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d", [64, 128])
def test_tiles_of_several_launches(siso, dtype, d):  # noqa: F811
    """65,535 sequences, all empty but three, 256 heads: more than 2^23 workgroups, in both kernels."""
    print(f"case: several launches {dtype} d={d}", flush=True)
    n, heads = 65535, 256
    rows = {0: 130, 40000: 2, n - 1: 131}  # (two of them are chunks)
    length = {0: 140, 40000: 30, n - 1: 131}
    kv = siso.PagedKV(heads, d, 21, page_tokens=16, dtype=siso.FP8 if dtype == "fp8" else siso.BF16)
    first, lengths, table = torch.zeros(n + 1, dtype=torch.int32), torch.zeros(n, dtype=torch.int32), torch.zeros(n, 9, dtype=torch.int32)
    for b in rows:
        first[b + 1:] += rows[b]
        lengths[b] = length[b]
    table[0], table[40000, :2], table[n - 1] = torch.arange(0, 9), torch.tensor([9, 10]), torch.arange(11, 20)
    g = torch.Generator(device=DEV).manual_seed(170)
    total = sum(length.values())
    k, v = (torch.randn(total, heads, d, generator=g, device=DEV).bfloat16() for _ in range(2))
    q = torch.randn(sum(rows.values()), heads, d, generator=g, device=DEV).bfloat16()
    three = list(rows)
    at = torch.tensor([0, *torch.tensor(list(length.values())).cumsum(0).tolist()], dtype=torch.int32, device=DEV)
    some = kv.batch(at, ints(list(length.values())), table[three].to(DEV).contiguous())
    kv.write(some, k, v)
    new = torch.tensor([0, *torch.tensor(list(rows.values())).cumsum(0).tolist()], dtype=torch.int32, device=DEV)
    want = kv.attend(kv.batch(new, ints(list(length.values())), table[three].to(DEV).contiguous()), q, with_lse=True)
    got = kv.attend(kv.batch(first.to(DEV), lengths.to(DEV), table.to(DEV), rows=sum(rows.values())), q, with_lse=True)
    # against the same rows by themselves (which the tests of smaller batches check): other parts, the same bar of roundings
    assert torch.isfinite(got[0].float()).all() and torch.isfinite(got[1]).all()
    assert ((got[0].double() - want[0].double()).abs() <= 2 * 1.02 * 2.0 ** -8 * (want[0].double().abs() + float(v.abs().max()))).all()
    assert ((got[1] - want[1]).abs() <= 1e-4).all()
    # and the definition, for some rows and heads
    fine_k, fine_v = (x.double() for x in kv.read(some, dtype=torch.float32))
    for b, row in ((0, 0), (0, 129), (1, 1), (2, 0), (2, 130)):
        seen = int(at[b]) + list(length.values())[b] - list(rows.values())[b] + row + 1
        for h in (0, 3, 255):
            kk, vv = fine_k[int(at[b]):seen, h], fine_v[int(at[b]):seen, h]
            s = (kk @ q[int(new[b]) + row, h].double()) * d ** -0.5
            p = torch.softmax(s, 0)
            out = got[0][int(new[b]) + row, h].double()
            assert ((out - p @ vv).abs() <= 1.1 * 2.0 ** -8 * ((p @ vv).abs() + p @ vv.abs()) + 1e-4).all()
            assert abs(float(got[1][int(new[b]) + row, h]) - float(torch.logsumexp(s, 0))) <= 1e-4
    assert kv.bad_pages() == 0
