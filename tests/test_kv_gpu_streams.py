"""The paged cache's calls on a stream that is not torch's current one and has much to do already."""

import pytest
import torch

import kv_oracle
from gpu_util import DEV
from test_gpu_kv import Setup, siso  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("rows", [1, 150])
def test_rows_given_up_while_they_wait_to_be_copied(siso, dtype, rows):  # noqa: F811
    print(f"case: copies that wait {dtype} {rows}", flush=True)
    s = Setup(siso, dtype, 64, 2, 16, [rows, 1], [400, 90], seed=130)
    s.write()
    q = s.queries(4).to(DEV)
    want = s.kv.attend(s.batch, q, with_lse=True)
    wide = torch.randn(4096, 4096, device=DEV).bfloat16()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    s.kv.set_stream(side)
    for _ in range(3):
        views = [x.to(DEV).transpose(0, 2).contiguous().transpose(0, 2) for x in (s.k, s.v)] + [q.transpose(0, 2).contiguous().transpose(0, 2)]
        shapes = [v.shape for v in views]
        with torch.cuda.stream(side):
            for _ in range(40):  # some milliseconds
                torch.mm(wide, wide)
        side.wait_stream(torch.cuda.current_stream())
        s.kv.write(s.all, views[0], views[1])
        out, lse = s.kv.attend(s.batch, views[2], with_lse=True)
        back = s.kv.read(s.all)
        del views
        junk = [torch.full(shape, float("nan"), dtype=torch.bfloat16, device=DEV) for shape in shapes for _ in range(3)]
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
        for got, x in zip(back, (s.k, s.v)):
            assert torch.equal(got.double().cpu(), kv_oracle.held(x, dtype).bfloat16().double())
        del junk
