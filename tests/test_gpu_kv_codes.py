"""Every quotient that the 8-bit storage of the paged cache can meet within a binade: all mantissas of a vector's largest element against
all smaller bfloat16 numbers down to those that round to zero, at scales from the smallest to the largest."""

import pytest
import torch

import kv_oracle
from gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [-126, -90, -60, 0, 40, 100, 126])
def test_codes_are_those_of_a_correctly_rounded_quotient(power):
    from paper_2508_18736_amd import siso
    print(f"case: codes at 2^{power}", flush=True)
    mantissas = (1 + torch.arange(128, dtype=torch.float64) / 128) * 2.0 ** power
    rows = []
    for top in mantissas:
        # 19 binades below the largest element: E4M3 reaches 2^-10 * 2^-8 below it
        x = torch.cat([mantissas * 2.0 ** -e for e in range(20)])
        x = x[x <= top]
        x = torch.cat([x, torch.zeros(-len(x) % 255, dtype=torch.float64)]).view(-1, 255)
        rows.append(torch.cat([torch.full((len(x), 1), float(top), dtype=torch.float64), x], 1))
    x = torch.cat(rows)
    x[1::2] *= -1
    x = x.bfloat16()
    t = len(x)
    kv = siso.PagedKV(1, 256, -(-t // 1024), page_tokens=1024, dtype=siso.FP8)
    pages = torch.arange(kv.pages, dtype=torch.int32, device=DEV)[None].contiguous()
    batch = kv.batch(torch.tensor([0, t], dtype=torch.int32, device=DEV), torch.tensor([t], dtype=torch.int32, device=DEV), pages)
    kv.write(batch, x[:, None].to(DEV), x.flip(0)[:, None].to(DEV))
    k, v = kv.read(batch, dtype=torch.float32)
    want = kv_oracle.held(x, "fp8").float()
    assert torch.equal(k[:, 0].cpu(), want) and torch.equal(v[:, 0].cpu(), want.flip(0))
