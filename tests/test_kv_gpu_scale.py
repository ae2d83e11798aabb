"""Attention under scales at the ends of single precision."""

import math

import pytest
import torch

from gpu_util import DEV
from test_gpu_kv import Setup, siso  # noqa: F401
from test_gpu_kv_heavy import Wide

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "fp8"])
@pytest.mark.parametrize("d,kind", [(64, Setup), (128, Setup), (64, Wide), (128, Wide)])
@pytest.mark.parametrize("scale", [3.4028234e38, -3.2e38, 2.9e38, 2.3e38, 1e-45])
def test_scores_of_zero_under_any_scale(siso, dtype, d, kind, scale):  # noqa: F811
    print(f"case: scale {scale} {dtype} d={d} {kind.__name__}", flush=True)
    s = kind(siso, dtype, d, 1, 16, [200, 3], [300, 40], seed=160)
    s.write()
    q = torch.zeros(203, 1, d, dtype=torch.bfloat16)
    out, lse = s.kv.attend(s.batch, q.to(DEV), scale=scale, with_lse=True)
    s.check(q, scale=0.0, got=(out, lse), label=f"scale {scale}")


def test_scales_that_are_not_finite_are_refused(siso):  # noqa: F811
    s = Setup(siso, "bf16", 64, 1, 16, [1], [20], seed=161)
    for scale in (math.inf, -math.inf, math.nan):
        with pytest.raises(siso.SisoError):
            s.kv.attend(s.batch, s.queries(1).to(DEV), scale=scale)
