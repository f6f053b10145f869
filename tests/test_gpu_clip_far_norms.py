"""Gradients whose norm is far above the one they are clipped to."""
import math

import pytest
import torch

import explore_util as ref
from paper_2001_08743_amd import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("dtype,scale,max_norm", [(torch.float32, 1e37, 1e-2), (torch.float32, 1e37, 1e-4), (torch.float32, 1e30, 1e-12), (torch.float32, 1e37, 1e-20),
                                                  (torch.bfloat16, 1e37, 1e-3), (torch.bfloat16, 1e37, 1e-30)])
def test_clip_by_a_factor_below_fp32s_normal_numbers(dtype, scale, max_norm):
    g = torch.Generator().manual_seed(3)
    ts = [(scale * torch.randn(n, generator=g)).to(dtype).to(DEV) for n in (1000, 7, 40001)]
    norm = math.sqrt(sum(float(t.double().square().sum()) for t in ts))
    factor = max_norm / (norm + 1e-6)
    assert factor < 2.0 ** -126
    keep = [t.clone() for t in ts]
    outs = [torch.empty_like(t) for t in ts]
    binding.cham_clip_grads(ts, max_norm, out=outs)
    binding.cham_clip_grads(ts, max_norm)
    for t, k, o in zip(ts, keep, outs):
        x = k.double() * factor
        # the factor and the product are rounded to fp32 at most, the result to its type
        assert (o.double() - x).abs().le(x.abs() * (2 * ref.U + ref.HALF[dtype]) * (1 + 1e-6) + ref.TINY[dtype]).all()
        assert torch.equal(t, o)
