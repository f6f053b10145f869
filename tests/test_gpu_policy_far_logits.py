"""Policy operators on logits far from 0: a softmax does not change when all logits of a head move together, and no bound of the
oracle depends on where they stand.  One shape for each kernel and way to join its sums."""
import math

import pytest
import torch

import explore_util as ref
from paper_2001_08743_amd import binding
from test_gpu_explore import COEF, DEV, _check_loss, _check_policy, _gen, _loss_inputs, _policy_inputs, _run_loss

pytestmark = pytest.mark.gpu

# lanes (four heads, one head), tiles, rows by a wave, 256, 512 and 1024 threads, groups of lanes, parts by a wave and by a workgroup, joined by
# themselves or beside the gradient
SHAPES = [(37, 24, 3), (33, 12, 24), (9, 1, 30), (3, 200, 7), (300, 1, 700), (600, 1, 2049), (40, 1, 16000), (270, 1, 70001), (1025, 3, 300),
          (3, 2, 1000), (2, 2, 9000), (5, 1, 50021), (40, 1, 70001)]
# an offset that the type's items have room beside
OFFSETS = [(torch.float32, 100.0), (torch.float32, -1e4), (torch.float32, 1e4), (torch.float32, 1e6), (torch.bfloat16, 100.0), (torch.bfloat16, -1e4),
           (torch.float16, -100.0), (torch.float16, 1e4)]


def _check_both(x, a, seed, G, V, **kw):
    got, want = _run_loss(x, a, _loss_inputs(x, a, 0, seed), **kw)
    _check_loss(got, want, G, V)
    lp, H, _ = ref.policy(x, a)
    _check_policy(binding.cham_policy_logp(x.to(DEV), a.to(DEV)), lp, H, G, V)


@pytest.mark.parametrize("dtype,offset", OFFSETS, ids=lambda v: str(v)[6:] if isinstance(v, torch.dtype) else f"{v:g}")
@pytest.mark.parametrize("R,G,V", SHAPES)
def test_heads_moved_together(R, G, V, dtype, offset):
    x, a = _policy_inputs(R, G, V, torch.float32, R + V, masked=R % 2 == 0)
    # heads by different amounts, so that none is another's
    x = (x + offset * (1 + 0.25 * (torch.arange(G) % 8))[:, None]).to(dtype)
    _check_both(x, a, R, G, V)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16], ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("R,G,V", SHAPES)
def test_uniform_heads_anywhere(R, G, V, dtype):
    """A head that is filled with a finite mask is uniform; log-probabilities and entropy are those of any other uniform head."""
    x, a = _policy_inputs(R, G, V, torch.float32, R + V)
    at = [-65504.0, 65504.0, 1e4] if dtype == torch.float16 else [-1e9, -1e30, 1e30, -1e12, 1e7, 3e38, -3e38, 1e10, torch.finfo(dtype).min, torch.finfo(dtype).max]
    for i in range(R * G):
        if i % 3 == 0 or R * G < 10:
            x[i // G, i % G] = at[i // (1 if R * G < 10 else 3) % len(at)]
    _check_both(x.to(dtype), a, R, G, V)


@pytest.mark.parametrize("mask", [-1e9, -1e30])
@pytest.mark.parametrize("R,G,V", SHAPES)
def test_choices_masked_by_a_finite_value(R, G, V, mask):
    x, a = _policy_inputs(R, G, V, torch.float32, R + V, masked=True)
    x = torch.where(x == -math.inf, torch.full_like(x, mask), x + 300.0)
    _check_both(x, a, R, G, V, entropy_coef=0.0 if V % 2 else 0.1)


@pytest.mark.parametrize("R,G,V", SHAPES)
def test_probabilities_of_a_gradient_add_up(R, G, V):
    """sum over a head of dL/dx = D - D sum p is 0; here D = -A exactly (a ratio of 1), and the sum of V items each off by its bound."""
    x, a = _policy_inputs(R, G, V, torch.float32, R + V)
    x += 1e5
    old = binding.cham_policy_logp(x.to(DEV), a.to(DEV))["logp"].cpu()
    got, want = _run_loss(x, a, dict(old=old, adv=torch.randn(R, generator=_gen(R))), use=(), value_coef=0.0, kl_coef=0.0, entropy_coef=0.0)
    off = got["grad_logits"].cpu().double().sum(-1).abs()
    assert off.le(want["tol"].sum(-1)).all(), float((off / want["tol"].sum(-1)).max())
