"""Several heads of up to 512 choices on both sides of where a wave takes a whole decision: decisions, heads and choices all count."""
import pytest
import torch

import explore_util as ref
from paper_2001_08743_amd import binding
from test_gpu_explore import DEV, TYPES, _check_loss, _check_policy, _gen, _loss_inputs, _policy_inputs, _run_loss

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("R,G,V", [(255, 2, 70), (256, 2, 70), (257, 7, 65), (300, 24, 130), (768, 24, 200), (1000, 64, 70), (1100, 100, 150), (1024, 64, 500), (520, 250, 40)])
def test_loss_and_logp_of_groups(R, G, V, dtype):
    x, a = _policy_inputs(R, G, V, dtype, R + G + V, masked=R % 2 == 0)
    weights = torch.rand(R, generator=_gen(7)) * (torch.rand(R, generator=_gen(8)) < 0.8)
    got, want = _run_loss(x, a, _loss_inputs(x, a, 0, R), weights=weights)
    _check_loss(got, want, G, V)
    lp, H, _ = ref.policy(x, a)
    _check_policy(binding.cham_policy_logp(x.to(DEV), a.to(DEV)), lp, H, G, V)
