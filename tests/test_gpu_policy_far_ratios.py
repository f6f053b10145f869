"""Ratios and divergences beyond fp32's range: a decision's differences, ratio, divergence and products have the range of a double."""
import pytest
import torch

from test_gpu_explore import _check_loss, _loss_inputs, _policy_inputs, _run_loss

pytestmark = pytest.mark.gpu

# every kernel that takes decisions: lanes, tiles, rows, groups, joins by themselves and beside the gradient
SHAPES = [(37, 24, 3), (33, 12, 24), (3, 200, 7), (300, 1, 700), (270, 1, 70001), (1025, 3, 300), (3, 2, 1000), (2, 2, 9000), (5, 1, 50021), (40, 1, 70001)]


@pytest.mark.parametrize("R,G,V", SHAPES)
def test_ratio_beyond_fp32(R, G, V):
    x, a = _policy_inputs(R, G, V, torch.float32, R + V)
    b = _loss_inputs(x, a, 0, R)
    far = torch.arange(R) % 2 == 0
    b["old"] = torch.where(far, b["old"] - 100.0, b["old"])         # e^100
    b["adv"][0] = 0.0                                               # 0 times it is 0
    got, want = _run_loss(x, a, b, weights=torch.full((R,), 1e-20), use=("values", "old_values"), kl_coef=0.0)
    assert torch.isfinite(want["terms"]).all()
    _check_loss(got, want, G, V)


@pytest.mark.parametrize("R,G,V", SHAPES)
def test_divergence_beyond_fp32(R, G, V):
    x, a = _policy_inputs(R, G, V, torch.float32, R + V)
    b = _loss_inputs(x, a, 0, R)
    b["ref"] = torch.where(torch.arange(R) % 2 == 0, b["ref"] + 100.0, b["ref"])
    got, want = _run_loss(x, a, b, weights=torch.full((R,), 1e-20))
    assert torch.isfinite(want["terms"]).all()
    _check_loss(got, want, G, V)


@pytest.mark.parametrize("R,G,V", SHAPES)
def test_ratio_and_divergence_that_are_infinite_or_nothing(R, G, V):
    x, a = _policy_inputs(R, G, V, torch.float32, R + V)
    b = _loss_inputs(x, a, 0, R)
    kw = dict(use=("ref",), value_coef=0.0, want_grad=False)
    clean, _ = _run_loss(x, a, b, **kw)
    b["adv"] = b["adv"].abs() + 0.5
    for old, ratio in ((-2000.0, float("inf")), (2000.0, 0.0)):
        b["old"][:] = old
        got, _ = _run_loss(x, a, b, kl_coef=0.0, **kw)
        # positive advantages: the ratio counts up to 1.3
        mean = float((b["adv"].double() * min(ratio, 1.3)).mean())
        assert abs(float(got["terms"][1]) + mean) <= 4e-7 * abs(mean)
    b["ref"][0] = float("inf")
    got, _ = _run_loss(x, a, b, **kw)
    assert got["terms"][4] == float("inf")
    b["ref"][0] = float("-inf")                                     # e^-inf + inf - 1
    got, _ = _run_loss(x, a, b, **kw)
    assert got["terms"][4] == float("inf")
    b["ref"][0] = float("nan")
    got, _ = _run_loss(x, a, b, **kw)
    assert torch.isnan(got["terms"][4]) and torch.equal(got["logp"], clean["logp"])
