"""Lists of tensors that share memory are refused."""
import pytest
import torch

from paper_2001_08743_amd import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", [torch.float32, torch.bfloat16])
def test_tensors_that_share_memory(kind):
    flat = torch.zeros(100, dtype=kind, device="cuda:0")
    for bad in ([flat[:60], flat[59:]], [flat[50:], flat[:51]], [flat, flat[99:]], [flat[10:20], flat], [flat[:7], torch.zeros(3, device="cuda:0"), flat[:7]]):
        with pytest.raises(binding.ChamError):
            binding.GradList(bad)
    # side by side in one buffer, empty ones in between
    both = binding.GradList([flat[60:], flat[30:30], flat[:60], flat[60:60]])
    flat += 1
    assert float(binding.cham_grad_norm(both)["norm"]) == 10.0
