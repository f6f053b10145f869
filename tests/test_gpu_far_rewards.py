"""Infinities far behind a step of a trajectory."""
import math

import pytest
import torch

from paper_2001_08743_amd import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


# by rows: a wave, several tiles, chunks; side by side: in one launch, in chunks, by 64
@pytest.mark.parametrize("B,S", [(3, 300), (600, 7000), (1, 60000), (20, 300), (20, 40001), (600, 3000)])
def test_an_infinite_reward_is_infinite_for_all_earlier_steps(B, S):
    """gamma lambda > 0 times an infinity is one, however many steps lie between, with episode ends to look for or without."""
    for place in (lambda t: t.to(DEV), lambda t: t.to(DEV).t().contiguous().t()):
        r, v = torch.zeros(B, S), torch.zeros(B, S)
        r[:, S - 2] = math.inf
        for dones in (None, torch.zeros(B, S, dtype=torch.uint8)):
            got = binding.cham_gae(place(r), place(v), 0.5, 0.5, dones=None if dones is None else place(dones))
            for k in ("advantages", "returns"):
                assert (got[k][:, :S - 1] == math.inf).all() and (got[k][:, S - 1] == 0).all(), k
