"""Calls of the agent's update whose outputs or workspace share memory with another argument are refused at the C entry points, before
anything is launched; addresses are placeholders."""
import ctypes as C

import pytest

from paper_2001_08743_amd import binding

DIM = -2
A = 1 << 24                          # arguments this far apart
ROWS = ["weights", "old", "adv", "ref", "values", "old_values", "returns"]
OUTS = ["terms", "logp", "entropy", "grad_values", "ws"]
R, G, V = 64, 3, 5


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def _loss(lib, **at):
    names = ["logits", "actions", *ROWS, *OUTS, "grad"]
    p = {n: A * (i + 1) for i, n in enumerate(names)}
    p.update(at)
    coef = binding._PolicyCoef(0.2, 0.2, 0.5, 0.1, 0.1, 0.2)
    need = binding.cham_policy_workspace_bytes(R, G, V, 0, True)
    return lib.cham_policy_loss(p["logits"], 0, R, G, V, G * V, V, p["actions"], 16, 0, *(p[n] for n in ROWS), C.byref(coef), p["terms"], p["logp"], p["entropy"],
                                p["grad"], G * V, V, p["grad_values"], p["ws"], need, None)


@pytest.mark.parametrize("out", OUTS + ["grad"])
@pytest.mark.parametrize("other", ROWS + OUTS + ["actions", "logits", "grad"])
def test_loss(lib, out, other):
    if out == other or (out, other) == ("grad", "logits"):
        return                                            # a gradient may be the logits themselves
    at = A * 40
    assert _loss(lib, **{out: at, other: at}) == DIM
    size = {"terms": 24, "actions": R * G, "logits": 4 * R * G * V, "grad": 4 * R * G * V, "ws": 256}.get(other, 4 * R)
    assert _loss(lib, **{out: at + (size - 8) // 256 * 256, other: at}) == DIM          # behind its beginning


@pytest.mark.parametrize("out", ["logp", "entropy", "ws"])
@pytest.mark.parametrize("other", ["logits", "actions", "weights", "logp", "entropy", "ws"])
def test_logp(lib, out, other):
    if out == other:
        return
    p = {n: A * (i + 1) for i, n in enumerate(["logits", "actions", "weights", "logp", "entropy", "ws"])}
    p[out] = p[other]
    need = binding.cham_policy_workspace_bytes(R, G, V, 0, False)
    assert lib.cham_policy_logp(p["logits"], 0, R, G, V, G * V, V, p["actions"], 16, 0, p["weights"], p["logp"], p["entropy"], p["ws"], need, None) == DIM


@pytest.mark.parametrize("strides", [(5000, 1), (1, 3), (10000, 2)])
@pytest.mark.parametrize("out", ["adv", "ret", "ws"])
@pytest.mark.parametrize("other", ["rewards", "values", "dones", "bootstrap", "lengths", "adv", "ret", "ws"])
def test_gae(lib, out, other, strides):
    B, S = 3, 5000
    if out == other:
        return
    p = {n: A * (i + 1) for i, n in enumerate(["rewards", "values", "dones", "bootstrap", "lengths", "adv", "ret", "ws"])}
    need = binding.cham_gae_workspace_bytes(B, S)
    assert need > 0
    call = lambda: lib.cham_gae(0, B, S, p["rewards"], *strides, p["values"], *strides, p["dones"], *strides, p["bootstrap"], p["lengths"], 0.9, 0.9, p["adv"],
                                p["ret"], *strides, p["ws"], need, None)
    p[out] = p[other]
    assert call() == DIM
    if strides[1] != 2 and other not in ("bootstrap", "lengths", "ws"):
        p[out] = p[other] + 256                           # behind its beginning: arrays without gaps
        assert call() == DIM


def test_gae_without_dones_does_not_look_at_their_strides(lib):
    far = (1 << 63) - 1
    assert lib.cham_gae(0, 3, 4, A, 4, 1, 2 * A, 4, 1, None, far, far, None, None, 0.9, 0.9, 3 * A, 3 * A, 4, 1, None, 0, None) == DIM
