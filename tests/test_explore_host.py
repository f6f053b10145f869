"""Refusals of the agent's update at the C entry points: nothing is launched, so no GPU is needed and device pointers are
placeholders that no host code looks behind."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

from paper_2001_08743_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
NULL, DIM, WORKSPACE, FLAG, TYPE, COEF = -1, -2, -6, -8, -11, -12
P = 1 << 20                          # a placeholder, aligned to everything
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    return binding.load()


def _logp(lib, logits=P, type=0, R=4, G=2, V=3, ld_r=6, ld_g=3, actions=P, action_type=16, first=-1, weights=None, logp=P, entropy=P, ws=0, ws_bytes=0):
    return lib.cham_policy_logp(logits, type, R, G, V, ld_r, ld_g, actions, action_type, first, weights, logp, entropy, ws, ws_bytes, None)


def test_codes_have_texts(lib):
    texts = {lib.cham_strerror(c) for c in range(-12, 0)}
    assert len(texts) == 12


@pytest.mark.parametrize("want,bad", [
    (DIM, dict(R=-1)), (DIM, dict(G=0)), (DIM, dict(G=65537)), (DIM, dict(V=0)), (DIM, dict(V=(1 << 24) + 1)), (DIM, dict(R=1 << 40, G=2)),
    (DIM, dict(ld_g=2)), (DIM, dict(ld_r=5)), (DIM, dict(ld_r=-6)), (DIM, dict(R=1 << 38, ld_r=1 << 39)), (DIM, dict(logits=P + 2)),
    (DIM, dict(type=1, logits=P + 1)), (DIM, dict(action_type=17, actions=P + 1)), (DIM, dict(action_type=18, actions=P + 4)),
    (DIM, dict(weights=P + 2)), (DIM, dict(logp=P + 2)), (DIM, dict(entropy=P + 1)),
    (TYPE, dict(type=3)), (TYPE, dict(type=-1)), (TYPE, dict(action_type=0)), (TYPE, dict(action_type=19)),
    (NULL, dict(logits=None)), (NULL, dict(actions=None)), (NULL, dict(logp=None)),
])
def test_logp_refuses(lib, want, bad):
    assert _logp(lib, **bad) == want


def test_logp_accepts_up_to_the_workspace(lib):
    # heads of a large vocabulary need a workspace: every check before it has passed
    assert _logp(lib, G=2, V=100000, ld_r=200000, ld_g=100000) == WORKSPACE
    assert _logp(lib, G=2, V=100000, ld_r=100000, ld_g=400000, entropy=None) == WORKSPACE          # heads first
    need = binding.cham_policy_workspace_bytes(4, 2, 100000, 0, False)
    assert _logp(lib, V=100000, ld_r=200000, ld_g=100000, ws=P, ws_bytes=need - 1) == WORKSPACE
    assert _logp(lib, V=100000, ld_r=200000, ld_g=100000, ws=P + 8, ws_bytes=need) == WORKSPACE
    assert _logp(lib, R=0, logits=None, actions=None, logp=None) == 0


def _loss(lib, coef=(), logits=P, type=0, R=4, G=2, V=3, ld_r=6, ld_g=3, actions=P, action_type=16, first=-1, weights=None, old=P, adv=P, ref=P,
          values=P, old_values=P, returns=P, terms=P, logp=P, entropy=P, grad=P + (1 << 16), gld_r=6, gld_g=3, grad_values=P, ws=0, ws_bytes=0,
          no_coef=False):
    c = binding._PolicyCoef(*{**dict(clip_low=0.2, clip_high=0.2, value=1.0, entropy=0.1, kl=0.1, value_clip=0.2), **dict(coef)}.values())
    return lib.cham_policy_loss(logits, type, R, G, V, ld_r, ld_g, actions, action_type, first, weights, old, adv, ref, values, old_values, returns,
                                None if no_coef else C.byref(c), terms, logp, entropy, grad, gld_r, gld_g, grad_values, ws, ws_bytes, None)


@pytest.mark.parametrize("want,bad", [
    (DIM, dict(R=-1)), (DIM, dict(V=0)), (TYPE, dict(type=9)), (TYPE, dict(action_type=2)),
    (NULL, dict(no_coef=True)), (NULL, dict(terms=None)), (NULL, dict(old=None)), (NULL, dict(adv=None)),
    (NULL, dict(ref=None)), (NULL, dict(values=None)), (NULL, dict(returns=None)), (NULL, dict(values=None, returns=None)),
    (NULL, dict(values=None, returns=None, coef=dict(value=0.0))),                                   # old values without values
    (COEF, dict(coef=dict(clip_low=-0.1))), (COEF, dict(coef=dict(clip_high=NAN))), (COEF, dict(coef=dict(kl=INF))),
    (COEF, dict(coef=dict(entropy=-1.0))), (COEF, dict(coef=dict(value=NAN))), (COEF, dict(coef=dict(value_clip=-1.0))),
    (DIM, dict(old=P + 1)), (DIM, dict(adv=P + 2)), (DIM, dict(ref=P + 2)), (DIM, dict(values=P + 2)), (DIM, dict(returns=P + 2)),
    (DIM, dict(terms=P + 2)), (DIM, dict(grad=P + (1 << 16) + 2)), (DIM, dict(gld_r=5)), (DIM, dict(gld_g=2)), (DIM, dict(grad_values=P + 1)),
    (DIM, dict(grad=P + 4)), (DIM, dict(grad=P + 4 * 23)), (DIM, dict(grad=P, gld_r=7)), (DIM, dict(logits=P + 4, grad=P)),   # overlap
])
def test_loss_refuses(lib, want, bad):
    assert _loss(lib, **bad) == want


def test_loss_accepts_up_to_the_workspace(lib):
    assert _loss(lib) == WORKSPACE
    assert _loss(lib, grad=P) == WORKSPACE                                     # in place
    assert _loss(lib, grad=P + 4 * 24) == WORKSPACE                            # right behind
    assert _loss(lib, grad=None, grad_values=None, logp=None, entropy=None) == WORKSPACE
    assert _loss(lib, coef=dict(kl=0.0, value=0.0, value_clip=NAN), ref=None, values=None, old_values=None, returns=None) == WORKSPACE


def _gae(lib, type=0, B=4, S=10, r=P, r_ld=(10, 1), v=P, v_ld=(10, 1), d=P, d_ld=(10, 1), boot=P, lengths=P, gamma=0.9, lam=0.99, adv=P, ret=P,
         o_ld=(10, 1), ws=0, ws_bytes=0):
    return lib.cham_gae(type, B, S, r, *r_ld, v, *v_ld, d, *d_ld, boot, lengths, gamma, lam, adv, ret, *o_ld, ws, ws_bytes, None)


@pytest.mark.parametrize("want,bad", [
    (TYPE, dict(type=16)), (DIM, dict(B=-1)), (DIM, dict(S=-1)), (DIM, dict(S=1 << 31)), (DIM, dict(B=1 << 30, S=1 << 20)),
    (COEF, dict(gamma=1.1)), (COEF, dict(gamma=NAN)), (COEF, dict(lam=-0.1)), (COEF, dict(lam=NAN)),
    (NULL, dict(r=None)), (NULL, dict(v=None)), (NULL, dict(adv=None)),
    (DIM, dict(r_ld=(-10, 1))), (DIM, dict(v_ld=(10, -1))), (DIM, dict(d_ld=(10, 1 << 41))), (DIM, dict(B=1 << 30, S=16, r_ld=(1 << 40, 1))),
    (DIM, dict(o_ld=(9, 1))), (DIM, dict(o_ld=(0, 1))), (DIM, dict(o_ld=(1, 3))),
    (DIM, dict(r=P + 2)), (DIM, dict(type=1, v=P + 1)), (DIM, dict(boot=P + 2)), (DIM, dict(lengths=P + 2)), (DIM, dict(adv=P + 2)), (DIM, dict(ret=P + 1)),
    (WORKSPACE, dict(B=1, S=1 << 20, r_ld=(0, 1), v_ld=(0, 1), d_ld=(0, 1), o_ld=(0, 1))),
])
def test_gae_refuses(lib, want, bad):
    assert _gae(lib, **bad) == want


def test_gae_of_nothing_is_no_error(lib):
    assert _gae(lib, B=0, r=None, v=None, adv=None) == 0
    assert _gae(lib, S=0, r=None, v=None, adv=None) == 0
    assert binding.cham_gae_workspace_bytes(0, 5) == 0


def _clip(lib, ptrs=(P, P), outs=None, numels=(5, 6), types=(0, 1), n=2, max_norm=1.0, norm=P, ws=0, ws_bytes=0, flags=0, fn="clip"):
    a = (C.c_void_p * 2)(*ptrs) if ptrs is not None else None
    o = (C.c_void_p * 2)(*outs) if outs is not None else None
    m = (C.c_int64 * 2)(*numels) if numels is not None else None
    t = (C.c_int32 * 2)(*types) if types is not None else None
    if fn == "norm":
        return lib.cham_grad_norm(a, m, t, n, norm, ws, ws_bytes, None)
    return lib.cham_clip_grads(a, o, m, t, n, max_norm, norm, ws, ws_bytes, flags, None)


@pytest.mark.parametrize("fn", ["norm", "clip"])
@pytest.mark.parametrize("want,bad", [
    (DIM, dict(n=-1)), (NULL, dict(numels=None)), (NULL, dict(types=None)), (TYPE, dict(types=(0, 16))), (DIM, dict(numels=(5, -1))),
    (DIM, dict(numels=(1 << 40, 1))), (NULL, dict(norm=None)), (DIM, dict(norm=P + 4)), (NULL, dict(ptrs=None)), (NULL, dict(ptrs=(P, None))),
    (DIM, dict(ptrs=(P + 2, P))), (DIM, dict(ptrs=(P, P + 1))), (WORKSPACE, dict()), (WORKSPACE, dict(ws=P, ws_bytes=8)),
])
def test_norm_and_clip_refuse(lib, fn, want, bad):
    assert _clip(lib, fn=fn, **bad) == want


@pytest.mark.parametrize("want,bad", [
    (FLAG, dict(flags=1)), (FLAG, dict(flags=33)), (COEF, dict(max_norm=-1.0)), (COEF, dict(max_norm=NAN)), (NULL, dict(outs=(P, None))),
    (DIM, dict(outs=(P + 2, P))), (WORKSPACE, dict(outs=(P, P))),
])
def test_clip_refuses(lib, want, bad):
    assert _clip(lib, **bad) == want


@pytest.mark.skipif(shutil.which("hipcc") is None and not os.path.exists("/opt/rocm/bin/hipcc"), reason="no hipcc")
def test_host_code_under_address_and_ub_sanitizers(tmp_path):
    from paper_2001_08743_amd import build as libbuild
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all"]
    so = libbuild.build_host_sanitized(str(tmp_path))
    exe = str(tmp_path / "explore_host_check")
    subprocess.run(["/opt/rocm/lib/llvm/bin/clang", "-O1", "-g", *san, "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "paper_2001_08743_amd", "csrc", "explore_host_check.c"), so,
                    "-Wl,-rpath," + os.path.dirname(so), "-Wl,-rpath,/opt/rocm/lib", "-o", exe], check=True)
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0", UBSAN_OPTIONS="print_stacktrace=1")   # the HIP runtime keeps its allocations until exit
    r = subprocess.run([exe], env=env, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-4000:])
    assert "explore_host_check ok" in r.stdout
