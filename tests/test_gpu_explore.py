"""The agent's update on the GPU against its definitions in 64 bits."""
import math

import pytest
import torch

import explore_util as ref
from paper_2001_08743_amd import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]


def _gen(seed):
    return torch.Generator().manual_seed(seed)


def _policy_inputs(R, G, V, dtype, seed, masked=False, first=0, adtype=torch.int64, head_axis=True):
    """Logits below 40 from a head's maximum, actions among the choices that are not masked; on the CPU."""
    g = _gen(seed)
    x = (3.0 * torch.randn(R, G, V, generator=g)).clamp(-15, 15)
    if masked:
        keep = torch.rand(R, G, V, generator=g) < 0.6
        keep[..., 0] |= ~keep.any(-1)
        x = x.masked_fill(~keep, -math.inf)
    score = torch.where(x == -math.inf, torch.full_like(x, -1.0), torch.rand(R, G, V, generator=g))
    a = score.argmax(-1)
    x = x.to(dtype)
    if not head_axis:
        x, a = x[:, 0], a[:, 0]
    return x, (a + first).to(adtype)


def _loss_inputs(x, a, first, seed, weights=None):
    """What a loss compares with: ratios away from the border of the clip, values in steps of 1/16 (comparisons exact)."""
    g = _gen(seed + 1)
    lp, _, _ = ref.policy(x, a, first)
    R = x.shape[0]
    lp = torch.where(torch.isfinite(lp), lp, torch.zeros(()).double())
    moved = torch.tensor([-0.7, -0.15, -0.02, 0.0, 0.05, 0.12, 0.5])[torch.randint(0, 7, (R,), generator=g)]
    v = torch.randint(-32, 32, (R,), generator=g) / 16
    o = v + torch.randint(-8, 9, (R,), generator=g) / 16
    t = v + torch.randint(-16, 17, (R,), generator=g) / 16
    return dict(old=(lp - moved).float(), adv=torch.randn(R, generator=g), ref=(lp + 0.3 * torch.randn(R, generator=g)).float(), values=v.float(),
                old_values=o.float(), returns=t.float())


COEF = dict(clip_low=0.2, clip_high=0.3, value_coef=0.5, entropy_coef=0.1, kl_coef=0.2, value_clip=0.25)


def _run_loss(x, a, b, first=0, weights=None, out=None, use=("ref", "values", "old_values"), **kw):
    coef = {**COEF, **kw}
    d = {k: v.to(DEV) for k, v in b.items()}
    got = binding.cham_policy_loss(x.to(DEV) if not x.is_cuda else x, a.to(DEV), d["old"], d["adv"], first_action=first,
                                   ref_logp=d["ref"] if "ref" in use else None, weights=None if weights is None else weights.to(DEV),
                                   values=d["values"] if "values" in use else None, old_values=d["old_values"] if "old_values" in use else None,
                                   returns=d["returns"] if "values" in use else None, out=out, **coef)
    want = ref.loss(x, a, b["old"], b["adv"], first, b["ref"] if "ref" in use else None, weights, b["values"] if "values" in use else None,
                    b["old_values"] if "old_values" in use else None, b["returns"] if "values" in use else None,
                    **{k: v for k, v in coef.items() if k != "want_grad"})
    return got, want


def _check_policy(got, lp, H, G, V):
    lp, H = lp.double(), H.double()
    assert (got["logp"].cpu().double() - lp).abs().le(ref.logp_error(V, G) + 2 * ref.U * lp.abs()).all()
    assert (got["entropy"].cpu().double() - H).abs().le(ref.entropy_error(V, G) + 2 * ref.U * H.abs()).all()


def _check_loss(got, want, G, V):
    _check_policy(got, want["logp"], want["entropy"], G, V)
    off = (got["terms"].cpu().double() - want["terms"]).abs()
    assert off.le(want["terms_tol"]).all(), (off, want["terms_tol"])
    grad = got["grad_logits"].cpu().double()
    bad = (grad - want["grad_logits"]).abs() > want["tol"]
    assert not bad.any(), (int(bad.sum()), ((grad - want["grad_logits"]).abs() / want["tol"]).max())
    if want["grad_values"] is not None:
        assert torch.equal(got["grad_values"].cpu(), want["grad_values"].float())


SHAPES = [(1, 1, 1), (1, 1, 2), (5, 3, 3), (130, 24, 3), (1037, 5, 3), (7, 64, 2), (33, 12, 24), (3, 200, 7), (2, 300, 3), (2, 1100, 4), (2, 1025, 9), (50, 7, 40), (4, 64, 64), (9, 5, 70), (6, 90, 130), (3, 1, 255), (4, 1, 256), (2, 1, 257),
          (17, 1, 1000), (300, 1, 33), (2, 3, 5000), (70, 2, 300), (3, 1, 4097), (5, 1, 8191), (600, 1, 2049), (2, 1, 50021), (1, 1, 131072),
          (3, 1, 140001), (1, 2, 270000), (600, 1, 33000), (270, 1, 70001), (260, 1, 140003), (1024, 2, 512), (1025, 3, 511), (4099, 2, 65), (1100, 7, 130), (1024, 2, 513), (1024, 256, 66)]


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("R,G,V", SHAPES)
def test_loss_and_logp_over_sizes(R, G, V, dtype):
    first, adtype = (-1, torch.int8) if V <= 100 else (0, torch.int64 if V % 2 else torch.int32)
    x, a = _policy_inputs(R, G, V, dtype, R + G + V, masked=V > 2 and (R + V) % 2 == 0, first=first, adtype=adtype, head_axis=G > 1 or R % 2 == 0)
    b = _loss_inputs(x, a, first, R)
    weights = None
    if R > 2:
        weights = torch.rand(R, generator=_gen(7)) * (torch.rand(R, generator=_gen(8)) < 0.8)
    got, want = _run_loss(x, a, b, first, weights)
    _check_loss(got, want, G, V)
    lp, H, _ = ref.policy(x, a, first)
    _check_policy(binding.cham_policy_logp(x.to(DEV), a.to(DEV), first_action=first), lp, H, G, V)


@pytest.mark.parametrize("entropy_coef", [0.0, 0.1])
@pytest.mark.parametrize("use", [(), ("ref",), ("values",), ("values", "old_values")], ids="-".join)
@pytest.mark.parametrize("R,G,V", [(37, 6, 3), (20, 1, 600), (3, 1, 40000)])
def test_loss_with_and_without_its_terms(R, G, V, use, entropy_coef):
    x, a = _policy_inputs(R, G, V, torch.float32, 3)
    b = _loss_inputs(x, a, 0, 5)
    got, want = _run_loss(x, a, b, use=use, entropy_coef=entropy_coef, kl_coef=0.2 if "ref" in use else 0.0, value_coef=0.5 if "values" in use else 0.0)
    _check_loss(got, want, G, V)
    assert (got["grad_values"] is None) == ("values" not in use)
    # forward only: the same terms
    only, _ = _run_loss(x, a, b, use=use, entropy_coef=entropy_coef, kl_coef=0.2 if "ref" in use else 0.0, value_coef=0.5 if "values" in use else 0.0,
                        want_grad=False)
    assert only["grad_logits"] is None and torch.equal(only["terms"], got["terms"]) and torch.equal(only["logp"], got["logp"])


@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("R,G,V", [(40, 4, 3), (21, 3, 50), (13, 1, 901), (3, 2, 4100), (4, 1, 20003), (1027, 3, 70), (5, 1, 70001), (20, 1, 70001)])
def test_strides_and_memory_between(R, G, V, dtype):
    x, a = _policy_inputs(R, G, V, dtype, 11, masked=V > 3)
    b = _loss_inputs(x, a, 0, 12)
    _, want = _run_loss(x, a, b)
    for order in ("rows", "heads"):
        shape = (R, G, V + 5) if order == "rows" else (G, R, V + 5)
        wide, to = (torch.full(shape, 7.0, dtype=dtype, device=DEV) for _ in range(2))
        view = wide[:, :, 3:3 + V] if order == "rows" else wide[:, :, 3:3 + V].transpose(0, 1)
        to_view = to[:, :, 1:1 + V] if order == "rows" else to[:, :, 1:1 + V].transpose(0, 1)
        view.copy_(x)
        out = dict(terms=torch.empty(6, device=DEV), logp=torch.empty(R, device=DEV), entropy=torch.empty(R, device=DEV), grad_logits=to_view,
                   grad_values=torch.empty(R, device=DEV))
        got, _ = _run_loss(view, a, b, out=out)
        _check_loss(got, want, G, V)
        assert (to[..., 0] == 7).all() and (to[..., 1 + V:] == 7).all()
        # in place
        out["grad_logits"] = view
        again, _ = _run_loss(view, a, b, out=out)
        assert torch.equal(again["grad_logits"], got["grad_logits"])
        assert (wide[..., :3] == 7).all() and (wide[..., 3 + V:] == 7).all()


@pytest.mark.parametrize("R,G,V", [(12, 5, 3), (12, 4, 90), (6, 1, 700), (6, 1, 40001), (6, 2, 9000), (1026, 5, 90)])
def test_left_out_heads_and_decisions(R, G, V):
    x, a = _policy_inputs(R, G, V, torch.float32, 21)
    w = torch.full((R,), 0.25)
    b = _loss_inputs(x, a, 0, 22)
    w[1] = 0.0                                            # a padded decision: nothing of it is read
    x[1] = math.nan
    for k in b:
        b[k][1] = math.nan
    a[1] = 1 << 40
    x[2] = -math.inf                                      # every choice of every head masked
    a[3] = -5                                             # no head of it counts
    x[3, 0, 0] = math.nan
    if G > 1:
        x[4, 1] = -math.inf                               # one head without a choice
        a[5, 0] = -1                                      # a knob that this decision does not have
    x[0, 0, 1:] = torch.finfo(torch.float32).min          # masked by the lowest value: one choice left
    a[0, 0] = 0
    got, want = _run_loss(x, a, b, weights=w)
    for r in (1, 2, 3):
        assert not want["on"][r]
        assert not got["grad_logits"][r].any() and got["grad_values"][r] == 0 and got["logp"][r] == 0 and got["entropy"][r] == 0
    _check_loss(got, want, G, V)
    logp = binding.cham_policy_logp(x.to(DEV), a.to(DEV), weights=w.to(DEV))
    _check_policy(logp, want["logp"], want["entropy"], G, V)
    # a head where all choices have the lowest value is uniform
    x[4, 0] = torch.finfo(torch.float32).min
    got = binding.cham_policy_logp(x[4:5].to(DEV), a[4:5].to(DEV))
    lp, H, _ = ref.policy(x[4:5], a[4:5])
    _check_policy(got, lp, H, G, V)


@pytest.mark.parametrize("R,G,V", [(50, 5, 3), (50, 1, 700), (5, 1, 40001), (5, 2, 9000), (1026, 5, 90)])
def test_weights_of_either_sign(R, G, V):
    x, a = _policy_inputs(R, G, V, torch.float32, 23)
    w = torch.randn(R, generator=_gen(24))
    got, want = _run_loss(x, a, _loss_inputs(x, a, 0, 25), weights=w)
    _check_loss(got, want, G, V)


@pytest.mark.parametrize("R,G,V", [(9, 5, 3), (9, 1, 700), (5, 1, 40001), (5, 2, 9000), (1026, 5, 90)])
def test_what_is_no_number_stays_in_its_decision(R, G, V):
    x, a = _policy_inputs(R, G, V, torch.float32, 31)
    b = _loss_inputs(x, a, 0, 32)
    clean, _ = _run_loss(x, a, b)
    y, c = x.clone(), a.clone()
    y[0, 0, V - 1] = math.nan
    y[1, G - 1, 0] = math.inf
    c[2, 0] = V                                           # outside the choices
    got, _ = _run_loss(y, c, b)
    for r in range(3):
        assert torch.isnan(got["logp"][r]) and torch.isnan(got["entropy"][r])
    assert torch.isnan(got["grad_logits"][0, 0]).all() and torch.isnan(got["grad_logits"][2, 0]).all()
    assert torch.isnan(got["terms"][0])
    assert torch.equal(got["logp"][3:], clean["logp"][3:]) and torch.equal(got["grad_logits"][3:], clean["grad_logits"][3:])


def test_terms_with_coefficient_zero_add_nothing_whatever_they_are():
    x, a = _policy_inputs(4, 2, 3, torch.float32, 41)
    b = _loss_inputs(x, a, 0, 42)
    b["ref"][:] = math.inf                                # the divergence is infinite
    got, _ = _run_loss(x, a, b, kl_coef=0.0)
    assert torch.isfinite(got["terms"][0]) and torch.isinf(got["terms"][4]) and torch.isfinite(got["grad_logits"]).all()


@pytest.mark.parametrize("R,G,V", [(4, 3, 3), (3, 1, 40)])
def test_gradient_against_differences(R, G, V):
    x, a = _policy_inputs(R, G, V, torch.float32, 51)
    b = _loss_inputs(x, a, 0, 52)
    got, want = _run_loss(x, a, b)
    h = 1e-5
    kw = {**COEF, "ref": b["ref"], "old_values": b["old_values"], "returns": b["returns"], "values": b["values"]}
    for i in range(0, x.numel(), 5):
        e = torch.zeros(x.numel(), dtype=torch.float64)
        e[i] = h
        e = e.reshape(x.shape)
        # third derivatives are below 100 here: h^2 / 6 of them, and the loss's rounding over h
        up, down = (ref.loss(_Exact(x.double() + s * e), a, b["old"], b["adv"], 0, **kw)["terms"][0] for s in (1, -1))
        slope = (up - down) / (2 * h)
        assert abs(float(got["grad_logits"].reshape(-1)[i]) - float(slope)) <= float(want["tol"].reshape(-1)[i]) + 100 * h * h / 6 + 2e-15 * 20 / h


class _Exact:
    """Logits in 64 bits with the interface of fp32 ones."""

    def __init__(self, x):
        self.x, self.dtype, self.shape = x, torch.float32, x.shape

    def double(self):
        return self.x


def test_no_decisions():
    z = torch.zeros(0, device=DEV)
    got = binding.cham_policy_loss(torch.zeros(0, 3, device=DEV), torch.zeros(0, dtype=torch.int64, device=DEV), z, z)
    assert got["terms"].tolist() == [0.0] * 6
    assert binding.cham_policy_logp(torch.zeros(0, 2, 3, device=DEV), torch.zeros(0, 2, dtype=torch.int64, device=DEV))["logp"].shape == (0,)


def test_rows_beyond_32_bit_offsets():
    # two decisions 2^32 items apart
    ld = (1 << 32) + 6
    flat = torch.zeros(ld + 4, dtype=torch.bfloat16, device=DEV)
    x, a = _policy_inputs(2, 1, 3, torch.bfloat16, 61, head_axis=False)
    view = flat.as_strided((2, 3), (ld, 1))
    view.copy_(x)
    b = _loss_inputs(x, a, 0, 62)
    out = dict(terms=torch.empty(6, device=DEV), logp=torch.empty(2, device=DEV), entropy=torch.empty(2, device=DEV), grad_logits=view,
               grad_values=torch.empty(2, device=DEV))
    got = binding.cham_policy_loss(view, a.to(DEV), b["old"].to(DEV), b["adv"].to(DEV), out=out, entropy_coef=0.1)
    want = ref.loss(x, a, b["old"], b["adv"], entropy_coef=0.1)
    bad = (got["grad_logits"].cpu().double() - want["grad_logits"]).abs() > want["tol"]
    assert not bad.any()


@pytest.mark.parametrize("R,G,V", [(500, 24, 3), (300, 1, 4000), (3, 1, 60001), (4200, 5, 100)])
def test_loss_is_the_same_run_to_run_and_on_another_stream(R, G, V):
    x, a = _policy_inputs(R, G, V, torch.float32, 71)
    b = _loss_inputs(x, a, 0, 72)
    one, _ = _run_loss(x, a, b)
    xd = x.to(DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        two, _ = _run_loss(xd, a, b)
    side.synchronize()
    for k in ("terms", "logp", "entropy", "grad_logits", "grad_values"):
        assert torch.equal(one[k], two[k]), k


def test_binding_refuses():
    x = torch.zeros(4, 3, device=DEV)
    a = torch.zeros(4, dtype=torch.int64, device=DEV)
    z = torch.zeros(4, device=DEV)
    bad = [lambda: binding.cham_policy_logp(x.double(), a), lambda: binding.cham_policy_logp(x, a.to(torch.int16)), lambda: binding.cham_policy_logp(x, a[:3]),
           lambda: binding.cham_policy_logp(x.t(), a[:3]), lambda: binding.cham_policy_logp(x.cpu(), a), lambda: binding.cham_policy_logp(x, a.cpu()),
           lambda: binding.cham_policy_logp(x, a, weights=z.double()), lambda: binding.cham_policy_loss(x, a, z[:3], z), lambda: binding.cham_policy_loss(x, a, z, z, kl_coef=0.1),
           lambda: binding.cham_policy_loss(x, a, z, z, value_coef=0.1), lambda: binding.cham_policy_loss(x, a, z, z, clip_low=-1.0),
           lambda: binding.cham_policy_loss(x.expand(4, 3)[:1].expand(4, 3), a, z, z),
           lambda: binding.cham_gae(x, x.bfloat16(), 0.9, 0.9), lambda: binding.cham_gae(x, x, 1.9, 0.9), lambda: binding.cham_gae(x, x, 0.9, 0.9, lengths=a),
           lambda: binding.cham_gae(x, x[:, :2], 0.9, 0.9), lambda: binding.cham_clip_grads([x.t()], 1.0), lambda: binding.cham_clip_grads([x, x.cpu()], 1.0),
           lambda: binding.cham_clip_grads([x], -1.0), lambda: binding.cham_clip_grads([x, z, x], 1.0), lambda: binding.cham_clip_grads([x], 1.0, out=[x, x]), lambda: binding.cham_clip_grads([x], 1.0, out=[x.half()]),
           lambda: binding.cham_clip_grads([x], 1.0, norm_given=True), lambda: binding.cham_grad_norm([a])]
    for f in bad:
        with pytest.raises(binding.ChamError):
            f()


# --- advantages

GAE_SHAPES = [(1, 1), (3, 2), (128, 500), (1, 2047), (2, 2048), (5, 2049), (70, 64), (130, 33), (300, 7), (1000, 1), (3, 20000), (1, 70001), (17, 9000), (2, 300), (512, 256), (513, 257), (777, 321), (530, 2100)]


def _gae_inputs(B, S, dtype, seed):
    g = _gen(seed)
    return dict(rewards=torch.randn(B, S, generator=g).to(dtype), values=torch.randn(B, S, generator=g).to(dtype), dones=(torch.rand(B, S, generator=g) < 0.05).to(torch.uint8),
                bootstrap=torch.randn(B, generator=g), lengths=torch.randint(0, S + 1, (B,), generator=g, dtype=torch.int32))


def _check_gae(got, want, there, before=0.0):
    for k, w in zip(("advantages", "returns"), want):
        x = got[k].cpu()
        # in double over the whole trajectory, rounded once
        assert (x.double() - w)[there].abs().le(ref.U * w[there].abs() * (1 + 1e-6) + 1e-9).all(), k
        assert (x[~there] == before).all(), k


@pytest.mark.parametrize("layout", ["by_row", "by_step", "odd"])
@pytest.mark.parametrize("dtype", TYPES, ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("B,S", GAE_SHAPES)
def test_gae_over_sizes_and_layouts(B, S, dtype, layout):
    i = _gae_inputs(B, S, dtype, B + S)
    lam = 1.0 if S % 2 else 0.97
    adv, ret, there = ref.gae(i["rewards"], i["values"], 0.99, lam, i["dones"], i["bootstrap"], i["lengths"])

    def place(t, fill):
        if layout == "by_row":
            return t.to(DEV)
        if layout == "by_step":
            return t.to(DEV).t().contiguous().t()
        wide = torch.full((B, 2 * S + 3), fill, dtype=t.dtype, device=DEV)
        view = wide[:, 1:1 + 2 * S:2]
        view.copy_(t)
        return view

    out = dict(advantages=place(torch.full((B, S), 5.0), 5.0), returns=place(torch.full((B, S), 5.0), 5.0))
    got = binding.cham_gae(place(i["rewards"], 9), place(i["values"], 9), 0.99, lam, dones=place(i["dones"], 1), bootstrap=i["bootstrap"].to(DEV),
                           lengths=i["lengths"].to(DEV), out=out)
    _check_gae(got, (adv, ret), there, 5.0)
    if layout == "odd":
        assert (out["advantages"]._base[:, 0::2] == 5).all()
    adv, ret, there = ref.gae(i["rewards"], i["values"], 0.9, 0.99)
    got = binding.cham_gae(place(i["rewards"], 9), place(i["values"], 9), 0.9, 0.99)
    _check_gae(got, (adv, ret), there)


def test_gae_steps_behind_a_length_are_not_read_and_lengths_are_held():
    i = _gae_inputs(6, 40, torch.float32, 3)
    i["lengths"] = torch.tensor([0, 1, 39, 40, 41, -3], dtype=torch.int32)
    adv, ret, there = ref.gae(i["rewards"], i["values"], 0.9, 0.9, None, i["bootstrap"], i["lengths"])
    r, v = (torch.where(there, t, torch.full_like(t, math.nan)) for t in (i["rewards"], i["values"]))
    for place in (lambda t: t.to(DEV), lambda t: t.to(DEV).t().contiguous().t()):
        got = binding.cham_gae(place(r), place(v), 0.9, 0.9, bootstrap=i["bootstrap"].to(DEV), lengths=i["lengths"].to(DEV))
        _check_gae(got, (adv, ret), there)
    only = binding.cham_gae(r.to(DEV), v.to(DEV), 0.9, 0.9, bootstrap=i["bootstrap"].to(DEV), lengths=i["lengths"].to(DEV),
                            out=dict(advantages=torch.zeros(6, 40, device=DEV), returns=None))
    assert torch.equal(only["advantages"], got["advantages"])


@pytest.mark.parametrize("B,S,at", [(9, 70, 33), (9, 70, 32), (2, 3000, 1999), (1, 60000, 40000), (600, 700, 300), (8, 400, 127)])
def test_gae_an_episode_keeps_its_nan(B, S, at):
    i = _gae_inputs(B, S, torch.float32, 91)
    i["dones"][:] = 0
    i["dones"][:, at] = 1                                 # the last step of the first episode
    for place in (lambda t: t.to(DEV), lambda t: t.to(DEV).t().contiguous().t()):
        run = lambda: binding.cham_gae(place(i["rewards"]), place(i["values"]), 1.0, 1.0, dones=place(i["dones"]))["advantages"]
        i["rewards"][:, S - 1] = 1.0
        clean = run()
        i["rewards"][:, S - 1] = math.nan                 # of the second
        got = run()
        assert torch.equal(got[:, :at + 1], clean[:, :at + 1])
        assert torch.isnan(got[:, at + 1:]).all()
        i["rewards"][:, S - 1] = 1.0
    # factors that become too small for a double do not end an episode
    v = torch.zeros(1, 20000, device=DEV)
    r = torch.zeros(1, 20000, device=DEV)
    r[0, -1] = math.nan
    assert torch.isnan(binding.cham_gae(r, v, 0.5, 0.5)["advantages"]).all()


@pytest.mark.parametrize("gamma,lam", [(0.0, 0.9), (0.9, 0.0)])
@pytest.mark.parametrize("B,S", [(9, 70), (600, 700), (1, 30000)])
def test_gae_without_a_sum_behind(B, S, gamma, lam):
    i = _gae_inputs(B, S, torch.float32, 92)
    adv, ret, there = ref.gae(i["rewards"], i["values"], gamma, lam, i["dones"], i["bootstrap"], None)
    for place in (lambda t: t.to(DEV), lambda t: t.to(DEV).t().contiguous().t()):
        r, v, d = place(i["rewards"]), place(i["values"]), place(i["dones"])
        _check_gae(binding.cham_gae(r, v, gamma, lam, dones=d, bootstrap=i["bootstrap"].to(DEV)), (adv, ret), there)
        d.zero_()
        r[:, S - 1] = math.nan                            # 0 times what is no number is none, with dones or without them
        for dones in (None, d):
            assert torch.isnan(binding.cham_gae(r, v, gamma, lam, dones=dones)["advantages"]).all()


def test_gae_side_by_side_in_many_chunks():
    B, S = 20, 40001
    i = _gae_inputs(B, S, torch.float32, 77)
    i["lengths"][:3] = torch.tensor([S, 1, 512])
    adv, ret, there = ref.gae(i["rewards"], i["values"], 1.0, 0.999, i["dones"], i["bootstrap"], i["lengths"])
    side = lambda t: t.to(DEV).t().contiguous().t()
    got = binding.cham_gae(side(i["rewards"]), side(i["values"]), 1.0, 0.999, dones=side(i["dones"]), bootstrap=i["bootstrap"].to(DEV), lengths=i["lengths"].to(DEV))
    assert got["advantages"].stride() == (1, B)
    _check_gae(got, (adv, ret), there)


def test_gae_shared_rewards_and_no_trajectories():
    r = torch.randn(1, 50, generator=_gen(1)).to(DEV).expand(9, 50)          # one reward row for all
    v = torch.randn(9, 51, generator=_gen(2)).to(DEV)[:, :50]
    adv, ret, there = ref.gae(r, v, 0.9, 0.95)
    _check_gae(binding.cham_gae(r, v, 0.9, 0.95, dones=torch.zeros(9, 50, dtype=torch.bool, device=DEV)), (adv, ret), there)
    assert binding.cham_gae(r[:0], v[:0], 0.9, 0.9)["advantages"].shape == (0, 50)
    assert binding.cham_gae(r[:, :0], v[:, :0], 0.9, 0.9)["advantages"].shape == (9, 0)


# --- gradients

def _tensors(sizes, types, seed, scale=1.0, offset=0):
    g = _gen(seed)
    out = []
    for i, n in enumerate(sizes):
        t = types[i % len(types)]
        base = torch.zeros(n + offset, dtype=t, device=DEV)
        base[offset:] = (scale * torch.randn(n, generator=g)).to(t)
        out.append(base[offset:])
    return out


def _norm64(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts))


@pytest.mark.parametrize("offset", [0, 1, 3])
@pytest.mark.parametrize("sizes", [[1], [0, 5, 0], [7, 8, 9, 16384, 16385], [1] * 300, [100003, 3, 0, 250000], [64 * 72, 72, 64 * 64, 64, 64 * 24, 64],
                                   [(i * 37) % 4001 for i in range(700)], [20000000]], ids=lambda s: f"{len(s)}x{max(s)}")
@pytest.mark.parametrize("types", [TYPES[:1], TYPES[1:2], TYPES], ids=["f32", "bf16", "mixed"])
def test_norm_and_clip_over_sizes(sizes, types, offset):
    ts = _tensors(sizes, types, 5, offset=offset)
    keep = [t.clone() for t in ts]
    want = _norm64(ts)
    n = max(sum(sizes), 1)
    got = binding.cham_grad_norm(ts)["norm"]
    assert abs(float(got) - want) <= want * n * 2.0 ** -52
    outs = _tensors(sizes, types, 6, offset=(offset * 2) % 5)
    r = binding.cham_clip_grads(ts, 0.3 * want, out=outs)
    assert torch.equal(r["norm"], got)
    factor = min(1.0, 0.3 * want / (want + 1e-6))
    for t, k, o in zip(ts, keep, outs):
        assert torch.equal(t, k)
        x = k.double() * factor
        # the factor and the product are rounded to fp32, the result to its type
        assert (o.double() - x).abs().le(x.abs() * (2 * ref.U + ref.HALF[t.dtype]) * (1 + 1e-6) + ref.TINY[t.dtype]).all()
    again = binding.GradList(ts)
    r = binding.cham_clip_grads(again, 0.3 * want)                        # in place: the same
    for t, o in zip(ts, outs):
        assert torch.equal(t, o)
    # nothing to clip: not touched, or copied
    r = binding.cham_clip_grads(again, 1e30)
    for t, o in zip(ts, outs):
        assert torch.equal(t, o)
    fresh = [torch.full_like(t, 3.0) for t in ts]
    binding.cham_clip_grads(again, math.inf, out=fresh)
    for t, o in zip(ts, fresh):
        assert torch.equal(t, o)


def test_norm_and_clip_of_many_chunks():
    # more than 128 MiB: a workgroup for every 32 KiB scales
    sizes = [5, 41_000_001, 0, 16384, 16_000_003]
    types = (torch.bfloat16, torch.bfloat16, torch.float32, torch.float16, torch.float32)
    g = torch.Generator(device=DEV).manual_seed(6)
    ts = [torch.randn(n, generator=g, device=DEV).to(t) for n, t in zip(sizes, types)]
    want = _norm64(ts)
    outs = [torch.empty_like(t) for t in ts]
    r = binding.cham_clip_grads(ts, 0.3 * want, out=outs)
    assert abs(float(r["norm"]) - want) <= want * sum(sizes) * 2.0 ** -52
    factor = 0.3 * want / (want + 1e-6)
    for t, o in zip(ts, outs):
        x = t.double() * factor
        assert (o.double() - x).abs().le(x.abs() * (2 * ref.U + ref.HALF[t.dtype]) * (1 + 1e-6) + ref.TINY[t.dtype]).all()
    binding.cham_clip_grads(ts, 0.3 * want)
    for t, o in zip(ts, outs):
        assert torch.equal(t, o)


def test_norm_of_values_whose_squares_leave_fp32():
    for scale in (1e30, 1e-30):
        ts = _tensors([1000, 77], TYPES[:2], 9, scale=scale)
        want = _norm64(ts)
        assert abs(float(binding.cham_grad_norm(ts)["norm"]) - want) <= want * 1e-12


def test_clip_of_what_is_no_number():
    ts = _tensors([1000, 50], TYPES[:1], 10)
    ts[1][3] = math.nan
    r = binding.cham_clip_grads(ts, 1.0)
    assert torch.isnan(r["norm"]).all() and all(torch.isnan(t).all() for t in ts)
    ts = _tensors([1000, 50], TYPES[:1], 10)
    ts[0][7] = math.inf
    r = binding.cham_clip_grads(ts, 1.0)
    assert torch.isinf(r["norm"]).all() and torch.isnan(ts[0][7]) and not ts[1].any() and int(torch.isnan(ts[0]).sum()) == 1
    z = [torch.zeros(10, device=DEV)]
    assert float(binding.cham_clip_grads(z, 0.0)["norm"]) == 0.0 and not z[0].any()
    ts = _tensors([100], TYPES[:1], 10)
    binding.cham_clip_grads(ts, 0.0)
    assert not ts[0].any()


def test_norm_given_and_no_tensors():
    ts = _tensors([1000, 50], TYPES[:1], 11)
    keep = [t.clone() for t in ts]
    norm = torch.tensor([10.0], dtype=torch.float64, device=DEV)
    r = binding.cham_clip_grads(ts, 5.0, norm=norm, norm_given=True)
    assert float(r["norm"]) == 10.0
    f = torch.tensor(5.0 / (10.0 + 1e-6), dtype=torch.float64).float().to(DEV)
    for t, k in zip(ts, keep):
        assert torch.equal(t, k * f)
    assert float(binding.cham_grad_norm([])["norm"]) == 0.0
    assert float(binding.cham_clip_grads([], 1.0)["norm"]) == 0.0
    assert float(binding.cham_clip_grads([torch.zeros(0, device=DEV)], 1.0)["norm"]) == 0.0
