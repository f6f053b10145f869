"""Workloads of the exploration agent's update, the operators beside the configuration updater: log-probabilities of
actions, the clipped policy loss with its gradients, advantages, and clipping of gradients by their global norm.

Decisions have one head per knob with three directions each (what ``cham_update_configs`` applies), one head per knob with
a choice each, or a single head of many choices (tokens of a policy that is a language model).  The plain form computes in 32
bits, per decision in 64 (ratios next to the border of the clip, differences of log-probabilities), and the recurrence and
the sum of squares in 64.
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # one step of the paper's 128 trajectories: log-probabilities of the directions just taken; latency is all there is
        dict(name="logp-step", op="logp", rows=128, heads=24, choices=3, type="f32"),
        # log-probabilities of a micro-batch of tokens under the old or the reference policy
        dict(name="logp-tokens", op="logp", rows=4096, heads=1, choices=32768, type="bf16"),
        # one epoch over an iteration of the explorer: 128 trajectories x 500 steps x 24 knobs, the paper's coefficients
        dict(name="loss-explorer", op="loss", rows=64000, heads=24, choices=3, type="f32", clip=0.3, kl=0.0, entropy=0.1, value=1.0, padded=0.0,
             masked=False),
        # a head of choices per knob, the smaller knobs' missing choices masked
        dict(name="loss-choices", op="loss", rows=4099, heads=12, choices=24, type="f32", clip=0.2, kl=0.05, entropy=0.01, value=0.5,
             padded=0.1, masked=True),
        # a handful of answered tokens, an odd vocabulary
        dict(name="loss-few-tokens", op="loss", rows=9, heads=1, choices=50021, type="f32", clip=0.2, kl=0.05, entropy=0.0, value=0.0, padded=0.0,
             masked=False),
        # a padded batch in half precision (the weights carry the scale of the loss), an odd vocabulary
        dict(name="loss-padded", op="loss", rows=6001, heads=1, choices=8191, type="f16", clip=0.2, kl=0.1, entropy=0.01, value=0.5, padded=0.3,
             masked=True),
        # a micro-batch of tokens over a large vocabulary: the largest call
        dict(name="loss-tokens", op="loss", rows=4096, heads=1, choices=131072, type="bf16", clip=0.2, kl=0.05, entropy=0.0, value=0.0,
             padded=0.0, masked=False),
        # the explorer's trajectories as the updater walks them: step by step, 128 side by side
        dict(name="gae-explorer", op="gae", rows=128, steps=500, by_step=True, type="f32", ragged=False, dones=True),
        # answers of uneven length, one row each
        dict(name="gae-tokens", op="gae", rows=512, steps=8192, by_step=False, type="bf16", ragged=True, dones=False),
        # few very long runs with episodes ending inside
        dict(name="gae-long", op="gae", rows=3, steps=200003, by_step=False, type="f32", ragged=False, dones=True),
        # the explorer's own small network: latency
        dict(name="clip-explorer", op="clip", model=64, layers=1, vocab=72, type="f32"),
        # the matrices and vectors of a language model
        dict(name="clip-model", op="clip", model=2048, layers=24, vocab=65536, type="bf16"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logp", "loss", "loss", "gae", "clip"])
    kind = rng.choice(["f32", "bf16", "f16"])
    if op in ("logp", "loss"):
        if rng.random() < 0.4:                              # knobs
            heads, choices = rng.randint(2, 40), rng.choice([2, 3, 3, rng.randint(4, 40)])
            rows = _log_int(rng, 16, 64000)
        else:                                               # tokens
            heads, choices = 1, _log_int(rng, 100, 131072)
            rows = _log_int(rng, 1, min(16384, (1 << 28) // choices))
        case = dict(op=op, rows=rows, heads=heads, choices=choices, type=kind)
        if op == "loss":
            case.update(clip=rng.choice([0.1, 0.2, 0.3]), kl=rng.choice([0.0, 0.05, 0.2]), entropy=rng.choice([0.0, 0.01, 0.1]),
                        value=rng.choice([0.0, 0.5, 1.0]), padded=rng.choice([0.0, 0.0, 0.2, 0.6]), masked=choices > 3 and rng.random() < 0.3)
        return case
    if op == "gae":
        rows = _log_int(rng, 1, 2048)
        return dict(op=op, rows=rows, steps=_log_int(rng, 1, min(200000, (1 << 22) // rows)), by_step=rng.random() < 0.5, type=rng.choice(["f32", "f32", kind]),
                    ragged=rng.random() < 0.5, dones=rng.random() < 0.5)
    return dict(op=op, model=_log_int(rng, 16, 1536), layers=rng.randint(1, 24), vocab=_log_int(rng, 30, 50000), type=kind)


def _shapes(case):
    """Gradients of a network: embedding, per layer four square and three wide matrices and two vectors, a last vector."""
    m = case["model"]
    wide = (8 * m // 3 + 7) // 8 * 8 + 1
    layer = [(m, m)] * 4 + [(wide, m)] * 2 + [(m, wide)] + [(m,)] * 2
    return [(case["vocab"], m)] + layer * case["layers"] + [(m,)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dev = "cuda"

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=dev)

    def uniform(*shape):
        return torch.rand(*shape, generator=gen, device=dev)

    kind = _TYPES[case["type"]]
    if case["op"] in ("logp", "loss"):
        R, G, V = case["rows"], case["heads"], case["choices"]
        logits = torch.empty(R, G, V, dtype=kind, device=dev)
        actions = torch.empty(R, G, dtype=torch.int64, device=dev)
        logp = torch.empty(R, dtype=torch.float32, device=dev)
        cards = torch.randint(2, V + 1, (G,), generator=gen, device=dev)
        part = max(1, (1 << 26) // (G * V))
        for r in range(0, R, part):                         # actions are drawn from the policy itself
            n = min(part, R - r)
            x = (2.0 * normal(n, G, V)).to(kind)
            if case.get("masked"):                          # each head has its own number of choices
                x = x.masked_fill(torch.arange(V, device=dev) >= cards[:, None], -math.inf)
            logits[r:r + n] = x
            a = (x.float() - torch.log(-torch.log(uniform(n, G, V).clamp(1e-7, 1.0 - 1e-7)))).argmax(-1)
            actions[r:r + n] = a
            x = x.float()
            logp[r:r + n] = (x.gather(-1, a[..., None])[..., 0] - x.logsumexp(-1)).sum(-1)
        first = 0
        if V == 3:                                          # directions, as the updater takes them
            actions, first = (actions - 1).to(torch.int8), -1
        state = dict(case=case, logits=logits, actions=actions, first=first)
        if case["op"] == "loss":
            # how far the policy has moved since the actions were taken.  A ratio that falls on the border of the clip itself belongs to
            # either side, by its last rounding: it is put to one
            moved = 0.15 * normal(R)
            for border in (math.log1p(case["clip"]), math.log1p(-case["clip"])):
                moved = torch.where((moved - border).abs() < 2e-4, moved + 1e-3, moved)
            weights = torch.ones(R, device=dev)
            if case["padded"] > 0:
                weights = (uniform(R) >= case["padded"]).float()
            scale = 65536.0 if case["type"] == "f16" else 1.0
            state["weights"] = weights * scale / weights.sum().clamp(min=1.0)
            state["old"] = logp - moved
            state["adv"] = normal(R)
            state["ref"] = logp + 0.2 * normal(R) if case["kl"] > 0 else None
            if case["value"] > 0:
                state["values"] = normal(R)
                state["old_values"] = state["values"] + 0.3 * normal(R)
                state["returns"] = state["values"] + normal(R)
        return state
    if case["op"] == "gae":
        B, S = case["rows"], case["steps"]
        shape = (S, B) if case["by_step"] else (B, S)
        view = (lambda t: t.t()) if case["by_step"] else (lambda t: t)
        state = dict(case=case, rewards=view((0.1 * normal(*shape)).to(kind)), values=view(normal(*shape).to(kind)), bootstrap=normal(B))
        state["dones"] = view((uniform(*shape) < 4.0 / S).to(torch.uint8)) if case["dones"] else None
        state["lengths"] = torch.randint(1, S + 1, (B,), generator=gen, device=dev, dtype=torch.int32) if case["ragged"] else None
        state["out"] = dict(advantages=view(torch.zeros(*shape, device=dev)), returns=view(torch.zeros(*shape, device=dev)))
        return state
    # gradients in one buffer, as a program that reduces them keeps them; every tensor begins at a multiple of 256 bytes
    shapes = _shapes(case)
    sizes = [math.prod(s) for s in shapes]
    step = 256 // torch.finfo(kind).bits * 8
    starts = np.concatenate([[0], np.cumsum([(n + step - 1) // step * step for n in sizes])]).tolist()
    flat, clipped = (torch.zeros(starts[-1], dtype=kind, device=dev) for _ in range(2))
    grads = [flat[s:s + n].view(shape) for s, n, shape in zip(starts, sizes, shapes)]
    outs = [clipped[s:s + n].view(shape) for s, n, shape in zip(starts, sizes, shapes)]
    for i, g in enumerate(grads):
        g.copy_(normal(*g.shape) * (1e-3 * (1 + i % 7)))
    return dict(case=case, grads=grads, outs=outs, clipped=clipped, max_norm=0.5 * 1e-3 * 4 * math.sqrt(sum(sizes)))


# What the explorer's update is run with (discount and trace of the paper's table of hyper-parameters), and how far values are clipped
_GAMMA, _LAMBDA, _VALUE_CLIP = 0.9, 0.99, 0.2


def _plain_softmax(state):
    """exp(x - max), its sum, log-probabilities (0 where a choice is masked) and what actions choose, in 32 bits."""
    x = state["logits"].float()
    a = (state["actions"].long() - state["first"])[..., None]
    z = x - x.amax(-1, keepdim=True)
    e = torch.exp(z)
    s = e.sum(-1, keepdim=True)
    logp = torch.where(e > 0, z - torch.log(s), torch.zeros_like(z))
    p = e / s
    entropy = -(p * logp).sum(-1)
    return a, p, logp, logp.gather(-1, a)[..., 0].double().sum(-1), entropy


def _plain_logp(state):
    _, _, _, lp, entropy = _plain_softmax(state)
    return dict(logp=lp.float(), entropy=entropy.double().sum(-1).float())


def _plain_loss(state):
    case = state["case"]
    a, p, logp, lp, entropy = _plain_softmax(state)
    H = entropy.double().sum(-1)
    w, adv = state["weights"].double(), state["adv"].double()
    ratio = torch.exp(lp - state["old"].double())
    free = ratio * adv
    held = ratio.clamp(1.0 - case["clip"], 1.0 + case["clip"]) * adv
    policy = -torch.minimum(free, held)
    d = torch.where(free <= held, -free, torch.zeros_like(free))
    kl = torch.zeros_like(lp)
    if case["kl"] > 0:
        gap = state["ref"].double() - lp
        kl = torch.expm1(gap) - gap
        d = d - case["kl"] * torch.expm1(gap)
    value, grad_values = torch.zeros_like(lp), None
    if case["value"] > 0:
        v, o, t = (state[k].double() for k in ("values", "old_values", "returns"))
        near = (v - t).square()
        kept = (o + (v - o).clamp(-_VALUE_CLIP, _VALUE_CLIP) - t).square()
        value = 0.5 * torch.maximum(near, kept)
        grad_values = torch.where(near >= kept, w * case["value"] * (v - t), torch.zeros_like(v)).float()
    parts = torch.stack([policy, value, H, kl, (free > held).double()])
    sums = (torch.where(w != 0, parts, torch.zeros_like(parts)) * w).sum(-1)
    total = sums[0] + case["value"] * sums[1] - case["entropy"] * sums[2] + case["kl"] * sums[3]
    d = torch.where(w != 0, w * d, torch.zeros_like(d)).float()[:, None, None]
    grad = -d * p
    grad.scatter_add_(-1, a, d.expand_as(a))
    if case["entropy"] > 0:
        grad += (case["entropy"] * w).float()[:, None, None] * p * (logp + entropy[..., None])
    on = (w != 0).float()
    return dict(terms=torch.cat([total[None], sums]).float(), logp=lp.float() * on, entropy=H.float() * on,
                grad_logits=grad.to(state["logits"].dtype), grad_values=grad_values)


def _plain_gae(state):
    r, v = state["rewards"].double(), state["values"].double()
    B, S = r.shape
    at = torch.arange(S, device=r.device)
    n = torch.full((B,), S, device=r.device) if state["lengths"] is None else state["lengths"].long()
    inside = at < n[:, None]
    going = torch.ones_like(r) if state["dones"] is None else 1.0 - state["dones"].double()
    after = torch.where(at == n[:, None] - 1, state["bootstrap"].double()[:, None], torch.nn.functional.pad(v[:, 1:], (0, 1)))
    b = torch.where(inside, r + _GAMMA * going * after - v, torch.zeros_like(r))
    c = _GAMMA * _LAMBDA * going
    # A_t = b_t + c_t A_(t+1): runs of 1, 2, 4, ... steps are joined until one reaches the end
    span = 1
    while span < S:
        b = b + c * torch.nn.functional.pad(b[:, span:], (0, span))
        c = c * torch.nn.functional.pad(c[:, span:], (0, span))
        span *= 2
    out = state["out"]
    out["advantages"].copy_(torch.where(inside, b.float(), out["advantages"]))
    out["returns"].copy_(torch.where(inside, (b + v).float(), out["returns"]))
    return dict(out)


def _plain_clip(state):
    norm = torch.stack([g.double().square().sum() for g in state["grads"]]).sum().sqrt()
    scale = (state["max_norm"] / (norm + 1e-6)).clamp(max=1.0).float()
    [o.copy_(g.float() * scale) for o, g in zip(state["outs"], state["grads"])]
    return dict(norm=norm.reshape(1), clipped=state["clipped"])


def _own(state):
    from paper_2001_08743_amd import binding
    case = state["case"]
    kept = state.setdefault("kept", {})                     # output buffers, workspace and list of tensors, as a program keeps them
    if case["op"] == "logp":
        r = binding.cham_policy_logp(state["logits"], state["actions"], first_action=state["first"], out=kept.get("out"), workspace=kept.get("workspace"))
        kept.update(out=r, workspace=r["workspace"])
        return dict(logp=r["logp"], entropy=r["entropy"])
    if case["op"] == "loss":
        r = binding.cham_policy_loss(state["logits"], state["actions"], state["old"], state["adv"], first_action=state["first"],
                                     ref_logp=state["ref"], weights=state["weights"], values=state.get("values"),
                                     old_values=state.get("old_values"), returns=state.get("returns"), clip_low=case["clip"],
                                     clip_high=case["clip"], kl_coef=case["kl"], entropy_coef=case["entropy"], value_coef=case["value"],
                                     value_clip=_VALUE_CLIP, out=kept.get("out"), workspace=kept.get("workspace"))
        kept.update(out=r, workspace=r["workspace"])
        return {k: r[k] for k in ("terms", "logp", "entropy", "grad_logits", "grad_values")}
    if case["op"] == "gae":
        r = binding.cham_gae(state["rewards"], state["values"], _GAMMA, _LAMBDA, dones=state["dones"], bootstrap=state["bootstrap"],
                             lengths=state["lengths"], out=state["out"], workspace=kept.get("workspace"))
        kept["workspace"] = r["workspace"]
        return dict(advantages=r["advantages"], returns=r["returns"])
    if "grads" not in kept:
        kept.update(grads=binding.GradList(state["grads"]), outs=binding.GradList(state["outs"]))
    r = binding.cham_clip_grads(kept["grads"], state["max_norm"], out=kept["outs"], norm=kept.get("norm"), workspace=kept.get("workspace"))
    kept.update(norm=r["norm"], workspace=r["workspace"])
    return dict(norm=r["norm"], clipped=state["clipped"])


def run(state):
    if own:
        return _own(state)
    return {"logp": _plain_logp, "loss": _plain_loss, "gae": _plain_gae, "clip": _plain_clip}[state["case"]["op"]](state)


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}[case["type"]]
    if case["op"] in ("logp", "loss"):
        R, n = case["rows"], case["rows"] * case["heads"] * case["choices"]
        acts = case["rows"] * case["heads"] * (1 if case["choices"] == 3 else 8)
        if case["op"] == "logp":                            # maximum, difference, exponential, two sums
            return dict(bytes=n * size + acts + 8 * R, flops=6 * n)
        # decisions that do not count are written (zeros), not read
        read = n * (1.0 - case["padded"])
        rows = R * (20 + (4 if case["kl"] > 0 else 0) + (16 if case["value"] > 0 else 0))
        return dict(bytes=(read + n) * size + acts + rows, flops=read * (6 + 4 + (3 if case["entropy"] > 0 else 0)))
    if case["op"] == "gae":
        n = case["rows"] * case["steps"] * (0.5 if case["ragged"] else 1.0)
        return dict(bytes=n * (2 * size + 8 + (1 if case["dones"] else 0)) + 8 * case["rows"], flops=7 * n)
    n = sum(math.prod(s) for s in _shapes(case))
    return dict(bytes=2 * n * size + 8, flops=3 * n)


def exact(case, seed):
    """From the definitions, in 64 bits: gradients by differentiation, the recurrence step by step."""
    state = prepare(case, seed)
    if case["op"] in ("logp", "loss"):
        return _exact_policy(case, state)
    if case["op"] == "gae":
        r, v = (state[k].double().cpu().numpy() for k in ("rewards", "values"))
        B, S = r.shape
        n = np.full(B, S) if state["lengths"] is None else state["lengths"].cpu().numpy()
        go = np.ones((B, S)) if state["dones"] is None else 1.0 - state["dones"].cpu().numpy()
        r, v, go = (np.ascontiguousarray(x.T) for x in (r, v, go))
        adv, ret = np.zeros((S, B)), np.zeros((S, B))
        a, nxt = np.zeros(B), np.zeros(B)
        boot = state["bootstrap"].double().cpu().numpy()
        for t in range(S - 1, -1, -1):
            live = t < n
            nxt = np.where(t == n - 1, boot, nxt)
            a = np.where(live, r[t] + _GAMMA * go[t] * nxt - v[t] + _GAMMA * _LAMBDA * go[t] * a, 0.0)
            nxt = v[t]
            adv[t], ret[t] = a, np.where(live, a + v[t], 0.0)
        return dict(advantages=torch.from_numpy(adv.T.copy()), returns=torch.from_numpy(ret.T.copy()))
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in state["grads"]))
    flat = torch.zeros(state["clipped"].shape, dtype=torch.float64, device="cuda")
    base = state["grads"][0].storage_offset()
    for g in state["grads"]:
        at = g.storage_offset() - base
        flat[at:at + g.numel()] = g.double().reshape(-1) * min(1.0, state["max_norm"] / (norm + 1e-6))
    return dict(norm=torch.tensor([norm], dtype=torch.float64), clipped=flat)


def _exact_policy(case, state):
    R, G, V = state["logits"].shape
    part = max(1, (1 << 27) // (G * V))
    got = {k: [] for k in ("logp", "entropy", "grad_logits", "grad_values")}
    terms = torch.zeros(6, dtype=torch.float64, device="cuda")
    for r in range(0, R, part):
        rows = slice(r, r + part)
        x = state["logits"][rows].double().requires_grad_()
        taken = state["actions"][rows].long() - state["first"]
        logs = torch.log_softmax(x, -1)
        lp = logs.gather(-1, taken[..., None]).sum((-1, -2))
        masked = torch.isneginf(x)
        H = -(torch.exp(logs) * logs.masked_fill(masked, 0.0)).sum((-1, -2))
        if case["op"] == "logp":
            got["logp"].append(lp.detach())
            got["entropy"].append(H.detach())
            continue
        w = state["weights"][rows].double()
        A = state["adv"][rows].double()
        rho = torch.exp(lp - state["old"][rows].double())
        bounded = torch.clamp(rho, 1 - case["clip"], 1 + case["clip"])
        pg = torch.maximum(-rho * A, -bounded * A)
        kl = torch.zeros_like(lp)
        if case["kl"] > 0:
            diff = state["ref"][rows].double() - lp
            kl = torch.exp(diff) - diff - 1
        vl = torch.zeros_like(lp)
        if case["value"] > 0:
            v = state["values"][rows].double().requires_grad_()
            o, t = state["old_values"][rows].double(), state["returns"][rows].double()
            moved = torch.minimum(torch.maximum(v, o - _VALUE_CLIP), o + _VALUE_CLIP)
            vl = torch.maximum((v - t) ** 2 / 2, (moved - t) ** 2 / 2)
        loss = (w * (pg + case["value"] * vl - case["entropy"] * H + case["kl"] * kl)).sum()
        loss.backward()
        g = x.grad
        terms += torch.stack([loss, (w * pg).sum(), (w * vl).sum(), (w * H).sum(), (w * kl).sum(), (w * (-bounded * A > -rho * A)).sum()]).detach()
        got["grad_logits"].append(torch.where(masked, torch.zeros_like(g), g))
        if case["value"] > 0:
            # where both are alike the derivative of the maximum halves: inside the clip both have that of the first
            got["grad_values"].append(v.grad)
        got["logp"].append(lp.detach() * (w != 0))
        got["entropy"].append(H.detach() * (w != 0))
    out = {k: torch.cat(v) if v else None for k, v in got.items()}
    return dict(out, terms=terms) if case["op"] == "loss" else dict(logp=out["logp"], entropy=out["entropy"])
