"""A round of the exploration agent as a program runs it: actions of a policy through the configuration updater, advantages,
the clipped loss, gradients of the networks, clipping; by itself and captured into a graph."""
import torch
import pytest

import explore_util as ref
from paper_2001_08743_amd import binding

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
STEPS, B, KNOBS, HIDDEN = 30, 16, 7, 32
COEF = dict(clip_low=0.3, clip_high=0.3, value_coef=1.0, entropy_coef=0.1, value_clip=0.2)


def _net(seed):
    g = torch.Generator().manual_seed(seed)
    shapes = [(HIDDEN, KNOBS), (HIDDEN,), (3 * KNOBS, HIDDEN), (3 * KNOBS,), (1, HIDDEN), (1,)]
    return [(0.3 * torch.randn(*s, generator=g)).to(DEV).requires_grad_() for s in shapes]


def _forward(p, theta, cards):
    h = torch.tanh((theta.to(p[0].dtype) / cards.to(p[0].dtype)) @ p[0].t() + p[1])
    return (h @ p[2].t() + p[3]).reshape(-1, KNOBS, 3), (h @ p[4].t() + p[5])[:, 0]


def _explore(p, seed):
    """States, actions and their log-probabilities along B trajectories, through the updater."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    cards = torch.randint(3, 20, (KNOBS,), generator=g, device=DEV)
    theta = torch.zeros(B, KNOBS, dtype=torch.uint8, device=DEV)
    table = binding.cham_visited_table_clear(torch.zeros(1 << 14, dtype=torch.int64, device=DEV))
    rows = torch.zeros(1 << 12, KNOBS, dtype=torch.uint8, device=DEV)
    count = torch.zeros(1, dtype=torch.int32, device=DEV)
    states, actions, logps, values = [], [], [], []
    for _ in range(STEPS):
        with torch.no_grad():
            logits, v = _forward(p, theta, cards)
            logits = logits.contiguous()
            u = torch.rand(logits.shape, generator=g, device=DEV).clamp(1e-6, 1 - 1e-6)
            a = ((logits - torch.log(-torch.log(u))).argmax(-1) - 1).to(torch.int8)
        states.append(theta.clone())
        actions.append(a)
        logps.append(binding.cham_policy_logp(logits, a, first_action=-1)["logp"])
        values.append(v)
        binding.cham_update_configs(theta, a, cards.to(torch.int16), 1, table, rows, count)
    assert 0 < int(count) <= STEPS * B
    return cards, torch.stack(states), torch.stack(actions), torch.stack(logps), torch.stack(values), theta


def test_a_round_gives_the_gradients_of_its_definition():
    p = _net(1)
    cards, states, actions, old, values, last = _explore(p, 2)
    g = torch.Generator(device=DEV).manual_seed(3)
    rewards = torch.randn(STEPS, B, generator=g, device=DEV)
    with torch.no_grad():
        bootstrap = _forward(p, last, cards)[1]
    # steps are stored first: trajectories side by side
    r = binding.cham_gae(rewards.t(), values.t(), 0.9, 0.99, bootstrap=bootstrap)
    adv, ret, there = ref.gae(rewards.t(), values.t(), 0.9, 0.99, bootstrap=bootstrap)
    assert (r["advantages"].cpu().double() - adv).abs().le(ref.U * adv.abs() * 1.01 + 1e-9).all()
    adv, ret = (r[k].t().reshape(-1) for k in ("advantages", "returns"))
    # an epoch later the networks have moved
    with torch.no_grad():
        for t in p:
            t += 0.02 * torch.randn(t.shape, generator=g, device=DEV)
    flat = states.reshape(-1, KNOBS)
    logits, v = _forward(p, flat, cards)
    out = binding.cham_policy_loss(logits.detach(), actions.reshape(-1, KNOBS), old.reshape(-1), adv, first_action=-1, values=v.detach(),
                                   old_values=values.reshape(-1), returns=ret, **COEF)
    torch.autograd.backward([logits, v], [out["grad_logits"], out["grad_values"]])
    norm = binding.cham_grad_norm([t.grad for t in p])["norm"]
    before = [t.grad.clone() for t in p]
    binding.cham_clip_grads([t.grad for t in p], 0.5 * float(norm), norm=norm, norm_given=True)

    q = [t.detach().double().cpu().requires_grad_() for t in p]
    logits64, v64 = _forward(q, flat.cpu(), cards.cpu())
    logs = torch.log_softmax(logits64, -1)
    lp = logs.gather(-1, (actions.reshape(-1, KNOBS).long().cpu() + 1)[..., None]).sum((-1, -2))
    rho = torch.exp(lp - old.reshape(-1).double().cpu())
    A = adv.double().cpu()
    assert ((rho - 0.7).abs() > 1e-4).all() and ((rho - 1.3).abs() > 1e-4).all()      # no ratio on the border
    o, t = values.reshape(-1).double().cpu(), ret.double().cpu()
    kept = o + (v64 - o).clamp(-0.2, 0.2)
    vl = torch.maximum((v64 - t) ** 2, (kept - t) ** 2) / 2
    H = -(torch.exp(logs) * logs).sum((-1, -2))
    loss = (-torch.minimum(rho * A, rho.clamp(0.7, 1.3) * A) + vl - 0.1 * H).mean()
    loss.backward()
    # the networks run in fp32: 64 products a sum, and 480 decisions whose gradients are added
    assert abs(float(out["terms"][0]) - loss.item()) <= 1e-5 * (1 + abs(loss.item()))
    scale = max(float(t.grad.abs().max()) for t in q)
    for t, b, x in zip(p, before, q):
        assert (b.cpu().double() - x.grad).abs().max() <= 2e-5 * scale
        assert torch.equal(t.grad, b * torch.tensor(0.5 * float(norm) / (float(norm) + 1e-6), dtype=torch.float32, device=DEV))


@pytest.mark.parametrize("R,G,V", [(40, 6, 3), (6, 1, 30000), (64, 1, 2000)])
def test_captured_update_replays_as_the_eager_one(R, G, V):
    g = torch.Generator(device=DEV).manual_seed(4)
    x = torch.zeros(R, G, V, device=DEV)
    a = torch.zeros(R, G, dtype=torch.int32, device=DEV)
    old, adv, rew, val = (torch.zeros(R, device=DEV) for _ in range(4))
    outs = [torch.empty(R, G, V, device=DEV), torch.empty(R, device=DEV)]

    def update():
        lp = binding.cham_policy_logp(x, a)
        gae = binding.cham_gae(rew.reshape(1, R), val.reshape(1, R), 0.99, 0.95)
        r = binding.cham_policy_loss(x, a, old, gae["advantages"][0], values=val, returns=gae["returns"][0], value_coef=0.5, entropy_coef=0.01)
        c = binding.cham_clip_grads([r["grad_logits"], r["grad_values"]], 1e-3, out=outs)
        return [lp["logp"], gae["advantages"], r["terms"], r["grad_logits"], r["grad_values"], c["norm"], *outs]

    def fill():
        x.copy_(torch.randn(x.shape, generator=g, device=DEV))
        a.copy_(torch.randint(0, V, a.shape, generator=g, device=DEV))
        for t in (old, adv, rew, val):
            t.copy_(torch.randn(R, generator=g, device=DEV))
        old.mul_(0.1).add_(binding.cham_policy_logp(x, a)["logp"])

    fill()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        update()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        static = update()
    for _ in range(4):
        fill()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in static]
        for k, (s, e) in enumerate(zip(got, update())):
            assert torch.equal(s, e), k
