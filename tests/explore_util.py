"""The agent's update in 64 bits, written from its definitions, and how far fp32 kernels may be from it."""
import math

import torch

HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}    # of a value, rounding to the type
TINY = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25}
U = 2.0 ** -24


def heads(logits, actions, first):
    """Per head, in 64 bits: in or not, log-probabilities (-inf where masked), probabilities, choice (0 where not in)."""
    x = logits.double().cpu()
    if x.dim() == 2:
        x = x[:, None]
    a = actions.long().cpu().reshape(x.shape[:2]) - first
    V = x.shape[-1]
    bad = a >= V
    live = ((a >= 0) & (x != -math.inf).any(-1)) | bad
    m = x.amax(-1, keepdim=True)
    z = torch.where(live[..., None] & ~bad[..., None], x - m, torch.zeros_like(x))
    logs = z - torch.log(torch.exp(z).sum(-1, keepdim=True))
    logs = torch.where(bad[..., None], torch.full_like(logs, math.nan), logs)
    return live, logs, torch.exp(logs), a.clamp(0, V - 1)


def policy(logits, actions, first=0, weights=None):
    """logp, entropy [R] and whether a decision counts."""
    live, logs, p, a = heads(logits, actions, first)
    lp = torch.where(live, logs.gather(-1, a[..., None])[..., 0], torch.zeros(()).double()).sum(-1)
    plogp = torch.where(p == 0, torch.zeros_like(p), p * logs)
    H = torch.where(live, -plogp.sum(-1), torch.zeros(()).double()).sum(-1)
    on = live.any(-1)
    if weights is not None:
        on = on & (weights.cpu() != 0)
    zero = torch.zeros_like(lp)
    return torch.where(on, lp, zero), torch.where(on, H, zero), on


def loss(logits, actions, old, adv, first=0, ref=None, weights=None, values=None, old_values=None, returns=None, clip_low=0.2, clip_high=0.2,
         value_coef=0.0, entropy_coef=0.0, kl_coef=0.0, value_clip=0.2):
    """terms [6], logp, entropy, grad_logits, grad_values in 64 bits, and per item how far the kernel's gradient may be off."""
    live, logs, p, a = heads(logits, actions, first)
    lp, H, on = policy(logits, actions, first, weights)
    R, G, V = p.shape
    w = (torch.full((R,), 1.0 / max(R, 1), dtype=torch.float64) if weights is None else weights.cpu()).double()
    zero = torch.zeros(R, dtype=torch.float64)
    adv, old = adv.double().cpu(), old.double().cpu()
    rho = torch.exp(lp - old)
    free, held = rho * adv, rho.clamp(1 - clip_low, 1 + clip_high) * adv
    clipped = free > held
    D = torch.where(clipped, zero, -free)
    size = free.abs()
    kl = zero
    if ref is not None:
        d = ref.double().cpu() - lp
        kl = torch.where(torch.isposinf(torch.exp(d)), torch.exp(d), torch.exp(d) - d - 1)      # infinite where d is
        if kl_coef != 0:
            D = D + kl_coef * (1 - torch.exp(d))
            size = size + kl_coef * torch.exp(d)
    vl, gv = zero, None
    if values is not None:
        v, t = values.double().cpu(), returns.double().cpu()
        near = (v - t) ** 2
        kept = near if old_values is None else (old_values.double().cpu() + (v - old_values.double().cpu()).clamp(-value_clip, value_clip) - t) ** 2
        vl = torch.maximum(near, kept) / 2
        gv = torch.where(on & (near >= kept), w * value_coef * (v - t), zero)
    parts = torch.stack([-torch.minimum(free, held), vl, H, kl, clipped.double()])
    parts = torch.where(on, w * parts, zero)
    s = parts.sum(-1)
    # a term with coefficient 0 adds nothing, whatever it is
    total = s[0]
    for c, x in ((value_coef, s[1]), (-entropy_coef, s[2]), (kl_coef, s[3])):
        total = total + c * x if c != 0 else total
    counts = (on[:, None] & live)[..., None]
    one = torch.zeros_like(p).scatter_(-1, a[..., None], 1.0)
    Dw, Ew = (w * D)[:, None, None], (w * entropy_coef)[:, None, None]
    lg = logs.clamp(min=-800.0)
    Hg = -torch.where(p == 0, torch.zeros_like(p), p * logs).sum(-1, keepdim=True)
    grad = torch.where(counts, Dw * (one - p) + Ew * p * (lg + Hg), torch.zeros_like(p))
    e = lse_error(V)
    off = ((w * size).abs() * logp_error(V, G))[:, None, None] + Dw.abs() * 4 * U
    rel = e + (2 * lg.abs() + 6) * U
    tol = off * (one - p).abs() + p * (Dw.abs() + Ew.abs() * (lg.abs() + Hg)) * rel + Ew.abs() * p * (entropy_error(V, 1) + e + 4 * U * lg.abs())
    tol = tol + HALF[logits.dtype] * grad.abs() * (1 + 1e-6) + TINY[logits.dtype]
    terms_tol = torch.where(on, w.abs() * (size + 1) * logp_error(V, G) * 4 + w.abs() * entropy_error(V, G), zero).sum() + 2 * U * (s.abs().sum() + 1e-30)
    return dict(terms=torch.cat([total[None], s]), logp=lp, entropy=H, grad_logits=grad.reshape(logits.shape), grad_values=gv,
                tol=tol.reshape(logits.shape), terms_tol=terms_tol, on=on)


def lse_error(V):
    """Of a head's log-sum-exp.  An exponential e^z is off by (2 |z| + 3) U of itself (difference, product with log2 e, exp2 within an
    ulp), and sum e^z |z| / sum e^z <= log V; at most V / 64 additions and rescalings follow one another in a lane, and 30 join the lanes."""
    return (2 * math.log(V) + 3 + 2 * (V / 64 + 30)) * U + 2 * U * math.log(2 * V)


def logp_error(V, G):
    return G * (lse_error(V) + 40 * U)         # logits here are below 40 from their maximum, their differences rounded once


def entropy_error(V, G):
    return G * (1 + 2 * math.log(V + 1)) * 2 * lse_error(V)


def gae(rewards, values, gamma, lam, dones=None, bootstrap=None, lengths=None):
    """Advantages and returns in 64 bits, step by step, and which steps are there."""
    r, v = rewards.double().cpu(), values.double().cpu()
    B, S = r.shape
    n = torch.full((B,), S) if lengths is None else lengths.long().cpu().clamp(0, S)
    go = torch.ones(B, S, dtype=torch.float64) if dones is None else (dones.cpu() == 0).double()
    boot = torch.zeros(B, dtype=torch.float64) if bootstrap is None else bootstrap.double().cpu()
    adv = torch.zeros(B, S, dtype=torch.float64)
    a = torch.zeros(B, dtype=torch.float64)
    for t in range(S - 1, -1, -1):
        there = t < n
        nxt = torch.where(t == n - 1, boot, v[:, t + 1] if t + 1 < S else boot)
        a = torch.where(there, r[:, t] + gamma * go[:, t] * nxt - v[:, t] + gamma * lam * go[:, t] * a, torch.zeros(()).double())
        adv[:, t] = a
    return adv, adv + v, torch.arange(S) < n[:, None]
